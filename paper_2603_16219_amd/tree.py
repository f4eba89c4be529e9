"""Binding of trees of drafted tokens (include/specsteer_tree.h): argument marshalling only.

As in ``binding``, arguments that need nothing done to them go to native code (csrc/tree/tree_calls.cpp), others through ctypes here.

A block of drafts that branches: its tree grows from the specialist's likeliest tokens (``losses.token_alternatives``), ``attention`` scores its
rows over the cache in each of a model's layers, ``verify`` walks it as ``binding.verify_block`` does a chain, and ``commit`` keeps the
keys and values of the accepted path:

    out = tree.attention(q, k, v, k_cache, v_cache, block_table, cache_len, parents)            # per layer, [B, N + 1, heads, dim]
    step = tree.verify(G, S_ctx, S_noctx, tokens, uniforms, parents, lam=0.5, beta=1.0)          # logits [B, N + 1, V]
    cache_len = tree.commit(k, v, k_cache, v_cache, block_table, cache_len, step["accepted_len"], step["path"])   # per layer

parents [B, N] holds each node's parent, an earlier node or -1 for the last token, which is row 0 of everything that has N + 1 rows; without it
trees are chains, and with N = 0 there is the last token alone.  All work is done by ``libspecsteer_tree.so`` (hand-written HIP for
gfx950) on torch's current stream.  There is no CPU or PyTorch fallback, and no gradient.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional

import torch  # imported before the library so both share one HIP runtime

from . import build as _build
from .binding import SS_FLAG_GREEDY, SpecSteerError, SSParams, _ptr, _ready, _refuse_repeated_rows, _stream, load_wrappers, make_params

_DTYPES = {torch.bfloat16: 1, torch.float16: 2}


class SSTreeParams(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("nodes", ctypes.c_int32),
        ("heads", ctypes.c_int32),
        ("kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("pages", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("table_width", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("q_stride", ctypes.c_int64 * 3),
        ("k_stride", ctypes.c_int64 * 3),
        ("out_stride", ctypes.c_int64 * 3),
        ("cache_stride", ctypes.c_int64 * 3),
        ("table_stride", ctypes.c_int64),
    ]


_lib = None
_calls = None  # the native wrappers, once the library is loaded and if they can be


def library() -> ctypes.CDLL:
    """Load libspecsteer_tree.so from the package directory (building it only if absent)."""
    global _lib, _calls
    if _lib is None:
        path = _build.TREE_LIBRARY
        if not os.path.exists(path):
            _build.build_tree_library()
        lib = ctypes.CDLL(path)
        p, params, block = ctypes.c_void_p, ctypes.POINTER(SSTreeParams), ctypes.POINTER(SSParams)
        lib.specsteer_tree_attention_workspace_bytes.restype = ctypes.c_size_t
        lib.specsteer_tree_attention_workspace_bytes.argtypes = [params]
        lib.specsteer_tree_verify_workspace_bytes.restype = ctypes.c_size_t
        lib.specsteer_tree_verify_workspace_bytes.argtypes = [block]
        lib.specsteer_tree_attention.argtypes = [p] * 9 + [params] + [p] * 2 + [ctypes.c_size_t, p]
        lib.specsteer_tree_verify.argtypes = [p] * 7 + [block] + [p] * 5 + [ctypes.c_size_t, p]
        lib.specsteer_tree_commit.argtypes = [p] * 8 + [params] + [p] * 2
        for name in ("attention", "verify", "commit"):
            getattr(lib, "specsteer_tree_" + name).restype = ctypes.c_int
        lib.specsteer_tree_status_string.restype = ctypes.c_char_p
        lib.specsteer_tree_status_string.argtypes = [ctypes.c_int]
        _lib = lib
        _calls = load_wrappers("_tree_calls", _build.tree_calls_path, _build.build_tree_calls, lambda: (
            lib.specsteer_tree_attention_workspace_bytes, lib.specsteer_tree_attention, lib.specsteer_tree_verify_workspace_bytes,
            lib.specsteer_tree_verify, lib.specsteer_tree_commit))
    return _lib


def _native(name: str, *args):
    """What the native wrapper of this name returns for arguments that it takes, None for others."""
    if _lib is None:
        library()
    if _calls is None:
        return None
    out = getattr(_calls, name)(*args)
    if type(out) is int:
        raise SpecSteerError(out, status_string(out))
    return out


def status_string(status: int) -> str:
    return library().specsteer_tree_status_string(int(status)).decode()


def attention_workspace_bytes(params: SSTreeParams) -> int:
    return int(library().specsteer_tree_attention_workspace_bytes(ctypes.byref(params)))


def verify_workspace_bytes(params: SSParams) -> int:
    return int(library().specsteer_tree_verify_workspace_bytes(ctypes.byref(params)))


def _call(function, device: torch.device, *args) -> None:
    """A call of the library on the device's current stream, with that device the current one."""
    if torch.cuda.current_device() == device.index:
        rc = function(*args, _stream(device))
    else:
        with torch.cuda.device(device):
            rc = function(*args, _stream(device))
    if rc != 0:
        raise SpecSteerError(rc, status_string(rc))


def _strides(t: torch.Tensor, what: str) -> list:
    """Strides of [.., .., heads, dim] for the library: 0 where a dimension of size 1 or none makes one meaningless."""
    if t.numel():
        if t.stride(3) != 1:
            raise ValueError(f"{what} must have its last dimension contiguous")
        if any(n > 1 and s == 0 for n, s in zip(t.shape[:3], t.stride()[:3])):
            raise ValueError(f"{what} must not repeat the same memory (an expanded tensor): pass a contiguous copy")
        if any(n > 1 and s % 8 for n, s in zip(t.shape[:3], t.stride()[:3])) or t.data_ptr() % 16:
            raise ValueError(f"{what} must have all its rows at multiples of 16 bytes")
    return [s if n > 1 else 0 for n, s in zip(t.shape[:3], t.stride()[:3])]


def _ints(t: Optional[torch.Tensor], what: str, shape: tuple, device: torch.device) -> Optional[torch.Tensor]:
    if t is None:
        return None
    if t.dtype.is_floating_point or t.dtype.is_complex or t.dtype in (torch.bool, torch.uint32, torch.uint64):
        raise TypeError(f"{what} must be integers, got {t.dtype}")
    if tuple(t.shape) != shape:
        raise ValueError(f"{what} must be {list(shape)}, got {list(t.shape)}")
    if t.dtype is torch.int64:  # a number beyond 32 bits must not come out as another, valid one: the least is none, the largest may be a length
        t = torch.where((t < 2**31) & (t >= -2**31), t, -2**31)
    return _ready(t, device, torch.int32)


def _scratch(workspace: Optional[torch.Tensor], need: int, device: torch.device) -> torch.Tensor:
    if workspace is None:
        return torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    if not workspace.is_contiguous() or workspace.device != device:
        raise ValueError("workspace must be a contiguous tensor on the arguments' device")
    return workspace


def _bytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


def _cache_params(k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, block_table: torch.Tensor) -> tuple:
    """Params of a call with the cache, those of the queries left out, and the table as it is passed."""
    if k.dim() != 4 or k.shape != v.shape:
        raise ValueError("k and v must both be [B, N + 1, kv_heads, dim]")
    B, R, H, D = k.shape
    if R < 1:
        raise ValueError("k and v must have a row for the last token")
    if k_cache.dim() != 4 or k_cache.shape != v_cache.shape or tuple(k_cache.shape[2:]) != (H, D) or k_cache.shape[1] < 1:
        raise ValueError(f"k_cache and v_cache must both be [pages, page_size, {H}, {D}]")
    code = _DTYPES.get(k.dtype)
    if code is None:
        raise TypeError(f"keys and values must be bfloat16 or float16, got {k.dtype}")
    if not (k.dtype == v.dtype == k_cache.dtype == v_cache.dtype):
        raise ValueError("keys, values and their caches must share a dtype")
    if not k.is_cuda:
        raise ValueError("trees need device tensors; there is no CPU path")
    if not (k.device == v.device == k_cache.device == v_cache.device):
        raise ValueError("keys, values and their caches must be on one device")
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError(f"block_table must be [B, pages of a sequence] with B = {B}, got {list(block_table.shape)}")
    ks, cs = _strides(k, "k"), _strides(k_cache, "k_cache")
    if ks != _strides(v, "v"):
        raise ValueError("k and v must share strides")
    if cs != _strides(v_cache, "v_cache"):
        raise ValueError("k_cache and v_cache must share strides")
    width = block_table.shape[1]
    if not (block_table.dtype is torch.int32 and block_table.device == k.device and (width <= 1 or block_table.stride(1) == 1) and
            (B <= 1 or block_table.stride(0) >= width)):
        block_table = _ints(block_table, "block_table", (B, width), k.device)
    p = SSTreeParams(batch=B, nodes=R - 1, heads=H, kv_heads=H, head_dim=D, dtype=code, pages=k_cache.shape[0], page_size=k_cache.shape[1],
                     table_width=width, scale=0.0, table_stride=block_table.stride(0) if B > 1 and width else 0)
    p.k_stride[:], p.cache_stride[:] = ks, cs
    return p, block_table


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, block_table: torch.Tensor,
              cache_len: torch.Tensor, parents: Optional[torch.Tensor] = None, *, tree_len: Optional[torch.Tensor] = None,
              scale: Optional[float] = None, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """specsteer_tree_attention of q [B, N + 1, heads, dim] with the block's own k and v [B, N + 1, kv_heads, dim] over caches [pages, page_size,
    kv_heads, dim] in bfloat16 or float16, dim 64 or 128: [B, N + 1, heads, dim], into `out` if given.  block_table [B, pages of a sequence],
    cache_len [B], parents [B, N] or None for chains, tree_len [B] or None for N are integers.  scale is 1 / sqrt(dim) unless given."""
    res = _native("attention", q, k, v, k_cache, v_cache, block_table, cache_len, parents, tree_len, scale, out, workspace)
    if res is not None:
        return res
    p, table = _cache_params(k, v, k_cache, v_cache, block_table)
    B, R, H, D = k.shape
    dev = k.device
    if q.dim() != 4 or tuple(q.shape[:2]) != (B, R) or q.shape[3] != D or q.shape[2] < 1 or q.shape[2] % H:
        raise ValueError(f"q must be [{B}, {R}, a multiple of {H}, {D}], got {list(q.shape)}")
    if D not in (64, 128):
        raise ValueError(f"heads must have 64 or 128 elements, got {D}")
    if q.dtype != k.dtype or q.device != dev:
        raise ValueError("q must have the keys' dtype and device")
    cache_len = _ints(cache_len, "cache_len", (B,), dev)
    parents = _ints(parents, "parents", (B, R - 1), dev)
    tree_len = _ints(tree_len, "tree_len", (B,), dev)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=dev)
    elif out.shape != q.shape or out.dtype != q.dtype or out.device != dev:
        raise ValueError("out must have q's shape, dtype and device")
    elif out.numel() and out.untyped_storage().data_ptr() in [t.untyped_storage().data_ptr() for t in (q, k, v, k_cache, v_cache)]:
        raise ValueError("out must not share memory with an input")
    p.heads, p.scale = q.shape[2], 1 / math.sqrt(D) if scale is None else scale
    p.q_stride[:], p.out_stride[:] = _strides(q, "q"), _strides(out, "out")
    workspace = _scratch(workspace, attention_workspace_bytes(p), dev)
    _call(library().specsteer_tree_attention, dev, _ptr(q), _ptr(k), _ptr(v), _ptr(k_cache), _ptr(v_cache), _ptr(table), _ptr(cache_len),
          _ptr(parents), _ptr(tree_len), ctypes.byref(p), _ptr(out), _ptr(workspace), _bytes(workspace))
    torch.autograd.graph.increment_version(out)
    return out


def verify(G: torch.Tensor, S_ctx: torch.Tensor, S_noctx: torch.Tensor, tokens: torch.Tensor, uniforms: torch.Tensor,
           parents: Optional[torch.Tensor] = None, *, lam: float = 0.5, beta: float = 1.0, temperature: float = 1.0,
           tree_len: Optional[torch.Tensor] = None, greedy: bool = False, workspace: Optional[torch.Tensor] = None) -> dict:
    """specsteer_tree_verify on logits [B, N + 1, V] (vocab stride 1), tokens [B, N] and uniforms [B, N + 1]: {"accepted_len" [B], "path" [B, N],
    "next_token" [B] int32, "next_token_logprob" [B] float32}.  parents [B, N], or None for chains."""
    res = _native("verify", G, S_ctx, S_noctx, tokens, uniforms, parents, lam, beta, temperature, tree_len, greedy, workspace)
    if res is not None:
        return res
    if not (G.shape == S_ctx.shape == S_noctx.shape) or G.dim() != 3 or G.shape[1] < 1:
        raise ValueError("logit tensors must share a [B, N + 1, V] shape")
    if not (G.dtype == S_ctx.dtype == S_noctx.dtype):
        raise ValueError("logit tensors must share a dtype")
    if not (G.is_cuda and G.device == S_ctx.device == S_noctx.device):
        raise ValueError("trees need device tensors on one device; there is no CPU path")
    B, R, V = G.shape
    lead = [n > 1 for n in (B, R)]
    if any([s for s, m in zip(t.stride(), lead) if m] != [s for s, m in zip(G.stride(), lead) if m] or (V > 1 and t.stride(2) != 1) for t in (G, S_ctx, S_noctx)):
        raise ValueError("logit tensors must share strides, with the vocabulary contiguous")
    if (B > 1 and G.stride(0) == 0) or (R > 1 and G.stride(1) == 0):
        _refuse_repeated_rows()
    dev = G.device
    if tuple(uniforms.shape) != (B, R) or not uniforms.dtype.is_floating_point:
        raise ValueError(f"uniforms must be floating point, [B, N + 1] = [{B}, {R}], got {list(uniforms.shape)}")
    tokens = _ints(tokens, "tokens", (B, R - 1), dev)
    parents = _ints(parents, "parents", (B, R - 1), dev)
    tree_len = _ints(tree_len, "tree_len", (B,), dev)
    uniforms = _ready(uniforms, dev, torch.float32)
    params = make_params(B, R - 1, V, G.dtype, lam=lam, beta=beta, temperature=temperature, stride_b=G.stride(0) if B > 1 else 0,
                         stride_t=G.stride(1) if R > 1 else 0, flags=SS_FLAG_GREEDY if greedy else 0)
    workspace = _scratch(workspace, verify_workspace_bytes(params), dev)
    out = {"accepted_len": torch.empty(B, dtype=torch.int32, device=dev), "path": torch.empty(B, R - 1, dtype=torch.int32, device=dev),
           "next_token": torch.empty(B, dtype=torch.int32, device=dev), "next_token_logprob": torch.empty(B, dtype=torch.float32, device=dev)}
    _call(library().specsteer_tree_verify, dev, _ptr(G), _ptr(S_ctx), _ptr(S_noctx), _ptr(tokens), _ptr(parents), _ptr(tree_len), _ptr(uniforms),
          ctypes.byref(params), _ptr(out["accepted_len"]), _ptr(out["path"]), _ptr(out["next_token"]), _ptr(out["next_token_logprob"]), _ptr(workspace),
          _bytes(workspace))
    return out


def commit(k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, block_table: torch.Tensor, cache_len: torch.Tensor,
           accepted_len: torch.Tensor, path: Optional[torch.Tensor] = None) -> torch.Tensor:
    """specsteer_tree_commit: rows 0 and path + 1 of k and v [B, N + 1, kv_heads, dim] to the ends of the cached sequences, in place.  path [B, N] and
    accepted_len [B] are what verify returned; without a path the rows are a chain's, whose accepted_len verify_block returns.  Returns the new
    cache lengths [B] int32, -1 for sequences of which nothing was written."""
    res = _native("commit", k, v, k_cache, v_cache, block_table, cache_len, accepted_len, path)
    if res is not None:
        return res
    p, table = _cache_params(k, v, k_cache, v_cache, block_table)
    B, R, _, D = k.shape
    if D % 8 or not 8 <= D <= 1024:
        raise ValueError(f"heads must have a multiple of 8 elements, up to 1024, got {D}")
    dev = k.device
    caches = [t.untyped_storage().data_ptr() for t in (k_cache, v_cache) if t.numel()]
    if any(t.numel() and t.untyped_storage().data_ptr() in caches for t in (k, v)):
        raise ValueError("k and v must not share memory with the caches")
    cache_len = _ints(cache_len, "cache_len", (B,), dev)
    accepted_len = _ints(accepted_len, "accepted_len", (B,), dev)
    path = _ints(path, "path", (B, R - 1), dev)
    new_len = torch.empty(B, dtype=torch.int32, device=dev)
    _call(library().specsteer_tree_commit, dev, _ptr(k), _ptr(v), _ptr(k_cache), _ptr(v_cache), _ptr(table), _ptr(cache_len), _ptr(accepted_len),
          _ptr(path), ctypes.byref(p), _ptr(new_len))
    torch.autograd.graph.increment_version(k_cache)
    torch.autograd.graph.increment_version(v_cache)
    return new_len
