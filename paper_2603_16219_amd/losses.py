"""Binding of the losses over full-vocabulary logits (include/specsteer_loss.h), and of their rows' entropies and likeliest tokens
(include/specsteer_alternatives.h): argument marshalling only.

As in ``binding``, arguments that need nothing done to them go to native code (csrc/loss/loss_calls.cpp), others through ctypes here.

Every sum, loss and gradient is formed inside ``libspecsteer_loss.so`` (hand-written HIP for gfx950) on torch's current
stream; PyTorch supplies device memory and the stream.  There is no CPU or PyTorch fallback.

A loss comes with the gradient of the logits it was given, which the model's own backward pass goes on from:

    out = losses.policy_loss(logits, tokens, old_logprobs, advantages, mask=mask, ref_logprobs=ref, kl_coef=0.05)
    logits.backward(out["grad_logits"])

Logits may have any strides with the vocabulary contiguous and each sequence's rows before the next one's (logits[:, :-1] of a padded
vocabulary; not [T, B, V].transpose(0, 1)).

The gradient may go to a tensor of the caller's, `grad_logits=`, which may be the logits themselves.  Autograd takes that for an operation in
place: the backward pass of a model whose last operation keeps its output (a tanh, say) refuses logits that were replaced.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch  # imported before the library so both share one HIP runtime

from . import build as _build
from .binding import SpecSteerError, _ptr, _ready, _refuse_repeated_rows, _stream, load_wrappers

SS_LOSS_SUM = 1
SS_LOSS_SEQ_MEAN = 2
SS_LOSS_SEQ_ADVANTAGES = 4

_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


class SSLossParams(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("length", ctypes.c_int32),
        ("vocab", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("stride_b", ctypes.c_int64),
        ("stride_t", ctypes.c_int64),
        ("grad_stride_b", ctypes.c_int64),
        ("grad_stride_t", ctypes.c_int64),
        ("temperature", ctypes.c_float),
        ("grad_scale", ctypes.c_float),
    ]


class SSPolicyParams(ctypes.Structure):
    _fields_ = [("clip_low", ctypes.c_float), ("clip_high", ctypes.c_float), ("kl_coef", ctypes.c_float), ("flags", ctypes.c_uint32)]


class SSPreferenceParams(ctypes.Structure):
    _fields_ = [("beta", ctypes.c_float), ("label_smoothing", ctypes.c_float), ("flags", ctypes.c_uint32)]


_lib = None
_calls = None  # the native wrappers, once the library is loaded and if they can be


def library() -> ctypes.CDLL:
    """Load libspecsteer_loss.so from the package directory (building it only if absent)."""
    global _lib, _calls
    if _lib is None:
        path = _build.LOSS_LIBRARY
        if not os.path.exists(path):
            _build.build_loss_library()
        lib = ctypes.CDLL(path)
        p, params = ctypes.c_void_p, ctypes.POINTER(SSLossParams)
        lib.specsteer_loss_workspace_bytes.restype = ctypes.c_size_t
        lib.specsteer_loss_workspace_bytes.argtypes = [params]
        lib.specsteer_token_logprobs.argtypes = [p] * 3 + [params] + [p] * 3 + [ctypes.c_size_t, p]
        lib.specsteer_token_logprobs_grad.argtypes = [p] * 5 + [params] + [p] * 2
        lib.specsteer_policy_loss.argtypes = [p] * 7 + [params, ctypes.POINTER(SSPolicyParams)] + [p] * 5 + [ctypes.c_size_t, p]
        lib.specsteer_preference_loss.argtypes = [p] * 4 + [params, ctypes.POINTER(SSPreferenceParams)] + [p] * 6 + [ctypes.c_size_t, p]
        lib.specsteer_token_alternatives_workspace_bytes.restype = ctypes.c_size_t
        lib.specsteer_token_alternatives_workspace_bytes.argtypes = [params, ctypes.c_int32]
        lib.specsteer_token_alternatives.argtypes = [p] * 3 + [params, ctypes.c_int32] + [p] * 6 + [ctypes.c_size_t, p]
        lib.specsteer_token_alternatives_grad.argtypes = [p] * 7 + [params] + [p] * 2
        for name in ("token_logprobs", "token_logprobs_grad", "policy_loss", "preference_loss", "token_alternatives", "token_alternatives_grad"):
            getattr(lib, "specsteer_" + name).restype = ctypes.c_int
        lib.specsteer_loss_status_string.restype = ctypes.c_char_p
        lib.specsteer_loss_status_string.argtypes = [ctypes.c_int]
        _lib = lib
        _calls = load_wrappers("_loss_calls", _build.loss_calls_path, _build.build_loss_calls, lambda: (
            lib.specsteer_loss_workspace_bytes, lib.specsteer_token_logprobs, lib.specsteer_token_logprobs_grad, lib.specsteer_policy_loss,
            lib.specsteer_preference_loss, lib.specsteer_token_alternatives_workspace_bytes, lib.specsteer_token_alternatives,
            lib.specsteer_token_alternatives_grad))
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
    return library().specsteer_loss_status_string(int(status)).decode()


def workspace_bytes(params: SSLossParams) -> int:
    return int(library().specsteer_loss_workspace_bytes(ctypes.byref(params)))


def _call(function, device: torch.device, *args) -> None:
    """A call of the library on the device's current stream, with that device the current one."""
    if torch.cuda.current_device() == device.index:
        rc = function(*args, _stream(device))
    else:
        with torch.cuda.device(device):
            rc = function(*args, _stream(device))
    if rc != 0:
        raise SpecSteerError(rc, status_string(rc))


def _strides(t: torch.Tensor, what: str) -> tuple:
    """Strides for the library: 0 where a dimension of size 1 or none makes one meaningless."""
    B, T, V = t.shape
    sb, st, sv = t.stride()
    if sv != 1 and V > 1:
        raise ValueError(f"{what} must have the vocabulary contiguous")
    if t.numel() and ((B > 1 and sb == 0) or (T > 1 and st == 0)):
        _refuse_repeated_rows()
    return (sb if B > 1 and T > 0 else 0, st if T > 1 else 0)


def _make_params(logits: torch.Tensor, tokens: torch.Tensor, temperature: float, grad_scale: float = 1.0,
                 grad_logits: Optional[torch.Tensor] = None) -> SSLossParams:
    if logits.dim() != 3:
        raise ValueError("logits must be [B, T, V]")
    code = _DTYPES.get(logits.dtype)
    if code is None:
        raise TypeError(f"logits must be float32 or bfloat16, got {logits.dtype}")
    if not logits.is_cuda:
        raise ValueError("the losses need device tensors; there is no CPU path")
    if tuple(tokens.shape) != tuple(logits.shape[:2]):
        raise ValueError(f"tokens must be [B, T] = {list(logits.shape[:2])}, got {tuple(tokens.shape)}")
    sb, st = _strides(logits, "logits")
    gsb, gst = (0, 0) if grad_logits is None else _strides(grad_logits, "grad_logits")
    return SSLossParams(*logits.shape, code, sb, st, gsb, gst, temperature, grad_scale)


def _ready_tokens(tokens: torch.Tensor, device: torch.device) -> torch.Tensor:
    if tokens.dtype is torch.int64:  # an id beyond 32 bits must not come out as another, valid one
        tokens = tokens.clamp(-1, 2**31 - 1)
    elif tokens.dtype.is_floating_point or tokens.dtype.is_complex or tokens.dtype in (torch.bool, torch.uint64):
        raise TypeError(f"tokens must be integers that int64 holds, got {tokens.dtype}")
    return _ready(tokens, device, torch.int32)


def _ready_mask(mask: Optional[torch.Tensor], tokens: torch.Tensor, device: torch.device) -> Optional[torch.Tensor]:
    if mask is None:
        return None
    if mask.dtype not in (torch.bool, torch.uint8):
        raise TypeError(f"mask must be bool or uint8, got {mask.dtype}")
    if mask.shape != tokens.shape:
        raise ValueError(f"mask must be [B, T] = {list(tokens.shape)}, got {tuple(mask.shape)}")
    return _ready(mask, device, mask.dtype)


def _ready_rows(t: Optional[torch.Tensor], what: str, tokens: torch.Tensor, device: torch.device) -> Optional[torch.Tensor]:
    if t is None:
        return None
    if t.shape != tokens.shape:
        raise ValueError(f"{what} must be [B, T] = {list(tokens.shape)}, got {tuple(t.shape)}")
    if not t.dtype.is_floating_point:
        raise TypeError(f"{what} must be floating point, got {t.dtype}")
    return _ready(t, device, torch.float32)


def _gradient(logits: torch.Tensor, want: bool, out: Optional[torch.Tensor], ref_logits: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """The tensor that the gradient goes to."""
    if out is None:
        return torch.empty(logits.shape, dtype=logits.dtype, device=logits.device) if want else None
    if not want:
        raise ValueError("grad_logits was given but no gradient is wanted")
    if out.shape != logits.shape or out.dtype != logits.dtype or out.device != logits.device:
        raise ValueError("grad_logits must have the logits' shape, type and device")
    storage = out.untyped_storage().data_ptr()
    if out.numel() and storage == logits.untyped_storage().data_ptr() and not (
            out.data_ptr() == logits.data_ptr() and out.stride() == logits.stride()):
        raise ValueError("grad_logits must be the logits themselves or memory of its own")
    if out.numel() and ref_logits is not None and storage == ref_logits.untyped_storage().data_ptr():
        raise ValueError("grad_logits must not share memory with ref_logits")
    return out


def _written(grad_logits: Optional[torch.Tensor]) -> None:
    """Autograd learns that the gradient was written to a tensor, which may be one that a backward pass has saved."""
    if grad_logits is not None:
        torch.autograd.graph.increment_version(grad_logits)


def _scratch(workspace: Optional[torch.Tensor], params: SSLossParams, device: torch.device, need=None) -> torch.Tensor:
    if workspace is None:
        return torch.empty(max(workspace_bytes(params) if need is None else need, 256), dtype=torch.uint8, device=device)
    if not workspace.is_contiguous() or workspace.device != device:
        raise ValueError("workspace must be a contiguous tensor on the logits' device")
    return workspace


def _bytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, *, mask: Optional[torch.Tensor] = None, temperature: float = 1.0,
                   want_stats: bool = False, workspace: Optional[torch.Tensor] = None) -> dict:
    """specsteer_token_logprobs on logits [B, T, V] and tokens [B, T]: {"logprobs" [B, T] float32, 0 where `mask` [B, T] is
    false, "stats" [B, T, 2] or None}.  The stats are what token_logprobs_grad takes."""
    out = _native("token_logprobs", logits, tokens, mask, temperature, want_stats, workspace)
    if out is not None:
        return out
    params = _make_params(logits, tokens, temperature)
    dev = logits.device
    mask = _ready_mask(mask, tokens, dev)
    tokens = _ready_tokens(tokens, dev)
    workspace = _scratch(workspace, params, dev)
    logprobs = torch.empty(tokens.shape, dtype=torch.float32, device=dev)
    stats = torch.empty(*tokens.shape, 2, dtype=torch.float32, device=dev) if want_stats else None
    _call(library().specsteer_token_logprobs, dev, _ptr(logits), _ptr(tokens), _ptr(mask), ctypes.byref(params), _ptr(logprobs), _ptr(stats),
          _ptr(workspace), _bytes(workspace))
    return {"logprobs": logprobs, "stats": stats}


def token_logprobs_grad(logits: torch.Tensor, tokens: torch.Tensor, stats: torch.Tensor, grad_logprobs: torch.Tensor, *,
                        mask: Optional[torch.Tensor] = None, temperature: float = 1.0, grad_scale: float = 1.0,
                        grad_logits: Optional[torch.Tensor] = None) -> torch.Tensor:
    """specsteer_token_logprobs_grad: the gradient [B, T, V] with respect to the logits, in their type, of a loss whose gradient with
    respect to their log-probs is grad_logprobs [B, T].  It goes to `grad_logits` if given, which may be the logits."""
    out = _native("token_logprobs_grad", logits, tokens, stats, grad_logprobs, mask, temperature, grad_scale, grad_logits)
    if out is not None:
        return out
    grad_logits = _gradient(logits, True, grad_logits)
    params = _make_params(logits, tokens, temperature, grad_scale, grad_logits)
    dev = logits.device
    if tuple(stats.shape) != (*tokens.shape, 2) or stats.dtype is not torch.float32 or stats.device != dev:
        raise ValueError("stats must be what token_logprobs(..., want_stats=True) returned for these logits")
    mask = _ready_mask(mask, tokens, dev)
    grad_logprobs = _ready_rows(grad_logprobs, "grad_logprobs", tokens, dev)
    tokens, stats = _ready_tokens(tokens, dev), stats.contiguous()
    _call(library().specsteer_token_logprobs_grad, dev, _ptr(logits), _ptr(tokens), _ptr(mask), _ptr(stats), _ptr(grad_logprobs),
          ctypes.byref(params), _ptr(grad_logits))
    _written(grad_logits)
    return grad_logits


MAX_TOPK = 64


def alternatives_workspace_bytes(params: SSLossParams, topk: int) -> int:
    return int(library().specsteer_token_alternatives_workspace_bytes(ctypes.byref(params), topk))


def token_alternatives(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, *, topk: int = 0, mask: Optional[torch.Tensor] = None,
                       temperature: float = 1.0, want_stats: bool = False, workspace: Optional[torch.Tensor] = None) -> dict:
    """specsteer_token_alternatives on logits [B, T, V] and, if given, tokens [B, T]: {"logprobs" [B, T] float32 or None without tokens,
    "entropy" [B, T] float32, "top_tokens" [B, T, topk] int32 and "top_logprobs" [B, T, topk] float32 or None for topk 0, "stats" [B, T, 2]
    or None}.  Alternatives come by decreasing logit, ties by increasing id; -1 and -inf where there is none."""
    out = _native("token_alternatives", logits, tokens, topk, mask, temperature, want_stats, workspace)
    if out is not None:
        return out
    if isinstance(topk, bool) or not isinstance(topk, int) or not 0 <= topk <= MAX_TOPK:
        raise ValueError(f"topk must be an integer in 0..{MAX_TOPK}, got {topk!r}")
    if logits.dim() != 3:
        raise ValueError("logits must be [B, T, V]")
    dev, rows = logits.device, logits.shape[:2]
    like = torch.empty(rows, dtype=torch.int32, device="meta") if tokens is None else tokens
    params = _make_params(logits, like, temperature)
    mask = _ready_mask(mask, like, dev)
    tokens = None if tokens is None else _ready_tokens(tokens, dev)
    workspace = _scratch(workspace, params, dev, alternatives_workspace_bytes(params, topk))
    logprobs = None if tokens is None else torch.empty(rows, dtype=torch.float32, device=dev)
    entropy = torch.empty(rows, dtype=torch.float32, device=dev)
    top_tokens = torch.empty(*rows, topk, dtype=torch.int32, device=dev) if topk else None
    top_logprobs = torch.empty(*rows, topk, dtype=torch.float32, device=dev) if topk else None
    stats = torch.empty(*rows, 2, dtype=torch.float32, device=dev) if want_stats else None
    _call(library().specsteer_token_alternatives, dev, _ptr(logits), _ptr(tokens), _ptr(mask), ctypes.byref(params), topk, _ptr(logprobs), _ptr(entropy),
          _ptr(top_tokens), _ptr(top_logprobs), _ptr(stats), _ptr(workspace), _bytes(workspace))
    return {"logprobs": logprobs, "entropy": entropy, "top_tokens": top_tokens, "top_logprobs": top_logprobs, "stats": stats}


def token_alternatives_grad(logits: torch.Tensor, tokens: Optional[torch.Tensor], stats: torch.Tensor, entropy: Optional[torch.Tensor],
                            grad_logprobs: Optional[torch.Tensor], grad_entropy: Optional[torch.Tensor], *, mask: Optional[torch.Tensor] = None,
                            temperature: float = 1.0, grad_scale: float = 1.0, grad_logits: Optional[torch.Tensor] = None) -> torch.Tensor:
    """specsteer_token_alternatives_grad: the gradient [B, T, V] with respect to the logits, in their type, of a loss whose gradients with
    respect to their log-probs and entropies are grad_logprobs and grad_entropy [B, T] (None: 0, not both).  stats and entropy are what
    token_alternatives(..., want_stats=True) returned.  It goes to `grad_logits` if given, which may be the logits."""
    out = _native("token_alternatives_grad", logits, tokens, stats, entropy, grad_logprobs, grad_entropy, mask, temperature, grad_scale, grad_logits)
    if out is not None:
        return out
    if grad_logprobs is None and grad_entropy is None:
        raise ValueError("give grad_logprobs, grad_entropy or both")
    if (grad_logprobs is not None and tokens is None) or (grad_entropy is not None and entropy is None):
        raise ValueError("grad_logprobs needs the tokens, grad_entropy the entropy")
    if logits.dim() != 3:
        raise ValueError("logits must be [B, T, V]")
    grad_logits = _gradient(logits, True, grad_logits)
    dev, rows = logits.device, logits.shape[:2]
    like = torch.empty(rows, dtype=torch.int32, device="meta") if tokens is None else tokens
    params = _make_params(logits, like, temperature, grad_scale, grad_logits)
    if tuple(stats.shape) != (*rows, 2) or stats.dtype is not torch.float32 or stats.device != dev:
        raise ValueError("stats must be what token_alternatives(..., want_stats=True) returned for these logits")
    mask = _ready_mask(mask, like, dev)
    grad_logprobs = _ready_rows(grad_logprobs, "grad_logprobs", like, dev)
    grad_entropy = _ready_rows(grad_entropy, "grad_entropy", like, dev)
    entropy = _ready_rows(entropy, "entropy", like, dev)
    tokens, stats = None if tokens is None else _ready_tokens(tokens, dev), stats.contiguous()
    _call(library().specsteer_token_alternatives_grad, dev, _ptr(logits), _ptr(tokens), _ptr(mask), _ptr(stats), _ptr(entropy), _ptr(grad_logprobs),
          _ptr(grad_entropy), ctypes.byref(params), _ptr(grad_logits))
    _written(grad_logits)
    return grad_logits


_REDUCTIONS = {"token_mean": 0, "sum": SS_LOSS_SUM, "seq_mean": SS_LOSS_SEQ_MEAN}


def policy_loss(logits: torch.Tensor, tokens: torch.Tensor, old_logprobs: torch.Tensor, advantages: torch.Tensor, *,
                mask: Optional[torch.Tensor] = None, ref_logits: Optional[torch.Tensor] = None,
                ref_logprobs: Optional[torch.Tensor] = None, clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0,
                temperature: float = 1.0, reduction: str = "token_mean", grad_scale: float = 1.0, want_grad: bool = True,
                grad_logits: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> dict:
    """specsteer_policy_loss: the clipped policy loss with a KL term to a reference given by its log-probs of the tokens or by its
    logits.  advantages is [B, T], or [B] for one a sequence; reduction "token_mean", "seq_mean" or "sum".  Returns {"loss" [],
    "logprobs" [B, T], "kl" [B, T] or None without a reference, "grad_logits" [B, T, V] in the logits' type or None}."""
    flags = _REDUCTIONS.get(reduction)
    if flags is None:
        raise ValueError(f"reduction must be one of {sorted(_REDUCTIONS)}, got {reduction!r}")
    out = _native("policy_loss", logits, tokens, old_logprobs, advantages, mask, ref_logits, ref_logprobs, clip_low, clip_high, kl_coef, temperature,
                  flags, grad_scale, want_grad, grad_logits, workspace)
    if out is not None:
        return out
    if ref_logits is not None and ref_logprobs is not None:
        raise ValueError("give the reference by its logits or by its log-probs, not both")
    has_ref = ref_logits is not None or ref_logprobs is not None
    if kl_coef != 0.0 and not has_ref:
        raise ValueError("a KL term needs ref_logits or ref_logprobs")
    if ref_logits is not None and (logits.dim() != 3 or ref_logits.shape != logits.shape or ref_logits.dtype != logits.dtype or
                                   _strides(ref_logits, "ref_logits") != _strides(logits, "logits") or ref_logits.device != logits.device):
        raise ValueError("ref_logits must have the logits' shape, type, strides and device")
    grad_logits = _gradient(logits, want_grad, grad_logits, ref_logits)
    params = _make_params(logits, tokens, temperature, grad_scale, grad_logits)
    dev = logits.device
    if advantages.dim() == 1 and advantages.shape[0] == logits.shape[0]:
        flags |= SS_LOSS_SEQ_ADVANTAGES
        if not advantages.dtype.is_floating_point:
            raise TypeError(f"advantages must be floating point, got {advantages.dtype}")
        advantages = _ready(advantages, dev, torch.float32)
    else:
        advantages = _ready_rows(advantages, "advantages, unless [B],", tokens, dev)
    old_logprobs = _ready_rows(old_logprobs, "old_logprobs", tokens, dev)
    ref_logprobs = _ready_rows(ref_logprobs, "ref_logprobs", tokens, dev)
    mask = _ready_mask(mask, tokens, dev)
    tokens = _ready_tokens(tokens, dev)
    workspace = _scratch(workspace, params, dev)
    loss = torch.empty((), dtype=torch.float32, device=dev)
    logprobs = torch.empty(tokens.shape, dtype=torch.float32, device=dev)
    kl = torch.empty(tokens.shape, dtype=torch.float32, device=dev) if has_ref else None
    _call(library().specsteer_policy_loss, dev, _ptr(logits), _ptr(ref_logits), _ptr(tokens), _ptr(mask), _ptr(old_logprobs),
          _ptr(ref_logprobs), _ptr(advantages), ctypes.byref(params),
          ctypes.byref(SSPolicyParams(clip_low, clip_high, kl_coef, flags)), _ptr(loss), _ptr(logprobs), _ptr(kl), _ptr(grad_logits),
          _ptr(workspace), _bytes(workspace))
    _written(grad_logits)
    return {"loss": loss, "logprobs": logprobs, "kl": kl, "grad_logits": grad_logits}


def preference_loss(logits: torch.Tensor, tokens: torch.Tensor, *, mask: Optional[torch.Tensor] = None,
                    ref_logprobs: Optional[torch.Tensor] = None, beta: float = 0.1, label_smoothing: float = 0.0,
                    temperature: float = 1.0, reduction: str = "mean", grad_scale: float = 1.0, want_grad: bool = True,
                    grad_logits: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> dict:
    """specsteer_preference_loss: sequence i of the first half of the batch is preferred to sequence i of the second.  reduction "mean"
    or "sum" over the pairs.  Returns {"loss" [], "pair_loss" [B/2], "margin" [B/2], "logprobs" [B, T], "grad_logits" [B, T, V] in
    the logits' type or None}."""
    if reduction not in ("mean", "sum"):
        raise ValueError(f"reduction must be 'mean' or 'sum', got {reduction!r}")
    flags = SS_LOSS_SUM if reduction == "sum" else 0
    out = _native("preference_loss", logits, tokens, mask, ref_logprobs, beta, label_smoothing, temperature, flags, grad_scale, want_grad, grad_logits,
                  workspace)
    if out is not None:
        return out
    grad_logits = _gradient(logits, want_grad, grad_logits)
    params = _make_params(logits, tokens, temperature, grad_scale, grad_logits)
    dev = logits.device
    if params.batch & 1:
        raise ValueError(f"pairs need an even batch, got {params.batch}")
    ref_logprobs = _ready_rows(ref_logprobs, "ref_logprobs", tokens, dev)
    mask = _ready_mask(mask, tokens, dev)
    tokens = _ready_tokens(tokens, dev)
    workspace = _scratch(workspace, params, dev)
    loss = torch.empty((), dtype=torch.float32, device=dev)
    pair_loss = torch.empty(params.batch // 2, dtype=torch.float32, device=dev)
    margin = torch.empty_like(pair_loss)
    logprobs = torch.empty(tokens.shape, dtype=torch.float32, device=dev)
    _call(library().specsteer_preference_loss, dev, _ptr(logits), _ptr(tokens), _ptr(mask), _ptr(ref_logprobs), ctypes.byref(params),
          ctypes.byref(SSPreferenceParams(beta, label_smoothing, flags)), _ptr(loss), _ptr(pair_loss),
          _ptr(margin), _ptr(logprobs), _ptr(grad_logits), _ptr(workspace), _bytes(workspace))
    _written(grad_logits)
    return {"loss": loss, "pair_loss": pair_loss, "margin": margin, "logprobs": logprobs, "grad_logits": grad_logits}
