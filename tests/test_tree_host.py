"""CPU checks of the calls with trees: what the header declares and the binding mirrors, and what is refused before anything is enqueued."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, DTYPE, PARAM, STRIDE, WORKSPACE = range(7)
NAMES = ["specsteer_tree_attention", "specsteer_tree_attention_workspace_bytes", "specsteer_tree_commit", "specsteer_tree_status_string",
         "specsteer_tree_verify", "specsteer_tree_verify_workspace_bytes"]


@pytest.fixture(scope="module")
def tree():
    from paper_2603_16219_amd import tree as m

    m.library()
    return m


def test_library_exports_every_declared_symbol(tree):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "specsteer_tree.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(specsteer_\w+)\s*\(", text))) == NAMES
    for n in NAMES:
        assert getattr(tree.library(), n) is not None
    assert len({tree.status_string(i) for i in range(8)}) == 8 and tree.status_string(99) == "unknown status"


@pytest.mark.parametrize("compiler,std", [("gcc", "-std=c99"), ("g++", "-std=c++17")])
def test_header_compiles_alone_and_has_the_binding_s_layout(tree, tmp_path, compiler, std):
    src = tmp_path / ("t.c" if compiler == "gcc" else "t.cpp")
    fields = [f"(int)offsetof(ss_tree_params, {n})" for n, _ in tree.SSTreeParams._fields_]
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "specsteer_tree.h"\nint main(void) { printf("%d' + " %d" * len(fields)
                   + '\\n", (int)sizeof(ss_tree_params), ' + ", ".join(fields) + "); return 0; }\n")
    subprocess.run([compiler, std, "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-o", tmp_path / "t", src], check=True)
    got = [int(v) for v in subprocess.run([tmp_path / "t"], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(tree.SSTreeParams)] + [getattr(tree.SSTreeParams, n).offset for n, _ in tree.SSTreeParams._fields_]


AT = 1 << 20
ORDER = {"attention": ["q", "k", "v", "k_cache", "v_cache", "block_table", "cache_len", "parents", "tree_len", "params", "out", "workspace", "bytes", "stream"],
         "verify": ["G", "S_ctx", "S_noctx", "tokens", "parents", "tree_len", "uniforms", "params", "accepted_len", "path", "next_token",
                    "next_token_logprob", "workspace", "bytes", "stream"],
         "commit": ["k", "v", "k_cache", "v_cache", "block_table", "cache_len", "accepted_len", "path", "params", "new_len", "stream"]}


def params(tree, **more):
    p = tree.SSTreeParams(batch=2, nodes=5, heads=8, kv_heads=2, head_dim=64, dtype=1, pages=10, page_size=16, table_width=4, scale=0.1)
    for k, v in more.items():
        if k.endswith("_stride") and k != "table_stride":
            getattr(p, k)[:] = v
        else:
            setattr(p, k, v)
    return p


def call(tree, name, **spoiled):
    """A call with arguments in range (addresses that are only looked at), some of them spoiled."""
    args = {a: AT * (i + 1) for i, a in enumerate(ORDER[name])}
    own = {k: v for k, v in spoiled.items() if k not in args}
    if name == "verify":
        p = tree.SSParams(2, 5, 100, 1, 0, 0, 0.5, 1.0, 1.0, 0)
        for k, v in own.items():
            setattr(p, k, v)
    else:
        p = params(tree, **own)
    args.update(params=ctypes.byref(p), stream=None)
    if "bytes" in args:
        args["bytes"] = 1 << 40
    args.update({k: v for k, v in spoiled.items() if k in args})
    return getattr(tree.library(), "specsteer_tree_" + name)(*args.values())


@pytest.mark.parametrize("name", ["attention", "commit"])
@pytest.mark.parametrize("status,spoiled", [
    (NULL, dict(params=None)), *[(NULL, {k: None}) for k in ("k", "v", "k_cache", "v_cache", "block_table", "cache_len")],
    (SHAPE, dict(batch=-1)), (SHAPE, dict(nodes=-1)), (SHAPE, dict(nodes=1025)), (SHAPE, dict(kv_heads=0)), (SHAPE, dict(kv_heads=1025)),
    (SHAPE, dict(head_dim=0)), (SHAPE, dict(head_dim=68)), (SHAPE, dict(head_dim=2048)), (SHAPE, dict(pages=-1)), (SHAPE, dict(page_size=0)),
    (SHAPE, dict(table_width=-1)), (SHAPE, dict(table_width=1 << 16, page_size=1 << 16)), (SHAPE, dict(batch=1 << 20)),
    (DTYPE, dict(dtype=0)), (DTYPE, dict(dtype=3)),
    (STRIDE, dict(k_stride=(-8, 0, 0))), (STRIDE, dict(k_stride=(0, 12, 0))), (STRIDE, dict(cache_stride=(0, 0, 100))),
    (STRIDE, dict(cache_stride=(1 << 60, 0, 0))), (STRIDE, dict(k_stride=(1 << 62, 0, 0))), (STRIDE, dict(table_stride=-1)),
    *[(STRIDE, {k: AT + 8}) for k in ("k", "v", "k_cache", "v_cache")]])
def test_refusals_of_the_calls_with_a_cache(tree, name, status, spoiled):
    assert call(tree, name, **spoiled) == status


@pytest.mark.parametrize("name,status,spoiled", [
    *[("attention", NULL, {k: None}) for k in ("q", "out")], *[("commit", NULL, {k: None}) for k in ("accepted_len", "new_len")],
    ("attention", SHAPE, dict(heads=7)), ("attention", SHAPE, dict(heads=0)), ("attention", SHAPE, dict(heads=2048)), ("attention", SHAPE, dict(head_dim=96)),
    ("attention", PARAM, dict(scale=math.nan)), ("attention", PARAM, dict(scale=math.inf)),
    ("attention", STRIDE, dict(q_stride=(0, 4, 0))), ("attention", STRIDE, dict(q=AT + 2)), ("attention", STRIDE, dict(out=AT + 8)),
    ("attention", STRIDE, dict(out_stride=(0, 64, 0))), ("attention", STRIDE, dict(out_stride=(8, 0, 0))),
    ("attention", WORKSPACE, dict(workspace=None)), ("attention", WORKSPACE, dict(workspace=AT + 128)), ("attention", WORKSPACE, dict(bytes=0)),
    ("commit", STRIDE, dict(cache_stride=(64, 0, 0))), ("commit", STRIDE, dict(cache_stride=(0, 64, 0))), ("commit", SHAPE, dict(head_dim=1032)),
    ("commit", PARAM, dict(new_len=AT, cache_len=AT)),
    *[("verify", NULL, {k: None}) for k in ("params", "G", "S_ctx", "S_noctx", "tokens", "uniforms", "accepted_len", "path", "next_token")],
    *[("verify", SHAPE, {k: v}) for k, v in (("batch", -1), ("k_max", -1), ("k_max", 1025), ("vocab", 0), ("vocab", (1 << 20) + 1), ("batch", 1 << 20))],
    *[("verify", DTYPE, dict(dtype=d)) for d in (-1, 2)],
    *[("verify", PARAM, {k: v}) for k in ("lambda_", "temperature") for v in (0.0, -1.0, math.nan, math.inf)],
    ("verify", PARAM, dict(beta=math.nan)), ("verify", PARAM, dict(flags=2)), ("verify", PARAM, dict(flags=4)), ("verify", PARAM, dict(temperature=1e-40)),
    *[("verify", STRIDE, {k: v}) for k, v in (("stride_t", 99), ("stride_b", 599), ("stride_b", -1), ("stride_t", 1 << 60), ("G", AT + 1))],
    ("verify", WORKSPACE, dict(workspace=None)), ("verify", WORKSPACE, dict(bytes=0)), ("verify", WORKSPACE, dict(workspace=AT + 64))])
def test_refusals_of_single_calls(tree, name, status, spoiled):
    assert call(tree, name, **spoiled) == status


@pytest.mark.parametrize("name", list(ORDER))
def test_no_sequences_need_no_arrays(tree, name):
    assert call(tree, name, batch=0, **{k: None for k in ORDER[name] if k not in ("params", "stream", "bytes")}) == OK


def test_commit_refuses_one_cache_for_keys_and_values(tree):
    assert call(tree, "commit", k_cache=AT, v_cache=AT) == PARAM


def test_accepted_layouts(tree):
    """Refused for the workspace only, which is looked at last: pages of [heads, slots, dim], gaps, strides of dimensions of one element."""
    for more in (dict(cache_stride=(2048, 64, 1024)), dict(k_stride=(8192, 512, 64), q_stride=(1 << 20, 1024, 128)), dict(out_stride=(64, 1024, 128)),
                 dict(nodes=0, q_stride=(0, 8, 0))):
        assert call(tree, "attention", workspace=None, **more) == WORKSPACE
    assert call(tree, "verify", workspace=None, stride_t=101, stride_b=10000) == WORKSPACE
    assert tree.attention_workspace_bytes(params(tree)) >= 256 and tree.attention_workspace_bytes(params(tree, head_dim=65)) == 0
    assert tree.verify_workspace_bytes(tree.SSParams(2, 5, 100, 1, 0, 0, 0.5, 1.0, 1.0, 0)) >= 256
    assert tree.verify_workspace_bytes(tree.SSParams(2, 5, 100, 1, 0, 0, 0.5, 1.0, 0.0, 0)) == 0


def test_binding_refuses(tree):
    bf = torch.bfloat16
    q, k, c = torch.zeros(2, 4, 8, 64, dtype=bf), torch.zeros(2, 4, 2, 64, dtype=bf), torch.zeros(5, 16, 2, 64, dtype=bf)
    t, n = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="no CPU path"):
        tree.attention(q, k, k, c, c, t, n)
    with pytest.raises(ValueError, match="no CPU path"):
        tree.commit(k, k, c, c, t, n, n)
    with pytest.raises(ValueError, match="k and v"):
        tree.attention(q, k, k[:, :2], c, c, t, n)
    with pytest.raises(ValueError, match="caches|cache"):
        tree.attention(q, k, k, c[..., :32], c, t, n)
    with pytest.raises(TypeError, match="bfloat16 or float16"):
        tree.commit(k.float(), k.float(), c.float(), c.float(), t, n, n)
    g = torch.zeros(2, 4, 50)
    with pytest.raises(ValueError, match="no CPU path"):
        tree.verify(g, g, g, t, torch.zeros(2, 4))
    with pytest.raises(ValueError, match="dtype"):
        tree.verify(g, g, g.to(bf), t, torch.zeros(2, 4))
