"""CPU checks of the alternatives' calls: what the header declares, what is refused before anything is enqueued, the scratch, and the 64-bit
reference against automatic differentiation."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

import alternatives_reference as A

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, DTYPE, PARAM, STRIDE, WORKSPACE = range(7)
NAMES = ["specsteer_token_alternatives", "specsteer_token_alternatives_grad", "specsteer_token_alternatives_workspace_bytes"]


@pytest.fixture(scope="module")
def losses():
    from paper_2603_16219_amd import losses as m

    m.library()
    return m


def test_library_exports_every_declared_symbol(losses):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "specsteer_alternatives.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(specsteer_\w+)\s*\(", text))) == NAMES
    for n in NAMES:
        assert getattr(losses.library(), n) is not None


@pytest.mark.parametrize("compiler,std", [("gcc", "-std=c99"), ("g++", "-std=c++17")])
def test_header_compiles_alone(tmp_path, compiler, std):
    src = tmp_path / ("t.c" if compiler == "gcc" else "t.cpp")
    src.write_text('#include "specsteer_alternatives.h"\nint main(void) { return SS_MAX_TOPK == 64 ? 0 : 1; }\n')
    subprocess.run([compiler, std, "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-o", tmp_path / "t", src], check=True)
    subprocess.run([tmp_path / "t"], check=True)


def call(losses, name, **spoiled):
    """A call with arguments in range (addresses that are only looked at), some of them spoiled."""
    name = name.removeprefix("specsteer_")
    p = losses.SSLossParams(4, 8, 100, 1, 0, 0, 0, 0, 1.0, 1.0)
    order = {"token_alternatives": ["logits", "tokens", "mask", "params", "topk", "logprobs", "entropy", "top_tokens", "top_logprobs", "stats", "workspace",
                                    "bytes", "stream"],
             "token_alternatives_grad": ["logits", "tokens", "mask", "stats", "entropy", "grad_logprobs", "grad_entropy", "params", "grad_logits",
                                         "stream"]}[name]
    args = {a: 1 << 20 for a in order}
    args.update({"stream": None, "params": ctypes.byref(p)})
    if name == "token_alternatives":
        args.update({"topk": 8, "bytes": 1 << 30})
    for k, v in spoiled.items():
        if k in args:
            args[k] = v
        else:
            setattr(p, k, v)
    return getattr(losses.library(), "specsteer_" + name)(*args.values())


@pytest.mark.parametrize("name", NAMES[:2])
@pytest.mark.parametrize("status,spoiled", [
    (NULL, dict(params=None)), (NULL, dict(logits=None)), (NULL, dict(tokens=None)),
    (SHAPE, dict(batch=-1)), (SHAPE, dict(length=(1 << 20) + 1)), (SHAPE, dict(vocab=0)), (SHAPE, dict(vocab=(1 << 20) + 1)),
    (SHAPE, dict(batch=1 << 14, length=(1 << 10) + 1)), (DTYPE, dict(dtype=2)),
    (PARAM, dict(temperature=0.0)), (PARAM, dict(temperature=math.nan)), (PARAM, dict(grad_scale=math.inf)),
    (STRIDE, dict(stride_t=99)), (STRIDE, dict(stride_b=799)), (STRIDE, dict(grad_stride_t=99)), (STRIDE, dict(stride_t=1 << 61)),
    (STRIDE, dict(stride_b=100, stride_t=400)), (STRIDE, dict(logits=(1 << 20) + 1))])
def test_refusals_of_both_calls(losses, name, status, spoiled):
    assert call(losses, name, **spoiled) == status


@pytest.mark.parametrize("name,status,spoiled", [
    ("token_alternatives", PARAM, dict(topk=-1)), ("token_alternatives", PARAM, dict(topk=65)),
    ("token_alternatives", NULL, dict(top_tokens=None)), ("token_alternatives", NULL, dict(top_logprobs=None)),
    ("token_alternatives", WORKSPACE, dict(workspace=None)), ("token_alternatives", WORKSPACE, dict(workspace=(1 << 20) + 128)),
    ("token_alternatives", WORKSPACE, dict(bytes=64)),
    ("token_alternatives_grad", NULL, dict(stats=None)), ("token_alternatives_grad", NULL, dict(grad_logits=None)),
    ("token_alternatives_grad", NULL, dict(entropy=None)), ("token_alternatives_grad", NULL, dict(grad_logprobs=None, grad_entropy=None)),
    ("token_alternatives_grad", STRIDE, dict(grad_logits=(1 << 20) + 1))])
def test_refusals_of_single_calls(losses, name, status, spoiled):
    assert call(losses, name, **spoiled) == status


@pytest.mark.parametrize("name", NAMES[:2])
def test_no_rows_need_no_arrays(losses, name):
    none = dict(logits=None, tokens=None, mask=None, entropy=None, stats=None)
    assert call(losses, name, batch=0, **none) == OK
    assert call(losses, name, length=0, **none) == OK


def test_workspace_bytes(losses):
    p = lambda **k: losses.SSLossParams(**{**dict(batch=1, length=1, vocab=128256, dtype=1, temperature=1.0, grad_scale=1.0), **k})
    of = losses.alternatives_workspace_bytes
    assert of(p(), -1) == of(p(), 65) == of(p(vocab=0), 4) == 0
    assert of(p(batch=101), 64) == of(p(vocab=100), 64) == 256  # a workgroup a row needs none but the least
    slices = min(64, 1024, 128256 // 8 // 512)
    up = lambda n: -(-n // 256) * 256
    for k in (0, 1, 20, 64):
        assert of(p(), k) == up(slices * 24) + up(slices * k * 8) + 256


def test_reference_against_automatic_differentiation():
    g = torch.Generator().manual_seed(3)
    x = (3 * torch.randn(2, 3, 50, generator=g)).double()
    x[0, 0, 7:20] = -math.inf
    y = torch.randint(20, 50, (2, 3), generator=g)
    a, b = torch.randn(2, 3, generator=g).double(), torch.randn(2, 3, generator=g).double()
    rows = A.Rows(x, y, 0.7)
    leaf = x.clone().requires_grad_()
    log_p = torch.log_softmax(leaf / rows.tau, -1)
    entropy = -(log_p.exp() * torch.where(x > -math.inf, log_p, 0.0)).sum(-1)
    grad, = torch.autograd.grad((log_p.gather(-1, y[..., None])[..., 0] * a + entropy * b).sum(), leaf)
    torch.testing.assert_close(rows.entropy, entropy.detach(), rtol=1e-12, atol=1e-12)
    torch.testing.assert_close(rows.gradient2(a, b), grad.nan_to_num(0.0), rtol=1e-10, atol=1e-12)
    ids, lp, _ = rows.top(x, 60)
    assert ids[0, 0].tolist()[37:] == [-1] * 23 and torch.all(lp[0, 0, 37:] == -math.inf) and torch.all(lp[..., :36].diff(dim=-1) <= 0)


def test_binding_refuses(losses):
    x, y = torch.zeros(2, 3, 40), torch.zeros(2, 3, dtype=torch.int32)
    for bad in (dict(topk=65), dict(topk=-1), dict(topk=2.5), dict(topk=True)):
        with pytest.raises(ValueError, match="topk"):
            losses.token_alternatives(x, y, **bad)
    with pytest.raises(ValueError, match="no CPU path"):
        losses.token_alternatives(x, y, topk=3)
    with pytest.raises(ValueError, match="B, T, V"):
        losses.token_alternatives(x[0])
    s, h = torch.zeros(2, 3, 2), torch.zeros(2, 3)
    for args in ((x, y, s, h, None, None), (x, None, s, h, h, None), (x, y, s, None, None, h)):
        with pytest.raises(ValueError, match="grad_"):
            losses.token_alternatives_grad(*args)
