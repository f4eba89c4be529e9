"""CPU checks of the losses' library and binding: what it exports, what it refuses before anything is enqueued, and the 64-bit
reference that the GPU tests compare with, against automatic differentiation."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

import loss_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "specsteer_loss.h")
OK, NULL, SHAPE, DTYPE, PARAM, STRIDE, WORKSPACE = range(7)
NAMES = ["specsteer_loss_status_string", "specsteer_loss_workspace_bytes", "specsteer_policy_loss", "specsteer_preference_loss",
         "specsteer_token_logprobs", "specsteer_token_logprobs_grad"]


@pytest.fixture(scope="module")
def losses():
    from paper_2603_16219_amd import losses as m

    m.library()
    return m


def test_library_exports_every_declared_symbol(losses):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(specsteer_\w+)\s*\(", text))) == NAMES
    for n in NAMES:
        assert getattr(losses.library(), n) is not None
    assert len({losses.status_string(i) for i in range(8)}) == 8 and losses.status_string(99) == "unknown status"


@pytest.mark.parametrize("compiler,std", [("gcc", "-std=c99"), ("g++", "-std=c++17")])
def test_header_compiles_alone_and_has_the_binding_s_layout(losses, tmp_path, compiler, std):
    src = tmp_path / ("t.c" if compiler == "gcc" else "t.cpp")
    fields = [f"(int)offsetof(ss_loss_params, {n})" for n, _ in losses.SSLossParams._fields_]
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "specsteer_loss.h"\nint main(void) { printf("%d %d %d'
                   + " %d" * len(fields) + '\\n", (int)sizeof(ss_loss_params), (int)sizeof(ss_policy_params), (int)sizeof(ss_preference_params), '
                   + ", ".join(fields) + "); return 0; }\n")
    exe = tmp_path / "t"
    subprocess.run([compiler, std, "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-o", exe, src], check=True)
    got = [int(v) for v in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    want = [ctypes.sizeof(c) for c in (losses.SSLossParams, losses.SSPolicyParams, losses.SSPreferenceParams)]
    assert got == want + [getattr(losses.SSLossParams, n).offset for n, _ in losses.SSLossParams._fields_]


class Call:
    """One of the calls with arguments in range (addresses that are only looked at), to be spoiled one at a time."""

    def __init__(self, losses, name):
        self.losses, self.name = losses, name
        self.p = losses.SSLossParams(4, 8, 100, 1, 0, 0, 0, 0, 1.0, 1.0)
        self.q = losses.SSPolicyParams(0.2, 0.2, 0.1, 0) if name == "policy_loss" else losses.SSPreferenceParams(0.1, 0.0, 0)
        at = 1 << 20
        args = {"token_logprobs": ["logits", "tokens", "mask", "params", "logprobs", "stats", "workspace", "bytes", "stream"],
                "token_logprobs_grad": ["logits", "tokens", "mask", "stats", "grad_logprobs", "params", "grad_logits", "stream"],
                "policy_loss": ["logits", "ref_logits", "tokens", "mask", "old_logprobs", "ref_logprobs", "advantages", "params", "own", "loss",
                                "logprobs", "kl", "grad_logits", "workspace", "bytes", "stream"],
                "preference_loss": ["logits", "tokens", "mask", "ref_logprobs", "params", "own", "loss", "pair_loss", "margin", "logprobs",
                                    "grad_logits", "workspace", "bytes", "stream"]}[name]
        self.args = {a: at for a in args}
        self.args.update({"bytes": 1 << 30, "stream": None, "params": ctypes.byref(self.p)})
        if "own" in self.args:
            self.args["own"] = ctypes.byref(self.q)
        if name == "policy_loss":
            self.args["ref_logits"] = None

    def __call__(self, **spoiled):
        args = dict(self.args)
        for k, v in spoiled.items():
            if k in args:
                args[k] = v
            else:
                setattr(self.q if hasattr(self.q, k) else self.p, k, v)
        return getattr(self.losses.library(), "specsteer_" + self.name)(*args.values())


CALLS = ["token_logprobs", "token_logprobs_grad", "policy_loss", "preference_loss"]


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("status,spoiled", [
    (NULL, dict(params=None)), (NULL, dict(logits=None)), (NULL, dict(tokens=None)),
    (SHAPE, dict(batch=-1)), (SHAPE, dict(length=-1)), (SHAPE, dict(length=(1 << 20) + 1)), (SHAPE, dict(vocab=0)),
    (SHAPE, dict(vocab=(1 << 20) + 1)), (SHAPE, dict(batch=1 << 14, length=(1 << 10) + 1)), (SHAPE, dict(batch=(1 << 24) + 2, length=0)),
    (DTYPE, dict(dtype=2)), (DTYPE, dict(dtype=-1)),
    (PARAM, dict(temperature=0.0)), (PARAM, dict(temperature=-1.0)), (PARAM, dict(temperature=math.nan)), (PARAM, dict(temperature=math.inf)),
    (PARAM, dict(temperature=1e-40)), (PARAM, dict(grad_scale=math.inf)), (PARAM, dict(grad_scale=math.nan)),
    (STRIDE, dict(stride_t=99)), (STRIDE, dict(stride_t=-100)), (STRIDE, dict(stride_b=-800)), (STRIDE, dict(stride_b=799)),
    (STRIDE, dict(stride_t=1 << 61)), (STRIDE, dict(stride_b=1 << 61)), (STRIDE, dict(grad_stride_t=99)), (STRIDE, dict(grad_stride_b=799)),
    (STRIDE, dict(logits=(1 << 20) + 1))])
def test_refusals_of_every_call(losses, name, status, spoiled):
    assert Call(losses, name)(**spoiled) == status


@pytest.mark.parametrize("name,status,spoiled", [
    ("token_logprobs", NULL, dict(logprobs=None)), ("token_logprobs_grad", NULL, dict(stats=None)),
    ("token_logprobs_grad", NULL, dict(grad_logprobs=None)), ("token_logprobs_grad", NULL, dict(grad_logits=None)),
    ("token_logprobs_grad", STRIDE, dict(grad_logits=(1 << 20) + 1)), ("token_logprobs_grad", STRIDE, dict(dtype=0, logits=(1 << 20) + 2)),
    *[("policy_loss", NULL, {k: None}) for k in ("old_logprobs", "advantages", "loss", "own", "ref_logprobs")],
    ("policy_loss", PARAM, dict(ref_logits=1 << 20)), ("policy_loss", STRIDE, dict(ref_logits=(1 << 20) + 1, ref_logprobs=None)),
    *[("policy_loss", PARAM, {k: v}) for k in ("clip_low", "clip_high", "kl_coef") for v in (-0.1, math.nan, math.inf)],
    ("policy_loss", PARAM, dict(clip_low=1.5)), ("policy_loss", PARAM, dict(flags=3)), ("policy_loss", PARAM, dict(flags=8)),
    ("policy_loss", STRIDE, dict(grad_logits=(1 << 20) + 1)), ("preference_loss", STRIDE, dict(grad_logits=(1 << 20) + 1)),
    ("preference_loss", NULL, dict(loss=None)), ("preference_loss", NULL, dict(own=None)), ("preference_loss", SHAPE, dict(batch=3)),
    *[("preference_loss", PARAM, {k: v}) for k, v in (("beta", math.nan), ("beta", math.inf), ("label_smoothing", -0.1), ("label_smoothing", 0.6),
                                                      ("label_smoothing", math.nan), ("flags", 2))],
    *[(n, WORKSPACE, s) for n in ("token_logprobs", "policy_loss", "preference_loss")
      for s in (dict(workspace=None), dict(workspace=(1 << 20) + 128), dict(bytes=64))]])
def test_refusals_of_single_calls(losses, name, status, spoiled):
    assert Call(losses, name)(**spoiled) == status


def test_workspace_bytes(losses):
    p = losses.SSLossParams(4, 8, 100, 1, 0, 0, 0, 0, 1.0, 1.0)
    small = losses.workspace_bytes(p)
    assert small > 0 and small % 256 == 0
    p.length = 4096
    assert losses.workspace_bytes(p) > small
    p.vocab = 0
    assert losses.workspace_bytes(p) == 0 and losses.library().specsteer_loss_workspace_bytes(None) == 0


def test_calls_on_host_tensors_and_wrong_shapes_are_refused(losses):
    x, y, f = torch.zeros(2, 3, 10), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3)
    for call in (lambda: losses.token_logprobs(x, y), lambda: losses.token_logprobs_grad(x, y, torch.zeros(2, 3, 2), f),
                 lambda: losses.policy_loss(x, y, f, f), lambda: losses.preference_loss(x, y)):
        with pytest.raises(ValueError, match="no CPU path"):
            call()
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        losses.token_logprobs(x.half(), y)
    with pytest.raises(ValueError, match=r"\[B, T, V\]"):
        losses.token_logprobs(x[0], y)
    with pytest.raises(ValueError, match="reduction"):
        losses.policy_loss(x, y, f, f, reduction="mean")
    with pytest.raises(ValueError, match="reduction"):
        losses.preference_loss(x, y, reduction="token_mean")
    with pytest.raises(ValueError, match="not both"):
        losses.policy_loss(x, y, f, f, ref_logits=x, ref_logprobs=f)
    with pytest.raises(ValueError, match="KL term needs"):
        losses.policy_loss(x, y, f, f, kl_coef=0.1)
    with pytest.raises(ValueError, match="ref_logits must have"):
        losses.policy_loss(x, y, f, f, ref_logits=x[:, :2])


def test_the_reference_s_gradients_are_those_of_its_losses():
    g = torch.Generator().manual_seed(5)
    B, T, V = 4, 5, 13
    x = torch.randn(B, T, V, generator=g).double().requires_grad_()
    z = torch.randn(B, T, V, generator=g).double()
    y = torch.randint(0, V, (B, T), generator=g)
    mask = torch.rand(B, T, generator=g) < 0.7
    mask[1] = False
    tau = R.f32(0.7)
    lp = torch.log_softmax(x / tau, -1)
    at = lp.gather(-1, y[..., None])[..., 0]
    kl = (lp.exp() * (lp - torch.log_softmax(z / tau, -1))).sum(-1)
    old = (at + 0.3 * torch.randn(B, T, generator=g)).detach().float()
    ref = (at + 0.3 * torch.randn(B, T, generator=g)).detach().float()
    adv = torch.randn(B, generator=g)
    rows = R.Rows(x.detach(), y, 0.7, z)
    assert torch.allclose(rows.lp, at.detach(), atol=1e-13) and torch.allclose(rows.kl, kl.detach(), atol=1e-13)
    for reduction in ("token_mean", "seq_mean", "sum"):
        for with_ref in (False, True):
            r = torch.exp(at - old.double())
            a = adv.double()[:, None]
            est = torch.exp(ref.double() - at) - 1 - (ref.double() - at)
            term = -torch.minimum(r * a, torch.clip(r, 1 - R.f32(0.2), 1 + R.f32(0.3)) * a) + R.f32(0.1) * (kl if with_ref else est)
            loss = (R.norms(mask, reduction) * term).sum()
            want, = torch.autograd.grad(loss, x, retain_graph=True)
            rr = R.Rows(x.detach(), y, 0.7, z if with_ref else None)
            got = R.policy(rr, mask, old, adv, clip_low=0.2, clip_high=0.3, kl_coef=0.1, reduction=reduction, ref_logprobs=None if with_ref else ref)
            assert got["loss"].item() == pytest.approx(loss.item(), abs=1e-13)
            assert torch.allclose(torch.where(mask[..., None], rr.gradient(got["w"], got["k"]), 0.0), want, atol=1e-13)
    for reduction in ("mean", "sum"):
        d = ((at - ref.double()) * mask).sum(1)
        h = R.f32(0.4) * (d[:2] - d[2:])
        pair = -(1 - R.f32(0.1)) * torch.log(torch.sigmoid(h)) - R.f32(0.1) * torch.log(torch.sigmoid(-h))
        loss = pair.mean() if reduction == "mean" else pair.sum()
        want, = torch.autograd.grad(loss, x, retain_graph=True)
        got = R.preference(rows, mask, ref, beta=0.4, label_smoothing=0.1, reduction=reduction)
        assert got["loss"].item() == pytest.approx(loss.item(), abs=1e-13)
        assert torch.allclose(rows.gradient(got["w"]), want, atol=1e-13)


def test_waves_that_hold_a_row(tmp_path):
    """csrc/loss/loss_plan.h: a workgroup holds all of a row that fits, and no other number of waves would hold more on a compute unit."""
    src = tmp_path / "waves.cpp"
    src.write_text('#include <cstdio>\n#include <initializer_list>\n#include "loss_plan.h"\nint main() { for (int held : {kHeldVecs, kHeldPairs}) for (int n = 0; n < 140000; n = n < 4000 ? n + 1 : n * 17 / 16)'
                   ' std::printf("%d %d %d\\n", held, n, row_waves(n, held)); }\n')
    exe = tmp_path / "waves"
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-Wno-unused-function", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2603_16219_amd", "csrc", "loss"), "-o", exe, src], check=True)
    for line in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines():
        held, n, got = map(int, line.split())
        on_unit = lambda w: (16 // w) * min((w - 1) * 64 * held, n)
        assert 2 <= got <= 16 and on_unit(got) == max(on_unit(w) for w in range(2, 17)), (held, n)


def test_slices_of_calls_with_few_rows(tmp_path, losses):
    """csrc/loss/loss_plan.h: slices are as many as a wave joins, none is empty, and the workspace holds them."""
    src = tmp_path / "slices.cpp"
    src.write_text('#include <cstdio>\n#include "loss_plan.h"\nint main() { for (long r = 0; r < 300; r += r < 8 ? 1 : 7) for (int n = 0; n < 300000; n = n < 1100 ? n + 37 : n * 5 / 4)'
                   ' std::printf("%ld %d %d %d\\n", r, n, row_slices(r, n), score_slices(r, n)); }\n')
    exe = tmp_path / "slices"
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-Wno-unused-function", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2603_16219_amd", "csrc", "loss"), "-o", exe, src], check=True)
    seen = set()
    for line in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines():
        rows, vecs, n, scored = map(int, line.split())
        seen.add(n)
        assert 1 <= n <= 64 and scored in (1, n) and (n == 1 or vecs // n >= 512) and (n == 1 or rows <= 100)
        if n > 1:
            p = losses.SSLossParams(1, rows, 8 * vecs, 1, 0, 0, 0, 0, 1.0, 1.0)
            if p.vocab <= 1 << 20:
                assert losses.workspace_bytes(p) >= rows * (n * 32 + 4 + 16)
    assert {1, 2, 64} <= seen


def test_token_ids_beyond_32_bits_do_not_become_others(losses):
    cpu = torch.device("cpu")
    big = torch.tensor([[7, 2**32 + 7, -1, -2**33]])
    assert losses._ready_tokens(big, cpu).tolist() == [[7, 2**31 - 1, -1, -1]]
    assert losses._ready_tokens(torch.tensor([[2**32 - 1, 7]]).to(torch.uint32), cpu).tolist() == [[-1, 7]]
    with pytest.raises(TypeError):
        losses._ready_tokens(big.abs().to(torch.uint64), cpu)
