"""GPU tests of the losses where their arguments or values are at a limit of what they may be."""
import math

import pytest
import torch

import loss_reference as R
from test_gpu_losses import U_of, check_policy, check_preference, check_score, close, gen, losses, make, ragged_mask  # noqa: F401

pytestmark = pytest.mark.gpu

# one workgroup a row for both; in slices; many rows, one workgroup each
ROWS = [(2, 5, 3001), (2, 5, 50257), (2, 60, 3001)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("low", ["-inf", "lowest"])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("scale,coef,tau", [(2.0 ** 16, 0.05, 1.0), (2.0 ** 20, 0.1, 0.6), (1.0, 1e4, 1.0)])
def test_masked_tokens_under_a_large_weight_of_the_kl(losses, rows, low, dtype, scale, coef, tau):
    """A token that the policy masks counts nothing, whatever the reference says of it, also where the KL's weight times the largest
    difference of two logits passes fp32."""
    inp, g = make(*rows, dtype, ref=True)
    x, z, y = inp["logits"], inp["ref_logits"], inp["tokens"]
    value = -math.inf if low == "-inf" else torch.finfo(x.dtype).min
    x[..., :100] = value
    z[..., :50] = value  # both mask these, the policy alone the next
    y.clamp_(min=200)
    x[0, 1, 150] = x[0, 1, 200:].float().amin() - 500  # nothing of it is left in the policy, and the reference masks it
    z[0, 1, 150] = torch.finfo(x.dtype).min
    check_policy(losses, inp, g, kl="full", tau=tau, reduction="sum", kl_coef=coef, scale=scale)


@pytest.mark.parametrize("rows", [(4, 3), (4, 513), (34, 2)])  # one workgroup for all pairs, and one each
@pytest.mark.parametrize("beta", [0.25, -0.25])
def test_pairs_with_a_token_of_probability_zero(losses, rows, beta):
    """Pair 0 rejects such a sequence, pair 1 prefers one: margins of +-inf, whose losses are 0 and inf, and finite gradients."""
    B, T = rows
    P, V = B // 2, 50
    inp, _ = make(B, T, V, "f32")
    x, y = inp["logits"], inp["tokens"]
    good, bad = (0, 1) if beta > 0 else (1, 0)
    for row, t in ((P, 0), (1, T - 1)):
        y[row, t] = 7
        x[row, t, 7] = -math.inf
    out = losses.preference_loss(x, y, beta=beta)
    assert out["margin"][good] == math.inf and out["pair_loss"][good] == 0.0
    assert out["margin"][bad] == -math.inf and out["pair_loss"][bad] == math.inf
    assert out["loss"] == math.inf and out["pair_loss"][2:].isfinite().all()
    grad = out["grad_logits"]
    assert grad.isfinite().all() and not grad[[good, P + good]].any()
    assert grad[1, T - 1, 7] == (-beta / P if bad == 1 else 0.0)  # the whole weight, at a token without probability
    smooth = losses.preference_loss(x, y, beta=beta, label_smoothing=0.25)
    assert (smooth["pair_loss"][:2] == math.inf).all() and smooth["grad_logits"].isfinite().all()
    fine = torch.arange(B, device="cuda") % P != bad  # without the pair whose loss is infinite
    pairs = fine[:P]
    out = losses.preference_loss(x[fine].contiguous(), y[fine].contiguous(), beta=beta)
    want = losses.preference_loss(x, y, beta=beta)["pair_loss"][pairs].double().mean()
    assert abs(out["loss"].item() - want.item()) <= 2 * R.U * (want.item() + 1)  # each is rounded to fp32 once


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", ROWS)
def test_the_sampled_kl_of_a_token_of_probability_zero(losses, rows, dtype):
    """e^d - d - 1 grows with d without bound: +inf, and so is a loss with that term."""
    inp, g = make(*rows, dtype)
    x, y = inp["logits"], inp["tokens"]
    zero = torch.zeros(y.shape, dtype=torch.bool, device="cuda")
    zero[0, 1] = zero[1, 4] = True
    y[zero] = 7
    x[0, 1, 7] = x[1, 4, 7] = -math.inf
    old, ref = torch.full(y.shape, -8.0, device="cuda"), torch.full(y.shape, -9.0, device="cuda")
    adv = torch.randn(y.shape, generator=g, device="cuda")
    want = losses.policy_loss(x, y, old, adv)
    got = losses.policy_loss(x, y, old, adv, ref_logprobs=ref)
    assert (got["kl"][zero] == math.inf).all() and got["kl"][~zero].isfinite().all()
    assert torch.equal(got["loss"], want["loss"]) and torch.equal(got["grad_logits"], want["grad_logits"])
    assert losses.policy_loss(x, y, old, adv, ref_logprobs=ref, kl_coef=0.1)["loss"] == math.inf


@pytest.mark.parametrize("native", [True, False])
def test_autograd_learns_of_a_gradient_in_place_of_the_logits(losses, monkeypatch, native):
    """The backward pass of a model that saved its output refuses an output that was replaced; one that did not goes on."""
    if not native:
        monkeypatch.setattr(losses, "_calls", None)
    g = gen(3)
    hidden = torch.randn(4, 6, 32, generator=g, device="cuda")
    head = torch.randn(515, 32, generator=g, device="cuda").requires_grad_()
    y = torch.randint(0, 515, (4, 6), generator=g, device="cuda", dtype=torch.int32)
    old, adv = torch.zeros(4, 6, device="cuda") - 8, torch.randn(4, 6, generator=g, device="cuda")
    stats = losses.token_logprobs((hidden @ head.T).detach(), y, want_stats=True)["stats"]
    calls = [lambda x, to: losses.policy_loss(x, y, old, adv, grad_logits=to)["grad_logits"],
             lambda x, to: losses.preference_loss(x, y, grad_logits=to)["grad_logits"],
             lambda x, to: losses.token_logprobs_grad(x, y, stats, adv, grad_logits=to)]
    for call in calls:
        grads = []
        for place in (False, True):
            head.grad = None
            logits = hidden @ head.T
            before = logits._version
            logits.backward(call(logits, logits if place else None))
            assert logits._version == before + place
            grads.append(head.grad)
        assert torch.equal(*grads)
        saved = torch.tanh(hidden @ head.T)
        with pytest.raises(RuntimeError, match="inplace operation"):
            saved.backward(call(saved, saved))
        other = torch.tanh(hidden @ head.T)  # saved, and given for the gradient of something else
        call(logits.detach(), other.detach())
        with pytest.raises(RuntimeError, match="inplace operation"):
            other.sum().backward()
        with torch.inference_mode():  # tensors without a version
            x = logits.detach().clone()
            assert call(x, x) is x
        before = logits._version
        with pytest.raises(losses.SpecSteerError):  # refused, and nothing written
            losses.policy_loss(logits, y, old, adv, clip_low=2.0, grad_logits=logits)
        assert logits._version == before


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tau", [3e38, 1e35, 1e20, 1e13, 1e-13, 1e-20, 1e-30])
@pytest.mark.parametrize("rows", [(2, 3, 3001), (2, 3, 70001), (2, 60, 515)])
def test_temperatures_far_from_1(losses, rows, tau, dtype):
    """Logits as large or small as the temperature: distributions as any others."""
    inp, g = make(*rows, dtype, sigma=1.0, ref=True)
    unit = min(tau, 6e37)  # the largest logits of these, about 5, are numbers of the type still
    inp["logits"], inp["ref_logits"] = ((inp[k].float() * unit).to(inp[k].dtype) for k in ("logits", "ref_logits"))
    check_score(losses, inp, tau=tau)
    check_preference(losses, inp, g, tau=tau)
    for kl in ("none", "sampled", "full"):
        check_policy(losses, inp, g, kl=kl, tau=tau)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [(2, 6, 97), (2, 5, 50257), (2, 60, 3001), (1, 101, 70003)])
@pytest.mark.parametrize("shift", [100.0, -100.0, 700.0])
@pytest.mark.parametrize("of", ["policy", "reference"])
def test_a_common_offset_of_policy_or_reference(losses, rows, shift, of, dtype):
    """Logits are defined up to a constant a row: whole-vocabulary KL and gradient are as near to their definition as without the offset,
    by the bounds of the unshifted rows.  Logits on a grid of the type's steps at the offset, so that shifting rounds nothing."""
    inp, g = make(*rows, dtype, sigma=1.0, ref=True)
    x, y = inp["logits"], inp["tokens"]
    grid = 2.0 ** math.floor(math.log2(abs(shift) + 64)) * torch.finfo(x.dtype).eps
    h = (torch.randn(x.shape, generator=g, device="cuda").double() * max(1.0, 4 * grid) / grid).round() * grid
    z = h + (torch.randn(x.shape, generator=g, device="cuda").double() * max(0.2, grid) / grid).round() * grid
    tau = max(1.0, 2 * grid)
    plain = R.Rows(h, y, tau, z)
    h, z = (h + shift, z) if of == "policy" else (h, z + shift)
    assert torch.equal(h.to(x.dtype).double(), h) and torch.equal(z.to(x.dtype).double(), z)
    old = adv = torch.zeros(y.shape, device="cuda")  # the KL alone
    out = losses.policy_loss(h.to(x.dtype), y, old, adv, ref_logits=z.to(x.dtype), kl_coef=1.0, temperature=tau)
    close(out["kl"], plain.kl, plain.kl_err + U_of(plain.kl), "kl")
    none = torch.zeros_like(plain.lp)
    k = none + 1 / y.numel()
    exact = plain.gradient(none, k)
    bound = plain.gradient_bound(none, exact, x.dtype, k)
    if dtype == "bf16":  # formed from whole differences in fp32: the offset's and the mean's roundings, a half step each, and the product's
        bound = bound + 3 * R.U * abs(shift) / tau * (k[..., None] * plain.p) / tau
    close(out["grad_logits"], exact, bound, "grad_logits")


@pytest.mark.parametrize("kl", ["none", "full"])
@pytest.mark.parametrize("rows,V", [(100, 128256), (64, 50257), (300, 50257)])
def test_rows_of_nan_take_no_sweeps_of_their_own(losses, rows, V, kl):
    """What a diverged model gives: NaN wherever it reaches, at the time of other rows (those far from zero are swept one after the other, some
    hundred times slower)."""
    inp, g = make(1, rows, V, "bf16", ref=True)
    x, y = inp["logits"], inp["tokens"]
    more = {"ref_logits": inp["ref_logits"], "kl_coef": 0.1} if kl == "full" else {}
    old = torch.full(y.shape, -10.0, device="cuda")

    def call(t):
        return losses.policy_loss(t, y, old, old, **more)

    def time(t):
        best = math.inf
        for _ in range(5):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            for _ in range(5):
                call(t)
            end.record()
            end.synchronize()
            best = min(best, start.elapsed_time(end))
        return best

    bad = torch.full_like(x, math.nan)
    out = call(bad)
    assert out["loss"].isnan() and out["logprobs"].isnan().all() and out["grad_logits"].isnan().all()
    assert kl == "none" or out["kl"].isnan().all()
    scored = losses.token_logprobs(bad, y, want_stats=True)
    assert scored["logprobs"].isnan().all()
    assert losses.token_logprobs_grad(bad, y, scored["stats"], old).isnan().all()
    assert time(bad) <= 5 * time(x)
    if kl == "full":  # NaN in the reference alone: the log-probs are what they are, also of rows far from zero
        x[0, 3] = 3e6
        want = losses.policy_loss(x, y, old, old)
        out = losses.policy_loss(x, y, old, old, ref_logits=bad, kl_coef=0.1)
        assert torch.allclose(out["logprobs"], want["logprobs"], rtol=0, atol=2e-6) and out["kl"].isnan().all() and out["loss"].isnan()
        assert out["grad_logits"].isnan().all()


@pytest.mark.parametrize("B,T,V", [(16, 300, 32000), (4, 1025, 50257)])
@pytest.mark.parametrize("kept", [0.0, 0.3, 0.68, 0.72, 1.0])
def test_what_a_mask_keeps_decides_about_the_caches_only(losses, B, T, V, kept):
    """Preference losses of more than the caches hold: the same log-probs and gradient whichever way the rows are read."""
    inp, g = make(B, T, V, "bf16")
    x, y = inp["logits"], inp["tokens"]
    mask = torch.rand(B, T, generator=g, device="cuda") < kept
    scored = losses.token_logprobs(x, y, mask=mask, want_stats=True)
    out = losses.preference_loss(x, y, mask=mask, beta=0.01)
    assert torch.equal(out["logprobs"], scored["logprobs"])
    d = torch.where(mask, out["logprobs"], 0.0).double().sum(1)
    margin = R.f32(0.01) * (d[:B // 2] - d[B // 2:])  # of sums of log-probs as they are before they are rounded, by half a step each
    close(out["margin"], margin, 0.01 * 2 * T * R.U * 32 + U_of(margin), "margin")
    w = (-R.f32(0.01) / (B // 2) * torch.sigmoid(-out["margin"].double()))
    w = torch.cat([w, -w])[:, None].expand(B, T).float().contiguous()
    grad = losses.token_logprobs_grad(x, y, scored["stats"], w, mask=mask)
    # both round w (1[v = y] - p) to bf16 once, from weights that differ by a few steps of fp32
    assert ((out["grad_logits"].float() - grad.float()).abs() <= 2.0 ** -7 * grad.float().abs() + 1e-30).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("low", ["-inf", "lowest"])
@pytest.mark.parametrize("rows", [(1, 90, 50257), (1, 300, 3001)])
def test_tokens_of_no_probability_that_the_reference_masks(losses, rows, low, dtype):
    """Padding that the policy only holds far down and the reference masks: nothing of it counts, and no row is swept again for it."""
    inp, g = make(*rows, dtype, ref=True)
    x, z, y = inp["logits"], inp["ref_logits"], inp["tokens"]
    old, adv = torch.zeros(y.shape, device="cuda") - 9, torch.randn(y.shape, generator=g, device="cuda")

    def time():
        best = math.inf
        for _ in range(5):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            for _ in range(5):
                losses.policy_loss(x, y, old, adv, ref_logits=z, kl_coef=0.1)
            end.record()
            end.synchronize()
            best = min(best, start.elapsed_time(end))
        return best

    plain = time()
    x[..., :64] = -2000.0
    z[..., :64] = -math.inf if low == "-inf" else torch.finfo(z.dtype).min
    y.clamp_(min=64)
    check_policy(losses, inp, g, kl="full")
    check_policy(losses, inp, g, kl="full", mask=ragged_mask(*rows[:2], g, "lengths"), reduction="sum", scale=2.0 ** 16)
    assert time() <= 5 * plain


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", ROWS)
def test_a_token_that_the_reference_alone_has_at_the_lowest_value(losses, rows, dtype):
    """A KL as large as that value, or beyond fp32: no finite loss of ordinary size comes of it.  Other rows keep theirs."""
    inp, g = make(*rows, dtype, ref=True)
    x, z, y = inp["logits"], inp["ref_logits"], inp["tokens"]
    old, adv = torch.zeros(y.shape, device="cuda") - 9, torch.randn(y.shape, generator=g, device="cuda")
    want = losses.policy_loss(x, y, old, adv, ref_logits=z, kl_coef=0.1)
    x7 = x[0, 1, 7].clone()
    z[0, 1, 7] = torch.finfo(z.dtype).min
    got = losses.policy_loss(x, y, old, adv, ref_logits=z, kl_coef=0.1)
    assert x[0, 1, 7] == x7 and got["kl"][0, 1] > 1e30 and got["loss"] > 1e24
    others = torch.ones(y.shape, dtype=torch.bool, device="cuda")
    others[0, 1] = False
    assert torch.equal(got["kl"][others], want["kl"][others]) and torch.equal(got["grad_logits"][others], want["grad_logits"][others])
    assert torch.equal(got["logprobs"], want["logprobs"])
