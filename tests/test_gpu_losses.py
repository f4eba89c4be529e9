"""GPU tests of the losses over full-vocabulary logits against their definitions in 64 bits (tests/loss_reference.py has the bounds)."""
import math

import pytest
import torch

import loss_reference as R

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def losses():
    from paper_2603_16219_amd import losses as m

    assert torch.cuda.is_available(), "GPU tests need a device"
    m.library()
    return m


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def make(B, T, V, dtype, seed=0, sigma=2.0, ref=False):
    g = gen(1000 * seed + V + 7 * T + B)
    x = torch.randn(B, T, V, generator=g, device="cuda") * sigma
    out = {"logits": x.to(DTYPES[dtype]), "tokens": torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)}
    if ref:
        out["ref_logits"] = (x + 0.3 * torch.randn(B, T, V, generator=g, device="cuda")).to(DTYPES[dtype])
    return out, g


def ragged_mask(B, T, g, kind):
    if kind == "none":
        return None
    t = torch.arange(T, device="cuda")[None]
    if kind == "empty_sequence":  # the first sequence has no token that counts
        m = torch.rand(B, T, generator=g, device="cuda") < 0.6
        m[0] = False
        return m
    assert kind == "lengths"
    return t < torch.randint(0, T + 1, (B, 1), generator=g, device="cuda")


def close(got, want, bound, what):
    got, want = got.double(), want.double()
    assert torch.equal(got.isnan(), want.isnan()), f"{what}: NaN in other places"
    inf = want.isinf()
    assert torch.equal(got[inf], want[inf]), f"{what}: infinities"
    err = torch.where(want.isfinite(), (got - want).abs(), 0.0)
    worst = (err / bound).nan_to_num(0.0).max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} times its bound"


def check_grad(got, rows, w, kept, dtype, k=None):
    exact = torch.where(kept[..., None], rows.gradient(w, k), 0.0)
    close(got, exact, rows.gradient_bound(w, exact, got.dtype, k), "grad_logits")
    assert torch.all(got[~kept] == 0), "rows that do not count have a gradient"


def check_score(losses, inp, mask=None, tau=1.0, seed=0, logits=None, grad_logits=None):
    x, y = inp["logits"] if logits is None else logits, inp["tokens"]
    rows, kept = R.Rows(x, y, tau), R.kept_of(mask, y)
    out = losses.token_logprobs(x, y, mask=mask, temperature=tau, want_stats=True)
    close(out["logprobs"], torch.where(kept, rows.lp, 0.0), rows.lp_err, "logprobs")
    assert out["stats"].shape == (*y.shape, 2) and torch.all(out["stats"][~kept] == torch.tensor([0.0, 1.0], device="cuda"))
    w = torch.randn(y.shape, generator=gen(seed + 5), device="cuda")
    got = losses.token_logprobs_grad(x, y, out["stats"], w, mask=mask, temperature=tau, grad_scale=0.5, grad_logits=grad_logits)
    check_grad(got, rows, torch.where(kept, 0.5 * w.double(), 0.0), kept, x.dtype)
    return out


# Rows shorter than a vector, than a wave and than a workgroup, around those edges and around whole unrolled rounds of a workgroup, the
# odd vocabulary, and the smallest one there is.
EDGES = [1, 2, 3, 7, 8, 9, 15, 17, 31, 511, 512, 513, 2047, 2048, 2049, 4095, 4097, 8192, 16383, 16384, 16392, 32769, 50257, 65543]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", EDGES)
def test_token_logprobs_at_the_edges_of_vectors_and_workgroups(losses, V, dtype):
    inp, g = make(3, 5, V, dtype)
    check_score(losses, inp)
    check_score(losses, inp, mask=ragged_mask(3, 5, g, "empty_sequence"), tau=0.7)


@pytest.mark.parametrize("dtype,V", [("bf16", 128256), ("bf16", 151936), ("bf16", 256000), ("bf16", 131073), ("f32", 128256), ("f32", 100003),
                                     ("f32", 256000)])
def test_token_logprobs_of_large_vocabularies(losses, dtype, V):
    inp, _ = make(1, 3, V, dtype, sigma=3.0)
    check_score(losses, inp, tau=0.6)


@pytest.mark.parametrize("B,T", [(1, 1), (1, 700), (300, 1), (17, 33)])
def test_token_logprobs_of_few_and_many_rows(losses, B, T):
    inp, g = make(B, T, 1003, "bf16")
    check_score(losses, inp, mask=ragged_mask(B, T, g, "lengths"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1, 3, 4])
@pytest.mark.parametrize("pad", [0, 1, 5])
def test_views_with_strides_and_offsets(losses, dtype, offset, pad):
    """Rows that start anywhere, as logits[:, :-1] of a padded vocabulary do, with a gradient of other strides and alignment; what lies
    between and around the gradient's rows stays as it was."""
    B, T, V = 3, 6, 1037
    g = gen(offset * 10 + pad)
    store = torch.randn(offset + B * (T + 1) * (V + pad), generator=g, device="cuda").to(DTYPES[dtype])
    x = store[offset:].view(B, T + 1, V + pad)[:, :-1, :V]
    inp = {"tokens": torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)}
    for goff, gpad in ((0, 0), (offset, pad), (2, 3)):
        gstore = torch.full((goff + B * (T + 2) * (V + gpad) + 9,), 77.0, dtype=x.dtype, device="cuda")
        grad = gstore[goff:goff + B * (T + 2) * (V + gpad)].view(B, T + 2, V + gpad)[:, 1:-1, :V]
        check_score(losses, inp, logits=x, grad_logits=grad)
        touched = torch.zeros_like(gstore, dtype=torch.bool)
        touched[goff:goff + B * (T + 2) * (V + gpad)].view(B, T + 2, V + gpad)[:, 1:-1, :V] = True
        assert torch.all(gstore[~touched] == 77.0)


def policy_inputs(B, T, V, dtype, kl, g, inp, tau, per_token):
    rows = R.Rows(inp["logits"], inp["tokens"], tau)
    delta = 0.3 * torch.randn(B, T, generator=g, device="cuda", dtype=torch.float64)
    # where the ratio meets a border of the clipping the gradient jumps: the log-prob's own error may decide, so none is that near
    ratio = delta.exp()
    near = ((ratio - 0.8).abs() < 1e-3) | ((ratio - 1.28).abs() < 1e-3)
    old = (rows.lp - delta.masked_fill(near, 0.0)).float()
    adv = torch.randn((B, T) if per_token else (B,), generator=g, device="cuda")
    ref_lp = (rows.lp + 0.4 * torch.randn(B, T, generator=g, device="cuda")).float() if kl == "sampled" else None
    return old, adv, ref_lp


def check_policy(losses, inp, g, *, kl, mask=None, tau=1.0, per_token=True, reduction="token_mean", kl_coef=0.1, scale=1.0, grad_logits=None,
                 want_grad=True, poison=False):
    x, y = inp["logits"], inp["tokens"]
    B, T, V = x.shape
    z = inp["ref_logits"] if kl == "full" else None
    old, adv, ref_lp = policy_inputs(B, T, V, x.dtype, kl, g, inp, tau, per_token)
    rows, kept = R.Rows(x, y, tau, z), R.kept_of(mask, y)
    want = R.policy(rows, kept, old, adv, clip_low=0.2, clip_high=0.28, kl_coef=kl_coef if kl != "none" else 0.0, reduction=reduction,
                    ref_logprobs=ref_lp, scale=scale)
    if poison:  # nothing of a row that does not count is read
        x = x.clone()
        x[~kept] = math.nan
        y, old = y.masked_fill(~kept, -5), old.masked_fill(~kept, math.nan)
        if z is not None:
            z = z.masked_fill(~kept[..., None], math.nan)
        if ref_lp is not None:
            ref_lp = ref_lp.masked_fill(~kept, math.nan)
        if per_token:
            adv = adv.masked_fill(~kept, math.nan)
    out = losses.policy_loss(x, y, old, adv, mask=mask, ref_logits=z, ref_logprobs=ref_lp, clip_low=0.2, clip_high=0.28,
                             kl_coef=kl_coef if kl != "none" else 0.0, temperature=tau, reduction=reduction, grad_scale=scale,
                             want_grad=want_grad, grad_logits=grad_logits)
    close(out["logprobs"], torch.where(kept, rows.lp, 0.0), rows.lp_err, "logprobs")
    worst = torch.where(kept, rows.lp_err, 0.0).max().item()
    if kl == "full":
        close(out["kl"], want["kl"], rows.kl_err + U_of(want["kl"]), "kl")
        worst = max(worst, torch.where(kept, rows.kl_err, 0.0).max().item())
    elif kl == "sampled":  # its slope in the log-prob is 1 - e^d
        d = torch.where(kept, (ref_lp.double() - rows.lp).exp() + 1, 1.0)
        close(out["kl"], want["kl"], rows.lp_err * d + U_of(want["kl"]), "kl")
        worst *= d.max().item()
    else:
        assert out["kl"] is None
    close(out["loss"], want["loss"], 2 * worst * want["size"] + U_of(want["loss"]) + 1e-300, "loss")
    if not want_grad:
        assert out["grad_logits"] is None
        return out
    # the weight of a row moves with its log-prob: by lp_err of the ratio, and of the estimate's e^d
    w, k = want["w"], want["k"]
    exact = torch.where(kept[..., None], rows.gradient(w, k), 0.0)
    n = R.norms(kept, reduction) * scale
    adv2 = adv if adv.dim() == 2 else adv[:, None]
    dw = torch.where(kept, n * want["ratio"] * adv2.abs().double().nan_to_num(), 0.0)
    if ref_lp is not None:
        dw = dw + torch.where(kept, n * kl_coef * (ref_lp.double() - rows.lp).exp(), 0.0)
    moved = (dw * torch.where(kept, rows.lp_err, 0.0))[..., None] * (rows.onehot + rows.p) / rows.tau
    close(out["grad_logits"], exact, rows.gradient_bound(w, exact, x.dtype, k) + 2 * moved, "grad_logits")
    assert torch.all(out["grad_logits"][~kept] == 0)
    return out


def U_of(t):
    return R.U * t.abs() + 1e-37


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kl", ["none", "sampled", "full"])
@pytest.mark.parametrize("V", [1, 5, 8, 19, 513, 2048, 4099, 16391, 50257])
def test_policy_loss_at_the_edges(losses, V, kl, dtype):
    inp, g = make(3, 4, V, dtype, ref=True)
    check_policy(losses, inp, g, kl=kl)
    check_policy(losses, inp, g, kl=kl, mask=ragged_mask(3, 4, g, "empty_sequence"), tau=0.7, reduction="seq_mean", per_token=False, scale=3.0)


@pytest.mark.parametrize("mask", ["none", "lengths", "empty_sequence"])
@pytest.mark.parametrize("reduction", ["token_mean", "seq_mean", "sum"])
@pytest.mark.parametrize("per_token", [True, False])
def test_policy_loss_reductions_and_masks(losses, mask, reduction, per_token):
    for kl in ("none", "sampled", "full"):
        inp, g = make(7, 19, 331, "bf16", ref=True)
        check_policy(losses, inp, g, kl=kl, mask=ragged_mask(7, 19, g, mask), reduction=reduction, per_token=per_token, poison=mask != "none")


@pytest.mark.parametrize("dtype,V", [("bf16", 128256), ("bf16", 151936), ("bf16", 256000), ("bf16", 200001), ("f32", 128256), ("f32", 256000)])
@pytest.mark.parametrize("kl", ["none", "full"])
def test_policy_loss_of_large_vocabularies(losses, dtype, V, kl):
    inp, g = make(1, 3, V, dtype, sigma=3.0, ref=True)
    check_policy(losses, inp, g, kl=kl, tau=0.8)


# More rows than are cut into slices: one workgroup holds a row.  Around what it holds of short and long rows, and rows it holds a part of.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kl", ["none", "full"])
@pytest.mark.parametrize("V", [5, 1023, 4099, 8191, 8193, 16391, 30721, 61447, 122879, 122881, 200003])
def test_policy_loss_of_rows_held_by_a_workgroup(losses, V, kl, dtype):
    inp, g = make(2, 52, V, dtype, ref=True)
    check_policy(losses, inp, g, kl=kl, tau=0.9, mask=ragged_mask(2, 52, g, "lengths"))


@pytest.mark.parametrize("kl", ["none", "sampled", "full"])
def test_policy_loss_over_more_rows_than_units(losses, kl):
    inp, g = make(3, 300, 6007, "bf16", ref=True)
    check_policy(losses, inp, g, kl=kl, mask=ragged_mask(3, 300, g, "empty_sequence"), poison=True)
    inp, g = make(1, 17000, 211, "bf16", ref=True)  # more than count the mask's tokens themselves
    check_policy(losses, inp, g, kl=kl, mask=ragged_mask(1, 17000, g, "lengths"))


@pytest.mark.parametrize("offset", [1, 3, 15])
@pytest.mark.parametrize("T", [1, 5, 40, 700])
def test_tokens_counted_from_a_mask_at_any_address(losses, offset, T):
    inp, g = make(1, T, 67, "f32")
    store = torch.zeros(T + 64, dtype=torch.uint8, device="cuda")
    store[offset:offset + T] = (torch.rand(T, generator=g, device="cuda") < 0.5).byte() * torch.randint(1, 256, (T,), generator=g, device="cuda").byte()
    store[:offset], store[offset + T:] = 1, 1
    check_policy(losses, inp, g, kl="none", mask=store[offset:offset + T].view(1, T))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [4099, 50257, 70001])
def test_token_logprobs_of_many_long_rows(losses, V, dtype):
    inp, g = make(4, 75, V, dtype)
    check_score(losses, inp, mask=ragged_mask(4, 75, g, "lengths"), tau=0.8)
    check_score(losses, {k: v[:, :30] for k, v in inp.items()} | {"tokens": inp["tokens"][:, :30].contiguous()})


def test_policy_loss_without_gradient(losses):
    for kl in ("none", "sampled", "full"):
        inp, g = make(4, 9, 4099, "bf16", ref=True)
        check_policy(losses, inp, g, kl=kl, want_grad=False)


def check_preference(losses, inp, g, *, mask=None, tau=1.0, beta=0.3, smoothing=0.1, reference=True, reduction="mean", scale=1.0, want_grad=True):
    x, y = inp["logits"], inp["tokens"]
    rows, kept = R.Rows(x, y, tau), R.kept_of(mask, y)
    ref = (rows.lp + 0.3 * torch.randn(y.shape, generator=g, device="cuda")).float() if reference else None
    want = R.preference(rows, kept, ref, beta=beta, label_smoothing=smoothing, reduction=reduction, scale=scale)
    given = None if ref is None else ref.masked_fill(~kept, math.nan)
    out = losses.preference_loss(x, y, mask=mask, ref_logprobs=given, beta=beta, label_smoothing=smoothing, temperature=tau, reduction=reduction,
                                 grad_scale=scale, want_grad=want_grad)
    close(out["logprobs"], torch.where(kept, rows.lp, 0.0), rows.lp_err, "logprobs")
    close(out["margin"], want["margin"], want["margin_err"] + U_of(want["margin"]), "margin")
    close(out["pair_loss"], want["pair_loss"], want["margin_err"] + U_of(want["pair_loss"]), "pair_loss")  # its slope is at most 1
    close(out["loss"], want["loss"], want["margin_err"].sum() * want["factor"] + U_of(want["loss"]), "loss")
    if want_grad:
        w = want["w"]
        exact = torch.where(kept[..., None], rows.gradient(w), 0.0)
        # the weight's slope in the margin is at most 1/4 of beta times the pair's factor
        dw = (abs(beta) * want["factor"] * scale * want["margin_err"]).repeat(2)[:, None, None] * kept[..., None]
        close(out["grad_logits"], exact, rows.gradient_bound(w, exact, x.dtype) + dw * (rows.onehot + rows.p) / rows.tau, "grad_logits")
        assert torch.all(out["grad_logits"][~kept] == 0)
    else:
        assert out["grad_logits"] is None
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 7, 8, 513, 4099, 50257, 128256])
def test_preference_loss_at_the_edges(losses, V, dtype):
    inp, g = make(4, 5, V, dtype)
    check_preference(losses, inp, g)
    check_preference(losses, inp, g, mask=ragged_mask(4, 5, g, "empty_sequence"), tau=0.7, reduction="sum", scale=0.25)


@pytest.mark.parametrize("B,T", [(2, 1), (2, 2000), (32, 7), (34, 5), (2, 512), (2, 513), (600, 3)])
@pytest.mark.parametrize("reference", [True, False])
def test_preference_loss_of_few_and_many_pairs(losses, B, T, reference):
    inp, g = make(B, T, 403, "bf16")
    check_preference(losses, inp, g, mask=ragged_mask(B, T, g, "lengths"), reference=reference, beta=0.05, smoothing=0.0)
    check_preference(losses, inp, g, beta=-0.2, smoothing=0.5, reference=reference, want_grad=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("low", ["-inf", "lowest"])
def test_masked_vocabulary(losses, dtype, low):
    """A mask shared by policy and reference, one of the policy's own, a row with a single token left, and a row of lowest values only
    (uniform) or of -inf only (no distribution: NaN)."""
    dt = DTYPES[dtype]
    value = -math.inf if low == "-inf" else torch.finfo(dt).min
    inp, g = make(4, 6, 3001, dtype, ref=True)
    x, z, y = inp["logits"], inp["ref_logits"], inp["tokens"]
    off = torch.rand(3001, generator=g, device="cuda") < 0.5
    off.scatter_(0, y.flatten().long(), False)
    x[:, :, off] = value
    z[:, :, off] = value
    x[1, 2] = value  # one token left
    x[1, 2, 17] = 0.5
    y[1, 2] = 17
    x[2, 1, :1500] = value
    y[2, 1] = 1700
    x[3, 3] = value
    whole = torch.zeros(4, 6, dtype=torch.bool, device="cuda")
    whole[3, 3] = True
    for tau in (1.0, 0.6, 0.7, 0.9, 1.3):
        check_score(losses, {"logits": x, "tokens": y}, mask=None if low == "lowest" else ~whole, tau=tau)
    if low == "-inf":
        out = losses.token_logprobs(x, y, want_stats=True)
        assert out["logprobs"].isnan().sum() == 1 and out["logprobs"][3, 3].isnan()
        grad = losses.token_logprobs_grad(x, y, out["stats"], torch.ones(4, 6, device="cuda"))
        assert grad[3, 3].isnan().all() and not grad[~whole].isnan().any()
    z[1, 2, 17], z[3, 3] = 0.25, 0.0  # the reference's own masks differ in these rows
    for kl in ("none", "sampled", "full"):
        for tau in (1.0, 0.6, 0.9, 1.3):
            check_policy(losses, {"logits": x, "tokens": y, "ref_logits": z}, g, kl=kl, mask=~whole, tau=tau)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [(2, 5, 1003), (2, 5, 50257), (4, 30, 1003)])
def test_tokens_that_the_reference_alone_masks(losses, rows, dtype):
    """Their rows' KL is infinite and so is the loss; without a coefficient the KL is reported and loss and gradient are those without a reference."""
    inp, g = make(*rows, dtype, ref=True)
    x, y, z = inp["logits"], inp["tokens"], inp["ref_logits"]
    z[0, :2, 7] = -math.inf
    x[0, 1, 7] = x[0, 0].float().amin() - 500  # a token whose term is nothing: no matter what the reference says of it
    y[0, 1] = 8
    x[1, 3, 9] = -math.inf
    y[1, 3] = 8
    old, adv = torch.zeros(rows[:2], device="cuda") - 8, torch.randn(rows[:2], generator=g, device="cuda")
    want = losses.policy_loss(x, y, old, adv)
    got = losses.policy_loss(x, y, old, adv, ref_logits=z)
    assert torch.equal(got["loss"], want["loss"]) and torch.equal(got["logprobs"], want["logprobs"])
    half = torch.finfo(x.dtype).eps
    assert ((got["grad_logits"].float() - want["grad_logits"].float()).abs() <= half * want["grad_logits"].float().abs() + 1e-30).all()
    assert got["kl"][0, 0] == math.inf and got["kl"].flatten()[1:].isfinite().all()
    with_kl = losses.policy_loss(x, y, old, adv, ref_logits=z, kl_coef=0.1)
    assert not with_kl["loss"].isfinite() and not with_kl["grad_logits"][0, 0].isfinite().all()
    assert with_kl["grad_logits"].flatten(0, 1)[1:].isfinite().all()


@pytest.mark.parametrize("B,T", [(20000, 1), (2000, 40), (300, 65)])
def test_means_over_many_sequences(losses, B, T):
    inp, g = make(B, T, 37, "f32")
    mask = torch.rand(B, T, generator=g, device="cuda") < 0.4
    for reduction in ("token_mean", "seq_mean"):
        check_policy(losses, inp, g, kl="none", mask=mask, reduction=reduction)


@pytest.mark.parametrize("rows", [(3, 4, 2051), (3, 4, 70003), (2, 60, 1999)])  # one workgroup a row, slices, and the same of many rows
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift", [700.0, -7e5, 9e5, 3e7, -1e30])
def test_rows_far_from_zero(losses, dtype, shift, rows):
    """Logits around a common offset, on both sides of the limit up to which rows are summed by exponents, some of them masked."""
    inp, g = make(*rows, dtype, sigma=1.0, ref=True)
    x, z, y = inp["logits"], inp["ref_logits"], inp["tokens"]
    step = max(1.0, abs(shift)) * torch.finfo(x.dtype).eps  # differences of a few steps of the type there
    x.copy_(x.float() * step + shift)
    z.copy_(z.float() * step + shift)
    x[..., 1900:] = torch.finfo(x.dtype).min
    y[:] = y % 1900
    tau = max(1.0, step)
    check_score(losses, inp, tau=tau)
    for kl in ("none", "sampled", "full"):
        check_policy(losses, inp, g, kl=kl, tau=tau)
    check_preference(losses, inp | {"logits": x[:2], "tokens": y[:2]}, g, tau=tau)
    if abs(shift) < 1e7:  # differences of a few steps are many units here: rows of one token, nearly
        check_score(losses, inp)
        check_policy(losses, inp, g, kl="none")


def test_token_of_probability_zero_and_tokens_outside_the_vocabulary(losses):
    inp, g = make(4, 5, 777, "bf16")
    x, y = inp["logits"], inp["tokens"]
    x[0, 1, 5], y[0, 1] = -math.inf, 5
    y[1, 2], y[2, 3] = -1, 777
    out = losses.token_logprobs(x, y, want_stats=True)
    assert out["logprobs"][0, 1] == -math.inf
    bad = torch.zeros(4, 5, dtype=torch.bool, device="cuda")
    bad[1, 2] = bad[2, 3] = True
    assert torch.equal(out["logprobs"].isnan(), bad)
    grad = losses.token_logprobs_grad(x, y, out["stats"], torch.ones(4, 5, device="cuda"))
    assert grad[bad].isnan().all() and not grad[~bad].isnan().any()
    zeros = torch.zeros(4, 5, device="cuda")
    got = losses.policy_loss(x, y, zeros, zeros + 1, mask=None)
    assert got["loss"].isnan() and got["grad_logits"][bad].isnan().all() and not got["grad_logits"][~bad].isnan().any()
    fine = losses.policy_loss(x, y, zeros, zeros + 1, mask=~bad)
    assert not fine["loss"].isnan() and not fine["grad_logits"].isnan().any()
    y[0, 1] = 6
    pref = losses.preference_loss(x, y)  # bad tokens in sequences 1 and 2: pair 1 (1 and 3) and pair 0 (0 and 2)
    assert pref["margin"].isnan().all() and pref["loss"].isnan()
    y[2, 3] = 3
    pref = losses.preference_loss(x, y)
    assert torch.equal(pref["margin"].isnan().cpu(), torch.tensor([False, True]))
    assert pref["grad_logits"][[1, 3]].isnan().all() and not pref["grad_logits"][[0, 2]].isnan().any()


@pytest.mark.parametrize("T", [4, 51])
@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [9, 4099, 50257, 128256, 256000])
def test_gradient_in_place_of_the_logits(losses, V, dtype, far, T):
    inp, g = make(2, T, V, dtype, ref=True)
    x, y, z = inp["logits"], inp["tokens"], inp["ref_logits"]
    if far:
        x[1, ::2] = 2e6
    zeros, adv = torch.zeros(2, T, device="cuda") - 5, torch.randn(2, T, generator=g, device="cuda")
    mask = torch.tensor([[1, 1, 0, 1], [0, 1, 1, 1]], dtype=torch.bool, device="cuda").repeat(1, (T + 3) // 4)[:, :T]
    calls = [lambda t, **k: losses.policy_loss(t, y, zeros, adv, mask=mask, **k),
             lambda t, **k: losses.policy_loss(t, y, zeros, adv, mask=mask, ref_logits=z, kl_coef=0.2, **k),
             lambda t, **k: losses.preference_loss(t, y, mask=mask, beta=0.4, **k)]
    for call in calls:
        want = call(x)
        inplace = x.clone()
        got = call(inplace, grad_logits=inplace)
        assert got["grad_logits"] is inplace
        for k in want:
            assert want[k] is None or torch.equal(want[k], got[k]), k
    stats = losses.token_logprobs(x, y, want_stats=True)["stats"]
    inplace = x.clone()
    assert torch.equal(losses.token_logprobs_grad(inplace, y, stats, adv, grad_logits=inplace), losses.token_logprobs_grad(x, y, stats, adv))


def test_empty_calls(losses):
    for B, T in ((0, 5), (4, 0), (0, 0)):
        x = torch.empty(B, T, 100, device="cuda")
        y = torch.empty(B, T, dtype=torch.int32, device="cuda")
        f = torch.empty(B, T, device="cuda")
        assert losses.token_logprobs(x, y)["logprobs"].shape == (B, T)
        out = losses.policy_loss(x, y, f, f)
        assert out["loss"].item() == 0.0 and out["grad_logits"].shape == (B, T, 100)
        out = losses.preference_loss(x, y)
        assert out["loss"].item() == pytest.approx(math.log(2) if B else 0.0, rel=1e-7) and out["margin"].shape == (B // 2,)
    inp, g = make(4, 6, 211, "bf16")
    none = torch.zeros(4, 6, dtype=torch.bool, device="cuda")
    for reduction in ("token_mean", "seq_mean", "sum"):
        out = losses.policy_loss(inp["logits"], inp["tokens"], torch.zeros(4, 6, device="cuda"), torch.ones(4, device="cuda"), mask=none,
                                 reduction=reduction)
        assert out["loss"].item() == 0.0 and not out["grad_logits"].any() and not out["logprobs"].any()
    out = losses.preference_loss(inp["logits"], inp["tokens"], mask=none)
    assert out["loss"].item() == pytest.approx(math.log(2), rel=1e-7) and not out["grad_logits"].any()


def test_same_bits_on_every_call_on_dirty_workspaces(losses):
    inp, g = make(6, 40, 50257, "bf16", ref=True)
    x, y, z = inp["logits"], inp["tokens"], inp["ref_logits"]
    old, adv, mask = torch.zeros(6, 40, device="cuda") - 9, torch.randn(6, generator=g, device="cuda"), ragged_mask(6, 40, g, "lengths")
    params = losses._make_params(x, y, 1.0)
    need = losses.workspace_bytes(params)
    first = None
    for fill in (0, 255, 127):
        ws = torch.full((need + 512,), fill, dtype=torch.uint8, device="cuda")
        out = [losses.policy_loss(x, y, old, adv, mask=mask, ref_logits=z, kl_coef=0.1, workspace=ws[:need]),
               losses.preference_loss(x, y, mask=mask, workspace=ws[:need]), losses.token_logprobs(x, y, mask=mask, workspace=ws[:need])]
        assert torch.all(ws[need:] == fill), "written behind the workspace"
        flat = [t for o in out for t in o.values() if t is not None]
        first = first or flat
        assert all(torch.equal(a, b) for a, b in zip(first, flat))


def test_captured_and_replayed(losses):
    """One graph of a whole update, replayed between eager calls on other inputs."""
    inp, g = make(4, 12, 20011, "bf16", ref=True)
    x, y, z = inp["logits"], inp["tokens"], inp["ref_logits"]
    mask = ragged_mask(4, 12, g, "empty_sequence")
    old, adv = torch.zeros(4, 12, device="cuda") - 9, torch.randn(4, generator=g, device="cuda")

    def update(x):
        ref = losses.token_logprobs(z, y, mask=mask, want_stats=True)
        return [ref["logprobs"], losses.token_logprobs_grad(z, y, ref["stats"], old, mask=mask),
                *losses.policy_loss(x, y, old, adv, mask=mask, ref_logprobs=ref["logprobs"], kl_coef=0.1).values(),
                *losses.policy_loss(x, y, old, adv, mask=mask, ref_logits=z, kl_coef=0.1, reduction="seq_mean").values(),
                *losses.preference_loss(x, y, mask=mask, ref_logprobs=ref["logprobs"]).values()]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        update(x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        static = update(x)
    for i in range(4):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda") * 2)
        want = [t.clone() for t in update(x)]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, static)), i


def test_on_another_stream(losses):
    inp, g = make(4, 30, 50257, "bf16")
    x, y = inp["logits"], inp["tokens"]
    want = losses.preference_loss(x, y)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        busy = torch.randn(2048, 2048, device="cuda")
        for _ in range(20):
            busy = busy @ busy * 1e-3
        late = torch.zeros_like(x).add_(x)  # ready only behind the products
        got = losses.preference_loss(late, y)
    side.synchronize()
    assert all(torch.equal(want[k], got[k]) for k in want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_rows_than_one_dimension_of_a_grid_holds(losses, dtype):
    B, T, V = 2, 70001, 11
    inp, g = make(B, T, V, dtype, ref=True)
    mask = ragged_mask(B, T, g, "lengths")
    check_score(losses, inp, mask=mask)
    check_policy(losses, inp, g, kl="none", mask=mask)
    check_policy(losses, inp, g, kl="full", reduction="seq_mean", mask=mask)
    check_preference(losses, inp, g, mask=mask, beta=0.01)


@pytest.mark.parametrize("rows", [1, 101])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_vocabulary(losses, dtype, rows):
    inp, g = make(2 if rows == 1 else 1, rows, 1 << 20, dtype, ref=True)
    if rows == 1:
        check_score(losses, inp)
        check_preference(losses, inp, g)
    for kl in ("none", "full"):
        check_policy(losses, inp, g, kl=kl)


def test_calls_from_several_threads_and_streams_at_once(losses):
    """Four threads, each with a stream, inputs and a workspace of its own, and each of the calls over and over: what they give alone."""
    import threading

    def work(k):
        inp, g = make(2, 3 + 30 * k, 5003, "bf16", seed=k, ref=True)
        x, y, z = inp["logits"], inp["tokens"], inp["ref_logits"]
        old, adv = torch.zeros(y.shape, device="cuda") - 8, torch.randn(y.shape, generator=g, device="cuda")
        return lambda: [t for o in (losses.policy_loss(x, y, old, adv), losses.policy_loss(x, y, old, adv, ref_logits=z, kl_coef=0.1),
                                    losses.preference_loss(x, y), losses.token_logprobs(x, y)) for t in o.values() if t is not None]

    calls = [work(k) for k in range(4)]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    wrong = []

    def run(k):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                got = calls[k]()
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(want[k], got)):
                    wrong.append(k)

    threads = [threading.Thread(target=run, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_offsets_beyond_32_bits(losses):
    """Logits of more than 2^31 elements: rows at the end against the same rows on their own."""
    T, V = 8400, 256000
    assert T * V > 2**31
    x = torch.zeros(1, T, V, dtype=torch.bfloat16, device="cuda")
    g = gen(3)
    tail = torch.randn(1, 3, V, generator=g, device="cuda").bfloat16()
    x[:, -3:] = tail
    y = torch.randint(0, V, (1, T), generator=g, device="cuda", dtype=torch.int32)
    mask = torch.zeros(1, T, dtype=torch.bool, device="cuda")
    mask[:, -3:] = True
    old, adv = torch.zeros(1, T, device="cuda") - 12, torch.ones(1, device="cuda")
    want = losses.policy_loss(tail, y[:, -3:], old[:, -3:], adv)
    got = losses.policy_loss(x, y, old, adv, mask=mask, grad_logits=x)
    assert torch.equal(got["logprobs"][:, -3:], want["logprobs"]) and torch.equal(got["loss"], want["loss"])
    assert torch.equal(x[:, -3:], want["grad_logits"]) and not x[:, 4000:4003].any()
    x = x.view(2, T // 2, V)
    x[:, -3:] = tail
    y, mask, two = y.view(2, T // 2), mask.view(2, T // 2), torch.cat([tail, tail])
    mask[:, -3:] = True
    short = y[:, -3:].contiguous()
    want = losses.preference_loss(two, short)
    stats = losses.token_logprobs(two, short, want_stats=True)
    w = torch.randn(2, T // 2, generator=g, device="cuda")
    want_grad = losses.token_logprobs_grad(two, short, stats["stats"], w[:, -3:].contiguous())
    got = losses.token_logprobs(x, y, mask=mask, want_stats=True)
    # few rows are summed by other workgroups than many.  Log-probs of about -13: each result is rounded by 4.8e-7 at most, the sums before
    # differ by less; gradients: each is rounded to bf16, by 2^-8 at most.
    assert (got["logprobs"][:, -3:] - stats["logprobs"]).abs().max() <= 2e-6
    grad = losses.token_logprobs_grad(x, y, got["stats"], w, mask=mask)
    assert ((grad[:, -3:].float() - want_grad.float()).abs() <= 2.0 ** -7 * want_grad.float().abs() + 1e-30).all() and not grad[1, 2000:2003].any()
    del grad
    got = losses.preference_loss(x, y, mask=mask, grad_logits=x)
    assert (got["margin"] - want["margin"]).abs().max() <= 2e-6
    assert ((x[:, -3:].float() - want["grad_logits"].float()).abs() <= 2.0 ** -7 * want["grad_logits"].float().abs() + 1e-30).all()


@pytest.mark.parametrize("kl", ["sampled", "full"])
def test_gradients_against_differences(losses, kl):
    """Central differences of the loss itself along a direction, steps 2^-6.  The loss is fp32: its roundings and the sums' are
    about 8 u of it each side over 2^-5, and the step's own error is of the third derivative, 2^-12 / 6 times a few."""
    inp, g = make(2, 6, 97, "f32", sigma=1.0, ref=True)
    x, y, z = inp["logits"], inp["tokens"], inp["ref_logits"]
    rows = R.Rows(x, y, 1.0)
    old = (rows.lp + 0.05 * torch.randn(2, 6, generator=g, device="cuda")).float()
    adv, step = torch.randn(2, 6, generator=g, device="cuda"), 2.0 ** -6
    refs = {"ref_logits": z} if kl == "full" else {"ref_logprobs": (rows.lp + 0.2).float()}
    calls = [lambda t: losses.policy_loss(t, y, old, adv, kl_coef=0.5, clip_low=0.9, clip_high=5.0, **refs),
             lambda t: losses.preference_loss(t, y, ref_logprobs=old, beta=0.7, label_smoothing=0.2)]
    for call in calls:
        base = call(x)
        for _ in range(3):
            d = torch.randn(x.shape, generator=g, device="cuda")
            d /= d.norm()
            slope = (base["grad_logits"].double() * d).sum().item()
            diff = (call(x + step * d)["loss"].double() - call(x - step * d)["loss"].double()).item() / (2 * step)
            assert abs(diff - slope) <= 16 * R.U * max(1.0, abs(base["loss"].item())) / step + step * step


def test_a_training_step_through_a_model(losses):
    """Scoring by a frozen reference, the loss and its gradient, and the model's own backward pass from it: the weights' gradient is
    that of the whole step by automatic differentiation in 64 bits."""
    g = gen(11)
    B, T, D, V = 4, 8, 32, 1001
    hidden = torch.randn(B, T, D, generator=g, device="cuda")
    head = (torch.randn(V, D, generator=g, device="cuda") * 0.3).requires_grad_()
    frozen = torch.randn(V, D, generator=g, device="cuda") * 0.3
    y = torch.randint(0, V, (B, T), generator=g, device="cuda")
    mask = ragged_mask(B, T, g, "lengths")
    adv = torch.randn(B, generator=g, device="cuda")
    ref_logits = hidden @ frozen.T
    ref = losses.token_logprobs(ref_logits, y, mask=mask)["logprobs"]
    old = losses.token_logprobs((hidden @ head.T).detach(), y, mask=mask)["logprobs"]

    def by_definition(kind):
        w = head.detach().double().requires_grad_()
        lp = torch.log_softmax(hidden.double() @ w.T, -1)
        at = lp.gather(-1, y[..., None])[..., 0]
        if kind == "preference":
            d = ((at - ref.double()) * mask).sum(1)
            loss = -torch.nn.functional.logsigmoid(R.f32(0.1) * (d[:2] - d[2:])).mean()
        else:
            ratio = torch.exp(at - old.double())
            a = adv.double()[:, None]
            term = -torch.minimum(ratio * a, ratio.clamp(1 - R.f32(0.2), 1 + R.f32(0.2)) * a)
            if kind == "full":
                q = torch.log_softmax(ref_logits.double(), -1)
                term = term + R.f32(0.1) * (lp.exp() * (lp - q)).sum(-1)
            else:
                r = ref.double() - at
                term = term + R.f32(0.1) * (r.exp() - 1 - r)
            loss = (term * mask).sum() / mask.sum()
        loss.backward()
        return loss.item(), w.grad

    for kind in ("sampled", "full", "preference"):
        head.grad = None
        logits = hidden @ head.T
        if kind == "preference":
            out = losses.preference_loss(logits, y, mask=mask, ref_logprobs=ref, beta=0.1)
        else:
            refs = {"ref_logits": ref_logits} if kind == "full" else {"ref_logprobs": ref}
            out = losses.policy_loss(logits, y, old, adv, mask=mask, kl_coef=0.1, **refs)
        logits.backward(out["grad_logits"])
        loss, grad = by_definition(kind)
        # logits of 32 products in fp32 (32 u of a few), the gradients' sums over B T rows: 1e-5 of the largest is several times that
        assert out["loss"].item() == pytest.approx(loss, abs=1e-5)
        assert (head.grad.double() - grad).abs().max() <= 1e-5 * grad.abs().max() + 1e-7
