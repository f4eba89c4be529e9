"""GPU tests of entropies, top alternatives and their gradient against the definitions in 64 bits (tests/alternatives_reference.py has the bounds)."""
import math

import pytest
import torch

import alternatives_reference as A
from test_gpu_losses import close, gen, make, ragged_mask

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def losses():
    from paper_2603_16219_amd import losses as m

    assert torch.cuda.is_available(), "GPU tests need a device"
    m.library()
    return m


def check(losses, x, y, *, topk, mask=None, tau=1.0, seed=0, grad_logits=None, grad=True):
    rows = A.Rows(x, y, tau)
    kept = torch.ones_like(y, dtype=torch.bool) if mask is None else mask.bool()
    out = losses.token_alternatives(x, y, topk=topk, mask=mask, temperature=tau, want_stats=True)
    close(out["logprobs"], torch.where(kept, rows.lp, 0.0), rows.lp_err, "logprobs")
    close(out["entropy"], torch.where(kept, rows.entropy, 0.0), rows.entropy_err, "entropy")
    if topk:
        ids, lp, err = rows.top(x, topk)
        assert torch.equal(out["top_tokens"], torch.where(kept[..., None], ids, -1)), "top_tokens"
        close(out["top_logprobs"], torch.where(kept[..., None], lp, -math.inf), err, "top_logprobs")
    else:
        assert out["top_tokens"] is None and out["top_logprobs"] is None
    assert torch.all(out["stats"][~kept] == torch.tensor([0.0, 1.0], device="cuda"))
    if grad:
        g, k = (torch.randn(y.shape, generator=gen(seed + i), device="cuda") for i in (5, 6))
        for a, b in ((g, k), (None, k), (g, None)):
            got = losses.token_alternatives_grad(x, y, out["stats"], out["entropy"], a, b, mask=mask, temperature=tau, grad_scale=0.5, grad_logits=grad_logits)
            da, db = (torch.zeros_like(rows.lp) if t is None else torch.where(kept, 0.5 * t.double(), 0.0) for t in (a, b))
            exact = torch.where(kept[..., None], rows.gradient2(da, db), 0.0)
            close(got, exact, rows.gradient2_bound(da, db, exact, got.dtype), "grad_logits")
            assert torch.all(got[~kept] == 0)
    return out


# Around vectors, waves, workgroups, whole rounds and slices.
EDGES = [1, 2, 7, 8, 9, 31, 64, 511, 513, 2047, 2049, 4095, 4096, 4104, 4111, 8193, 16383, 16392, 32769, 50257, 65543]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", EDGES)
def test_edges_of_vectors_workgroups_and_slices(losses, V, dtype):
    inp, g = make(3, 5, V, dtype)
    check(losses, inp["logits"], inp["tokens"], topk=9)
    check(losses, inp["logits"], inp["tokens"], topk=64, mask=ragged_mask(3, 5, g, "empty_sequence"), tau=0.7)
    inp, g = make(7, 30, V, dtype, seed=1)  # a workgroup a row
    check(losses, inp["logits"], inp["tokens"], topk=17, mask=ragged_mask(7, 30, g, "lengths"), grad=V < 20000)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 16, 100, 101])
@pytest.mark.parametrize("topk", [0, 1, 2, 4, 5, 8, 16, 17, 32, 33, 63, 64])
def test_every_number_of_groups(losses, topk, rows, dtype):
    inp, _ = make(1, rows, 32003, dtype, seed=topk)
    check(losses, inp["logits"], inp["tokens"], topk=topk, grad=False)


@pytest.mark.parametrize("dtype,V", [("bf16", 128256), ("bf16", 256000), ("bf16", 131073), ("f32", 151936), ("bf16", 1 << 20)])
def test_long_rows(losses, dtype, V):
    for T in (2, 120):
        inp, _ = make(1, T, V, dtype)
        check(losses, inp["logits"], inp["tokens"], topk=20, tau=0.6, grad=T == 2)


def arranged(kind, V, dtype, g):
    x = torch.randn(V, generator=g, device="cuda") * 3
    if kind == "rising":
        x = x.sort().values
    elif kind == "falling":
        x = x.sort(descending=True).values
    elif kind == "uniform":
        x = torch.full_like(x, 1.25)
    elif kind == "zeros_of_both_signs":
        x = torch.where(torch.rand(V, generator=g, device="cuda") < 0.5, 0.0, -0.0)
    elif kind == "two_values":
        x = torch.where(torch.rand(V, generator=g, device="cuda") < 0.3, 2.0, -1.0)
    elif kind == "negative_ties":
        x = -torch.randint(3, 6, (V,), generator=g, device="cuda").float()
    elif kind == "top_at_one_end":
        x[-70:] += 50
    elif kind == "one_block":
        x[V // 2:V // 2 + 40] += 30
    elif kind == "certain":
        x[V // 3] = 60
    return x.to(dtype)


KINDS = ["rising", "falling", "uniform", "zeros_of_both_signs", "two_values", "negative_ties", "top_at_one_end", "one_block", "certain"]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [2, 130])
@pytest.mark.parametrize("kind", KINDS)
def test_orders_and_ties(losses, kind, rows, dtype):
    g = gen(len(kind) + rows)
    for V, topk in ((32000, 64), (50257, 7), (6001, 33)):
        x = arranged(kind, V, dtype, g)[None, None].expand(1, rows, V).contiguous()
        y = torch.randint(0, V, (1, rows), generator=g, device="cuda", dtype=torch.int32)
        check(losses, x, y, topk=topk, grad=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lead", [0, 1])
@pytest.mark.parametrize("rows", [1, 5, 100])
@pytest.mark.parametrize("tied", ["lowest", 1.25, 14.0])
@pytest.mark.parametrize("part", ["first", "last", "middle"])
def test_ties_in_one_part_of_a_row(losses, part, tied, rows, lead, dtype):
    """Of rows in slices only one has more ties than its lists hold, and the elements outside of vectors are among the likeliest."""
    V, vec, g = 50257, 8 if dtype is torch.bfloat16 else 4, gen(rows + lead)
    each = -(-(V // vec) // min(64, -(-1024 // rows), V // vec // 512)) * vec  # elements of a slice
    x = torch.full((1, rows, V + 7 + lead), math.nan, dtype=dtype, device="cuda")[:, :, lead:lead + V]
    x.copy_(torch.randn(1, rows, V, generator=g, device="cuda") * 3)
    at = {"first": 0, "middle": 3 * each, "last": V - 1 - each}[part]
    x[:, :, at:at + each] = torch.finfo(dtype).min if tied == "lowest" else tied
    x[:, :, [V - 1, V - 2, 1, 0]] = torch.tensor([16.0, 15.0, 15.5, 14.5], dtype=dtype, device="cuda")
    y = torch.randint(0, V, (1, rows), generator=g, device="cuda", dtype=torch.int32)
    y[0, 0] = V - 1
    for topk in (1, 7, 64):
        check(losses, x, y, topk=topk, grad=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [3, 120])
@pytest.mark.parametrize("low", ["inf", "lowest"])
def test_masked_tokens(losses, low, rows, dtype):
    g = gen(rows)
    V = 20011
    x = (torch.randn(1, rows, V, generator=g, device="cuda") * 3).to(dtype)
    v = -math.inf if low == "inf" else torch.finfo(dtype).min
    x[:, :, 12000:] = v                                   # padding
    x[0, 0, 5:] = v                                       # five tokens left
    x[0, 1] = torch.where(torch.rand(V, generator=g, device="cuda") < 0.999, torch.full((), v, dtype=dtype, device="cuda"), x[0, 1])
    y = torch.randint(0, 5, (1, rows), generator=g, device="cuda", dtype=torch.int32)
    check(losses, x, y, topk=20)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [2, 110])
def test_rows_without_a_distribution_and_far_ones(losses, rows, dtype):
    g = gen(3)
    V = 9000
    x = torch.randn(1, rows, V, generator=g, device="cuda").to(dtype)
    x[0, 0] = -math.inf
    y = torch.randint(0, V, (1, rows), generator=g, device="cuda", dtype=torch.int32)
    out = losses.token_alternatives(x, y, topk=4)
    assert out["logprobs"][0, 0].isnan() and out["entropy"][0, 0].isnan() and torch.all(out["top_tokens"][0, 0] == -1)
    assert torch.all(out["top_logprobs"][0, 0] == -math.inf) and not out["entropy"][0, 1:].isnan().any()
    x[0, 0] = torch.finfo(dtype).min  # a uniform row
    x[0, 1] = (x[0, 1].float() * 1e6 + 3e7).to(dtype)
    check(losses, x, y, topk=33)
    check(losses, x, y, topk=3, tau=1e-13)
    check(losses, x[:, 1:].contiguous(), y[:, 1:].contiguous(), topk=3, tau=1e13)
    x[0, 0] = math.nan  # unspecified, but it comes back
    out = losses.token_alternatives(x, y, topk=64, want_stats=True)
    assert torch.all(out["top_tokens"][0, 0] == -1)
    losses.token_alternatives_grad(x, y, out["stats"], out["entropy"], out["entropy"], out["entropy"])
    x[0, 0, ::2] = 1.0
    out = losses.token_alternatives(x, y, topk=64)
    assert out["top_tokens"][0, 0].tolist() == list(range(0, 128, 2))


def test_tokens_out_of_the_vocabulary_and_none(losses):
    inp, _ = make(2, 3, 1000, "f32")
    x, y = inp["logits"], inp["tokens"]
    y[0, 0], y[1, 2] = -1, 1000
    out = losses.token_alternatives(x, y, topk=2, want_stats=True)
    assert out["logprobs"].isnan().tolist() == [[True, False, False], [False, False, True]] and not out["entropy"].isnan().any()
    g = torch.ones(2, 3, device="cuda")
    grad = losses.token_alternatives_grad(x, y, out["stats"], out["entropy"], g, g)
    assert grad[0, 0].isnan().all() and grad[1, 2].isnan().all() and not grad[0, 1:].isnan().any()
    alone = losses.token_alternatives(x, topk=2, want_stats=True)
    assert alone["logprobs"] is None and all(torch.equal(alone[k], out[k]) for k in ("entropy", "top_tokens", "top_logprobs", "stats"))
    assert torch.equal(losses.token_alternatives_grad(x, None, out["stats"], out["entropy"], None, g), losses.token_alternatives_grad(x, y, out["stats"], out["entropy"], None, g))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [(2, 3), (9, 13)])
@pytest.mark.parametrize("lead,pad", [(0, 3), (1, 0), (3, 6)])
def test_strides_and_alignments(losses, dtype, rows, lead, pad):
    B, T = rows
    V = 5003
    g = gen(lead + pad)
    big = torch.full((B, T + 2, lead + V + pad), math.nan, dtype=dtype, device="cuda")
    x = big[:, 1:-1, lead:lead + V]
    x.copy_(torch.randn(B, T, V, generator=g, device="cuda") * 3)
    y = torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)
    around = torch.full((B, T + 1, V + 7), 5.0, dtype=dtype, device="cuda")
    check(losses, x, y, topk=12, mask=ragged_mask(B, T, g, "lengths"), grad_logits=around[:, :T, 2:2 + V])
    assert torch.all(around[:, T] == 5) and torch.all(around[:, :, :2] == 5) and torch.all(around[:, :, 2 + V:] == 5)


def test_gradient_in_place_and_masked_positions_unread(losses):
    inp, g = make(4, 40, 3001, "bf16")
    x, y, mask = inp["logits"], inp["tokens"], ragged_mask(4, 40, g, "empty_sequence")
    clean = losses.token_alternatives(x, y, topk=5, mask=mask, want_stats=True)
    w = torch.randn(4, 40, generator=g, device="cuda")
    want = losses.token_alternatives_grad(x, y, clean["stats"], clean["entropy"], w, w, mask=mask)
    x[~mask] = math.nan
    y[~mask] = 1 << 30
    out = losses.token_alternatives(x, y, topk=5, mask=mask, want_stats=True)
    for k in out:
        assert torch.equal(out[k], clean[k]), k
    got = losses.token_alternatives_grad(x, y, out["stats"], out["entropy"], torch.where(mask, w, math.nan), w, mask=mask, grad_logits=x)
    assert got is x and torch.equal(got, want)


def test_statistics_are_those_of_the_log_probs(losses):
    """The gradient of log-probs alone takes either call's statistics."""
    for dtype in ("bf16", "f32"):
        inp, _ = make(3, 50, 20000, dtype)
        x, y = inp["logits"], inp["tokens"]
        rows, w = A.Rows(x, y, 0.7), torch.randn(3, 50, generator=gen(2), device="cuda")
        for out in (losses.token_alternatives(x, y, temperature=0.7, want_stats=True), losses.token_logprobs(x, y, temperature=0.7, want_stats=True)):
            exact = rows.gradient(w.double())
            for got in (losses.token_logprobs_grad(x, y, out["stats"], w, temperature=0.7),
                        losses.token_alternatives_grad(x, y, out["stats"], None, w, None, temperature=0.7)):
                close(got, exact, rows.gradient_bound(w.double(), exact, got.dtype), "grad_logits")


def test_gradient_against_differences(losses):
    g = gen(9)
    x = torch.randn(2, 3, 500, generator=g, device="cuda") * 2
    y = torch.randint(0, 500, (2, 3), generator=g, device="cuda", dtype=torch.int32)
    a, b = torch.randn(2, 3, generator=g, device="cuda"), torch.randn(2, 3, generator=g, device="cuda")

    def loss(t):
        out = losses.token_alternatives(t, y, temperature=0.9)
        return (out["logprobs"].double() * a).sum() + (out["entropy"].double() * b).sum()

    out = losses.token_alternatives(x, y, temperature=0.9, want_stats=True)
    grad = losses.token_alternatives_grad(x, y, out["stats"], out["entropy"], a, b, temperature=0.9).double()
    for i in range(6):
        d = torch.randn(x.shape, generator=g, device="cuda")
        h = 2.0 ** -7
        # the outputs' rounding, some 1e-6 in all, over the step; the third derivative times the step squared, which halving it shows
        rough, fine = ((loss(x + s * d) - loss(x - s * d)) / (2 * s) for s in (2 * h, h))
        assert abs((grad * d).sum() - fine) <= abs(rough - fine) + 2e-6 / h, i


def test_native_and_general_path_agree(losses, monkeypatch):
    assert losses._calls is not None
    inp, g = make(3, 40, 4099, "bf16")
    x, y, mask = inp["logits"], inp["tokens"], ragged_mask(3, 40, g, "lengths")
    w = torch.randn(3, 40, generator=g, device="cuda")
    calls = [lambda: losses.token_alternatives(x, y, topk=5, mask=mask, temperature=0.8, want_stats=True),
             lambda: losses.token_alternatives(x, topk=0),
             lambda: losses.token_alternatives(x[:1, :2], y[:1, :2], topk=64, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))]
    out = calls[0]()
    calls += [lambda: {"g": losses.token_alternatives_grad(x, y, out["stats"], out["entropy"], w, w, mask=mask, temperature=0.8, grad_scale=2)},
              lambda: {"g": losses.token_alternatives_grad(x, None, out["stats"], out["entropy"], None, w, temperature=0.8)}]
    for c in calls:
        taken = []
        with monkeypatch.context() as m:
            m.setattr(losses, "_native", lambda *a, f=losses._native: taken.append(f(*a)) or taken[-1])
            native = c()
        assert taken[-1] is not None
        with monkeypatch.context() as m:
            m.setattr(losses, "_calls", None)
            general = c()
        assert list(native) == list(general)
        for k in native:
            assert (native[k] is None and general[k] is None) or torch.equal(native[k], general[k]), k
    # what has to be converted: tokens of 64 bits, weights of 16, a mask of bytes
    conv = losses.token_alternatives(x, y.long(), topk=5, mask=mask.to(torch.uint8), temperature=0.8)
    assert all(torch.equal(conv[k], out[k]) for k in ("logprobs", "entropy", "top_tokens", "top_logprobs"))


def test_replays_and_other_streams(losses):
    for rows in (3, 150):
        inp, _ = make(1, rows, 30011, "bf16")
        x, y = inp["logits"], inp["tokens"]
        w = torch.randn(1, rows, generator=gen(1), device="cuda")

        def step():
            out = losses.token_alternatives(x, y, topk=16, want_stats=True)
            return {**out, "grad": losses.token_alternatives_grad(x, y, out["stats"], out["entropy"], w, w)}

        want = step()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                got = step()
        for i in range(4):
            x.copy_(torch.randn(x.shape, generator=gen(20 + i), device="cuda") * 3)
            want = step()
            graph.replay()
            torch.cuda.synchronize()
            for k in want:
                assert torch.equal(got[k], want[k]), (rows, i, k)
        with torch.cuda.stream(side):
            again = step()
        torch.cuda.synchronize()
        assert all(torch.equal(again[k], want[k]) for k in want)


def test_offsets_past_32_bits(losses):
    V, rows = 1 << 20, 2100
    x = torch.empty(1, rows, V, dtype=torch.bfloat16, device="cuda")
    few = [0, 1, 2047, 2048, 2099]
    mask = torch.zeros(1, rows, dtype=torch.bool, device="cuda")
    mask[0, few] = True
    for t in few:
        x[0, t] = torch.randn(V, generator=gen(t), device="cuda") * 3
    y = torch.randint(0, V, (1, rows), generator=gen(1), device="cuda", dtype=torch.int32)
    out = losses.token_alternatives(x, y, topk=6, mask=mask)
    part, z = x[:, few].contiguous(), y[:, few].contiguous()
    r = A.Rows(part, z, 1.0)
    close(out["entropy"][:, few], r.entropy, r.entropy_err, "entropy")
    assert torch.equal(out["top_tokens"][:, few], r.top(part, 6)[0])
