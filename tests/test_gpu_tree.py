"""GPU tests of trees of drafts against their definitions in 64 bits (tests/tree_reference.py has the bounds)."""
import math

import pytest
import torch

import tree_reference as R
from test_gpu_losses import close, gen

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def tree():
    from paper_2603_16219_amd import tree as m

    assert torch.cuda.is_available(), "GPU tests need a device"
    m.library()
    assert m._calls is not None
    return m


def make(B, N, Hq, H, D, lens, page, dtype="bf16", seed=0, kind="random", ragged=False, spare=3):
    """Everything a call of attention takes; what no call may read is NaN."""
    g, dt, dev = gen(17 * seed + B + 7 * N + 31 * Hq + D + page), DTYPES[dtype], "cuda"
    lens = torch.tensor(lens if isinstance(lens, (list, tuple)) else [lens] * B, dtype=torch.int32, device=dev)
    width = max(1, -(-(int(lens.max()) + N + 1) // page))
    pages = B * width + spare
    normal = lambda *s: torch.randn(*s, generator=g, device=dev).to(dt)
    i = {"q": normal(B, N + 1, Hq, D), "k": normal(B, N + 1, H, D), "v": normal(B, N + 1, H, D) + 0.5, "cache_len": lens,
         "table": torch.randperm(pages, generator=g, device=dev)[:B * width].to(torch.int32).view(B, width).contiguous(),
         "parents": R.random_trees(B, N, g, dev, kind) if kind != "none" else None,
         "tree_len": torch.randint(0, N + 1, (B,), generator=g, device=dev, dtype=torch.int32) if ragged else None}
    kc, vc = normal(pages, page, H, D), normal(pages, page, H, D) + 0.5
    held = torch.zeros(pages, page, dtype=torch.bool, device=dev)
    for b in range(B):
        t = torch.arange(int(lens[b]), device=dev)
        held[i["table"][b, t // page].long(), t % page] = True
        if ragged:
            for x in (i["q"], i["k"], i["v"]):
                x[b, int(i["tree_len"][b]) + 1:] = math.nan
    kc[~held], vc[~held] = math.nan, math.nan
    return {**i, "k_cache": kc, "v_cache": vc}


def run(tree, i, **more):
    return tree.attention(i["q"], i["k"], i["v"], i["k_cache"], i["v_cache"], i["table"], i["cache_len"], i["parents"], tree_len=i["tree_len"], **more)


def check(tree, i, scale=None, **more):
    got = run(tree, i, scale=scale, **more)
    want, bound = R.attention(i["q"], i["k"], i["v"], i["k_cache"], i["v_cache"], i["table"], i["cache_len"], i["parents"], i["tree_len"],
                              1 / math.sqrt(i["q"].shape[3]) if scale is None else scale)
    close(got, want, bound.clamp(min=1e-30), "out")
    return got


LENGTHS = [0, 1, 2, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 700]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L", LENGTHS)
def test_single_tokens_at_the_edges_of_tiles(tree, L, D, dtype):
    check(tree, make(3, 0, 8, 2, D, [L, max(0, L - 1), L + 1], 16, dtype, kind="none"))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [1, 3, 16, 24, 100, 1000])
def test_pages_that_end_anywhere(tree, page, D):
    check(tree, make(2, 6, 8, 4, D, [517, 96], page))


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("kind", ["none", "chain", "random", "wide", "star"])
@pytest.mark.parametrize("N", [1, 2, 7, 8, 15, 16, 30, 31, 32, 33, 63, 64, 100])
def test_trees(tree, N, kind, dtype, D):
    check(tree, make(2, N, 4, 2, D, [75, 300], 16, dtype, kind=kind))
    check(tree, make(3, N, 2, 2, D, [0, 40, 129], 16, dtype, kind=kind, ragged=True, seed=1))


@pytest.mark.parametrize("Hq,H", [(1, 1), (3, 1), (16, 1), (5, 5), (14, 2), (64, 4), (40, 8), (33, 11), (128, 1)])
@pytest.mark.parametrize("N", [0, 3, 20])
def test_heads(tree, Hq, H, N):
    check(tree, make(2, N, Hq, H, 128, [200, 33], 16))
    check(tree, make(1, N, Hq, H, 64, [70], 16, "f16"))


@pytest.mark.parametrize("N,kind", [(255, "random"), (256, "wide"), (400, "none"), (1023, "chain"), (1024, "random")])
def test_large_trees(tree, N, kind):
    check(tree, make(1, N, 4, 2, 64, [130], 16, kind=kind))
    check(tree, make(2, N, 2, 1, 128, [0, 777], 16, kind=kind, ragged=True))


@pytest.mark.parametrize("L,B,Hq,H", [(20000, 1, 8, 2), (5000, 3, 16, 2), (70001, 1, 4, 1)])
def test_long_caches(tree, L, B, Hq, H):
    check(tree, make(B, 12, Hq, H, 128, [L - 137 * b for b in range(B)], 64))
    check(tree, make(B, 0, Hq, H, 64, [L - 1111 * b for b in range(B)], 16, "f16", kind="none"))


@pytest.mark.parametrize("N,Hq,H", [(40, 8, 2), (70, 16, 2), (130, 3, 1)])
@pytest.mark.parametrize("page", [1, 7, 64])
def test_wide_trees_over_long_caches(tree, N, Hq, H, page):
    """More columns than a workgroup of four waves has; with small pages a sequence's table comes in pieces, a new one inside of a share."""
    check(tree, make(2, N, Hq, H, 128, [5003, 1100], page, kind="random"))
    check(tree, make(3, N, Hq, H, 64, [2500, 0, 3333], page, "f16", kind="wide", ragged=True))


@pytest.mark.parametrize("B", [1, 2, 31, 64, 257, 600])
def test_batches_of_any_lengths(tree, B):
    g = torch.Generator().manual_seed(B)
    lens = (torch.rand(B, generator=g) ** 3 * 900).int().tolist()
    lens[0] = 0
    check(tree, make(B, 5, 4, 2, 128, lens, 16, ragged=True))
    lens[-1] = 3000
    check(tree, make(B, 0, 2, 2, 64, lens, 16, "f16", kind="none"))


def test_an_empty_batch(tree):
    i = make(1, 2, 4, 2, 64, 5, 16)
    e = {k: (v[:0] if k in ("q", "k", "v", "table", "cache_len", "parents") else v) for k, v in i.items()}
    assert run(tree, e).shape == (0, 3, 4, 64)


def test_no_cache_at_all(tree):
    i = make(2, 9, 4, 2, 64, 0, 16)
    i["k_cache"], i["v_cache"], i["table"] = i["k_cache"][:0], i["v_cache"][:0], i["table"][:, :0]
    check(tree, i)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scores_of_any_size(tree, dtype):
    i = make(2, 10, 8, 2, 128, [400, 77], 16, dtype)
    for scale in (0.0, -0.3, 1e-8, 3.0, 40.0):
        check(tree, i, scale=scale)
    i["q"] = (i["q"].float() * 30).to(i["q"].dtype)  # one key takes all, the maximum moves often
    check(tree, i, scale=1.0)
    i["q"].zero_()
    i["v"], i["v_cache"] = i["v"] * 0 + 3, i["v_cache"] * 0 + 3  # all weights alike
    assert torch.equal(run(tree, i), torch.full_like(i["q"], 3))


@pytest.mark.parametrize("scale,q,k", [(0.0, 1e15, 1e13), (1e-36, 1e18, 1e17), (-2e-38, 1e18, 3e18), (1e30, 1e-15, 1e-15), (-3.4e38, 0.0, 1.0), (3.4e38, 0.0, 1.0)])
def test_scales_at_the_ends_of_their_type(tree, scale, q, k):
    i = make(2, 10, 8, 2, 128, [400, 77], 16)
    i["q"], i["k"], i["k_cache"] = (i["q"].float() * q).to(torch.bfloat16), (i["k"].float() * k).to(torch.bfloat16), (i["k_cache"].float() * k).to(torch.bfloat16)
    check(tree, i, scale=scale)


def test_rising_and_falling_scores(tree):
    for sign in (1, -1):
        i = make(1, 3, 4, 1, 64, 3000, 16, "bf16")
        t = torch.arange(3000, device="cuda")
        at = (i["table"][0, t // 16].long(), t % 16)
        i["k_cache"][at] = (sign * (t[:, None, None] - 1500.0) / 40 * torch.ones(1, 64, device="cuda")).to(torch.bfloat16)
        i["q"] = i["q"].abs()
        check(tree, i)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_may_hold_anything(tree, bad):
    """Nodes that are no ancestors: their keys and values, one element or all."""
    for N, kind, Hq in ((12, "star", 4), (40, "random", 2), (70, "wide", 16)):
        i = make(2, N, Hq, 2, 128, [60, 0], 16, kind=kind, seed=3)
        want, bound = R.attention(*(i[k] for k in ("q", "k", "v", "k_cache", "v_cache", "table", "cache_len", "parents", "tree_len")), 1 / math.sqrt(128))
        for whole in (True, False):
            j = {k: (t.clone() if torch.is_tensor(t) else t) for k, t in i.items()}
            spoiled = [3, 7, N - 1]
            for n in spoiled:
                j["k"][:, n + 1, 0, :None if whole else 1] = bad
                j["v"][:, n + 1, 0, 5:None if whole else 6] = bad
                j["v"][:, n + 1, 1, -1:] = bad
            got = run(tree, j)
            for b in range(2):
                seen = R.sees(i["parents"][b].tolist(), N)
                clean = ~seen[:, [n + 1 for n in spoiled]].any(1)
                assert clean.sum() > 1
                close(got[b, clean.cuda()], want[b, clean.cuda()], bound[b, clean.cuda()], "rows that see none of them")


def test_strides(tree):
    B, N, Hq, H, D = 2, 5, 8, 2, 64
    i = make(B, N, Hq, H, D, [100, 37], 16)
    want = run(tree, i)
    fused = torch.full((B, N + 1, Hq + 2 * H + 1, D), math.nan, dtype=torch.bfloat16, device="cuda")
    fused[:, :, :Hq], fused[:, :, Hq:Hq + H], fused[:, :, Hq + H:Hq + 2 * H] = i["q"], i["k"], i["v"]
    j = dict(i, q=fused[:, :, :Hq], k=fused[:, :, Hq:Hq + H], v=fused[:, :, Hq + H:Hq + 2 * H])
    assert torch.equal(run(tree, j), want)
    both = torch.stack([i["k_cache"], i["v_cache"]], 1)  # [pages, 2, slots, heads, dim]
    assert torch.equal(run(tree, dict(i, k_cache=both[:, 0], v_cache=both[:, 1])), want)
    hnd = [i[k].transpose(1, 2).contiguous().transpose(1, 2) for k in ("k_cache", "v_cache")]  # pages of [heads, slots, dim]
    assert torch.equal(run(tree, dict(i, k_cache=hnd[0], v_cache=hnd[1])), want)
    wide = torch.full((B, i["table"].shape[1] + 5), -7, dtype=torch.int32, device="cuda")
    wide[:, :-5] = i["table"]
    assert torch.equal(run(tree, dict(i, table=wide[:, :-5])), want)
    assert torch.equal(run(tree, dict(i, table=i["table"].long(), cache_len=i["cache_len"].long(), parents=i["parents"].to(torch.int16))), want)
    around = torch.full((B, N + 2, Hq, D + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    out = around[:, :N + 1, :, :D]
    assert run(tree, i, out=out) is out and torch.equal(out, want)
    assert torch.all(around[:, N + 1] == 5) and torch.all(around[..., D:] == 5)
    turned = torch.empty(N + 1, B, Hq, D, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    assert torch.equal(run(tree, i, out=turned), want)


def test_refusals(tree):
    i = make(2, 5, 8, 2, 64, [100, 37], 16)
    ok = lambda **k: run(tree, dict(i, **k))
    with pytest.raises(ValueError, match="16 bytes"):
        big = torch.empty(2 * 6 * 8 * 64 + 1, dtype=torch.bfloat16, device="cuda")
        ok(q=big[1:].view(2, 6, 8, 64))
    with pytest.raises(ValueError, match="contiguous"):
        ok(q=torch.empty(2, 6, 64, 8, dtype=torch.bfloat16, device="cuda").transpose(2, 3))
    with pytest.raises(ValueError, match="expanded"):
        ok(k_cache=i["k_cache"][:1].expand_as(i["k_cache"]), v_cache=i["v_cache"][:1].expand_as(i["v_cache"]))
    with pytest.raises(ValueError, match="share strides"):
        ok(v_cache=torch.stack([i["v_cache"]] * 2, 1)[:, 0])
    with pytest.raises(ValueError, match="dtype"):
        ok(q=i["q"].half())
    with pytest.raises(ValueError, match="q must be"):
        ok(q=i["q"][:, :, :7])
    with pytest.raises(ValueError, match="cache_len"):
        ok(cache_len=i["cache_len"][:1])
    with pytest.raises(TypeError, match="integers"):
        ok(cache_len=i["cache_len"].float())
    with pytest.raises(ValueError, match="share memory"):
        run(tree, i, out=i["q"])
    with pytest.raises(ValueError, match="64 or 128"):
        d = make(1, 1, 2, 1, 96, 3, 16)
        run(tree, d)
    with pytest.raises(ValueError, match="workspace"):
        run(tree, i, workspace=torch.empty(100, 2, dtype=torch.uint8, device="cuda")[:, 0])
    from paper_2603_16219_amd.binding import SpecSteerError

    with pytest.raises(SpecSteerError, match="workspace"):
        run(tree, i, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("what", ["cache_len", "negative_len", "tree_len", "negative_tree", "parent", "self_parent", "low_parent", "page", "negative_page", "late_page"])
def test_bad_data_marks_its_sequence_alone(tree, what):
    for N, Hq, L in ((6, 4, 300), (50, 8, 1500)):
        i = make(3, N, Hq, 2, 128, [L, L - 50, L], 16, ragged=True, seed=9)
        i["tree_len"][1] = N
        want, bound = R.attention(*(i[k] for k in ("q", "k", "v", "k_cache", "v_cache", "table", "cache_len", "parents", "tree_len")), 1 / math.sqrt(128))
        width = i["table"].shape[1]
        at, v = {"cache_len": ("cache_len", width * 16 + 1), "negative_len": ("cache_len", -1), "tree_len": ("tree_len", N + 1), "negative_tree": ("tree_len", -3),
                 "parent": ("parents", N - 1), "self_parent": ("parents", 2), "low_parent": ("parents", -2), "page": ("table", i["k_cache"].shape[0]),
                 "negative_page": ("table", -1), "late_page": ("table", 1 << 30)}[what]
        if at in ("cache_len", "tree_len"):
            i[at][1] = v
        else:
            i[at][1, {"parent": N - 2, "late_page": (L - 51) // 16}.get(what, 2)] = v
        got = run(tree, i)
        assert got[1].isnan().all()
        close(got[::2], want[::2], bound[::2], "the others")  # lengths say where all sequences' sums are cut


@pytest.mark.parametrize("B,Hq,H", [(1, 32, 32), (7, 16, 8), (300, 4, 4)])
def test_a_bad_page_marks_every_head(tree, B, Hq, H):
    """Waves over their own keys, chains, heads whose pages are looked up once: the sequence's rows are NaN for each, and no other's are."""
    i = make(B, 0, Hq, H, 64, [900 + 7 * b % 100 for b in range(B)], 64, kind="none")
    want = run(tree, i)
    assert not want.isnan().any()
    for b in sorted({0, B // 2, B - 1}):
        for at in (0, 3, 14):
            table = i["table"].clone()
            table[b, at] = i["k_cache"].shape[0]
            got = run(tree, dict(i, table=table))
            assert got[b].isnan().all()
            others = torch.arange(B, device="cuda") != b
            assert torch.equal(got[others], want[others])


def test_pages_and_parents_that_are_not_needed_may_be_anything(tree):
    i = make(2, 8, 4, 2, 64, [33, 16], 16, ragged=True)
    want = run(tree, i)
    for b in range(2):
        i["table"][b, -(-int(i["cache_len"][b]) // 16):] = -5
        i["parents"][b, int(i["tree_len"][b]):] = 1 << 20
    assert torch.equal(run(tree, i), want)


def test_shared_pages_and_the_same_page_twice(tree):
    i = make(3, 4, 4, 2, 64, [64, 64, 64], 16, spare=20)
    i["table"][1, :2] = i["table"][0, :2]  # a common prompt
    i["table"][2, 1] = i["table"][2, 0]
    i["k_cache"], i["v_cache"] = i["k_cache"].nan_to_num(0.5), i["v_cache"].nan_to_num(0.5)
    check(tree, i)


def test_the_same_call_gives_the_same_bits(tree):
    i = make(5, 9, 16, 4, 128, [3000, 10, 0, 777, 1600], 16, ragged=True)
    need = 1 << 28
    for fill in (0, 255):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        got = run(tree, i, workspace=ws)
        assert torch.equal(got, run(tree, i))


def test_offsets_past_32_bits(tree):
    pages, page, H, D = 1 << 17, 16, 16, 128  # 2^32 elements, 8 GiB each
    kc = torch.empty(pages, page, H, D, dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    i = make(1, 3, 16, 16, 128, 200, 16)
    far = torch.randint(pages - 4000, pages, (i["table"].shape[1],), generator=gen(4), device="cuda", dtype=torch.int32)[None].contiguous()
    for j in range(i["table"].shape[1]):
        kc[far[0, j]], vc[far[0, j]] = i["k_cache"][i["table"][0, j]], i["v_cache"][i["table"][0, j]]
    i.update(k_cache=kc, v_cache=vc, table=far)
    check(tree, i)


def test_positions_up_to_the_last_of_31_bits(tree):
    """Shared pages of one position; the last 900 lie in pages of their own and weigh about a third of the row."""
    L = 2**31 - 1
    table = torch.zeros(1, L, dtype=torch.int32, device="cuda")
    table[0, -900:] = 1
    zeros = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    q, k, v, kc, vc = zeros(1, 1, 1, 64), zeros(1, 1, 1, 64), zeros(1, 1, 1, 64), zeros(5, 1, 1, 64), zeros(5, 1, 1, 64)
    q[..., 0], kc[1, ..., 0] = 1, 14
    v[:] = 3
    vc[0], vc[1] = 3, -5
    for length in (L, L - 130, L - 1000):
        last = max(0, 900 - (L - length)) * math.exp(14)
        rest = length - max(0, 900 - (L - length)) + 1
        want = (3.0 * rest - 5.0 * last) / (rest + last)
        got = tree.attention(q, k, v, kc, vc, table, torch.tensor([length], dtype=torch.int32, device="cuda"), scale=1.0).double()
        # half a step for the weights of either value and for the output
        assert (got - want).abs().max() <= 2.0 ** -8 * (3 + 5) + 2.0 ** -8 * abs(want), length
    # the last three positions; the next one has no place
    table[0, -3:] = torch.tensor([2, 3, 4], dtype=torch.int32, device="cuda")
    rows = torch.arange(4.0, device="cuda").to(torch.bfloat16)[None, :, None, None].expand(1, 4, 1, 64).contiguous() + 1
    at = lambda n: torch.tensor([n], dtype=torch.int32, device="cuda")
    assert tree.commit(rows, -rows, kc, vc, table, at(L - 3), at(3)).tolist() == [-1]
    assert torch.all(kc[2:] == 0)
    assert tree.commit(rows, -rows, kc, vc, table, at(L - 3), at(2)).tolist() == [L]
    assert kc[2:, 0, 0, 0].tolist() == [1, 2, 3] and vc[2:, 0, 0, 5].tolist() == [-1, -2, -3]
    table[0, -1] = 5
    assert tree.commit(rows, -rows, kc, vc, table, at(L - 3), at(2)).tolist() == [-1]


def test_native_and_general_path_agree(tree, monkeypatch):
    i = make(2, 5, 8, 2, 64, [100, 37], 16, ragged=True)
    v = verify_inputs(3, 9, 1000, "f32")
    kc = lambda: {k: (t.clone() if k.endswith("cache") else t) for k, t in i.items()}
    acc, path = torch.tensor([2, 5], dtype=torch.int32, device="cuda"), torch.arange(5, dtype=torch.int32, device="cuda").expand(2, 5).contiguous()

    def commit():
        j = kc()
        n = tree.commit(j["k"], j["v"], j["k_cache"], j["v_cache"], j["table"], j["cache_len"], acc, path)
        return [n, j["k_cache"].nan_to_num(9), j["v_cache"].nan_to_num(9)]

    calls = [lambda: [run(tree, i)], lambda: [run(tree, dict(i, parents=None, tree_len=None), scale=0.2, out=torch.empty_like(i["q"]))],
             lambda: list(walk(tree, v).values()), lambda: list(walk(tree, v, greedy=True, temperature=0.7).values()), commit]
    for c in calls:
        taken = []
        with monkeypatch.context() as m:
            m.setattr(tree, "_native", lambda *a, f=tree._native: taken.append(f(*a)) or taken[-1])
            native = c()
        assert taken[-1] is not None
        with monkeypatch.context() as m:
            m.setattr(tree, "_calls", None)
            general = c()
        for a, b in zip(native, general):
            assert a.dtype == b.dtype and torch.equal(a.nan_to_num(7), b.nan_to_num(7))


# ------------------------------------------------------------------ verify


def verify_inputs(B, N, V, dtype, seed=0, kind="random", ragged=False, spread=1.0):
    g, dev = gen(100 * seed + B + 13 * N + V), "cuda"
    base = torch.randn(B, N + 1, V, generator=g, device=dev) * 2 * spread
    t = [(base + 0.4 * spread * torch.randn(B, N + 1, V, generator=g, device=dev)).to(DTYPES[dtype]) for _ in range(3)]
    parents = None if kind == "none" else R.random_trees(B, N, g, dev, kind)
    return {"G": t[0], "Sp": t[1], "Sm": t[2], "tokens": torch.randint(0, V, (B, N), generator=g, device=dev, dtype=torch.int32),
            "uniforms": torch.rand(B, N + 1, generator=g, device=dev), "parents": parents,
            "tree_len": torch.randint(0, N + 1, (B,), generator=g, device=dev, dtype=torch.int32) if ragged else None}


def walk(tree, i, **more):
    return tree.verify(i["G"], i["Sp"], i["Sm"], i["tokens"], i["uniforms"], i["parents"], tree_len=i["tree_len"], **more)


def check_walk(tree, i, lam=0.5, beta=1.0, temperature=1.0, greedy=False):
    got = walk(tree, i, lam=lam, beta=beta, temperature=temperature, greedy=greedy)
    want = R.verify(*(i[k] for k in ("G", "Sp", "Sm", "tokens", "uniforms", "parents", "tree_len")), lam=lam, beta=beta, temperature=temperature, greedy=greedy)
    sure = torch.tensor([n > 1e-6 for n in want["near"]])
    assert sure.float().mean() >= 0.9
    for k in ("accepted_len", "path") + (("next_token",) if greedy else ()):
        assert torch.equal(got[k].cpu()[sure], torch.tensor(want[k], dtype=torch.int32).view(got[k].shape)[sure]), k
    tokens, lps = got["next_token"].tolist(), got["next_token_logprob"].tolist()
    for b in sure.nonzero()[:, 0].tolist():
        lp, cdf, u = want["rows"][b]
        t = tokens[b]
        assert greedy or (cdf[t] > u - 1e-6 and (t == 0 or cdf[t - 1] <= u + 1e-6) and lp[t] > -math.inf), (b, t, want["next_token"][b])
        assert abs(lps[b] - float(lp[t])) <= 1e-5, (b, lps[b], float(lp[t]))
    return got, want


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 9, 100, 511, 513, 2049, 4097, 8200, 32000, 50257, 131073])
def test_walk_over_vocabularies(tree, V, dtype):
    check_walk(tree, verify_inputs(3, 6, V, dtype), beta=0.8, temperature=0.7)
    check_walk(tree, verify_inputs(2, 5, V, dtype, seed=1, kind="wide"), greedy=True)


@pytest.mark.parametrize("kind", ["none", "chain", "random", "wide", "star"])
@pytest.mark.parametrize("N", [0, 1, 2, 15, 64, 65, 200])
def test_walk_down_trees(tree, N, kind):
    for seed, lam in ((0, 0.01), (1, 0.5), (2, 1.5)):
        check_walk(tree, verify_inputs(4, N, 700, "f32", seed, kind, ragged=seed == 1), lam=lam)


def test_walk_down_deep_and_large_trees(tree):
    for N, kind in ((1024, "chain"), (1024, "none"), (1000, "random"), (700, "star")):
        i = verify_inputs(2, N, 40, "f32", 1, kind)
        i["uniforms"][:, :-1] *= 0.02
        got, _ = check_walk(tree, i, lam=0.3)
        if kind in ("chain", "none"):
            assert int(got["accepted_len"].max()) > 50


@pytest.mark.parametrize("B", [1, 5, 64, 300, 1500])
def test_walk_of_batches(tree, B):
    check_walk(tree, verify_inputs(B, 8, 3001, "bf16", B, ragged=True), lam=0.2, beta=0.5, temperature=0.8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,V", [(1, 2, 32000), (1, 1, 128256), (1, 7, 151936), (2, 20, 262147), (1, 3, 1 << 20)])
def test_walk_counts_all_of_a_long_row(tree, B, N, V, dtype):
    """Each model's mass lies in another part of the row; all of a few rows are shared by many workgroups."""
    for seed in range(3):
        i = verify_inputs(B, N, V, dtype, seed, "random")
        i["G"][..., V - V // 8:] += 4
        i["Sm"][..., :V // 8] += 4
        i["tokens"][:] = torch.randint(0, V // 8, i["tokens"].shape, generator=gen(seed), device="cuda") + V // 2
        i["uniforms"][:, :-1] *= 0.9
        check_walk(tree, i, lam=0.7, beta=0.5)


def test_walk_with_peaked_rows(tree):
    """Rows as models have them: few likely tokens, which the drafts are; long paths."""
    for B, N, V, kind in ((16, 31, 32000, "random"), (3, 12, 128256, "wide"), (40, 16, 20000, "chain")):
        i = verify_inputs(B, N, V, "bf16", 5, kind)
        up = i["parents"].long()
        at = torch.arange(B, device="cuda")[:, None]
        for t in ("G", "Sp", "Sm"):
            i[t][at, up + 1, i["tokens"].long()] = (9 + torch.rand(B, N, generator=gen(3), device="cuda") + 0.5 * torch.randn(B, N, generator=gen(ord(t[-1])), device="cuda")).to(torch.bfloat16)
        got, want = check_walk(tree, i)
        assert sum(want["accepted_len"]) > B


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("greedy", [False, True])
def test_a_chain_is_the_block(tree, dtype, greedy):
    from paper_2603_16219_amd import binding

    for B, K, V in ((1, 4, 32000), (9, 16, 5003), (70, 8, 20000), (4, 0, 1000)):
        i = verify_inputs(B, K, V, dtype, 4, "none", ragged=K > 0)
        want = binding.verify_block(i["G"], i["Sp"], i["Sm"], i["tokens"], i["uniforms"], lam=0.3, beta=0.7, temperature=0.9, draft_len=i["tree_len"], greedy=greedy)
        for parents in (None, R.chain(B, K, "cuda")):
            got = walk(tree, dict(i, parents=parents), lam=0.3, beta=0.7, temperature=0.9, greedy=greedy)
            assert torch.equal(got["accepted_len"], want["accepted_len"]) and torch.equal(got["next_token"], want["next_token"])
            torch.testing.assert_close(got["next_token_logprob"], want["next_token_logprob"], rtol=0, atol=1e-5)
            n = torch.arange(K, device="cuda")
            assert torch.equal(got["path"], torch.where(n < want["accepted_len"][:, None], n, -1).to(torch.int32))


def test_walk_with_masked_tokens(tree):
    for V in (1000, 50257):
        i = verify_inputs(6, 9, V, "f32", 2)
        dead = torch.rand(V, generator=gen(1), device="cuda") < 0.3
        dead[:20] = False
        for t in ("G", "Sp", "Sm"):
            i[t][:, :, dead] = -math.inf
        i["tokens"] %= 20
        i["tokens"][0] = int(dead.nonzero()[0])
        i["uniforms"][0] = 0.0  # a masked token is not accepted by the least uniform either
        for greedy in (False, True):
            got, _ = check_walk(tree, i, beta=0.6, greedy=greedy)
            assert got["accepted_len"][0] == 0 and not dead[got["next_token"].long()].any()
        i["G"][1, :, 25:] = -math.inf
        check_walk(tree, i)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_walk_without_steering_reads_no_specialist_with_context(tree, dtype):
    i = verify_inputs(5, 7, 3000, dtype, 8)
    i["Sp"].fill_(math.nan)
    check_walk(tree, i, beta=0.0)


def test_uniforms_at_the_ends(tree):
    i = verify_inputs(4, 6, 513, "f32")
    last = 1.0 - 2.0 ** -24
    for u in (0.0, last):
        i["uniforms"][:, :-1] = 0.3
        i["uniforms"][:, -1] = u
        got = walk(tree, i)
        assert torch.all((got["next_token"] >= 0) & (got["next_token"] < 513))
        if u == 0.0:
            assert torch.all(got["next_token"] == 0)
    i["uniforms"][:, -1] = 1.0  # out of range: the last token with any probability
    i["G"][:, :, 500:] = -math.inf
    assert torch.all(walk(tree, i)["next_token"] == 499)


@pytest.mark.parametrize("what", ["len", "negative_len", "parent", "self_parent", "low_parent", "token", "negative_token"])
def test_bad_data_marks_its_walk_alone(tree, what):
    for B, N, V in ((3, 10, 3000), (200, 10, 700)):
        i = verify_inputs(B, N, V, "bf16", 6, ragged=True)
        i["tree_len"][1] = N
        want = walk(tree, i)
        at, v = {"len": ("tree_len", N + 1), "negative_len": ("tree_len", -1), "parent": ("parents", N - 1), "self_parent": ("parents", N - 2), "low_parent": ("parents", -2),
                 "token": ("tokens", V), "negative_token": ("tokens", -1)}[what]
        if at == "tree_len":
            i[at][1] = v
        else:
            i[at][1, N - 2] = v
        got = walk(tree, i)
        assert got["accepted_len"][1] == -1 and got["next_token"][1] == -1 and torch.all(got["path"][1] == -1) and got["next_token_logprob"][1].isnan()
        rest = [b for b in range(B) if b != 1]
        for k in want:
            assert torch.equal(got[k][rest], want[k][rest]), k


def test_walk_ignores_what_belongs_to_nobody(tree):
    for B in (3, 150):
        i = verify_inputs(B, 9, 2500, "bf16", 3, ragged=True)
        want = walk(tree, i)
        for b in range(B):
            n = int(i["tree_len"][b])
            i["tokens"][b, n:], i["parents"][b, n:] = -9, 1 << 29
            i["uniforms"][b, n:-1] = math.nan
            for t in ("G", "Sp", "Sm"):
                i[t][b, n + 1:] = math.nan
        got = walk(tree, i)
        assert all(torch.equal(got[k], want[k]) for k in want)


def test_walk_over_strided_logits(tree):
    for dtype in ("bf16", "f32"):
        i = verify_inputs(3, 6, 1001, dtype, 1)
        want = walk(tree, i)
        j = dict(i)
        for t in ("G", "Sp", "Sm"):
            big = torch.full((3, 9, 1010), math.nan, dtype=i[t].dtype, device="cuda")
            big[:, 1:8, 3:1004] = i[t]
            j[t] = big[:, 1:8, 3:1004]
        got = walk(tree, j)
        for k in ("accepted_len", "path", "next_token"):
            assert torch.equal(got[k], want[k]), k
        torch.testing.assert_close(got["next_token_logprob"], want["next_token_logprob"], rtol=0, atol=2e-6)


def test_walk_offsets_past_32_bits(tree):
    B, N, V = 3, 1023, 1 << 20
    G = torch.zeros(B, N + 1, V, dtype=torch.bfloat16, device="cuda")
    few = [0, 5, 1023]
    i = {"G": G, "Sp": G, "Sm": G, "tokens": torch.zeros(B, N, dtype=torch.int32, device="cuda"), "uniforms": torch.rand(B, N + 1, generator=gen(2), device="cuda"),
         "parents": torch.full((B, N), -1, dtype=torch.int32, device="cuda"), "tree_len": None}
    i["uniforms"][:, :-1] = 1.0  # refused
    for b in range(B):
        i["uniforms"][b, 1022] = 0.0
        for r in few:
            G[b, r] = torch.randn(V, generator=gen(10 * b + r), device="cuda") * 4
    got = walk(tree, i, lam=1.5)
    assert got["path"][:, 0].tolist() == [1022] * B and got["accepted_len"].tolist() == [1] * B
    for b in range(B):
        lp = torch.log_softmax(G[b, 1023].double(), 0)
        cdf = lp.exp().cumsum(0)
        u = i["uniforms"][b, -1].double()
        t = int(got["next_token"][b])
        assert (cdf[t] > u - 1e-6) and (t == 0 or cdf[t - 1] <= u + 1e-6) and abs(got["next_token_logprob"][b].double() - lp[t]) < 1e-5


# ------------------------------------------------------------------ commit


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,H,page", [(128, 8, 16), (64, 1, 1), (8, 3, 5), (72, 2, 24), (1024, 2, 16)])
def test_commit(tree, D, H, page, dtype):
    for B, N in ((1, 0), (3, 5), (20, 40)):
        i = make(B, N, H, H, D, [7 * b % 60 for b in range(B)], page, dtype)
        g = gen(5)
        acc = torch.randint(0, N + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        path = torch.full((B, N), -1, dtype=torch.int32, device="cuda")
        for b in range(B):
            n = int(acc[b])
            path[b, :n] = torch.randperm(N, generator=g, device="cuda")[:n].sort().values.to(torch.int32)
        for p in (path, None):
            want = R.commit(i["k"], i["v"], i["k_cache"], i["v_cache"], i["table"], i["cache_len"], acc, p)
            kc, vc = i["k_cache"].clone(), i["v_cache"].clone()
            versions = kc._version, vc._version
            new = tree.commit(i["k"], i["v"], kc, vc, i["table"], i["cache_len"], acc, p)
            assert torch.equal(new, want[2]) and torch.equal(kc.nan_to_num(9), want[0].nan_to_num(9)) and torch.equal(vc.nan_to_num(9), want[1].nan_to_num(9))
            assert kc._version > versions[0] and vc._version > versions[1]


@pytest.mark.parametrize("what", ["accepted", "negative_accepted", "cache_len", "negative_len", "room", "path", "negative_path", "page", "negative_page"])
def test_commit_writes_nothing_of_a_bad_path(tree, what):
    N = 20
    i = make(3, N, 2, 2, 64, [30, 30, 30], 16)
    acc, path = torch.tensor([4, 17, 20], dtype=torch.int32, device="cuda"), torch.arange(N, dtype=torch.int32, device="cuda").expand(3, N).contiguous()
    want = R.commit(i["k"], i["v"], i["k_cache"], i["v_cache"], i["table"], i["cache_len"], acc, path)
    room, mine = i["table"].shape[1] * 16, i["table"][1].long()
    at, v = {"accepted": (acc, N + 1), "negative_accepted": (acc, -1), "cache_len": (i["cache_len"], room + 1), "negative_len": (i["cache_len"], -1),
             "room": (i["cache_len"], room - 17), "path": (path, N), "negative_path": (path, -1), "page": (i["table"], i["k_cache"].shape[0]),
             "negative_page": (i["table"], -1)}[what]
    if at.dim() == 1:
        at[1] = v
    else:
        at[1, 15 if at is path else (30 + 17) // 16] = v
    kc, vc = i["k_cache"].clone(), i["v_cache"].clone()
    new = tree.commit(i["k"], i["v"], kc, vc, i["table"], i["cache_len"], acc, path)
    assert new.tolist() == [want[2][0], -1, want[2][2]]
    keep = torch.ones(kc.shape[0], dtype=torch.bool, device="cuda")
    keep[mine] = False
    for a, b, before in ((kc, want[0], i["k_cache"]), (vc, want[1], i["v_cache"])):
        assert torch.equal(a[keep].nan_to_num(9), b[keep].nan_to_num(9)) and torch.equal(a[~keep].nan_to_num(9), before[~keep].nan_to_num(9))


def test_commit_to_strided_caches_and_other_integers(tree):
    i = make(2, 6, 3, 3, 64, [10, 33], 16)
    acc, path = torch.tensor([3, 6], dtype=torch.int32, device="cuda"), torch.arange(6, dtype=torch.int32, device="cuda").expand(2, 6).contiguous()
    want = R.commit(i["k"], i["v"], i["k_cache"], i["v_cache"], i["table"], i["cache_len"], acc, path)
    both = torch.stack([i["k_cache"].transpose(1, 2), i["v_cache"].transpose(1, 2)], 1).contiguous()
    kc, vc = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
    new = tree.commit(i["k"], i["v"], kc, vc, i["table"].long(), i["cache_len"].long(), acc.long(), path.long())
    assert torch.equal(new, want[2]) and torch.equal(kc.nan_to_num(9), want[0].nan_to_num(9)) and torch.equal(vc.nan_to_num(9), want[1].nan_to_num(9))
    with pytest.raises(ValueError, match="share memory"):
        tree.commit(kc[:2, :7], vc[:2, :7], kc, vc, i["table"], i["cache_len"], acc, path)


# ------------------------------------------------------------------ together


def test_replays_and_other_streams(tree):
    i, v = make(3, 9, 8, 2, 128, [700, 64, 0], 16, ragged=True), verify_inputs(3, 9, 20000, "bf16", 7, ragged=True)
    kc, vc = i["k_cache"].nan_to_num(0.5), i["v_cache"].nan_to_num(0.5)

    def step():
        k2, v2 = kc.clone(), vc.clone()
        out = run(tree, dict(i, k_cache=k2, v_cache=v2))
        w = walk(tree, v)
        new = tree.commit(i["k"], i["v"], k2, v2, i["table"], i["cache_len"], w["accepted_len"], w["path"])
        return [out, new, k2, v2, *w.values()]

    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = step()
    for r in range(4):
        i["q"].copy_(torch.randn(i["q"].shape, generator=gen(r), device="cuda"))
        v["uniforms"].copy_(torch.rand(v["uniforms"].shape, generator=gen(r), device="cuda"))
        i["cache_len"].copy_(torch.tensor([700 - r, 64, r], device="cuda"))
        i["v"].copy_(torch.randn(i["v"].shape, generator=gen(9 + r), device="cuda"))
        i["k"].nan_to_num_(0.1)
        i["q"].nan_to_num_(0.1)
        i["v"].nan_to_num_(0.1)
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a.nan_to_num(7), b.nan_to_num(7)), r
    with torch.cuda.stream(side):
        again = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a.nan_to_num(7), b.nan_to_num(7)) for a, b in zip(again, want))


def test_calls_from_two_streams_at_once(tree):
    a, b = make(4, 9, 8, 2, 128, [900, 64, 0, 333], 16), make(2, 20, 8, 4, 64, [1500, 64], 16, "f16")
    va, vb = verify_inputs(4, 9, 30000, "bf16", 1), verify_inputs(2, 15, 50257, "f32", 2)
    want = [run(tree, a), run(tree, b), *walk(tree, va).values(), *walk(tree, vb).values()]
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        with torch.cuda.stream(s):
            x = [run(tree, a), *walk(tree, va).values()]
        with torch.cuda.stream(t):
            y = [run(tree, b), *walk(tree, vb).values()]
        torch.cuda.synchronize()
        for p, q in zip([x[0], y[0], *x[1:], *y[1:]], want):
            assert torch.equal(p, q)


def test_calls_from_several_threads(tree):
    """Each thread with a stream of its own, all at once, from Python threads that switch inside of the calls."""
    import threading

    from paper_2603_16219_amd import losses

    made = [(make(3, 4 + 9 * n, 8, 2, 64 if n % 2 else 128, [300 * n, 64, 5], 16, seed=n), verify_inputs(3, 9 + n, 9000 + n, "bf16", n)) for n in range(4)]
    torch.cuda.synchronize()

    def block(i, v):
        kc, vc = i["k_cache"].clone(), i["v_cache"].clone()
        w = walk(tree, v)
        some = dict(accepted_len=w["accepted_len"].clamp(max=i["k"].shape[1] - 1))
        new = tree.commit(i["k"], i["v"], kc, vc, i["table"], i["cache_len"] // 2, some["accepted_len"])
        top = losses.token_alternatives(v["G"], topk=5)
        return [run(tree, i), new, kc, vc, *w.values(), top["top_tokens"], top["top_logprobs"], top["entropy"]]

    want = [block(*m) for m in made]
    torch.cuda.synchronize()
    wrong = []

    def work(n):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(15):
                    got = block(*made[n])
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(a.nan_to_num(7), b.nan_to_num(7)) for a, b in zip(got, want[n])):
                        wrong.append(n)
        except Exception as e:  # what ends a thread would be lost
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(n,)) for n in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong


def test_a_block_of_a_small_model(tree):
    """From the specialist's alternatives to the cache of the next block: a tree grown, scored through an attention layer, walked, kept; the cached
    sequence then gives what a single pass over it gives."""
    from paper_2603_16219_amd import losses

    g, dev, B, N, V, Hq, H, D, page = gen(77), "cuda", 4, 9, 997, 4, 2, 64, 16
    normal = lambda *s: torch.randn(*s, generator=g, device=dev)
    emb, head = normal(V, 128), normal(3, Hq * D, V) / 12
    wq, wk, wv = normal(128, Hq * D) / 11, normal(128, H * D) / 11, normal(128, H * D) / 11
    bf = torch.bfloat16
    pages = 40
    kc, vc = torch.zeros(pages, page, H, D, dtype=bf, device=dev), torch.zeros(pages, page, H, D, dtype=bf, device=dev)
    table = torch.randperm(pages, generator=g, device=dev).to(torch.int32)[:B * 8].view(B, 8).contiguous()
    length = torch.zeros(B, dtype=torch.int32, device=dev)
    text = [[int(t)] for t in torch.randint(0, V, (B,), generator=g, device=dev)]
    parents = (torch.arange(N, device=dev) // 3 - 1).to(torch.int32).expand(B, N).contiguous()

    rows_of = [(emb @ w).view(V, n, D).to(bf) for w, n in ((wq, Hq), (wk, H), (wv, H))]  # of every token, rounded once

    def project(ids):
        return [t[ids.long()] for t in rows_of]

    def logits(out):
        h = out.float().flatten(-2)
        return [(h @ head[m]).contiguous() for m in range(3)]

    for block in range(6):
        last = torch.tensor([[t[-1]] for t in text], dtype=torch.int32, device=dev)
        # the tree's levels: three alternatives of the root's row, then three of each of those that fit
        ids = torch.zeros(B, N, dtype=torch.int32, device=dev)
        for lo in range(0, N, 3):
            rows = torch.cat([last, ids], 1)
            q, k, v = project(rows)
            sp = logits(tree.attention(q, k, v, kc, vc, table, length, parents))[1]
            top = losses.token_alternatives(sp, topk=3)["top_tokens"]
            ids[:, lo:lo + 3] = top[:, lo // 3]
        rows = torch.cat([last, ids], 1)
        q, k, v = project(rows)
        G, Sp, Sm = logits(tree.attention(q, k, v, kc, vc, table, length, parents))
        u = torch.rand(B, N + 1, generator=g, device=dev)
        step = tree.verify(G, Sp, Sm, ids, u, parents, lam=0.2, beta=0.5)
        want = R.verify(G, Sp, Sm, ids, u, parents, None, lam=0.2, beta=0.5, temperature=1.0)
        assert step["path"].tolist() == want["path"] and step["next_token"].tolist() == want["next_token"]
        length = tree.commit(k, v, kc, vc, table, length, step["accepted_len"], step["path"])
        for b in range(B):
            text[b] += [int(ids[b, i]) for i in want["path"][b] if i >= 0] + [want["next_token"][b]]
        assert length.tolist() == [len(t) - 1 for t in text]
    # one more token for each sequence, over the cache; and the whole text as one chain over an empty one
    last = torch.tensor([[t[-1]] for t in text], dtype=torch.int32, device=dev)
    q, k, v = project(last)
    one = tree.attention(q, k, v, kc, vc, table, length)
    for b in range(B):
        q, k, v = project(torch.tensor([text[b]], dtype=torch.int32, device=dev))
        whole, bound = R.attention(q, k, v, kc[:0], vc[:0], table[:1, :0], length[:1] * 0, None, None, 1 / 8)
        close(one[b, 0], whole[0, -1], bound[0, -1], "the last token")
        close(tree.attention(q, k, v, kc[:0], vc[:0], table[:1, :0], length[:1] * 0), whole, bound, "the chain")
