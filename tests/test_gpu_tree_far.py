"""GPU tests of the walk down a tree where exponents h / T are large or far apart: low and high temperatures, rows far from zero, steering terms that
cancel, the type's lowest value.  Against the definitions in 64 bits, from differences of logits, which are exact there.

u = 2^-24, z a term's distance to the row's largest in powers of two.  A term formed in double is off by 1.4 z u (its exponent as one fp32 number) and 2 u; one
formed in fp32 by up to 3 u ln 2 times its steering term in powers of two, whose mean is at most 16 there.  Cumulated probabilities are off by
(2.1 E[z] + 2 + 34) u, 2.8e-6 for E[z] = 5, a log-prob by as much and half a step of its own."""
import math

import pytest
import torch

import tree_reference as R
from test_gpu_losses import gen
from test_gpu_tree import DTYPES, tree, verify_inputs, walk  # noqa: F401

pytestmark = pytest.mark.gpu
TOL = 4e-6


def reference(i, lam, beta, temperature, greedy):
    """As tree_reference.verify, by differences: {accepted_len, path, next_token, near, rows}."""
    f32 = lambda x: torch.tensor(x, dtype=torch.float32).item()
    lam, beta, tau = f32(lam), f32(beta), f32(temperature)
    B, N1, V = i["G"].shape
    up = R.chain(B, N1 - 1).tolist() if i["parents"] is None else i["parents"].tolist()
    ns = [N1 - 1] * B if i["tree_len"] is None else i["tree_len"].tolist()
    res = {"accepted_len": [], "path": [], "next_token": [], "near": [], "rows": []}
    for b in range(B):
        cur, path, near = -1, [], 1.0
        while True:
            kids = R.children(up[b], ns[b], cur)
            if not kids:
                break
            y = i["tokens"][b, kids].long()
            g, s = (i[t][b, cur + 1].double() for t in ("G", "Sm"))
            log_sum = lambda x: torch.logsumexp((x - x.max()) / tau, 0)
            ratio = ((g[y] - s[y]) - (g.max() - s.max())) / tau - (log_sum(g) - log_sum(s))
            alpha = torch.where(g[y] == -math.inf, -1.0, torch.exp(ratio) / lam).clamp(max=1.0).tolist()
            taken = None
            for k, a in zip(kids, alpha):
                u = i["uniforms"][b, k].double().item()
                if a < 1.0:
                    near = min(near, abs(u - a) / max(a, 1e-6))
                if u <= a:
                    taken = k
                    break
            if taken is None:
                break
            cur = taken
            path.append(cur)
        g, sp, sm = (i[t][b, cur + 1].double() for t in ("G", "Sp", "Sm"))
        h = g if beta == 0 else g + beta * torch.where(sp == sm, 0.0, sp - sm)
        z = (h - h.max()) / tau
        lp = z - torch.logsumexp(z, 0)
        cdf = lp.exp().cumsum(0)
        u = i["uniforms"][b, N1 - 1].double() * cdf[-1]
        res["accepted_len"].append(len(path))
        res["path"].append(path + [-1] * (N1 - 1 - len(path)))
        res["next_token"].append(int((h == h.max()).nonzero()[0]) if greedy else int((cdf <= u).sum().clamp(max=V - 1)))
        res["near"].append(near)
        res["rows"].append((lp, cdf, u))
    return res


def check(tree, i, lam=0.5, beta=0.5, temperature=1.0, greedy=False):
    got = walk(tree, i, lam=lam, beta=beta, temperature=temperature, greedy=greedy)
    want = reference(i, lam, beta, temperature, greedy)
    sure = torch.tensor([n > 1e-6 for n in want["near"]])
    assert sure.float().mean() >= 0.7
    for k in ("accepted_len", "path") + (("next_token",) if greedy else ()):
        assert torch.equal(got[k].cpu()[sure], torch.tensor(want[k], dtype=torch.int32).view(got[k].shape)[sure]), k
    tokens, lps = got["next_token"].tolist(), got["next_token_logprob"].tolist()
    for b in sure.nonzero()[:, 0].tolist():
        lp, cdf, u = want["rows"][b]
        t = tokens[b]
        assert greedy or (cdf[t] > u - TOL and (t == 0 or cdf[t - 1] <= u + TOL) and lp[t].exp() > 0), (b, t, want["next_token"][b])
        assert abs(lps[b] - float(lp[t])) <= TOL + abs(float(lp[t])) * 2.0 ** -24, (b, t, lps[b], float(lp[t]))
    return want


def likely_drafts(i, g, share=0.7):
    """Most drafts are what the specialist and the cloud like best at their row."""
    B, N = i["tokens"].shape
    up = i["parents"].long() if i["parents"] is not None else torch.arange(-1, N - 1, device="cuda").expand(B, N)
    rows = up + 1
    at = torch.arange(B, device="cuda")[:, None]
    for t, seed in (("G", 1), ("Sp", 2), ("Sm", 3)):
        add = (9 + torch.rand(B, N, generator=gen(seed), device="cuda")).to(i[t].dtype)
        some = torch.rand(B, N, generator=gen(7), device="cuda") < share
        i[t][at, rows, i["tokens"].long()] = torch.where(some, add, i[t][at, rows, i["tokens"].long()])
    return i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V", [(9, 3001), (100, 900), (0, 40003)])
@pytest.mark.parametrize("beta", [0.0, 0.5, -0.75])
@pytest.mark.parametrize("temperature", [3e38, 1e13, 50.0, 0.05, 0.01, 1e-3, 1e-4, 1e-6, 1e-8, 1e-10, 1e-13, 1e-30])
def test_temperatures(tree, temperature, beta, N, V, dtype):
    for seed in (0, 1):
        i = likely_drafts(verify_inputs(4, N, V, dtype, seed), gen(seed))
        for greedy in (False, True):
            check(tree, i, lam=0.7, beta=beta, temperature=temperature, greedy=greedy)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V", [(9, 3001), (100, 900), (2, 40003)])
@pytest.mark.parametrize("which", ["G", "Sm", "Sp", "G Sm", "G Sp Sm"])
@pytest.mark.parametrize("offset", [1e5, -1e5, 1e7, -3e9, 1e30])
def test_rows_far_from_zero(tree, offset, which, N, V, dtype):
    """Some rows of a tree, in some of its tensors."""
    for seed, temperature in ((0, 1.0), (1, 0.7)):
        i = likely_drafts(verify_inputs(4, N, V, dtype, seed), gen(seed))
        rows = torch.rand(4, N + 1, generator=gen(seed + 5), device="cuda") < 0.6
        rows[0, 0] = True
        for t in which.split():
            i[t] = torch.where(rows[..., None], (i[t].float() + offset).to(i[t].dtype), i[t])
        check(tree, i, temperature=temperature)
        check(tree, i, temperature=temperature, beta=1.0, greedy=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V", [(9, 3001), (100, 900), (1, 40003)])
@pytest.mark.parametrize("low", ["all", "G", "Sp", "Sm", "row"])
def test_the_type_s_lowest_value(tree, low, N, V, dtype):
    for seed in (0, 1):
        i = likely_drafts(verify_inputs(4, N, V, dtype, seed), gen(seed))
        dead = torch.rand(V, generator=gen(seed), device="cuda") < (1.5 / V if low == "Sm" else 0.3)
        if low == "Sm":
            dead[17] = True
        v = torch.finfo(i["G"].dtype).min
        if low == "row":
            i["G"][:2] = v
        else:
            for t in ("G", "Sp", "Sm") if low == "all" else (low,):
                i[t][:, :, dead] = v
        for greedy in (False, True):
            check(tree, i, greedy=greedy)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [3001, 40003])
def test_large_steering_terms_in_a_few_places(tree, V, dtype):
    """One token alone, in its own chunk of the row, has a steering term that cancels its logit; others are ordinary."""
    for seed, size in ((0, 40.0), (1, 3e3), (2, 2e5), (3, 1e9), (4, 1e12)):
        i = verify_inputs(6, 0, V, dtype, seed)
        at = torch.randint(0, V, (6,), generator=gen(seed), device="cuda")
        b = torch.arange(6, device="cuda")
        i["G"][b, 0, at] = -size
        i["Sp"][b, 0, at] = 2 * size  # in bf16 with what its 8 bits leave out of the cancelling
        i["Sm"][b, 0, at] = 0.0
        for beta in (0.5, 0.25):
            check(tree, i, beta=beta)
            check(tree, i, beta=beta, greedy=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("temperature", [0.05, 0.01, 1e-3])
def test_a_chain_is_the_block_at_low_temperatures(tree, temperature, dtype):
    from paper_2603_16219_amd import binding

    for B, K, V, beta in ((1, 4, 32000, 0.7), (9, 16, 5003, -0.7), (70, 8, 2000, 0.0), (4, 0, 1000, 1.0)):
        i = likely_drafts(verify_inputs(B, K, V, dtype, 4, "none"), gen(1), 0.9)
        a = binding.verify_block(i["G"], i["Sp"], i["Sm"], i["tokens"], i["uniforms"], lam=0.3, beta=beta, temperature=temperature)
        got = walk(tree, i, lam=0.3, beta=beta, temperature=temperature)
        assert torch.equal(got["accepted_len"], a["accepted_len"]) and torch.equal(got["next_token"], a["next_token"])
        torch.testing.assert_close(got["next_token_logprob"], a["next_token_logprob"], rtol=2.0 ** -23, atol=1e-5)
