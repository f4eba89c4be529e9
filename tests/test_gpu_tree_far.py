"""GPU tests of the walk down a tree where exponents h / T are large or far apart: low and high temperatures, rows far from zero, steering terms that
cancel, the type's lowest value.  Against the definitions in 64 bits, from differences of logits, which are exact there."""
import math

import pytest
import torch

import tree_reference as R
from test_gpu_losses import gen
from test_gpu_tree import DTYPES, tree, verify_inputs, walk  # noqa: F401

pytestmark = pytest.mark.gpu


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
    for k in ("accepted_len", "path"):
        assert torch.equal(got[k].cpu()[sure], torch.tensor(want[k], dtype=torch.int32).view(got[k].shape)[sure]), k
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
