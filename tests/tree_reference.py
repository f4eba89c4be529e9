"""Trees of drafts from their definitions in 64 bits, a sequence at a time, and how far the kernels may be off.

Attention, u = 2^-24, e half a step of the tensors' type: a score s = scale q.k is a sum of D products in fp32, off by (sqrt(D) + 8) u of the sum of
their sizes, and by 4 u of itself (the factor, its product, the subtraction of the maximum); a weight by as much of itself, by 4 u for the
exponential and by e for its rounding to the values' type, below the type's normal numbers (of fp16, with weights up to 2^10: 2^-24 of the
largest) by 2^-35; sums of n terms by (sqrt(n) + 16) u.  So with weights p_j that add up to 1

    out    sum_j p_j (|v_j| + |out|) (ds_j + (sqrt(n) + 20) u) + sum_j p_j |v_j| e + n 2^-35 max|v| + e |out|

A walk decides as in 64 bits unless a uniform lies within 1e-6 of its threshold, and draws the token whose share of the row, widened by 1e-6, holds
the uniform: with terms (3 z ln 2 + 2) u off, z their distances to the largest in powers of two, cumulated probabilities are off by (2.1 E[z] + 2) u,
8e-7 for E[z] = 5.
"""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24


def chain(B, N, device="cpu"):
    return (torch.arange(N, dtype=torch.int32, device=device) - 1).expand(B, N).contiguous()


def random_trees(B, N, g, device, kind="random"):
    i = torch.arange(N, device=device)
    if kind == "wide":
        return (i // 3 - 1).to(torch.int32).expand(B, N).contiguous()
    if kind == "star":
        return torch.full((B, N), -1, dtype=torch.int32, device=device)
    if kind == "chain":
        return chain(B, N, device)
    return ((torch.rand(B, N, generator=g, device=device) * (i + 1)).floor().clamp(max=i).to(torch.int32) - 1).contiguous()


def sees(parents, n):
    """[n + 1, n + 1]: which of the block's rows each row sees."""
    m = torch.zeros(n + 1, n + 1, dtype=torch.bool)
    m[:, 0] = True
    for i in range(n):
        m[i + 1] |= m[parents[i] + 1]
        m[i + 1, i + 1] = True
    return m


def attention(q, k, v, k_cache, v_cache, table, cache_len, parents, tree_len, scale):
    """(out, bound) in 64 bits; rows past a tree are 0."""
    B, R, Hq, D = q.shape
    H, page = k.shape[2], k_cache.shape[1]
    G, dev = Hq // H, q.device
    out = torch.zeros(q.shape, dtype=torch.float64, device=dev)
    bound = torch.zeros_like(out)
    e = torch.finfo(q.dtype).eps / 2
    up = chain(B, R - 1).tolist() if parents is None else parents.tolist()
    ns = [R - 1] * B if tree_len is None else tree_len.tolist()
    for b, L in enumerate(cache_len.tolist()):
        n = ns[b]
        at = torch.arange(L, device=dev)
        pages, slots = table[b, at // page].long(), at % page
        kk = torch.cat([k_cache[pages, slots], k[b, :n + 1]]).double().permute(1, 2, 0)  # H, D, L + n + 1
        vv = torch.cat([v_cache[pages, slots], v[b, :n + 1]]).double().permute(1, 0, 2)
        seen = torch.cat([torch.ones(n + 1, L, dtype=torch.bool), sees(up[b], n)], 1).to(dev)
        vv = vv.contiguous()
        qq = q[b, :n + 1].double().view(n + 1, H, G, D).permute(1, 2, 0, 3).reshape(H, G * (n + 1), D)
        s = (qq @ kk.contiguous()).view(H, G, n + 1, -1) * scale
        size = (qq.abs() @ kk.abs().contiguous()).view(H, G, n + 1, -1) * abs(scale)
        p = torch.softmax(s.masked_fill(~seen, -math.inf), -1)
        terms = s.shape[-1]
        top = s.masked_fill(~seen, -math.inf).amax(-1, keepdim=True)
        ds = (math.sqrt(D) + 8) * U * size + 4 * U * (s.abs() + (s - top).abs())
        w = p * (ds + (math.sqrt(terms) + 20) * U).masked_fill(~seen, 0.0)
        flat = lambda t: t.reshape(H, G * (n + 1), -1)
        o = flat(p) @ vv
        va = vv.abs().contiguous()
        err = flat(w) @ va + flat(w).sum(-1, keepdim=True) * o.abs() + flat(p) @ va * e + terms * 2.0 ** -35 * va.amax() + e * o.abs()
        back = lambda t: t.view(H, G, n + 1, D).permute(2, 0, 1, 3).reshape(n + 1, Hq, D)
        out[b, :n + 1], bound[b, :n + 1] = back(o), back(err)
    return out, bound


def children(parents, n, cur):
    return [i for i in range(n) if parents[i] == cur]


def verify(G, Sp, Sm, tokens, uniforms, parents, tree_len, *, lam, beta, temperature, greedy=False):
    """dict of accepted_len, path, next_token, of how near a decision was (the least |u - alpha| / alpha of the tests), and of the last row's
    log-probs, cumulated probabilities and scaled uniform."""
    f32 = lambda x: torch.tensor(x, dtype=torch.float32).item()
    lam, beta, tau = f32(lam), f32(beta), f32(temperature)
    B, R, V = G.shape
    up = chain(B, R - 1).tolist() if parents is None else parents.tolist()
    ns = [R - 1] * B if tree_len is None else tree_len.tolist()
    res = {"accepted_len": [], "path": [], "next_token": [], "near": [], "rows": []}
    for b in range(B):
        cur, path, near = -1, [], 1.0
        while True:
            kids = children(up[b], ns[b], cur)
            if not kids:
                break
            y = tokens[b, kids].long()
            lg, lm = (torch.log_softmax(t[b, cur + 1].double() / tau, -1)[y] for t in (G, Sm))
            alpha = torch.where(lg == -math.inf, -1.0, torch.exp(lg - lm) / lam).clamp(max=1.0).tolist()
            taken = None
            for i, a in zip(kids, alpha):
                u = uniforms[b, i].double().item()
                if a < 1.0:
                    near = min(near, abs(u - a) / max(a, 1e-6))
                if u <= a:
                    taken = i
                    break
            if taken is None:
                break
            cur = taken
            path.append(cur)
        g, sp, sm = (t[b, cur + 1].double() for t in (G, Sp, Sm))
        h = g if beta == 0 else g + beta * torch.where(sp == sm, 0.0, sp - sm)
        lp = torch.log_softmax(h / tau, -1)
        cdf = lp.exp().cumsum(0)
        u = uniforms[b, R - 1].double() * cdf[-1]
        token = int((h == h.max()).nonzero()[0]) if greedy else int((cdf <= u).sum().clamp(max=V - 1))
        res["accepted_len"].append(len(path))
        res["path"].append(path + [-1] * (R - 1 - len(path)))
        res["next_token"].append(token)
        res["near"].append(near)
        res["rows"].append((lp, cdf, u))
    return res


def commit(k, v, k_cache, v_cache, table, cache_len, accepted, path):
    """The caches and lengths afterwards."""
    kc, vc, new = k_cache.clone(), v_cache.clone(), []
    page = kc.shape[1]
    for b, (L, n) in enumerate(zip(cache_len.tolist(), accepted.tolist())):
        rows = [0] + [r + 1 for r in (range(n) if path is None else path[b, :n].tolist())]
        for j, r in enumerate(rows):
            p, s = int(table[b, (L + j) // page]), (L + j) % page
            kc[p, s], vc[p, s] = k[b, r], v[b, r]
        new.append(L + n + 1)
    return kc, vc, torch.tensor(new, dtype=torch.int32, device=k.device)
