"""Trees of drafted tokens: what they are grown from, scored by, verified and kept with.

Operators (``paper_2603_16219_amd.losses`` and ``paper_2603_16219_amd.tree``):
  alternatives       log-probs of given tokens with the entropy and the top alternatives of their rows, on logits [B, T, V]
  alternatives_grad  the same and the gradient of any loss of the log-probs and entropies with respect to the logits
  attention          attention of a tree's rows, the last token and the drafted ones behind it, over a paged cache and their
                     ancestors in the tree; a chain of drafts and a single token are trees too
  verify             the ratio test down a tree of drafts, and the token drawn from the recovery distribution where it ends
  commit             keys and values of the accepted path into the paged cache

Ranges (``draw``): alternatives of 1 .. 8192 rows, vocabularies 32000 .. 256000, odd ones among them, bf16 and fp32, 0 .. 64
alternatives, masks of prompts and padding, and ragged ones; 1 .. 256 sequences of 0 .. 255 drafted tokens, chains, random
trees and wide ones, all of a batch's trees full or ragged; caches of 0 .. 131072 tokens in pages of 1 .. 256, bf16 and fp16,
heads of 64 and 128, 1 .. 16 of them a key/value head.
"""
from __future__ import annotations

import math

import torch

own = False

# Vocabularies are those of the repository's workloads and tests; batches, draft lengths and the verification's parameters too.  Heads, pages
# and contexts are ordinary ones.
MAX_LOGITS = 1 << 29


def listed():
    return [
        # One token of one user, answered with its 20 likeliest alternatives: the smallest call, only launches and latency count.
        dict(name="alternatives_one_token", op="alternatives", batch=1, length=1, vocab=32000, dtype="f32", mask="full", topk=20, temperature=1.0),
        # The rows of a serving batch, the alternatives from which the next drafts' trees grow.
        dict(name="alternatives_batch", op="alternatives", batch=64, length=16, vocab=151936, dtype="bf16", mask="full", topk=16, temperature=1.0),
        # A few short answers with an entropy bonus, in fp32, with alternatives for the log of the run.
        dict(name="alternatives_grad_small", op="alternatives_grad", batch=2, length=24, vocab=50257, dtype="f32", mask="completion", topk=5,
             temperature=1.0),
        # A training step with an entropy bonus.
        dict(name="alternatives_grad_batch", op="alternatives_grad", batch=8, length=256, vocab=128256, dtype="bf16", mask="completion", topk=0,
             temperature=1.0),
        # One new token of one user, no drafts: latency.
        dict(name="attention_one_token", op="attention", batch=1, nodes=0, tree="chain", ragged=False, context=1024, heads=32, kv_heads=8, dim=128,
             page=16, dtype="bf16"),
        # A serving batch with a small tree for each user, contexts of any length.
        dict(name="attention_trees", op="attention", batch=32, nodes=24, tree="random", ragged=True, context=4096, heads=32, kv_heads=8, dim=128,
             page=16, dtype="bf16"),
        # Long documents with wide trees: the most arithmetic for each byte of the cache.
        dict(name="attention_long", op="attention", batch=4, nodes=63, tree="wide", ragged=False, context=65536, heads=32, kv_heads=8, dim=128,
             page=64, dtype="bf16"),
        # Chains, as verify_block takes them, a key/value head for every head, pages that end anywhere in a tile, in fp16.
        dict(name="attention_chains_f16", op="attention", batch=128, nodes=8, tree="chain", ragged=True, context=2000, heads=16, kv_heads=16, dim=64,
             page=24, dtype="f16"),
        # One user's small tree: a chain of dependent steps, latency.
        dict(name="verify_one_tree", op="verify", batch=1, nodes=12, tree="random", ragged=False, vocab=32000, dtype="f32", temperature=1.0),
        # A serving batch of trees of any size.
        dict(name="verify_trees", op="verify", batch=64, nodes=31, tree="random", ragged=True, vocab=128256, dtype="bf16", temperature=0.7),
        # One user's accepted path: latency.
        dict(name="commit_one_path", op="commit", batch=1, nodes=12, tree="random", ragged=False, context=1024, heads=8, kv_heads=8, dim=128, page=16,
             dtype="bf16"),
        # Those of a large batch.
        dict(name="commit_paths", op="commit", batch=256, nodes=24, tree="random", ragged=True, context=512, heads=8, kv_heads=8, dim=128, page=16,
             dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["alternatives", "alternatives", "alternatives_grad", "attention", "attention", "attention", "verify", "verify", "commit"])
        if op.startswith("alternatives"):
            case = dict(op=op, batch=_log_int(rng, 1, 64), length=_log_int(rng, 1, 1024), vocab=_log_int(rng, 32000, 256000),
                        dtype="f32" if rng.random() < 0.3 else "bf16", mask=rng.choice(["full", "completion", "ragged"]),
                        topk=rng.choice([0, 1, 4, 8, 20, 33, 64]), temperature=rng.choice([0.6, 0.7, 1.0, 1.0]))
            logits = case["batch"] * case["length"] * case["vocab"]
        else:
            case = dict(op=op, batch=_log_int(rng, 1, 256), nodes=_log_int(rng, 1, 256) - 1, tree=rng.choice(["chain", "random", "wide"]),
                        ragged=rng.random() < 0.5)
            if op == "verify":
                case.update(vocab=_log_int(rng, 32000, 256000), dtype="f32" if rng.random() < 0.3 else "bf16", temperature=rng.choice([0.6, 0.7, 1.0, 1.0]))
                logits = 3 * case["batch"] * (case["nodes"] + 1) * case["vocab"]
            else:
                kv = _log_int(rng, 1, 16)
                case.update(context=_log_int(rng, 1, 131073) - 1, heads=kv * rng.choice([1, 1, 2, 4, 7, 8, 16]), kv_heads=kv, dim=rng.choice([64, 128, 128]),
                            page=rng.choice([1, 16, 16, 24, 64, 100, 256]), dtype=rng.choice(["bf16", "bf16", "f16"]))
                logits = 0
                scores = case["batch"] * case["heads"] * (case["nodes"] + 1) * (case["context"] + case["nodes"] + 1)
                cache = case["batch"] * case["context"] * kv * case["dim"]
                if cache > (1 << 27 if op == "commit" else 1 << 30) or (op == "attention" and scores > 1 << 30):
                    continue
        if case.get("vocab") and rng.random() < 0.5:
            case["vocab"] &= ~63  # model heads are usually padded; the others stay odd or even as they fall
        if logits > MAX_LOGITS or case["batch"] * (case.get("nodes", 0) + 1) > 16384:
            continue
        if _cost(case) <= max(_cost(c) for c in listed()):
            return case


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 150)


LAM, BETA = 0.5, 0.8
_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _f32(v):
    return torch.tensor(v, dtype=torch.float32).item()  # parameters are passed in fp32


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    if case["op"].startswith("alternatives"):
        return _prepare_rows(case, gen, dev)
    s = {"case": case, **_prepare_trees(case, gen, dev)}
    return _prepare_verify(s, case, gen, dev) if case["op"] == "verify" else _prepare_cache(s, case, gen, dev)


def _chunks(rows, width):
    step = max(1, (64 << 20) // max(1, width))
    return [(r, min(rows, r + step)) for r in range(0, rows, step)]


def _prepare_rows(case, gen, dev):
    """Logits of a model (a Gaussian part over the vocabulary and some likely tokens), tokens drawn from them, the mask of the positions
    that count, and the gradients that a loss has left for log-probs and entropies."""
    B, T, V, tau = case["batch"], case["length"], case["vocab"], case["temperature"]
    logits = torch.empty(B * T, V, dtype=_DTYPES[case["dtype"]], device=dev)
    tokens = torch.empty(B * T, dtype=torch.int32, device=dev)
    for a, b in _chunks(B * T, V):
        x = torch.randn(b - a, V, generator=gen, device=dev) * 2.0
        at = torch.randint(0, V, (b - a, 24), generator=gen, device=dev)
        x.scatter_reduce_(1, at, 6 + 5 * torch.rand(b - a, 24, generator=gen, device=dev), "amax")
        logits[a:b] = x
        x = logits[a:b].float() / tau
        tokens[a:b] = (x - torch.empty_like(x).exponential_(generator=gen).log_()).argmax(-1)  # a draw, by Gumbel noise
    t = torch.arange(T, device=dev)[None, :]
    mask = None
    if case["mask"] == "completion":  # a prompt before the answer, padding behind it
        mask = (t >= torch.randint(0, T // 2 + 1, (B, 1), generator=gen, device=dev)) & (
            t < torch.randint(3 * T // 4, T + 1, (B, 1), generator=gen, device=dev))
    elif case["mask"] == "ragged":  # answers of any length from none on
        mask = t < torch.randint(0, T + 1, (B, 1), generator=gen, device=dev)
    s = {"case": case, "logits": logits.view(B, T, V), "tokens": tokens.view(B, T), "mask": mask}
    if case["op"] == "alternatives_grad":
        s["grad_logprobs"] = -torch.rand(B, T, generator=gen, device=dev) / (B * T)
        s["grad_entropy"] = -0.1 * torch.rand(B, T, generator=gen, device=dev) / (B * T)
    return s


def _prepare_trees(case, gen, dev):
    """Parents [B, N], each before its children, -1 for children of the last token; how many drafts each sequence has."""
    B, N = case["batch"], case["nodes"]
    i = torch.arange(N, device=dev)
    parents = None
    if case["tree"] == "random":  # each behind any of those before it
        parents = ((torch.rand(B, N, generator=gen, device=dev) * (i + 1)).floor().clamp(max=i).to(torch.int32) - 1).contiguous()
    elif case["tree"] == "wide":  # three behind each
        parents = (i // 3 - 1).to(torch.int32).expand(B, N).contiguous()
    tree_len = torch.randint(0, N + 1, (B,), generator=gen, device=dev, dtype=torch.int32) if case["ragged"] else None
    return {"parents": parents, "tree_len": tree_len}


def _prepare_verify(s, case, gen, dev):
    """Three models' logits of related contexts: the same likely tokens, weighted differently.  The k-th child of a row is the specialist's k-th
    likeliest of those."""
    B, N, V = case["batch"], case["nodes"], case["vocab"]
    rows = B * (N + 1)
    names = ("G", "S_ctx", "S_noctx")
    out = {n: torch.empty(rows, V, dtype=_DTYPES[case["dtype"]], device=dev) for n in names}
    likely = torch.randint(0, V, (rows, 16), generator=gen, device=dev)
    height = 8 + 5 * torch.rand(rows, 16, generator=gen, device=dev)
    for a, b in _chunks(rows, V):
        base = torch.randn(b - a, V, generator=gen, device=dev)
        for n in names:
            x = base + 0.5 * torch.randn(b - a, V, generator=gen, device=dev)
            x.scatter_reduce_(1, likely[a:b], height[a:b] + 0.7 * torch.randn(b - a, 16, generator=gen, device=dev), "amax")
            out[n][a:b] = x
    by_rank = likely.gather(1, out["S_ctx"].gather(1, likely).float().argsort(-1, descending=True)).view(B, N + 1, 16)
    parents = _parents(s, B, N, dev)
    rank = (torch.tril(parents[:, :, None] == parents[:, None, :]).sum(-1) - 1) % 16
    tokens = by_rank[torch.arange(B, device=dev)[:, None], parents + 1, rank]
    return {**s, **{n: out[n].view(B, N + 1, V) for n in names}, "tokens": tokens.to(torch.int32).contiguous(),
            "uniforms": torch.rand(B, N + 1, generator=gen, device=dev)}


def _prepare_cache(s, case, gen, dev):
    """A pool of pages in no order, contexts of half the longest to the longest where they differ, and the block's own rows."""
    B, N, L, page, H, D = case["batch"], case["nodes"], case["context"], case["page"], case["kv_heads"], case["dim"]
    dt = _DTYPES[case["dtype"]]
    cache_len = torch.full((B,), L, dtype=torch.int32, device=dev)
    if case["ragged"]:
        cache_len = torch.randint(L // 2, L + 1, (B,), generator=gen, device=dev, dtype=torch.int32)
    per = -(-(L + N + 1) // page)
    table = torch.randperm(B * per, generator=gen, device=dev).to(torch.int32).view(B, per)
    s.update(cache_len=cache_len, block_table=table)

    def normal(*size):
        flat = torch.empty(math.prod(size), dtype=dt, device=dev)
        for a, b in _chunks(flat.numel(), 1):
            flat[a:b] = torch.randn(b - a, generator=gen, device=dev)
        return flat.view(*size)

    s.update(k_cache=normal(B * per, page, H, D), v_cache=normal(B * per, page, H, D), k=normal(B, N + 1, H, D), v=normal(B, N + 1, H, D))
    if case["op"] == "attention":
        s["q"] = normal(B, N + 1, case["heads"], D)
        return s
    parents, length = _parents(s, B, N, dev), _lengths(s, B, N, dev)
    accepted = torch.rand(B, N, generator=gen, device=dev) < 0.7
    on_path = _walk(accepted & (torch.arange(N, device=dev) < length[:, None]), parents)
    return {**s, **_path(on_path)}


def _run_own(s):
    from paper_2603_16219_amd import losses, tree

    case = s["case"]
    op = case["op"]
    if op.startswith("alternatives"):
        given = dict(mask=s["mask"], temperature=case["temperature"])
        out = losses.token_alternatives(s["logits"], s["tokens"], topk=case["topk"], want_stats=op != "alternatives", **given)
        found = {k: out[k] for k in ("logprobs", "entropy", "top_tokens", "top_logprobs")}
        if op == "alternatives_grad":
            found["grad_logits"] = losses.token_alternatives_grad(s["logits"], s["tokens"], out["stats"], out["entropy"], s["grad_logprobs"],
                                                                  s["grad_entropy"], **given)
        return found
    if op == "attention":
        return tree.attention(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["block_table"], s["cache_len"], s["parents"],
                              tree_len=s["tree_len"])
    if op == "verify":
        return tree.verify(s["G"], s["S_ctx"], s["S_noctx"], s["tokens"], s["uniforms"], s["parents"], lam=LAM, beta=BETA,
                           temperature=case["temperature"], tree_len=s["tree_len"])
    new_len = tree.commit(s["k"], s["v"], s["k_cache"], s["v_cache"], s["block_table"], s["cache_len"], s["accepted_len"], s["path"])
    return {"cache_len": new_len, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def run(s):
    if own:
        return _run_own(s)
    op = s["case"]["op"]
    if op.startswith("alternatives"):
        return _plain_alternatives(s)
    return {"attention": _plain_attention, "verify": _plain_verify, "commit": _plain_commit}[op](s)


def _plain_alternatives(s):
    case, x, y = s["case"], s["logits"], s["tokens"].long()[..., None]
    tau, n, V = _f32(case["temperature"]), case["topk"], x.shape[-1]
    kept = torch.ones(y.shape[:2], dtype=torch.bool, device=x.device) if s["mask"] is None else s["mask"]
    z = x.float() / tau
    top = z.amax(-1, keepdim=True)
    e = (z - top).exp_()
    total = e.sum(-1, keepdim=True, dtype=torch.float64)
    lse = top.double() + total.log()
    entropy = lse - (e * z).sum(-1, keepdim=True, dtype=torch.float64) / total
    lp = x.gather(-1, y).double() / tau - lse
    out = {"logprobs": torch.where(kept, lp[..., 0], 0.0).float(), "entropy": torch.where(kept, entropy[..., 0], 0.0).float(),
           "top_tokens": None, "top_logprobs": None}
    if n:
        bits = x.float().view(torch.int32).long()
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) << 32 | (V - 1 - torch.arange(V, device=x.device))  # ties: the lowest index
        at = V - 1 - (order.topk(n, -1).values & 0xFFFFFFFF)
        out["top_tokens"] = torch.where(kept[..., None], at, -1).to(torch.int32)
        out["top_logprobs"] = torch.where(kept[..., None], x.gather(-1, at).double() / tau - lse, -math.inf).float()
    if case["op"] == "alternatives_grad":
        g, k = s["grad_logprobs"][..., None], s["grad_entropy"][..., None]
        log_p = z - lse.float()
        grad = log_p.exp().mul_(-g - k * (log_p + entropy.float()))
        grad.scatter_add_(-1, y, g)
        out["grad_logits"] = torch.where(kept[..., None], grad.div_(tau), 0.0).to(x.dtype)
    return out


def _parents(s, B, N, dev):
    if s["parents"] is None:
        return (torch.arange(N, device=dev) - 1).expand(B, N)
    return s["parents"].long()


def _lengths(s, B, N, dev):
    return torch.full((B,), N, device=dev) if s["tree_len"] is None else s["tree_len"].long()


def _ancestors(parents):
    """[B, N, N]: whether j is i or an ancestor of i.  Steps to the parent, doubled until they reach past any depth."""
    N = parents.shape[1]
    up = torch.eye(N, device=parents.device) + (parents[:, :, None] == torch.arange(N, device=parents.device))
    for _ in range(max(1, N).bit_length()):
        up = (torch.matmul(up, up) > 0).float()
    return up > 0


def _walk(accepted, parents):
    """Which nodes the walk from the root goes through: those whose ancestors are all the first accepted ones of their siblings."""
    before = torch.tril(parents[:, :, None] == parents[:, None, :], -1)
    first = accepted & ~(before & accepted[:, None, :]).any(-1)
    return ~(_ancestors(parents) & ~first[:, None, :]).any(-1)


def _path(on_path):
    B, N = on_path.shape
    accepted_len = on_path.sum(-1)
    order = torch.where(on_path, torch.arange(N, device=on_path.device), N).sort(-1).values
    return {"accepted_len": accepted_len.to(torch.int32), "path": torch.where(order < N, order, -1).to(torch.int32)}


def _plain_attention(s):
    case, q = s["case"], s["q"].float()
    B, R, Hq, D = q.shape
    H, dev, L = case["kv_heads"], q.device, case["context"]
    # the cache in order, and behind it the block's own rows
    at = torch.arange(L, device=dev)
    page = s["block_table"][:, at // case["page"]].long()
    k = torch.cat([s["k_cache"][page, at % case["page"]], s["k"]], 1).float().permute(0, 2, 3, 1)
    v = torch.cat([s["v_cache"][page, at % case["page"]], s["v"]], 1).float().permute(0, 2, 1, 3)
    seen = torch.ones(B, R, R, dtype=torch.bool, device=dev).tril() & (torch.arange(R, device=dev) == 0)  # every row sees the first one
    seen[:, 1:, 1:] = _ancestors(_parents(s, B, R - 1, dev))
    seen = torch.cat([(at < s["cache_len"][:, None])[:, None].expand(B, R, L), seen], 2)
    x = torch.matmul(q.view(B, R, H, Hq // H, D).permute(0, 2, 3, 1, 4).reshape(B, H, -1, D), k.contiguous()).view(B, H, Hq // H, R, L + R)
    x = x.mul_(1 / math.sqrt(D)).masked_fill_(~seen[:, None, None], -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True)).exp_()
    x = x.div_(x.sum(-1, keepdim=True))
    o = torch.matmul(x.view(B, H, -1, L + R), v.contiguous()).view(B, H, Hq // H, R, D).permute(0, 3, 1, 2, 4).reshape(B, R, Hq, D)
    kept = torch.arange(R, device=dev) <= _lengths(s, B, R - 1, dev)[:, None]
    return torch.where(kept[..., None, None], o, 0.0).to(s["q"].dtype)


def _plain_verify(s):
    tau = _f32(s["case"]["temperature"])
    B, R, V = s["G"].shape
    N, dev = R - 1, s["G"].device
    parents, b = _parents(s, B, N, dev), torch.arange(B, device=dev)
    y = s["tokens"].long()

    def token_logprobs(h):  # of every node, at its parent's row
        x = h.float() / tau
        top = x.amax(-1, keepdim=True)
        lse = (x.sub_(top).exp_().sum(-1, dtype=torch.float64).log() + top[..., 0]).gather(1, parents + 1)
        return h[b[:, None], parents + 1, y].double() / tau - lse

    alpha = (token_logprobs(s["G"]) - token_logprobs(s["S_noctx"])).exp() / _f32(LAM)
    drafted = torch.arange(N, device=dev) < _lengths(s, B, N, dev)[:, None]
    found = _path(_walk((s["uniforms"][:, :N].double() <= alpha.clamp(max=1)) & drafted, parents))
    last = torch.cat([torch.full((B, 1), -1, dtype=torch.int32, device=dev), found["path"]], 1).amax(-1).long() + 1  # the row where the walk ends
    h = s["G"][b, last].double() + _f32(BETA) * (s["S_ctx"][b, last].double() - s["S_noctx"][b, last].double())
    h = h / tau
    e = (h - h.amax(-1, keepdim=True)).exp()
    cdf = e.cumsum(-1)
    token = (cdf <= s["uniforms"][:, N:].double() * cdf[:, -1:]).sum(-1, keepdim=True).clamp(max=V - 1)
    logprob = (e.gather(1, token) / cdf[:, -1:]).log()
    return {**found, "next_token": token[:, 0].to(torch.int32), "next_token_logprob": logprob[:, 0].float()}


def _plain_commit(s):
    path, dev, page = s["path"].long(), s["k"].device, s["case"]["page"]
    B, N = path.shape
    row = torch.cat([torch.zeros(B, 1, dtype=torch.long, device=dev), path + 1], 1)
    j = torch.arange(N + 1, device=dev)
    kept = j <= s["accepted_len"][:, None]
    b, j = kept.nonzero(as_tuple=True)
    at = s["cache_len"].long()[b] + j
    where = (s["block_table"].long()[b, at // page], at % page)
    s["k_cache"][where] = s["k"][b, row[b, j]]
    s["v_cache"][where] = s["v"][b, row[b, j]]
    return {"cache_len": s["cache_len"] + s["accepted_len"] + 1, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def work(case):
    """Every input once and every output once: the logits of the kept rows, the rows of the accepted path, the keys and values of the cache.
    What is accepted goes by the data: about what these inputs give."""
    B, op = case["batch"], case["op"]
    esz = 4 if case["dtype"] == "f32" else 2
    if op.startswith("alternatives"):
        rows, V = B * case["length"], case["vocab"]
        kept = rows * {"full": 1.0, "completion": 0.625, "ragged": 0.5}[case["mask"]]
        grad = rows if op == "alternatives_grad" else 0
        return {"bytes": (kept + grad) * V * esz + rows * (12 + 8 * case["topk"]), "flops": (8 * kept + 7 * kept * (grad > 0)) * V}
    N = case["nodes"] * (0.5 if case["ragged"] else 1.0)
    steps = 0.7 * min(N, 3.0) if case["tree"] == "chain" else 0.8 * math.log(N + 1)
    if op == "verify":
        return {"bytes": B * (2 * steps + 3) * case["vocab"] * esz + B * 12 * (case["nodes"] + 1), "flops": B * (2 * steps + 3) * 5 * case["vocab"]}
    token = 2 * case["kv_heads"] * case["dim"] * esz
    if op == "commit":
        return {"bytes": 2 * B * (steps + 1) * token + 4 * B * (case["nodes"] + 3), "flops": B}
    L = case["context"] * (0.75 if case["ragged"] else 1.0)
    q = 2 * case["heads"] * case["dim"] * esz
    return {"bytes": B * (L * token + (N + 1) * (token + q)), "flops": 4 * case["dim"] * case["heads"] * B * (N + 1) * (L + 1 + steps)}


def exact(case, seed):
    """From the definitions, in 64 bits: a block of rows or a sequence at a time, the gradient by automatic differentiation, the walk down a tree
    node by node."""
    s = prepare(case, seed)
    if case["op"].startswith("alternatives"):
        return _exact_alternatives(case, s)
    B, N = case["batch"], case["nodes"]
    dev = (s["k"] if "k" in s else s["G"]).device
    parents = list(range(-1, N - 1)) if s["parents"] is None else None
    parents = [parents] * B if parents is not None else s["parents"].tolist()
    length = [N] * B if s["tree_len"] is None else s["tree_len"].tolist()
    if case["op"] == "verify":
        return _exact_verify(case, s, parents, length)
    table, filled = s["block_table"].long(), s["cache_len"].tolist()
    page, H = case["page"], case["kv_heads"]
    if case["op"] == "commit":
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        count, path = s["accepted_len"].tolist(), s["path"].tolist()
        table = table.tolist()
        to, rows = [], []
        for b in range(B):
            for j, node in enumerate([-1] + path[b][:count[b]]):
                t = filled[b] + j
                to.append((table[b][t // page], t % page))
                rows.append((b, node + 1))
        (p, o), (b, r) = zip(*to), zip(*rows)
        kc[list(p), list(o)], vc[list(p), list(o)] = s["k"].double()[list(b), list(r)], s["v"].double()[list(b), list(r)]
        return {"cache_len": torch.tensor([filled[i] + count[i] + 1 for i in range(B)], dtype=torch.int32, device=dev), "k_cache": kc, "v_cache": vc}
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
    group = case["heads"] // H
    for b in range(B):
        R, L = length[b] + 1, filled[b]
        sees = torch.zeros(R, R, dtype=torch.bool)
        for r in range(R):
            node = r - 1
            sees[r, r] = sees[r, 0] = True
            while node >= 0:
                sees[r, node + 1] = True
                node = parents[b][node]
        bias = torch.zeros(R, L + R, dtype=torch.float64, device=dev)
        bias[:, L:].masked_fill_(~sees.to(dev), -math.inf)
        used = table[b, :-(-L // page)]
        for h in range(H):
            k = torch.cat([s["k_cache"][used, :, h].reshape(-1, case["dim"])[:L], s["k"][b, :R, h]]).double()
            v = torch.cat([s["v_cache"][used, :, h].reshape(-1, case["dim"])[:L], s["v"][b, :R, h]]).double()
            q = s["q"][b, :R, h * group:(h + 1) * group].double()
            score = (q.reshape(R * group, -1) @ k.T.contiguous()).view(R, group, -1) / math.sqrt(case["dim"]) + bias[:, None]
            out[b, :R, h * group:(h + 1) * group] = (torch.softmax(score, -1).view(R * group, -1) @ v).view(R, group, -1)
    return out


def _exact_alternatives(case, s):
    B, T, V = s["logits"].shape
    tau, n, rows = _f32(case["temperature"]), case["topk"], B * T
    x, y = s["logits"].view(rows, V), s["tokens"].view(rows).long()
    dev = x.device
    kept = torch.ones(rows, dtype=torch.bool, device=dev) if s["mask"] is None else s["mask"].view(rows)
    out = {"logprobs": torch.zeros(rows, dtype=torch.float64, device=dev), "entropy": torch.zeros(rows, dtype=torch.float64, device=dev),
           "top_tokens": torch.full((rows, n), -1, dtype=torch.int32, device=dev) if n else None,
           "top_logprobs": torch.full((rows, n), -math.inf, dtype=torch.float64, device=dev) if n else None}
    with_grad = case["op"] == "alternatives_grad"
    if with_grad:
        out["grad_logits"] = torch.zeros(rows, V, dtype=torch.float64, device=dev)
    step = max(1, (16 << 20) // V)
    for a in range(0, rows, step):
        at = torch.arange(a, min(rows, a + step), device=dev)[kept[a:a + step]]
        with torch.enable_grad():
            leaf = x[at].double().requires_grad_(with_grad)
            log_p = torch.log_softmax(leaf / tau, -1)
            lp = log_p[torch.arange(len(at), device=dev), y[at]]
            entropy = -(log_p.exp() * log_p).sum(-1)
        if with_grad and len(at):
            loss = (lp * s["grad_logprobs"].view(rows)[at]).sum() + (entropy * s["grad_entropy"].view(rows)[at]).sum()
            out["grad_logits"][at], = torch.autograd.grad(loss, leaf)
        out["logprobs"][at], out["entropy"][at] = lp.detach(), entropy.detach()
        if n:
            first = torch.sort(x[at], dim=-1, descending=True, stable=True).indices[:, :n]
            out["top_tokens"][at], out["top_logprobs"][at] = first.to(torch.int32), log_p.detach().gather(1, first)
    return {k: None if v is None else v.view(B, T, *v.shape[1:]) for k, v in out.items()}


def _exact_verify(case, s, parents, length):
    B, N, tau, dev = case["batch"], case["nodes"], _f32(case["temperature"]), s["G"].device
    y, u = s["tokens"].tolist(), s["uniforms"].double()
    u_list, out = u.tolist(), {"accepted_len": [], "path": [], "next_token": [], "next_token_logprob": []}
    for b in range(B):
        cur, path = -1, []
        while True:
            children = [i for i in range(length[b]) if parents[b][i] == cur]
            if not children:
                break
            at = torch.tensor([y[b][i] for i in children], device=dev)
            ratio = [torch.log_softmax(s[name][b, cur + 1].double() / tau, -1)[at] for name in ("G", "S_noctx")]
            alpha = (torch.exp(ratio[0] - ratio[1]) / _f32(LAM)).tolist()
            taken = [i for i, a in zip(children, alpha) if u_list[b][i] <= min(1.0, a)]
            if not taken:
                break
            cur = taken[0]
            path.append(cur)
        g, plus, minus = (s[name][b, cur + 1].double() for name in ("G", "S_ctx", "S_noctx"))
        p = torch.softmax((g + _f32(BETA) * (plus - minus)) / tau, -1)
        token = int(torch.searchsorted(p.cumsum(0), u[b, N:], right=True).clamp(max=case["vocab"] - 1))
        out["accepted_len"].append(len(path))
        out["path"].append(path + [-1] * (N - len(path)))
        out["next_token"].append(token)
        out["next_token_logprob"].append(math.log(p[token].item()))
    return {k: torch.tensor(v, dtype=torch.float64 if k == "next_token_logprob" else torch.int32, device=dev).view(B, -1)
            if k == "path" else torch.tensor(v, dtype=torch.float64 if k == "next_token_logprob" else torch.int32, device=dev) for k, v in out.items()}
