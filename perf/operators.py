"""The losses over full-vocabulary logits, as calls of a training step, and the scoring of given tokens.

Operators (``paper_2603_16219_amd.losses``), on logits [B, T, V] whose row t scores ``tokens[:, t]``:
  score        token log-probs of given tokens, as a rollout or a frozen reference needs them
  score_grad   the same and the gradient of any loss of them with respect to the logits
  policy       the clipped policy loss with a KL term, and its gradient; the KL from the reference's log-probs of the
               same tokens ("sampled"), from the reference's logits over the whole vocabulary ("full"), or none
  preference   the loss of paired sequences' log ratios, and its gradient

Ranges (``draw``): 1 .. 16384 rows in 1 .. 64 sequences, vocabularies 32000 .. 256000, odd ones among them, bf16 and
fp32, masks of prompts and padding, and ragged ones that leave sequences empty, temperatures 0.6 .. 1.
"""
from __future__ import annotations

import math

import torch

own = False

# Sizes are those of the repository's workloads (vocabularies of 32000, 128256, 151936 and 256000, the odd 50257 of
# its tests; 1 .. 512 sequences, drafts of up to 16 tokens) and ordinary training lengths.
MAX_LOGITS = 1 << 30


def listed():
    return [
        # One drafted block of one user scored: the smallest call, only launches and latency count.
        dict(name="score_one_block", op="score", batch=1, length=4, vocab=32000, dtype="f32", mask="full", temperature=1.0),
        # A serving batch of drafts scored for the log-probs that a later policy update compares with.
        dict(name="score_rollout", op="score", batch=64, length=16, vocab=151936, dtype="bf16", mask="full", temperature=1.0),
        # A frozen reference over a batch of ragged completions, a vocabulary whose rows start at odd elements.
        dict(name="score_ragged_odd", op="score", batch=16, length=301, vocab=50257, dtype="bf16", mask="ragged", temperature=1.0),
        # Fine-tuning on few short answers: forward and gradient through a loss of the user's own, in fp32.
        dict(name="score_grad_small", op="score_grad", batch=2, length=24, vocab=50257, dtype="f32", mask="completion", temperature=1.0),
        # Fine-tuning at an ordinary size.
        dict(name="score_grad_batch", op="score_grad", batch=8, length=512, vocab=128256, dtype="bf16", mask="completion", temperature=1.0),
        # The policy loss of a single short answer: latency.
        dict(name="policy_one_answer", op="policy", batch=1, length=9, vocab=32000, dtype="bf16", mask="full", kl="sampled",
             per_token=False, reduction="token_mean", temperature=1.0),
        # A group of sampled answers, the usual training step: prompts masked, one advantage an answer.
        dict(name="policy_group", op="policy", batch=8, length=512, vocab=128256, dtype="bf16", mask="completion", kl="sampled",
             per_token=False, reduction="token_mean", temperature=0.7),
        # The whole-vocabulary KL to the generalist, whose logits are at hand anyway.
        dict(name="policy_full_kl", op="policy", batch=4, length=512, vocab=151936, dtype="bf16", mask="completion", kl="full",
             per_token=True, reduction="seq_mean", temperature=1.0),
        # The largest call: the largest vocabulary, every position kept.
        dict(name="policy_largest", op="policy", batch=16, length=256, vocab=256000, dtype="bf16", mask="full", kl="none",
             per_token=True, reduction="token_mean", temperature=1.0),
        # One pair of short answers in fp32: three dependent steps, latency.
        dict(name="preference_one_pair", op="preference", batch=2, length=7, vocab=32000, dtype="f32", mask="full", temperature=1.0),
        # Pairs of ordinary length, prompts masked.
        dict(name="preference_pairs", op="preference", batch=8, length=512, vocab=128256, dtype="bf16", mask="completion",
             temperature=1.0),
        # Many pairs of long answers on a small vocabulary, ragged, sequences of every length from none on.
        dict(name="preference_long", op="preference", batch=16, length=1024, vocab=32000, dtype="bf16", mask="ragged", temperature=1.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        case = dict(op=rng.choice(["score", "score_grad", "policy", "policy", "preference", "preference"]), batch=_log_int(rng, 1, 64),
                    length=_log_int(rng, 1, 2048), vocab=_log_int(rng, 32000, 256000), dtype="f32" if rng.random() < 0.3 else "bf16",
                    mask=rng.choice(["full", "completion", "ragged"]), temperature=rng.choice([0.6, 0.7, 1.0, 1.0]))
        if rng.random() < 0.5:
            case["vocab"] &= ~63  # model heads are usually padded; the others stay odd or even as they fall
        if case["op"] == "preference":
            case["batch"] += case["batch"] & 1
        if case["op"] == "policy":
            case.update(kl=rng.choice(["none", "sampled", "full"]), per_token=rng.random() < 0.5,
                        reduction=rng.choice(["token_mean", "seq_mean", "sum"]))
        rows = case["batch"] * case["length"]
        if rows > 16384 or rows * case["vocab"] * (2 if case.get("kl") == "full" else 1) > MAX_LOGITS:
            continue
        if work(case)["bytes"] <= max(work(c)["bytes"] for c in listed()):
            return case


CLIP_LOW, CLIP_HIGH, KL_COEF = 0.2, 0.28, 0.05
BETA, SMOOTHING = 0.1, 0.05


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _f32(v):
    return torch.tensor(v, dtype=torch.float32).item()  # parameters are passed in fp32


def _row_chunks(rows, vocab):
    step = max(1, (64 << 20) // vocab)
    return [(r, min(rows, r + step)) for r in range(0, rows, step)]


def prepare(case, seed):
    """Logits of a model (a Gaussian part over the vocabulary), tokens drawn from them, the mask of the positions that
    count, and what the rollout and the reference left: log-probs near the policy's, advantages."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    B, T, V, tau = case["batch"], case["length"], case["vocab"], case["temperature"]
    rows, dt, full = B * T, _dtype(case), case.get("kl") == "full"
    logits = torch.empty(rows, V, dtype=dt, device=dev)
    ref_logits = torch.empty(rows, V, dtype=dt, device=dev) if full else None
    tokens = torch.empty(rows, dtype=torch.int32, device=dev)
    lp = torch.empty(rows, device=dev)
    for a, b in _row_chunks(rows, V):
        x = torch.randn(b - a, V, generator=gen, device=dev) * 2.5
        if full:  # a policy that has moved a little from its reference
            ref_logits[a:b] = x
            x += 0.25 * torch.randn(b - a, V, generator=gen, device=dev)
        logits[a:b] = x
        x = logits[a:b].float() / tau
        e = torch.empty_like(x).exponential_(generator=gen)
        tokens[a:b] = (x - e.log_()).argmax(-1)  # a draw from the softmax, by Gumbel noise
        lp[a:b] = x.gather(1, tokens[a:b].long()[:, None])[:, 0] - torch.logsumexp(x, -1)
    t = torch.arange(T, device=dev)[None, :]
    mask = None
    if case["mask"] == "completion":  # a prompt before the answer, padding behind it
        lo = torch.randint(0, T // 2 + 1, (B, 1), generator=gen, device=dev)
        hi = torch.randint(3 * T // 4, T + 1, (B, 1), generator=gen, device=dev)
        mask = (t >= lo) & (t < hi)
    elif case["mask"] == "ragged":  # answers of any length from none on
        mask = t < torch.randint(0, T + 1, (B, 1), generator=gen, device=dev)
    s = {"case": case, "logits": logits.view(B, T, V), "ref_logits": ref_logits.view(B, T, V) if full else None,
         "tokens": tokens.view(B, T), "mask": mask}
    lp = lp.view(B, T)
    if case["op"] == "policy":
        delta = 0.15 * torch.randn(B, T, generator=gen, device=dev)
        ratio = delta.exp()
        at_border = ((ratio - (1 + CLIP_HIGH)).abs() < 1e-3) | ((ratio - (1 - CLIP_LOW)).abs() < 1e-3)
        s["old_logprobs"] = lp - delta.masked_fill(at_border, 0.0)
        s["ref_logprobs"] = lp + 0.2 * torch.randn(B, T, generator=gen, device=dev) if case["kl"] == "sampled" else None
        s["advantages"] = torch.randn((B, T) if case["per_token"] else (B,), generator=gen, device=dev)
    elif case["op"] == "preference":
        s["ref_logprobs"] = lp + 0.1 * torch.randn(B, T, generator=gen, device=dev)
    elif case["op"] == "score_grad":
        s["grad_logprobs"] = -torch.rand(B, T, generator=gen, device=dev) / (B * T)
    return s


def _run_own(s):
    from paper_2603_16219_amd import losses

    case = s["case"]
    op, tau = case["op"], case["temperature"]
    if op == "score":
        return losses.token_logprobs(s["logits"], s["tokens"], mask=s["mask"], temperature=tau)["logprobs"]
    if op == "score_grad":
        out = losses.token_logprobs(s["logits"], s["tokens"], mask=s["mask"], temperature=tau, want_stats=True)
        grad = losses.token_logprobs_grad(s["logits"], s["tokens"], out["stats"], s["grad_logprobs"], mask=s["mask"], temperature=tau)
        return {"logprobs": out["logprobs"], "grad_logits": grad}
    if op == "policy":
        out = losses.policy_loss(s["logits"], s["tokens"], s["old_logprobs"], s["advantages"], mask=s["mask"],
                                 ref_logits=s["ref_logits"], ref_logprobs=s["ref_logprobs"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH,
                                 kl_coef=0.0 if case["kl"] == "none" else KL_COEF, temperature=tau, reduction=case["reduction"])
        return {k: out[k] for k in _outputs(case)}
    out = losses.preference_loss(s["logits"], s["tokens"], mask=s["mask"], ref_logprobs=s["ref_logprobs"], beta=BETA,
                                 label_smoothing=SMOOTHING, temperature=tau)
    return {k: out[k] for k in _outputs(case)}


def _outputs(case):
    if case["op"] == "policy":
        return ("loss", "logprobs", "grad_logits") if case["kl"] == "none" else ("loss", "logprobs", "kl", "grad_logits")
    return ("loss", "pair_loss", "margin", "logprobs", "grad_logits")


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    op, tau, y = case["op"], case["temperature"], s["tokens"].long()[..., None]
    x, top, total = _plain_rows(s["logits"], tau)
    lse = top.double() + total.log()  # divergences and sums of hundreds of log-probs are small beside their terms: 64 bits
    lp = (s["logits"].gather(-1, y).double() / _f32(tau) - lse)[..., 0]
    kept = torch.ones_like(lp, dtype=torch.bool) if s["mask"] is None else s["mask"]
    logprobs = torch.where(kept, lp, 0.0).float()
    if op == "score":
        return logprobs
    if op == "score_grad":
        w, out = s["grad_logprobs"], {}
    elif op == "policy":
        kl = None
        if case["kl"] == "full":
            z, z_top, z_total = _plain_rows(s["ref_logits"], tau)
            diff, lse_diff = z.neg_().add_(x), lse - z_top.double() - z_total.log()
            kl = ((x - top).exp().mul_(diff).sum(-1, keepdim=True, dtype=torch.float64) / total - lse_diff)[..., 0]
        w, kl_weight, out = _plain_policy_weights(s, lp, kl, kept)
    else:
        w, out = _plain_preference_weights(s, lp, kept)
    p = x.sub_(lse.float()).exp_()
    grad = -w[..., None] * p
    if op == "policy" and case["kl"] == "full":
        grad += kl_weight[..., None] * p.mul_(diff.sub_((lse_diff + kl[..., None]).float()))
    grad.scatter_add_(-1, y, w[..., None])
    grad = torch.where(kept[..., None], grad.div_(tau), 0.0).to(s["logits"].dtype)
    return {**out, "logprobs": logprobs, "grad_logits": grad}


def _plain_rows(logits, tau):
    """The rows over the temperature, their maxima and sums of exponentials."""
    x = logits.float() / tau
    top = x.amax(-1, keepdim=True)
    return x, top, (x - top).exp_().sum(-1, keepdim=True, dtype=torch.float64)


def _plain_policy_weights(s, lp, full_kl, kept):
    """Weights of every token's log-prob and of a whole-vocabulary divergence in the gradient, and the loss."""
    case, a = s["case"], s["advantages"].double()
    a = a if a.dim() == 2 else a[:, None]
    n = kept.double()
    if case["reduction"] == "token_mean":
        n = n / n.sum().clamp(min=1)
    elif case["reduction"] == "seq_mean":
        count = n.sum(1, keepdim=True)
        n = n / count.clamp(min=1) / (count > 0).sum().clamp(min=1)
    ratio = (lp - s["old_logprobs"]).exp()
    plain, clipped = ratio * a, ratio.clamp(1 - _f32(CLIP_LOW), 1 + _f32(CLIP_HIGH)) * a
    term, w, kl, out = -torch.minimum(plain, clipped), torch.where(plain <= clipped, -plain, 0.0), full_kl, {}
    if case["kl"] == "sampled":
        d = s["ref_logprobs"] - lp
        kl, w = torch.expm1(d) - d, w - _f32(KL_COEF) * torch.expm1(d)
    if kl is not None:
        term = term + _f32(KL_COEF) * kl
        out["kl"] = torch.where(kept, kl, 0.0).float()
    out["loss"] = torch.where(kept, n * term, 0.0).sum().float()
    return (n * w).float(), (_f32(KL_COEF) * n).float(), out


def _plain_preference_weights(s, lp, kept):
    ratio = torch.where(kept, lp - s["ref_logprobs"], 0.0).sum(1)
    pairs = ratio.shape[0] // 2
    h = _f32(BETA) * (ratio[:pairs] - ratio[pairs:])
    softplus = lambda v: v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))
    e = _f32(SMOOTHING)
    pair_loss = (1 - e) * softplus(-h) + e * softplus(h)
    dh = ((e - 1) / (1 + torch.exp(h)) + e / (1 + torch.exp(-h))) * _f32(BETA) / pairs
    w = torch.cat([dh, -dh]).float()[:, None] * kept
    return w, {"loss": pair_loss.mean().float(), "pair_loss": pair_loss.float(), "margin": h.float()}


def work(case):
    """The logits of the kept rows are read once (the reference's too for the whole-vocabulary KL), the gradient is
    written for every row; about five operations a logit for the sum of exponentials and five for the gradient."""
    B, T, V, esz = case["batch"], case["length"], case["vocab"], 2 if case["dtype"] == "bf16" else 4
    kept = B * T * {"full": 1.0, "completion": 0.625, "ragged": 0.5}[case["mask"]]
    read = 2.0 if case.get("kl") == "full" else 1.0
    grad = 0.0 if case["op"] == "score" else 1.0
    small = B * T * (9 + (0 if case["op"] == "score" else 12))
    return {"bytes": (read * kept + grad * B * T) * V * esz + small, "flops": (5 * read + (5 + 3 * (read - 1)) * grad) * kept * V}


def exact(case, seed):
    """By automatic differentiation in 64 bits: the loss as a function of the rows' log-probs (and divergences), then a
    block of rows at a time."""
    s = prepare(case, seed)
    B, T, V = s["logits"].shape
    tau, rows, op = _f32(case["temperature"]), B * T, case["op"]
    x, y = s["logits"].view(rows, V), s["tokens"].view(rows, 1).long()
    r = s["ref_logits"].view(rows, V) if s["ref_logits"] is not None else None
    kept = torch.ones(B, T, dtype=torch.bool, device=x.device) if s["mask"] is None else s["mask"]
    keep = kept.double()
    lp = torch.zeros(rows, dtype=torch.float64, device=x.device)
    kl = torch.zeros_like(lp)

    def row_terms(a, b):
        leaf = x[a:b].double().requires_grad_()
        z = torch.log_softmax(leaf / tau, -1)
        k = None
        if r is not None:
            k = (z.exp() * (z - torch.log_softmax(r[a:b].double() / tau, -1))).sum(-1)
        return leaf, z.gather(1, y[a:b])[:, 0], k

    step = max(1, (24 << 20) // V)
    chunks = [(a, min(rows, a + step)) for a in range(0, rows, step)]
    with torch.no_grad():
        for a, b in chunks:
            _, lp[a:b], k = row_terms(a, b)
            if k is not None:
                kl[a:b] = k
    if op == "score":
        return lp.view(B, T) * keep
    out = {}
    lp_leaf, kl_leaf = lp.view(B, T).clone().requires_grad_(), kl.view(B, T).clone().requires_grad_()
    with torch.enable_grad():
        if op == "score_grad":
            loss = (lp_leaf * s["grad_logprobs"].double() * keep).sum()
        elif op == "policy":
            adv = s["advantages"].double()
            adv = adv if adv.dim() == 2 else adv[:, None].expand(B, T)
            ratio = torch.exp(lp_leaf - s["old_logprobs"].double())
            bounded = torch.clip(ratio, 1 - _f32(CLIP_LOW), 1 + _f32(CLIP_HIGH))
            term = -torch.minimum(ratio * adv, bounded * adv)
            if case["kl"] == "sampled":
                d = s["ref_logprobs"].double() - lp_leaf
                div = torch.exp(d) - 1 - d
            else:
                div = kl_leaf
            if case["kl"] != "none":
                out["kl"] = div.detach() * keep
                term = term + _f32(KL_COEF) * div
            term = term * keep
            if case["reduction"] == "sum":
                loss = term.sum()
            elif case["reduction"] == "token_mean":
                loss = term.sum() / max(1.0, keep.sum().item())
            else:
                full = keep.sum(1) > 0
                loss = (term.sum(1)[full] / keep.sum(1)[full]).sum() / max(1, int(full.sum()))
            out["loss"] = loss.detach()
        else:
            total = ((lp_leaf - s["ref_logprobs"].double()) * keep).sum(1)
            h = _f32(BETA) * (total[:B // 2] - total[B // 2:])
            pair = (-(1 - _f32(SMOOTHING)) * torch.nn.functional.logsigmoid(h)
                    - _f32(SMOOTHING) * torch.nn.functional.logsigmoid(-h))
            loss = pair.mean()
            out.update(loss=loss.detach(), pair_loss=pair.detach(), margin=h.detach())
        dlp, dkl = torch.autograd.grad(loss, (lp_leaf, kl_leaf), allow_unused=True)
    dlp = dlp.reshape(-1)
    grad = torch.empty(rows, V, dtype=torch.float64, device=x.device)
    for a, b in chunks:
        with torch.enable_grad():
            leaf, v, k = row_terms(a, b)
            target = (v * dlp[a:b]).sum()
            if k is not None and dkl is not None:
                target = target + (k * dkl.reshape(-1)[a:b]).sum()
        grad[a:b], = torch.autograd.grad(target, leaf)
    return {**out, "logprobs": lp.view(B, T) * keep, "grad_logits": grad.view(B, T, V)}
