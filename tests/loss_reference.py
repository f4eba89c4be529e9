"""The losses in 64 bits from their definitions, with the gradients written out, and how far the kernels may be off.

Error bounds (u = 2^-24, half a step of fp32).  A term 2^z, z = (h - m) c, is formed in fp32 from a subtraction, a product and
an exponential: the subtraction and the product are off by u each, c by u, the exponential by 2 u, so a term is off by
(3 |z| ln 2 + 2) u of itself.  A sum of n terms a lane adds about sqrt(n) u (the roundings are independent), its merging over lanes
10 u more.  So with n terms a lane

    log-prob   (sqrt(n) + 12 + 3 E|z|) u + u |lp|        E over the row's distribution, the last for its rounding to fp32
    gradient   half a step of its type + (3 |z_v| + 3 E|z| + sqrt(n) + 20) u of the term w p_v,
               and 4 u |w| / tau at the token, where w and w p_v cancel
    KL         the same bound times E|h - z| / tau + 1 for the cross term and twice that of a log-prob for the sums

n is V / 64 at most: a row is never left to less than a wave.
"""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24


def f32(v: float) -> float:
    return torch.tensor(v, dtype=torch.float32).item()


class Rows:
    """Everything a loss needs of rows of logits, in 64 bits."""

    def __init__(self, logits, tokens, tau, ref_logits=None):
        self.tau = f32(tau)
        x = logits.double()
        self.valid = (tokens >= 0) & (tokens < x.shape[-1])
        y = tokens.long().clamp(0, x.shape[-1] - 1)[..., None]
        m = x.amax(-1, keepdim=True)
        e = torch.exp((x - m) / self.tau)
        total = e.sum(-1, keepdim=True)
        self.p = e / total
        self.m, self.total = m[..., 0], total[..., 0]
        self.lse = (m / self.tau + total.log())[..., 0]
        self.lp = ((x.gather(-1, y) - m) / self.tau - total.log())[..., 0]
        self.lp = torch.where(self.valid, self.lp, math.nan)
        self.onehot = torch.zeros_like(x).scatter_(-1, y, 1.0)
        self.z = ((m - x) / self.tau / math.log(2)).clamp(max=1e6)  # how far below the maximum, in powers of two
        self.mean_z = (self.p * self.z).sum(-1)
        n = max(1, x.shape[-1] // 64)
        self.sum_err = (math.sqrt(n) + 12 + 3 * self.mean_z) * U
        self.lp_err = self.sum_err + U * self.lp.abs().nan_to_num(0, 0, 0)
        self.kl = None
        if ref_logits is not None:
            r = ref_logits.double()
            q = torch.log_softmax(r / self.tau, -1)
            log_p = (x - m) / self.tau - total.log()
            some = self.p > 0
            self.log_ratio = torch.where(some, log_p - q, 0.0)
            self.kl = (self.p * self.log_ratio).sum(-1)
            mr = r.amax(-1, keepdim=True)
            zr = ((mr - r) / self.tau / math.log(2)).clamp(max=1e6)
            diff = torch.where(some, (x - r).abs(), 0.0) / self.tau
            self.kl_err = self.sum_err * ((self.p * diff).sum(-1) + 1) + (math.sqrt(n) + 12 + 3 * (q.exp() * zr).sum(-1)) * U + 2 * U

    def gradient(self, w, k=None):
        """dL/dlogits for dL/dlp = w and dL/dKL = k, both [B, T]."""
        g = w[..., None] * (self.onehot - self.p)
        if k is not None:
            g = g + k[..., None] * self.p * (self.log_ratio - self.kl[..., None])
        return g / self.tau

    def gradient_bound(self, w, exact, dtype, k=None):
        w = w.abs()[..., None]
        rel = (3 * self.z + 20 + self.sum_err[..., None] / U) * U
        err = w * self.p * rel + 4 * U * w * self.onehot
        if k is not None:
            k = k.abs()[..., None]
            size = self.log_ratio.abs() + self.kl.abs()[..., None] + 1
            err = err + k * self.p * (rel + self.kl_err[..., None] + 8 * U) * size
        # below the smallest normal number a value is flushed or rounded absolutely
        return err / self.tau + torch.finfo(dtype).eps / 2 * 1.01 * exact.abs() + 2.0 ** -126


def kept_of(mask, tokens):
    return torch.ones_like(tokens, dtype=torch.bool) if mask is None else mask.bool()


def norms(kept, reduction):
    n = kept.double()
    if reduction == "sum":
        return n
    if reduction == "token_mean":
        return n / max(1.0, n.sum().item())
    count = n.sum(1, keepdim=True)
    return n / count.clamp(min=1) / max(1, int((count > 0).sum()))


def policy(rows: Rows, kept, old, adv, *, clip_low, clip_high, kl_coef, reduction, ref_logprobs=None, scale=1.0):
    """dict(loss, kl, w, k): w and k are the gradients of `scale` times the loss with respect to log-probs and whole-vocabulary KLs."""
    adv = adv.double()
    adv = adv if adv.dim() == 2 else adv[:, None].expand(kept.shape)
    n, lo, hi, coef = norms(kept, reduction), 1 - f32(clip_low), 1 + f32(clip_high), f32(kl_coef)
    ratio = torch.exp(rows.lp - old.double())
    plain, bound = ratio * adv, ratio.clamp(lo, hi) * adv
    clipped = plain > bound
    term = -torch.where(clipped, bound, plain)
    w = torch.where(clipped, 0.0, -plain)
    kl = k = None
    if rows.kl is not None:
        kl, k = rows.kl, coef * n
    elif ref_logprobs is not None:
        d = ref_logprobs.double() - rows.lp
        kl = torch.expm1(d) - d
        if coef:
            w = w - coef * torch.expm1(d)
    if kl is not None and coef:
        term = term + coef * kl
    zero = lambda t: torch.where(kept, t, 0.0)
    return {"loss": zero(n * term).sum(), "size": zero(n * (ratio * adv.abs() + (0 if kl is None else coef * (kl.abs() + 1)))).sum(),
            "kl": None if kl is None else zero(kl), "w": zero(n * w) * f32(scale), "k": None if k is None else zero(k) * f32(scale), "ratio": ratio}


def preference(rows: Rows, kept, ref_logprobs, *, beta, label_smoothing, reduction="mean", scale=1.0):
    zero = lambda t: torch.where(kept, t, 0.0)
    d = zero(rows.lp - (0.0 if ref_logprobs is None else ref_logprobs.double())).sum(1)
    P = d.shape[0] // 2
    h, e = f32(beta) * (d[:P] - d[P:]), f32(label_smoothing)
    log_s = torch.nn.functional.logsigmoid
    pair = -(1 - e) * log_s(h) - e * log_s(-h)
    factor = 1.0 if reduction == "sum" else 1.0 / P
    dh = f32(beta) * factor * (-(1 - e) * torch.sigmoid(-h) + e * torch.sigmoid(h))
    w = torch.cat([dh, -dh])[:, None] * kept * f32(scale)
    lp_err = zero(rows.lp_err).sum(1)
    margin_err = abs(f32(beta)) * (lp_err[:P] + lp_err[P:])
    return {"loss": pair.sum() * factor, "pair_loss": pair, "margin": h, "w": w, "margin_err": margin_err, "factor": factor}
