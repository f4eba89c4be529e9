"""Entropies, top alternatives and their gradient in 64 bits from the definitions, and how far the kernels may be off.

With loss_reference's u = 2^-24, z how far a logit lies below the row's largest in powers of two, n terms a lane, and H = (log2 s - x / s) ln 2:
a term's exponent t = h c - E, |t| <= z + 5, is off by (z + |t|) u; a term 2^t by (3 z ln 2 + 2) u of itself; the sums s and x by
(sqrt(n) + 12) u of their terms' sizes.  So

    entropy    ((sqrt(n) + 12) (E[z] + 6) + 3 E[z (z + E[z] + 6)]) u + u H
    gradient   of p_v (-g - k (log p_v + H)) / tau: p_v off by what it is in loss_reference, the bracket by k times (the entropy's error +
               (4 z + 40 + 8 (|log p_v| + H)) u) and 4 u |g|, half a step of its type, and 4 u |g| / tau at the token
"""
from __future__ import annotations

import math

import torch

import loss_reference as R
from loss_reference import U


class Rows(R.Rows):
    def __init__(self, logits, tokens, tau):
        super().__init__(logits, tokens, tau)
        x = logits.double()
        n = max(1, x.shape[-1] // 64)
        log_p = (x - self.m[..., None]) / self.tau - self.total.log()[..., None]
        self.log_p = log_p
        some = self.p > 0
        self.log_size = torch.where(some, log_p, 0.0)
        self.entropy = -(self.p * self.log_size).sum(-1)
        ez = self.mean_z
        self.entropy_err = ((math.sqrt(n) + 12) * (ez + 6) + 3 * (self.p * self.z * (self.z + ez[..., None] + 6)).sum(-1)) * U + U * self.entropy

    def top(self, logits, k):
        """(ids, log-probs, errors) of the k first by decreasing logit and increasing id; -1 and -inf where none is left."""
        x = logits.double() + 0.0
        masked = (x == -math.inf) | ((x == torch.finfo(logits.dtype).min) & (self.m[..., None] > torch.finfo(logits.dtype).min))
        x = torch.where(masked | x.isnan(), -math.inf, x)
        values, ids = torch.sort(x, dim=-1, descending=True, stable=True)
        values, ids = values[..., :k], ids[..., :k]
        pad = k - ids.shape[-1]
        if pad > 0:
            ids, values = torch.nn.functional.pad(ids, (0, pad)), torch.nn.functional.pad(values, (0, pad), value=-math.inf)
        none = values == -math.inf
        lp = torch.where(none, -math.inf, self.log_p.gather(-1, ids))
        return torch.where(none, -1, ids).to(torch.int32), lp, self.sum_err[..., None] + U * lp.abs().nan_to_num(0, 0, 0)

    def gradient2(self, g, k):
        b = -g[..., None] - k[..., None] * (self.log_size + self.entropy[..., None])
        return (g[..., None] * self.onehot + self.p * b) / self.tau

    def gradient2_bound(self, g, k, exact, dtype):
        g, k = g.abs()[..., None], k.abs()[..., None]
        rel = (3 * self.z + 20 + self.sum_err[..., None] / U) * U
        size = self.log_size.abs() + self.entropy[..., None]
        err = self.p * ((g + k * size) * rel + k * (self.entropy_err[..., None] + (4 * self.z + 40 + 8 * size) * U) + 4 * U * g) + 4 * U * g * self.onehot
        return err / self.tau + torch.finfo(dtype).eps / 2 * 1.01 * exact.abs() + 2.0 ** -126
