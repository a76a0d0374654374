"""Inputs and bounds for attention whose scores are far from zero, or far from one another: what the tolerance that grows with the largest score cannot tell from anything.

Two kinds:
  shifted   every score of every row is the same OFFSET away from zero, 5745 or -5745 units of log2 (reference points beyond 4096 are subtracted before scaling), and the
            weights are those of ordinary scores.  kv_helpers.tolerance with `big` about 4000 allows 2^-8 + 2 * 132 * 2^-24 * 4000 = 0.067 of the weighted sum of |V|.
  steep     scales so large that the key with the largest product has all the weight: a row whose largest product leads the second by more than both can be off
            (132 * 2^-24 of the sum of magnitudes each, as derived there) and by 40 / |scale| has the rest of its weights below e^-40, and its result is
            that key's V, within half a step of bf16 (its weight is a power of two and not rounded: it is the reference point, which every other score trails by
            more than it may lag).  Rows without such a lead are only held inside the range of the V that they see, give or take the rounding of
            their weights to bf16 (2^-8 of the largest |V|) and of the result."""
from __future__ import annotations

import math

import torch

D, SCALE = 128, 1 / math.sqrt(128)
QUERY, KEY = 256.0, 176.0                              # products of 45056, times the scale 3982: 5745 in log2


def rows(n_q, Hq, n_k, H, seed, sign=0):
    """q, k, v in bf16; sign: of the offset that every score has (0: none)."""
    g = torch.Generator().manual_seed(seed)
    q, k, v = ((s * torch.randn(n, h, D, generator=g)).to(torch.bfloat16) for n, h, s in ((n_q, Hq, 2.0), (n_k, H, 1.0), (n_k, H, 1.0)))
    if sign:
        q[..., 0], k[..., 0] = QUERY, sign * KEY
    return q, k, v


def steep(q, k, v, scale, seen):
    """q [Hq, 128], k, v [tokens, H, 128] of what one query token sees, in 64 bits.  Per query head: is there a lead, the leader's V, the least and largest V."""
    H, Hq = k.shape[1], q.shape[0]
    kk, vv = k[seen].transpose(0, 1), v[seen].transpose(0, 1)                      # [H, seen, 128]
    x = q.reshape(H, Hq // H, D)
    s = torch.matmul(x, kk.transpose(1, 2).contiguous()) * math.copysign(1.0, scale)
    size = torch.matmul(x.abs(), kk.abs().transpose(1, 2).contiguous()).amax(-1)
    top, at = s.max(-1)
    rest = s.scatter(-1, at[..., None], -math.inf).amax(-1)
    lead = top - rest > 2 * 132 * 2.0 ** -24 * size + 40 / abs(scale)
    leader = torch.gather(vv, 1, at[..., None].expand(*at.shape, D))
    low, high = (f(vv, 1).reshape(H, 1, D).expand_as(leader) for f in (torch.amin, torch.amax))
    return (t.reshape(Hq, *t.shape[2:]) for t in (lead, leader, low, high))


def steep_all(q, k, v, scale, sees):
    """The same for every query token: sees[i] are the tokens that it sees."""
    parts = [list(steep(q[i], k, v, scale, torch.as_tensor(s))) for i, s in enumerate(sees)]
    return [torch.stack([p[i] for p in parts]) for i in range(4)]


def wrong_steep(out, bounds):
    """How many elements are outside."""
    lead, leader, low, high = bounds
    exact = (out - leader).abs() <= 2.0 ** -8 * leader.abs()
    off = 2.01 * 2.0 ** -8 * torch.maximum(low.abs(), high.abs())
    inside = (out >= low - off) & (out <= high + off)
    return int((~torch.where(lead[..., None], exact, inside)).sum())


def wrong_shifted(out, want, tol):
    return int((~((out - want).abs() <= tol)).sum())


def mistaken(want):
    """Results that no bound may take: zeros, and the rows of other tokens."""
    return torch.zeros_like(want), want.roll(1, 0), want.roll(1, 1)
