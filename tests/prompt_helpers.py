"""Attention of packed sequences in plain torch and 64 bits: what the tests of tdk_prompt_attend compare with."""
from __future__ import annotations

import math

import torch

D = 128


def attend(lengths, q, k, v, scale, window=0, sink=0, part_out=None, part_lse=None):
    """lengths: (queries, keys) per sequence; q: float64 [n_q, Hq, 128], k, v: float64 [n_k, H, 128].  Returns out, lse and, for tolerances, the weighted sum
    of |V| and the largest scale * sum |q| |k| of a score."""
    H, Hq = k.shape[1], q.shape[1]
    group = Hq // H
    out, mass = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    big, q0, k0 = 0.0, 0, 0
    for n, m in lengths:
        if n and m:
            pos = torch.arange(m - n, m, device=q.device)[:, None]
            at = torch.arange(m, device=q.device)
            see = at <= pos
            if window:
                see = see & ((at > pos - window) | (at < sink))
            qq = q[q0:q0 + n].reshape(n, H, group, D).permute(1, 2, 0, 3)               # [H, group, n, D]
            kk, vv = k[k0:k0 + m].permute(1, 0, 2)[:, None], v[k0:k0 + m].permute(1, 0, 2)[:, None]
            score = torch.matmul(qq, kk.transpose(2, 3).contiguous()) * scale
            size = torch.matmul(qq.abs(), kk.abs().transpose(2, 3).contiguous()) * abs(scale)
            size = size[torch.isfinite(size) & see]
            big = max(big, float(size.max()) if size.numel() else 0.0)
            score = torch.where(see, score, torch.full((), -math.inf, dtype=torch.float64, device=q.device))
            top = score.amax(-1, keepdim=True)
            w = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
            tot = w.sum(-1, keepdim=True)
            w = torch.where(see, w / torch.where(tot == 0, torch.ones_like(tot), tot), torch.zeros_like(w))
            # what a query does not see does not reach it, whatever it holds
            odd = ~torch.isfinite(vv)
            fine = torch.where(odd, torch.zeros_like(vv), vv)
            o, ms = torch.matmul(w, fine), torch.matmul(w, fine.abs())
            if odd.any():
                for val, there in ((math.inf, vv == math.inf), (-math.inf, vv == -math.inf), (math.nan, torch.isnan(vv))):
                    hit = torch.matmul(see.double().expand_as(w), there.double()) > 0
                    o = torch.where(hit, o + val, o)
            out[q0:q0 + n] = o.permute(2, 0, 1, 3).reshape(n, Hq, D)
            mass[q0:q0 + n] = ms.permute(2, 0, 1, 3).reshape(n, Hq, D)
            lse[q0:q0 + n] = (top + tot.log()).permute(2, 0, 1, 3).reshape(n, Hq)
        q0, k0 = q0 + n, k0 + m
    if part_out is not None:
        both = torch.logaddexp(lse, part_lse)
        w, pw = torch.exp(lse - both), torch.exp(part_lse - both)
        w, pw = (torch.where(x == -math.inf, torch.zeros_like(y), y)[..., None] for x, y in ((lse, w), (part_lse, pw)))
        po = torch.where(pw == 0, torch.zeros_like(part_out), part_out)
        out, mass, lse = w * out + pw * po, w * mass + pw * po.abs(), both
    return out, lse, mass, big
