"""Paged caches that programs append to, in plain torch and 64 bits: what the tests of tdk_kv_* compare with.  Also builds batches."""
from __future__ import annotations

import math

import numpy as np
import torch

D = 128
GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def angles(pos, theta):
    """Cosines and sines of the positions' angles: 64 bits, rounded to 32 once."""
    j = np.arange(D // 2)
    inv = np.array([math.pow(theta, -(2.0 * k) / D) for k in j])
    a = np.asarray(pos, np.float64)[:, None] * inv[None]
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def rotate(x, pos, theta, interleaved):
    """x: float32 [n, heads, 128] -> float32, in the library's arithmetic (one product rounded, the other fused)."""
    c, s = (t[:, None, :].astype(np.float64) for t in angles(pos, theta))
    x = x.astype(np.float64)
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :64], x[..., 64:])
    ya = (a * c - (b * s).astype(np.float32)).astype(np.float32)
    yb = (b * c + (a * s).astype(np.float32)).astype(np.float32)
    out = np.empty(x.shape, np.float32)
    if interleaved:
        out[..., 0::2], out[..., 1::2] = ya, yb
    else:
        out[..., :64], out[..., 64:] = ya, yb
    return out


def to4(x):
    """float32 [..., 128] -> codes uint8 [..., 128], exponent bytes uint8 [..., 4]: block by block from the definition."""
    x = torch.as_tensor(x, dtype=torch.float64)
    b = x.reshape(*x.shape[:-1], 4, 32)
    bad = ~torch.isfinite(b).all(-1)
    b = torch.where(bad[..., None], torch.zeros_like(b), b)
    top = b.abs().amax(-1)
    mant, ex = torch.frexp(top)                                   # top = mant 2^ex, mant in [0.5, 1)
    e = ex - 1 - 2 + (mant >= 0.875).to(ex.dtype)
    e = torch.where(top == 0, torch.full_like(e, -126), e).clamp(-126, 127)
    y = b.abs() * torch.exp2(-e.double())[..., None]
    far = (y[..., None] - GRID).abs()
    least = far.amin(-1, keepdim=True)
    near = far == least                                           # one value, or two equally near: the even code
    code = torch.where(near[..., 0::2].any(-1), 2 * near[..., 0::2].to(torch.uint8).argmax(-1), 2 * near[..., 1::2].to(torch.uint8).argmax(-1) + 1)
    code = (code + 8 * torch.signbit(b).to(code.dtype)).to(torch.uint8)
    code = torch.where(bad[..., None], torch.zeros_like(code), code)
    byte = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    return code.reshape(x.shape), byte


def from4(code, byte):
    """float64 values of codes [..., 128] and bytes [..., 4]."""
    v = GRID[(code & 7).long()] * (1 - 2 * (code >> 3).double())
    unit = torch.exp2(byte.double() - 127)
    unit = torch.where(byte == 255, torch.full_like(unit, math.nan), unit)
    return (v.reshape(*code.shape[:-1], 4, 32) * unit[..., None]).reshape(code.shape)


def pack4(code, byte, T):
    """Tokens' rows [pages, T, H, 128] and [pages, T, H, 4] as pages [pages, H, T * 68]."""
    c = code.permute(0, 2, 1, 3).reshape(code.shape[0], code.shape[2], T * 64, 2)
    b = byte.permute(0, 2, 1, 3).reshape(byte.shape[0], byte.shape[2], T * 4)
    return torch.cat((c[..., 0] + 16 * c[..., 1], b), -1).contiguous()


def unpack4(pages, T):
    """The inverse: codes [pages, T, H, 128], bytes [pages, T, H, 4]."""
    p, H = pages.shape[:2]
    c = pages[..., :T * 64].reshape(p, H, T, 64)
    code = torch.stack((c & 15, c >> 4), -1).reshape(p, H, T, 128)
    return code.permute(0, 2, 1, 3), pages[..., T * 64:].reshape(p, H, T, 4).permute(0, 2, 1, 3)


class Batch:
    """Sequences (earlier tokens, new tokens) over a pool with its pages in random order, on the CPU; dev() gives the device's arrays."""

    def __init__(self, lengths, T, seed, spare=2, pad_tokens=0, extra_stride=1):
        g = np.random.default_rng(seed)
        self.T, self.lengths = T, lengths
        self.n_seqs = len(lengths)
        self.starts = np.concatenate([[0], np.cumsum([n for _, n in lengths])]).astype(np.int32)
        self.n = int(self.starts[-1])
        self.n_tokens = self.n + pad_tokens
        self.lens = np.array([h + n for h, n in lengths], np.int32)
        pages = [-(-int(l) // T) for l in self.lens]
        self.stride = max(pages + [0]) + extra_stride
        self.pool_pages = sum(pages) + spare
        order = g.permutation(self.pool_pages)
        self.table = np.full((self.n_seqs, self.stride), -1, np.int32)
        at = 0
        for s, p in enumerate(pages):
            self.table[s, :p] = order[at:at + p]
            at += p

    def positions(self):
        """Per new token: sequence, position."""
        return [(s, h + t) for s, (h, n) in enumerate(self.lengths) for t in range(n)]

    def dev(self):
        self.d = [torch.from_numpy(x).cuda() for x in (self.starts, self.lens, np.ascontiguousarray(self.table))]
        return self.d

    def struct(self, tdk, max_len=None):
        st, le, ta = self.dev()
        return tdk.kv_batch(self.n_seqs, self.n_tokens, int(self.lens.max()) if max_len is None else max_len, st, le, ta, self.stride)

    def slot(self, s, j):
        """(page, row) of a token, None where the table names no page."""
        lp = j // self.T
        if j < 0 or lp >= self.stride:
            return None
        p = int(self.table[s, lp])
        return (p, j % self.T) if 0 <= p < self.pool_pages else None


def attend(b: Batch, k, v, q, scale, window=0, sink=0, hole=None, part_out=None, part_lse=None):
    """k, v: float64 [pages, T, H, 128]; q: float64 [n, Hq, 128].  Per query token and head: softmax over what it sees, in 64 bits.
    Returns out [n, Hq, 128], lse [n, Hq] and, for tolerances, the weighted sum of |V| and the largest scale * sum |q| |k| of a score."""
    H, Hq = k.shape[2], q.shape[1]
    group = Hq // H
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    mass = torch.zeros(q.shape, dtype=torch.float64)
    big = 0.0
    for r, (s, p) in enumerate(b.positions()):
        seen = [j for j in range(p + 1) if (window == 0 or j > p - window or j < sink)
                and not (hole is not None and hole[s][0] <= j < hole[s][1]) and b.slot(s, j) is not None]
        if not seen:
            continue
        pg, at = (torch.tensor(x) for x in zip(*[b.slot(s, j) for j in seen]))
        kk, vv = k[pg, at].transpose(0, 1), v[pg, at].transpose(0, 1)          # [H, seen, 128]
        score = torch.matmul(kk, q[r].reshape(H, group, D).transpose(1, 2)).transpose(1, 2) * scale
        size = torch.matmul(kk.abs(), q[r].abs().reshape(H, group, D).transpose(1, 2)) * abs(scale)
        if torch.isfinite(size).any():
            big = max(big, float(size[torch.isfinite(size)].max()))
        top = score.amax(-1, keepdim=True)
        w = torch.exp(score - top)
        tot = w.sum(-1, keepdim=True)
        w = w / tot
        out[r] = torch.matmul(w, vv).reshape(Hq, D)
        mass[r] = torch.matmul(w, vv.abs()).reshape(Hq, D)
        lse[r] = (top + tot.log()).reshape(Hq)
    if part_out is not None:
        both = torch.logaddexp(lse, part_lse)
        w, pw = torch.exp(lse - both), torch.exp(part_lse - both)
        w, pw = torch.where(lse == -math.inf, torch.zeros_like(w), w)[..., None], torch.where(part_lse == -math.inf, torch.zeros_like(pw), pw)[..., None]
        po = torch.where(pw == 0, torch.zeros_like(part_out), part_out)
        out, mass, lse = w * out + pw * po, w * mass + pw * po.abs(), both
    return out, lse, mass, big


def tolerance(out, lse, mass, big, tokens):
    """How far a result in the library's arithmetic may be from the one in 64 bits, element by element: (out, lse).

    A score is a sum of 128 exact products in fp32 (each addition at most 2^-24 of the sum of magnitudes, `big`), times the scale and less the
    reference point (two roundings more, and one of the scale itself): at most e = 2^-24 (128 + 4) big.  A weight is then off by the factor
    e + 2^-22 (the exponential's last two places), and by 2^-8 more where it is rounded to bf16 for the second product; the sums over the
    tokens add 2^-24 a step.  Both the sum of weights and the weighted sum carry that.  The output is rounded to bf16, 2^-8 of the value (seven
    bits behind the leading one: in [1, 2) a step is 2^-7, and half of it 2^-8).
    Logarithm: two steps of fp32 at its result and at the sum's."""
    e = 2.0 ** -24 * 132 * big + 2.0 ** -22 + 2.0 ** -24 * tokens
    return 2.0 ** -8 * out.abs() + (2.0 ** -8 + 2 * e) * 1.01 * mass + 1e-30, e + 2.0 ** -22 * (2 + lse.abs())
