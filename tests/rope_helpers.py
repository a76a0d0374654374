"""Rotation by scaled frequencies and of part of the head, and pages of 8-bit values, in plain numpy / torch and 64 bits: what the tests compare with."""
from __future__ import annotations

import math

import numpy as np
import torch

D = 128
GRID8 = torch.tensor(sorted({(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)} | {m * 2.0 ** -9 for m in range(8)})[:127], dtype=torch.float64)


def frequencies(theta, rotary=D, scaling="none", factor=1.0, original=0.0, low=0.0, high=0.0, **_):
    """Radians per position of the pairs, one after the other from the definition."""
    out = []
    for j in range(rotary // 2):
        f = math.pow(theta, -(2.0 * j) / rotary)
        if scaling == "none":
            share = 0.0                               # of the frequency that is divided
        elif scaling == "linear":
            share = 1.0
        elif scaling == "turns":
            turns = original * f / (2 * math.pi)
            share = 1.0 if turns <= low else 0.0 if turns >= high else 1.0 - (turns - low) / (high - low)
        else:
            number = lambda turns: rotary * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(theta))      # noqa: E731
            a, b = max(math.floor(number(high)), 0), min(math.ceil(number(low)), rotary - 1)
            share = 0.0 if j <= a else 1.0 if j >= b else (j - a) / (b - a)
        out.append(f if share == 0.0 else f / factor * share + f * (1.0 - share))
    return np.array(out)


def rotate(x, pos, freq, rotary, interleaved, magnitude=1.0, back=False):
    """x: float32 [n, heads, 128] -> float32, in the library's arithmetic (angles in 64 bits, one product rounded, the other fused)."""
    a = np.asarray(pos, np.float64)[:, None] * freq[None]
    size = 1.0 / magnitude if back else magnitude
    c = (np.cos(a) * size).astype(np.float32).astype(np.float64)[:, None]
    s = (np.sin(a) * (-size if back else size)).astype(np.float32).astype(np.float64)[:, None]
    y = np.array(x, np.float32)
    h = rotary // 2
    at = (slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, h), slice(h, rotary))
    u, v = (x[..., i].astype(np.float64) for i in at)
    with np.errstate(invalid="ignore", over="ignore"):
        y[..., at[0]] = (u * c - (v * s).astype(np.float32)).astype(np.float32)
        y[..., at[1]] = (v * c + (u * s).astype(np.float32)).astype(np.float32)
    return y


def to8(x):
    """float32 [..., 128] -> codes uint8 [..., 128], exponent bytes uint8 [..., 4]: block by block from the definition."""
    x = torch.as_tensor(x, dtype=torch.float64)
    b = x.reshape(*x.shape[:-1], 4, 32)
    bad = ~torch.isfinite(b).all(-1)
    b = torch.where(bad[..., None], torch.zeros_like(b), b)
    top = b.abs().amax(-1)
    mant, ex = torch.frexp(top)                       # top = mant 2^ex, mant in [0.5, 1)
    e = ex - 1 - 8 + (mant > 0.90625).to(ex.dtype)
    e = torch.where(top == 0, torch.full_like(e, -124), e).clamp(min=-124)
    y = b.abs() * torch.exp2(-e.double())[..., None]
    up = torch.searchsorted(GRID8, y.contiguous()).clamp(max=126)
    dn = (up - 1).clamp(min=0)
    near_up, near_dn = GRID8[up] - y, y - GRID8[dn]
    code = torch.where((near_up < near_dn) | ((near_up == near_dn) & (up % 2 == 0)), up, dn)
    code = torch.where(y == 0, torch.zeros_like(code), code) + 128 * torch.signbit(b).to(code.dtype)
    code = torch.where(bad[..., None], torch.zeros_like(code), code).to(torch.uint8)
    byte = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    return code.reshape(x.shape), byte


def from8(code, byte):
    """float64 values of codes [..., 128] and bytes [..., 4], as bf16 has them (infinite from 2^128 on)."""
    k = (code & 127).long()
    v = torch.where(k == 127, torch.full(k.shape, math.nan, dtype=torch.float64), GRID8[k.clamp(max=126)]) * (1 - 2 * (code >> 7).double())
    unit = torch.exp2(byte.double() - 127)
    unit = torch.where(byte == 255, torch.full_like(unit, math.nan), unit)
    v = (v.reshape(*code.shape[:-1], 4, 32) * unit[..., None]).reshape(code.shape)
    return torch.where(v.abs() >= 2.0 ** 128, torch.sign(v) * math.inf, v)


def pack8(code, byte, T):
    """Tokens' rows [pages, T, H, 128] and [pages, T, H, 4] as pages [pages, H, T * 132]."""
    c = code.permute(0, 2, 1, 3).reshape(code.shape[0], code.shape[2], T * 128)
    b = byte.permute(0, 2, 1, 3).reshape(byte.shape[0], byte.shape[2], T * 4)
    return torch.cat((c, b), -1).contiguous()


def unpack8(pages, T):
    """The inverse: codes [pages, T, H, 128], bytes [pages, T, H, 4]."""
    p, H = pages.shape[:2]
    return pages[..., :T * 128].reshape(p, H, T, 128).permute(0, 2, 1, 3), pages[..., T * 128:].reshape(p, H, T, 4).permute(0, 2, 1, 3)
