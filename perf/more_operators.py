"""What a program does with a prompt before and after it enters the paged caches, and with caches in 8 bits.

Every case is one layer's worth of one call (two for the 8-bit store) on a batch of sequences:

  rotate    turn the new tokens' keys and queries for their positions, with nothing written into a cache: part of the head or all of
            it, either layout of the pairs, frequencies scaled for long contexts, or turned back again
  prompt    causal attention of rows that are not in pages: packed sequences whose last tokens are the queries, grouped heads,
            optionally a sliding window with first tokens that stay visible, optionally joined with a partial result over other tokens
  store8    rotate new tokens and write them into a cache in 8 bits (one sign, four exponent and three mantissa bits; 32 consecutive
            values share a power of two), then read the rows back as the next round's shared block does
  attend8   attention of the new tokens' queries over such a cache, with windows, spans that are attended to elsewhere, joined parts

Fields: seqs sequences; at most `new` new tokens each (ragged: 0..new); `hist` earlier tokens at most (half of that at
least); heads / q_heads; page tokens; style and theta of the rotation; rotary: elements of a head that turn; scaling: how the
frequencies are changed for contexts of `factor` times `original` tokens (low, high: turns over those tokens between which the change
fades; magnitude: of the cosines and sines); back: turned back; window (0: none), sink; hole: tokens of the shared span that is attended
to elsewhere (0: none); join: a partial result over tokens that are not here; fused: what enters are slices of one projection's output.

Inputs: keys, values and queries ~ N(0, 1), queries times 2 for attention (peaked weights); pages in random order;
pages that no call reads or writes all map to one page, as the repository's generator has it.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128
DEVICE = "cuda"


def _case(name, op, **kw):
    c = dict(name=name, op=op, seqs=1, new=1, ragged=False, hist=1000, heads=8, q_heads=40, page=16, style="half", theta=1.0e6,
             rotary=D, scaling="none", factor=1.0, original=0, low=0.0, high=0.0, magnitude=1.0, back=False, window=0, sink=0, hole=0,
             join=False, fused=False)
    c.update(kw)
    return c


def listed():
    return [
        # a scene with four agents, one token each: latency is all there is
        _case("rotate-tiny", "rotate", seqs=4, hist=256),
        # private prompts of a 25-agent session on their way to attention, frequencies slowed between two numbers of turns
        _case("rotate-prompts", "rotate", seqs=25, new=999, ragged=True, hist=4000, fused=True, theta=5.0e5, scaling="turns", factor=8.0, original=8192, low=1.0,
              high=4.0),
        # long documents, half of each head turned, pairs side by side, far positions, turned back to be kept without positions
        _case("rotate-part-far", "rotate", seqs=5, new=8000, ragged=True, hist=900001, style="interleaved", rotary=64, scaling="index", factor=32.0,
              original=32768, low=1.0, high=32.0, magnitude=1.3465735902799727, back=True, q_heads=16),
        # four short prompts in the four-agent scene
        _case("prompt-tiny", "prompt", seqs=4, new=33, hist=0),
        # private prompts of a 25-agent session, unequal lengths, straight from the projection
        _case("prompt-session", "prompt", seqs=25, new=999, ragged=True, hist=0, fused=True),
        # one long document
        _case("prompt-long", "prompt", new=8192, hist=0),
        # chunks of four documents behind the chunks before them, a window with four first tokens that stay, joined with a shared span's result
        _case("prompt-chunks", "prompt", seqs=4, new=2048, ragged=True, hist=6001, q_heads=64, theta=5.0e5, window=2048, sink=4, join=True),
        # a decode step of the 250-agent round
        _case("store8-decode250", "store8", seqs=250, hist=9000, fused=True),
        # whole outputs of 100 agents of an 80-layer model stored in 8 bits and read back as the next round's shared blocks
        _case("store8-outputs", "store8", seqs=100, new=400, ragged=True, hist=8000, q_heads=64, fused=True, theta=5.0e5, scaling="turns", factor=8.0, original=8192,
              low=1.0, high=4.0),
        # the four-agent scene's decode step
        _case("attend8-tiny", "attend8", seqs=4, hist=256),
        # the 250-agent round's decode step over private histories, joined with the shared span's partial result
        _case("attend8-decode250", "attend8", seqs=250, hist=4000, hole=5000),
        # private prompts of four agents behind their histories
        _case("attend8-prompts", "attend8", seqs=4, new=2048, ragged=True, hist=4000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def _dense(c):
    """Elements of the plain form's largest tables: keys, and scores."""
    if c["op"] in ("rotate", "store8"):
        return c["seqs"] * c["new"] * (c["q_heads"] + 2 * c["heads"]) * D, 0
    length = c["hist"] + c["hole"] + c["new"] + (2 * c["page"] if c["op"] == "attend8" else 0)
    return c["seqs"] * length * c["heads"] * D, c["seqs"] * c["q_heads"] * c["new"] * length


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _case("", rng.choice(["rotate", "rotate", "prompt", "prompt", "prompt", "store8", "store8", "attend8", "attend8", "attend8"]))
        del c["name"]
        c["seqs"] = _log(rng, 1, 256)
        c["new"] = rng.choice([1, 1, rng.randint(2, 8), _log(rng, 2, 8192)])
        c["ragged"] = c["new"] > 1 and rng.random() < 0.6
        c["hist"] = _log(rng, 1, 100000)
        c["heads"] = rng.choice([1, 2, 4, 8, 8, 8])
        c["q_heads"] = c["heads"] * rng.choice([1, 2, 4, 5, 5, 7, 8, 16])
        c["page"] = rng.choice([16, 16, 32])
        c["style"] = rng.choice(["half", "half", "interleaved"])
        c["theta"] = rng.choice([1.0e4, 5.0e5, 1.0e6])
        c["fused"] = rng.random() < 0.5
        if c["op"] in ("rotate", "store8"):
            c["rotary"] = rng.choice([16, 32, 64, 64, 96, 128, 128, 128, 128])
            c["scaling"] = rng.choice(["none", "linear", "turns", "index"])
            if c["scaling"] != "none":
                c["factor"] = rng.choice([2.0, 4.0, 8.0, 32.0, rng.uniform(1.0, 64.0)])
            if c["scaling"] in ("turns", "index"):
                c["original"] = rng.choice([4096, 8192, 32768])
                c["low"], c["high"] = rng.choice([(1.0, 4.0), (1.0, 32.0)])
                c["magnitude"] = rng.choice([1.0, 1.0, 0.1 * math.log(c["factor"]) + 1.0])
            if c["op"] == "rotate":
                c["hist"] = _log(rng, 1, 1000000)
                c["back"] = rng.random() < 0.3
        else:
            if c["op"] == "prompt":
                c["new"] = rng.choice([1, rng.randint(2, 64), _log(rng, 16, 8192), _log(rng, 16, 8192)])
                c["ragged"] = c["new"] > 1 and rng.random() < 0.6
                c["hist"] = rng.choice([0, 0, _log(rng, 1, 20000)])
                c["join"] = rng.random() < 0.3
            if rng.random() < 0.4:
                c["window"] = _log(rng, 16, 8192)
                c["sink"] = rng.choice([0, 1, 4, rng.randint(2, 64)])
            elif c["op"] == "attend8" and rng.random() < 0.4:
                c["hole"] = _log(rng, 16, 25600)
        keys, scores = _dense(c)
        if keys <= 2.5e9 and scores <= 3.0e9 and _cost(c) <= most:
            return c


def _lengths(c):
    """Per sequence: new tokens, earlier tokens before the span that is attended to elsewhere, the span, earlier tokens behind it."""
    rng = random.Random("%s %d %d %d %d" % (c["op"], c["seqs"], c["new"], c["hist"], c["hole"]))
    rows = []
    for i in range(c["seqs"]):
        new = c["new"] if not c["ragged"] or i == c["seqs"] - 1 else rng.randint(0, c["new"])
        hist = rng.randint(c["hist"] // 2, c["hist"])
        behind = min(hist, rng.randint(0, 200)) if c["hole"] else 0
        rows.append((new, hist - behind, c["hole"], behind))
    return rows


def _seen(c, new, before, hole, behind):
    """Tokens that some query of the sequence sees, and the sum over its queries of the tokens each sees."""
    length = before + hole + behind + new
    total, first = 0, None
    for p in range(length - new, length):
        lo = max(0, p + 1 - c["window"]) if c["window"] else 0
        first = lo if first is None else first
        total += p + 1 - hole if hole else p + 1 - lo + min(lo, c["sink"])
    if first is None:
        return 0, 0
    return (length - hole if hole else length - first + min(first, c["sink"])), total


def _joined(c):
    return bool(c["hole"] or c["join"])


def work(case):
    c, hd = case, case["heads"] * D
    lengths = _lengths(c)
    n = sum(r[0] for r in lengths)
    if c["op"] == "rotate":
        return {"bytes": n * 2 * 2 * (hd + c["q_heads"] * D), "flops": 0}
    row8 = c["heads"] * 132                                # one plane of a token in the cache
    if c["op"] == "store8":
        return {"bytes": n * (2 * 2 * hd + 2 * row8 + 2 * 2 * c["q_heads"] * D + 2 * row8 + 2 * 2 * hd), "flops": 0}
    seen = [_seen(c, *r) for r in lengths]
    per_query = c["q_heads"] * (2 * D + 2 * D + 4 + (4 * D + 4 if _joined(c) else 0))
    row = 2 * hd if c["op"] == "prompt" else row8
    return {"bytes": 2 * row * sum(s[0] for s in seen) + n * per_query, "flops": 4 * D * c["q_heads"] * sum(s[1] for s in seen)}


# ---- inputs ----

def _to8(x):
    """fp32 [..., 128] as an 8-bit row: 128 bytes of values and 4 of block exponents.

    The power of two of a block of 32 puts its largest magnitude into (232, 464]: 448 is the largest value, and what rounds to it
    lies up to 464.  2^-124 at least.  Values round to the nearest, ties to even."""
    b = x.reshape(*x.shape[:-1], 4, 32)
    top = b.abs().amax(-1, keepdim=True)
    mant, exp = torch.frexp(top)                       # top = mant 2^exp, mant in [0.5, 1)
    e = (exp - 1 - 8 + (mant > 0.90625)).clamp(-124, 120)
    e = torch.where(top == 0, torch.full_like(e, -124), e)
    code = torch.ldexp(b, -e).to(torch.float8_e4m3fn).view(torch.uint8)
    return code.reshape(x.shape), (e + 127).to(torch.uint8).reshape(*x.shape[:-1], 4)


def _from8(code, e):
    """The fp32 values of 8-bit rows [..., 128] with exponents [..., 4]."""
    v = code.view(torch.float8_e4m3fn).float().reshape(*code.shape[:-1], 4, 32)
    return torch.ldexp(v, e.int().unsqueeze(-1) - 127).reshape(code.shape)


def _table(c, lengths, rng):
    """Which page holds which tokens: page 0 stands for all that no call looks at."""
    T, rows, used = c["page"], [], 1
    reads = c["op"] == "attend8"
    stride = max(-(-sum(r) // T) for r in lengths) + 1
    for new, before, hole, behind in lengths:
        length = before + hole + behind + new
        first = length - new
        if reads:
            first = max(0, first + 1 - c["window"]) if c["window"] else 0
        row = []
        for p in range(-(-length // T)):
            live = (p + 1) * T > first or (reads and p * T < c["sink"])
            if hole and p * T >= before and (p + 1) * T <= before + hole:
                live = False
            row.append(used if live else 0)
            used += live
        rows.append(row)
    order = list(range(1, used))
    rng.shuffle(order)
    order = np.array([0] + order, dtype=np.int32)
    table = np.full((len(rows), stride), -1, np.int32)
    for i, row in enumerate(rows):
        table[i, :len(row)] = order[row]
    return torch.from_numpy(table).to(DEVICE), used, stride


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE).bfloat16()


def prepare(case, seed):
    c, g = case, torch.Generator(DEVICE)
    g.manual_seed(seed)
    rng = random.Random(seed)
    lengths, T, heads = _lengths(c), c["page"], c["heads"]
    n, wide, hd = sum(r[0] for r in lengths), c["q_heads"] * D, heads * D
    count = lambda xs: torch.tensor([0] + list(np.cumsum(xs)), dtype=torch.int32, device=DEVICE)      # noqa: E731
    s = dict(case=dict(c), n=n, longest=max(sum(r) for r in lengths), most=max(r[0] for r in lengths), starts=count([r[0] for r in lengths]),
             lens=torch.tensor([sum(r) for r in lengths], dtype=torch.int32, device=DEVICE))
    if c["op"] == "prompt":
        s["k_starts"] = count([sum(r) for r in lengths])
        s["nk"] = nk = sum(sum(r) for r in lengths)
        if c["fused"] and nk == n:
            s["q"], s["k"], s["v"] = torch.split(_randn(g, n, wide + 2 * hd), [wide, hd, hd], 1)
            s["q"].mul_(2)
        else:
            s["q"] = _randn(g, n, wide) * 2
            s["k"], s["v"] = torch.split(_randn(g, nk, 2 * hd), [hd, hd], 1) if c["fused"] else (_randn(g, nk, hd), _randn(g, nk, hd))
    elif c["op"] == "attend8":
        s["table"], s["pages"], s["stride"] = _table(c, lengths, rng)
        s["q"] = _randn(g, n, wide) * 2
        for name in ("pool_k", "pool_v"):
            pool = s[name] = torch.empty(s["pages"], heads, T * 132, dtype=torch.uint8, device=DEVICE)
            for at in range(0, s["pages"], 8192):      # (in pieces: the values in 32 bits take four times the room)
                m = min(8192, s["pages"] - at)
                code, e = _to8(torch.randn(m, heads, T, D, generator=g, device=DEVICE))
                pool[at:at + m] = torch.cat((code.reshape(m, heads, T * D), e.reshape(m, heads, T * 4)), -1)
    else:
        parts = torch.split(_randn(g, n, wide + 2 * hd), [wide, hd, hd], 1)
        s["q"], s["k"], s["v"] = parts if c["fused"] else [p.contiguous() for p in parts]
        s["q_out"], s["k_out"] = (torch.empty(n, h, D, dtype=torch.bfloat16, device=DEVICE) for h in (c["q_heads"], heads))
        if c["op"] == "store8":
            s["table"], s["pages"], s["stride"] = _table(c, lengths, rng)
            s["v_out"] = torch.empty(n, heads, D, dtype=torch.bfloat16, device=DEVICE)
            s["pool_k"], s["pool_v"] = (torch.zeros(s["pages"], heads, T * 132, dtype=torch.uint8, device=DEVICE) for _ in range(2))
        return s
    if c["hole"]:
        s["hole"] = torch.tensor([[r[1], r[1] + r[2]] for r in lengths], dtype=torch.int32, device=DEVICE)
    if _joined(c):
        s["part_out"] = torch.randn(n, c["q_heads"], D, generator=g, device=DEVICE) * 0.1
        s["part_lse"] = torch.randn(n, c["q_heads"], generator=g, device=DEVICE) + 8
    s["out"] = torch.empty(n, c["q_heads"], D, dtype=torch.bfloat16, device=DEVICE)
    s["lse"] = torch.empty(n, c["q_heads"], device=DEVICE)
    return s


# ---- the plain forms ----

def _frequencies(c):
    """Radians per position of every pair: theta^(-2 j / rotary), the slow ones divided by the factor."""
    R = c["rotary"]
    j = torch.arange(R // 2, dtype=torch.float64, device=DEVICE)
    f = c["theta"] ** (-2 * j / R)
    if c["scaling"] == "none":
        return f
    if c["scaling"] == "linear":
        return f / c["factor"]
    if c["scaling"] == "turns":                        # by the turns that a pair makes over the original length
        keep = ((c["original"] * f / (2 * math.pi) - c["low"]) / (c["high"] - c["low"])).clamp(0, 1)
    else:                                              # by the pair's number, between those whose turns are the borders
        at = lambda turns: R * math.log(c["original"] / (turns * 2 * math.pi)) / (2 * math.log(c["theta"]))      # noqa: E731
        first, last = max(math.floor(at(c["high"])), 0), min(math.ceil(at(c["low"])), R - 1)
        keep = 1 - ((j - first) / max(last - first, 0.001)).clamp(0, 1)
    return f / c["factor"] * (1 - keep) + f * keep


def _tokens(s):
    """Per new token: its sequence, its number in it, its position."""
    t = torch.arange(s["n"], device=DEVICE)
    seq = torch.searchsorted(s["starts"].long(), t, right=True) - 1
    i = t - s["starts"].long()[seq]
    return seq, i, s["lens"].long()[seq] - (s["starts"][1:] - s["starts"][:-1]).long()[seq] + i


def _rotate(c, x, pos):
    """Rows [n, heads, 128] rotated for their positions, in the arithmetic that the cache is defined by: the angles and their cosines and
    sines in 64 bits, those rounded to 32; one product rounded to 32 bits, the other inside a fused multiply-add (here in 64 bits, where
    it is exact)."""
    R = c["rotary"]
    angle = pos.double()[:, None] * _frequencies(c)
    size = 1 / c["magnitude"] if c["back"] else c["magnitude"]
    cos, sin = (torch.cos(angle) * size).float()[:, None, :], (torch.sin(angle) * (-size if c["back"] else size)).float()[:, None, :]
    x = x.reshape(x.shape[0], -1, D).float()
    y = x.clone()
    if c["style"] == "half":
        a, b, ya, yb = x[..., :R // 2], x[..., R // 2:R], y[..., :R // 2], y[..., R // 2:R]
    else:
        a, b, ya, yb = x[..., 0:R:2], x[..., 1:R:2], y[..., 0:R:2], y[..., 1:R:2]
    ya.copy_(a.double() * cos.double() - (b * sin).double())
    yb.copy_(b.double() * cos.double() + (a * sin).double())
    return y


def _plain_rotate(s):
    _, _, pos = _tokens(s)
    return {"k": _rotate(s["case"], s["k"], pos).bfloat16(), "q": _rotate(s["case"], s["q"], pos).bfloat16()}


def _plain_store(s):
    c, T = s["case"], s["case"]["page"]
    seq, _, pos = _tokens(s)
    page, at = s["table"][seq, pos // T].long(), pos % T
    k, q = _rotate(c, s["k"], pos), _rotate(c, s["q"], pos).bfloat16()
    out = {"q": q}
    for name, x in (("k", k), ("v", s["v"].reshape(s["n"], -1, D).float())):
        code, e = _to8(x)
        pool = s["pool_" + name]
        codes, es = pool[..., :T * D].unflatten(-1, (T, D)), pool[..., T * D:].unflatten(-1, (T, 4))
        codes[page, :, at], es[page, :, at] = code, e
        out[name] = _from8(codes[page, :, at], es[page, :, at]).bfloat16()
    return out


def _keys(s):
    """K and V as [seqs, heads, tokens, 128] in 32 bits, every sequence as long as the longest."""
    c, T, heads = s["case"], s["case"]["page"], s["case"]["heads"]
    planes = []
    if c["op"] == "prompt":
        row = (s["k_starts"][:-1].long()[:, None] + torch.arange(s["longest"], device=DEVICE)).clamp(max=s["nk"] - 1)
        for x in (s["k"], s["v"]):
            planes.append(x.reshape(s["nk"], heads, D)[row].float().transpose(1, 2))
        return planes
    table = s["table"].long().clamp(min=0)
    for pool in (s["pool_k"], s["pool_v"]):
        x = pool[table].permute(0, 2, 1, 3)
        planes.append(_from8(x[..., :T * D].unflatten(-1, (T, D)), x[..., T * D:].unflatten(-1, (T, 4))).flatten(2, 3))
    return planes


def _plain_attend(s):
    c, heads = s["case"], s["case"]["heads"]
    seqs, most, group = c["seqs"], s["most"], c["q_heads"] // heads
    k, v = _keys(s)
    i = torch.arange(most, device=DEVICE)
    news = (s["starts"][1:] - s["starts"][:-1]).long()
    q = s["q"].reshape(s["n"], heads, group, D)[(s["starts"][:-1].long()[:, None] + i).clamp(max=s["n"] - 1)]
    q = q.float().permute(0, 2, 1, 3, 4).reshape(seqs, heads, most * group, D) * (1 / math.sqrt(D))
    pos = (s["lens"].long() - news)[:, None] + i
    at = torch.arange(k.shape[2], device=DEVICE)
    see = at <= pos[..., None]
    if c["window"]:
        see = see & ((at > pos[..., None] - c["window"]) | (at < c["sink"]))
    if c["hole"]:
        see = see & ((at < s["hole"][:, :1]) | (at >= s["hole"][:, 1:]))[:, None, :]
    score = torch.matmul(q, k.transpose(2, 3)).reshape(seqs, heads, most, group, -1)
    score.masked_fill_(~see[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.reshape(seqs, heads, most * group, -1), v).reshape(seqs, heads, most, group, D)
    lse = top + total.log()
    out = (out / total).permute(0, 2, 1, 3, 4).reshape(seqs, most, c["q_heads"], D)
    lse = lse.permute(0, 2, 1, 3, 4).reshape(seqs, most, c["q_heads"])
    seq, num, _ = _tokens(s)
    out, lse = out[seq, num], lse[seq, num]
    if _joined(c):
        both = torch.logaddexp(lse, s["part_lse"])
        out = out * (lse - both).exp()[..., None] + s["part_out"] * (s["part_lse"] - both).exp()[..., None]
        lse = both
    return {"out": out.bfloat16(), "lse": lse}


# ---- the framework's calls ----

def _calls(s):
    """What a program keeps between steps: the handle of the geometry, the views of its buffers, the workspace."""
    from paper_2604_03143_amd import tdk
    c, op, wide, hd = s["case"], s["case"]["op"], s["case"]["q_heads"] * D, s["case"]["heads"] * D
    model = tdk.model(1, c["heads"], D, c["page"], c["theta"], tdk.ROPE_HALF if c["style"] == "half" else tdk.ROPE_INTERLEAVED)
    scaling = {"none": tdk.ROPE_SCALE_NONE, "linear": tdk.ROPE_SCALE_LINEAR, "turns": tdk.ROPE_SCALE_TURNS, "index": tdk.ROPE_SCALE_INDEX}[c["scaling"]]
    rope = tdk.rope(c["rotary"], scaling, c["factor"], c["original"], c["low"], c["high"], c["magnitude"])
    kv = tdk.tdk_kv_create_rope(model, rope, tdk.KV_BF16 if op in ("rotate", "prompt") else tdk.KV_MXFP8)
    got = dict(tdk=tdk, kv=kv)
    if op == "prompt":
        batch = got["batch"] = tdk.prompt_batch(c["seqs"], s["n"], s["nk"], s["longest"], s["starts"], s["k_starts"])
        need = tdk.tdk_prompt_attend_workspace_bytes(kv, batch, c["q_heads"])
        got["space"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEVICE)
        got["io"] = tdk.prompt_attend_io(s["q"], s["q"].stride(0), c["q_heads"], s["k"], s["k"].stride(0), s["v"], s["v"].stride(0), 1 / math.sqrt(D), s["out"],
                                         wide, s["lse"], got["space"], need, window=c["window"], n_sink=c["sink"], part_out=s.get("part_out"),
                                         part_lse=s.get("part_lse"))
        return got
    if op == "rotate":
        got["batch"] = tdk.kv_batch(c["seqs"], s["n"], s["longest"], s["starts"], s["lens"], None, 0)
        got["io"] = tdk.kv_rotate_io(s["k"], s["k"].stride(0), s["k_out"], hd, q=s["q"], q_stride=s["q"].stride(0), n_q_heads=c["q_heads"], q_out=s["q_out"],
                                     q_out_stride=wide, back=c["back"])
        return got
    got["cache"] = tdk.kv_cache(s["pool_k"], s["pool_v"], s["pages"])
    batch = got["batch"] = tdk.kv_batch(c["seqs"], s["n"], s["longest"], s["starts"], s["lens"], s["table"], s["stride"])
    if op == "store8":
        got["io"] = tdk.kv_rows(s["k"], s["v"], s["k"].stride(0), s["v"].stride(0), q=s["q"], q_stride=s["q"].stride(0), n_q_heads=c["q_heads"], q_out=s["q_out"],
                                q_out_stride=wide)
        got["rows"] = tdk.kv_rows(s["k_out"], s["v_out"], hd, hd)
        return got
    need = tdk.tdk_kv_attend_workspace_bytes(kv, batch, c["q_heads"])
    got["space"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEVICE)
    got["io"] = tdk.kv_attend_io(s["q"], s["q"].stride(0), c["q_heads"], 1 / math.sqrt(D), s["out"], wide, s["lse"], got["space"], need, window=c["window"],
                                 n_sink=c["sink"], hole=s.get("hole"), part_out=s.get("part_out"), part_lse=s.get("part_lse"))
    return got


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"rotate": _plain_rotate, "store8": _plain_store}.get(op, _plain_attend)(s)
    if "calls" not in s:
        s["calls"] = _calls(s)
    x = s["calls"]
    tdk, stream = x["tdk"], torch.cuda.current_stream().cuda_stream
    if op == "rotate":
        tdk.tdk_kv_rotate(x["kv"], x["batch"], x["io"], stream)
        return {"k": s["k_out"], "q": s["q_out"]}
    if op == "store8":
        tdk.tdk_kv_append(x["kv"], x["cache"], x["batch"], x["io"], stream)
        tdk.tdk_kv_read(x["kv"], x["cache"], x["batch"], x["rows"], stream)
        return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}
    if op == "prompt":
        tdk.tdk_prompt_attend(x["kv"], x["batch"], x["io"], stream)
    else:
        tdk.tdk_kv_attend(x["kv"], x["cache"], x["batch"], x["io"], stream)
    return {"out": s["out"], "lse": s["lse"]}


# ---- the definition in 64 bits ----

def _turn(c, x, seqs, starts, lens):
    """Rows as complex numbers times magnitude e^(i angle), sequence by sequence."""
    R, L = c["rotary"], c["original"]
    speed = []
    for j in range(R // 2):
        f = math.exp(-2 * j / R * math.log(c["theta"]))
        slow = f / c["factor"]
        if c["scaling"] == "linear":
            f = slow
        elif c["scaling"] == "turns":
            turns = L * f / (2 * math.pi)
            if turns < c["low"]:
                f = slow
            elif turns <= c["high"]:
                f = slow + (f - slow) * (turns - c["low"]) / (c["high"] - c["low"])
        elif c["scaling"] == "index":
            lo, hi = (R / 2 * math.log(L / (t * 2 * math.pi), c["theta"]) for t in (c["high"], c["low"]))
            lo, hi = max(0, math.floor(lo)), min(R - 1, math.ceil(hi))
            part = 0.0 if j <= lo else 1.0 if j >= hi else (j - lo) / (hi - lo)
            f = slow * part + f * (1 - part)
        speed.append(f)
    speed = torch.tensor(speed, dtype=torch.float64, device=DEVICE)
    done = []
    for i in range(seqs):
        a, b = starts[i], starts[i + 1]
        if a == b:
            continue
        y = x[a:b].reshape(b - a, -1, D).double()
        turned, rest = y[..., :R], y[..., R:]
        pairs = torch.stack(turned.chunk(2, -1), -1) if c["style"] == "half" else turned.unflatten(-1, (R // 2, 2))
        pos = torch.arange(lens[i] - (b - a), lens[i], dtype=torch.float64, device=DEVICE)
        w = torch.polar(torch.full((b - a, R // 2), c["magnitude"], dtype=torch.float64, device=DEVICE), pos[:, None] * speed)
        z = torch.view_as_complex(pairs.contiguous())
        z = torch.view_as_real(z / w[:, None] if c["back"] else z * w[:, None])
        z = torch.cat((z[..., 0], z[..., 1]), -1) if c["style"] == "half" else z.flatten(-2)
        done.append(torch.cat((z, rest), -1))
    return torch.cat(done)


def _nearest8(x):
    """The values that rows [..., 128] stand for in 8 bits: the nearest of the grid, the even one of two equally near."""
    grid = sorted({(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)} | {m * 2.0 ** -9 for m in range(8)})[:127]      # (the 128th is no number)
    grid = torch.tensor(grid, dtype=torch.float64, device=DEVICE)
    b = x.reshape(*x.shape[:-1], 4, 32)
    top = b.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -126)))
    e = (torch.where(top > 1.8125 * torch.exp2(e), e + 1, e) - 8).clamp(min=-124)
    y = b.abs() / torch.exp2(e)
    up = torch.searchsorted(grid, y.contiguous()).clamp(max=126)
    dn = (up - 1).clamp(min=0)
    du, dd = grid[up] - y, y - grid[dn]
    pick = torch.where((du < dd) | ((du == dd) & (up % 2 == 0)), up, dn)
    return (grid[pick] * torch.exp2(e) * torch.sign(b)).reshape(x.shape)


def _exact_attend(s):
    c, T, heads = s["case"], s["case"]["page"], s["case"]["heads"]
    group = c["q_heads"] // heads
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    out = torch.empty(s["n"], heads, group, D, dtype=torch.float64, device=DEVICE)
    lse = torch.empty(s["n"], heads, group, dtype=torch.float64, device=DEVICE)
    for i in range(c["seqs"]):
        n, length = starts[i + 1] - starts[i], lens[i]
        if not n:
            continue
        first = length - n
        keep = torch.arange(length, device=DEVICE)
        if c["hole"]:
            b, e = s["hole"][i].tolist()
            keep = torch.cat((keep[:b], keep[e:]))
        elif c["window"]:
            keep = keep[(keep < c["sink"]) | (keep > first - c["window"])]
        if c["op"] == "prompt":
            rows = keep + int(s["k_starts"][i])
            k, v = (s[x][rows].double().reshape(-1, heads, D) for x in ("k", "v"))
        else:
            page, at, kv = s["table"][i].long()[keep // T], keep % T, []
            for pool in (s["pool_k"], s["pool_v"]):
                code = pool[..., :T * D].unflatten(-1, (T, D))[page, :, at].int()
                e8 = pool[..., T * D:].unflatten(-1, (T, 4))[page, :, at].double()
                ex, m = (code >> 3 & 15).double(), (code & 7).double()
                x = torch.where(ex == 0, m * 2.0 ** -9, (8 + m) * torch.exp2(ex - 10)) * (1 - 2 * (code >> 7).double())
                kv.append(x * torch.exp2(e8 - 127).repeat_interleave(32, -1))
            k, v = kv
        pos = torch.arange(first, length, device=DEVICE)[:, None]
        see = keep <= pos
        if c["window"]:
            see = see & ((keep > pos - c["window"]) | (keep < c["sink"]))
        see = see.repeat_interleave(group, 0)
        for h in range(heads):
            x = s["q"][starts[i]:starts[i + 1]].reshape(n, heads, group, D)[:, h].double().reshape(n * group, D)
            score = (x @ k[:, h].T) / math.sqrt(D)
            score = torch.where(see, score, torch.full((), -math.inf, dtype=torch.float64, device=DEVICE))
            one = torch.logsumexp(score, -1)
            out[starts[i]:starts[i + 1], h] = (torch.exp(score - one[:, None]) @ v[:, h]).reshape(n, group, D)
            lse[starts[i]:starts[i + 1], h] = one.reshape(n, group)
    out, lse = out.reshape(s["n"], -1, D), lse.reshape(s["n"], -1)
    if _joined(c):
        pl, po = s["part_lse"].double(), s["part_out"].double()
        both = torch.logsumexp(torch.stack((lse, pl)), 0)
        out, lse = torch.exp(lse - both)[..., None] * out + torch.exp(pl - both)[..., None] * po, both
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("prompt", "attend8"):
        return _exact_attend(s)
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    k, q = (_turn(case, s[x], case["seqs"], starts, lens) for x in ("k", "q"))
    if case["op"] == "rotate":
        return {"k": k, "q": q}
    return {"q": q, "k": _nearest8(k), "v": _nearest8(s["v"].reshape(s["n"], -1, D).double())}
