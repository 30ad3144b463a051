"""Cases of rotary positions, of the paged cache in 4 bits, and of what joins them, with their plain forms.

kind      one pass is
rotary    query and key rows of a step or prompt turned by their positions, or their gradients turned back
append    packed new rows of one layer into the paged cache in 8 bits, keys (and queries) rotated on the way
store     the same into the cache in 4 bits, and the rows read back as bf16, as the next piece of a prompt takes them
attn      attention of the draft rows of one layer over the cache in 4 bits

The cache in 4 bits of one layer holds blocks of 64 tokens as e2m1 codes with a power of two per 32 of them:
of a key 32 channels of a token share one, of the values 32 tokens of a channel.  A block lies in the order in
which matrix instructions take it.  The block that is still open and the draft rows behind it are bf16 rows of a
ring of 128 per sequence and kv head (position p at row p % 128).

Sizes: the benchmark's configurations (2048 to 65536 cached keys, 8 / 2 to 64 / 8 heads, one to four
sequences), and batches of up to 32 sequences of unequal lengths as a server holds them.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

own = False

T, RING = 64, 128                  # tokens of a block, rows of the ring
DEV = "cuda:0"
F8 = torch.float8_e4m3fn
MOST_BYTES = 6.0e8                 # a drawn case moves no more than this
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}

ROTARY = dict(kind="rotary", rows=80, Hq=40, Hkv=8, D=128, dim=128, axes=1, interleaved=False, back=False, far=20000,
              dtype="bf16", factor=1.0)
APPEND = dict(kind="append", B=1, Hq=40, Hkv=8, n_lo=16384, n_hi=16384, start=0, draft=False, dim=128, axes=3,
              interleaved=False)
STORE = dict(APPEND, kind="store")
ATTN = dict(kind="attn", B=1, gamma=5, branches=1, Hq=40, Hkv=8, kv_lo=16384, kv_hi=16384, extras=False)


def listed():
    return [
        # queries and keys of a batch's draft rows, every step and layer
        dict(ROTARY, name="rotary-step"),
        # the prompt of one long video, three positions (time, height, width) a token
        dict(ROTARY, name="rotary-prompt", rows=16384, axes=3),
        # gradients of rows of small heads, a part of each turned, neighbours in pairs, a stretched context's factor
        dict(ROTARY, name="rotary-back", rows=5001, Hq=16, Hkv=16, D=80, dim=40, axes=2, interleaved=True, back=True,
             far=300000, factor=1.1386, dtype="fp32"),
        # the draft rows of a batch of 16 into the cache in 8 bits, with their queries: every step and layer
        dict(APPEND, name="append-drafts", B=16, n_lo=5, n_hi=5, start=16384, draft=True),
        # the prompt of one long video
        dict(APPEND, name="append-prompt", Hq=0),
        # pieces of prompts of unequal lengths behind rows that are there already, half of each head turned
        dict(APPEND, name="append-ragged", B=12, Hq=28, Hkv=4, n_lo=300, n_hi=9000, start=1100, dim=64, axes=1),
        # a long prompt's next piece into the cache in 4 bits, and back
        dict(STORE, name="store-piece", Hq=0, n_lo=2048, n_hi=2048, start=4133),
        # prompts of unequal lengths
        dict(STORE, name="store-ragged", B=12, n_lo=300, n_hi=9000, Hq=0, axes=1, interleaved=True),
        # plain decoding of one token over a short, odd context: the smallest attention
        dict(ATTN, name="decode-short", gamma=1, Hq=8, Hkv=2, kv_lo=777, kv_hi=777),
        # one layer of the 32B shape, five drafts, one user with a video of 16384 tokens
        dict(ATTN, name="verify-16k"),
        # a server's batch: sequences between a short clip and a long one, with log-sum-exp and video mass
        dict(ATTN, name="serve-ragged", B=16, kv_lo=2048, kv_hi=32768, extras=True),
        # long videos, four sequences, draft trees of two chains of four at the 72B shape
        dict(ATTN, name="long-video", B=4, gamma=8, branches=2, Hq=64, kv_lo=65536, kv_hi=65536),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["rotary"] * 3 + ["append"] * 2 + ["store"] * 2 + ["attn"] * 5)
        heads = rng.choice([(8, 2), (28, 4), (40, 8), (64, 8)])
        B = _log(rng, 1, 32)
        if kind == "rotary":
            D = rng.choice([64, 80, 96, 128, 128, 128, 256])
            c = dict(ROTARY, rows=_log(rng, 1, 20000), Hq=heads[0], Hkv=rng.choice([0, heads[1], heads[1]]), D=D,
                     dim=rng.choice([D, D, D // 2, D // 4 * 2, 2 * rng.randint(1, D // 2)]), axes=rng.choice([1, 1, 2, 3]),
                     interleaved=rng.random() < 0.4, back=rng.random() < 0.3, far=_log(rng, 100, 1000000),
                     dtype=rng.choice(["bf16", "bf16", "bf16", "fp16", "fp32"]), factor=rng.choice([1.0, 1.0, 1.1386]))
        elif kind == "attn":
            branches = rng.choice([1, 1, 1, 2, 3])
            hi = _log(rng, 1, 65536)
            c = dict(ATTN, B=B, Hq=heads[0], Hkv=heads[1], kv_hi=hi, branches=branches,
                     kv_lo=hi if rng.random() < 0.4 else max(1, int(hi * rng.uniform(0.02, 1))),
                     gamma=branches * rng.randint(2, 10) if branches > 1 else rng.choice([1, 1, rng.randint(2, 16)]),
                     extras=rng.random() < 0.3)
        else:
            draft = rng.random() < 0.3
            hi = rng.randint(1, 32) if draft else _log(rng, 1, 30000)
            c = dict(APPEND, kind=kind, B=B, Hq=rng.choice([0, heads[0]]), Hkv=heads[1], n_hi=hi, draft=draft,
                     start=rng.choice([0, _log(rng, 1, 20000)]), dim=rng.choice([128, 128, 64, 32, 96]),
                     axes=rng.choice([1, 3]), interleaved=rng.random() < 0.3,
                     n_lo=hi if rng.random() < 0.4 else max(1, int(hi * rng.uniform(0.02, 1))))
        if work(c)["bytes"] <= MOST_BYTES:
            return c


def _spread(n, lo, hi):
    """n lengths evenly over the logarithm between the two ends."""
    return [int(round(lo * (hi / lo) ** ((i + 0.5) / n))) for i in range(n)]


def _shift(v, seed):
    """The same lengths in another order for another seed."""
    return [v[(i * 7 + seed) % len(v) if len(v) % 7 else (i + seed) % len(v)] for i in range(len(v))]


def work(case):
    k = case["kind"]
    if k == "rotary":
        x = case["rows"] * (case["Hq"] + case["Hkv"])
        size = 4 if case["dtype"] == "fp32" else 2
        part = case["rows"] * 4.0 * case["axes"]
        return {"bytes": 2.0 * size * x * case["D"] + part, "flops": 3.0 * x * case["dim"]}
    B, H, D = case["B"], case["Hkv"], 128
    if k == "attn":
        g, nbytes, keys = case["gamma"], 0.0, 0
        for n in _spread(B, case["kv_lo"], case["kv_hi"]):
            full = n // T * T
            nbytes += H * (full * (1.0 * D + D / 16) + (n - full + g) * 4.0 * D) + full // T * 4
            keys += n + g
        nbytes += 4.0 * B * g * case["Hq"] * D + (8.0 * B * g * case["Hq"] if case["extras"] else 0)
        return {"bytes": nbytes, "flops": 4.0 * keys * g * case["Hq"] * D}
    nbytes = flops = 0.0
    of_block = T * 2.0 * D + 8 if k == "append" else T * (1.0 * D + D / 16)      # keys and values of a block
    for n in _spread(B, case["n_lo"], case["n_hi"]):
        start = case["start"]
        done = 0 if case["draft"] else (start + n) // T - start // T
        old = start % T if done else 0                       # rows of the open block, read back
        nbytes += H * (4.0 * D * (n + old) + done * of_block + (n + old - done * T) * 4.0 * D)
        nbytes += n * (4.0 * D * case["Hq"] + 4.0 * case["axes"])
        flops += 3.0 * n * (H + case["Hq"]) * case["dim"]
        if k == "store":                                     # the block that was open, and the new rows
            back = start % T + n
            nbytes += H * (4.0 * D * back + done * of_block + (back - done * T) * 4.0 * D)
    return {"bytes": nbytes, "flops": flops}


# ------------------------------------------------------------------------------ inputs
def _normal(gen, shape, gain=None, dtype=torch.bfloat16):
    """normal rows; `gain` per channel (keys of real models have a few large channels)."""
    x = torch.randn(shape, generator=gen, device=DEV)
    return (x if gain is None else x * gain).to(dtype)


def _gain(gen, D=128):
    return torch.exp(torch.randn((D,), generator=gen, device=DEV) * 0.5)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _frequencies(dim):
    return (10000.0 ** -(torch.arange(0, dim, 2, device=DEV, dtype=torch.float64) / dim)).float()


def _axis(dim, axes):
    """Which of a token's positions a frequency goes by: the first quarter by time, then height and width."""
    i = torch.arange(dim // 2, device=DEV)
    if axes == 1:
        return None
    return (i % 2 if axes == 2 else torch.where(i < dim // 8, 0, torch.where(i < dim * 5 // 16, 1, 2))).to(torch.uint8)


def _grid(gen, rows, axes, far):
    """int32 [axes, rows]: one position a token, or frame, row and column of a video's tokens behind some text."""
    t = torch.arange(rows, device=DEV) + int(torch.randint(max(1, far - rows + 1), (1,), generator=gen, device=DEV))
    if axes == 1:
        return t[None].to(torch.int32)
    w, first = 36, t[0]
    i = t - first
    return torch.stack([first + i // (w * 20), first + i // w % 20, first + i % w][3 - axes:]).to(torch.int32).contiguous()


def _to8(x):
    """[..., T, D] -> (e4m3 of x / s, s): s the smallest power of two with max |x| <= 448 s."""
    x = x.float()
    top = x.abs().amax(dim=(-2, -1))
    m, e = torch.frexp(top)
    s = torch.ldexp(torch.ones_like(top), torch.clamp(torch.where(m <= 0.875, e - 9, e - 8), min=-60))
    return (x / s[..., None, None]).to(F8), s


def _to4(x):
    """[..., 32] -> (e2m1 codes uint8 [..., 32], scale bytes uint8 [...]): the scale is the smallest power of
    two s with max |x| <= 7 s, its byte is the exponent + 127; rounded to nearest, ties to the even code."""
    x = x.float()
    m, e = torch.frexp(x.abs().amax(dim=-1))
    e = torch.clamp(torch.where(m <= 0.875, e - 3, e - 2), min=-60)
    y = torch.ldexp(x, -e[..., None])
    a = y.abs()
    # borders between neighbours; one on a border goes to the even code
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return code.to(torch.uint8) + 8 * torch.signbit(y).to(torch.uint8), (e + 127).to(torch.uint8)


def _pack(codes):
    return codes[..., 0::2] | codes[..., 1::2] << 4


def _pack_keys(x):
    """[..., 64 tokens, 128] -> bytes [..., 2, 64, 32] and scales [..., 2, 32, 4] of a block: channels in halves
    of 64; scale of tokens t and channels 64 a + 32 g .. + 31 at [g, t % 32, 2 (t / 32) + a]."""
    c, s = _to4(x.unflatten(-1, (2, 2, 32)))                  # [..., t, a, g, 32], [..., t, a, g]
    s = s.unflatten(-3, (2, 32)).movedim(-1, -4).movedim(-3, -2)              # [..., g, t % 32, t / 32, a]
    return _pack(c.flatten(-2)).movedim(-2, -3).contiguous(), s.flatten(-2).contiguous()


def _pack_values(x):
    """[..., 64 tokens, 128] -> bytes [..., 128, 32] and scales [..., 2, 32, 4]: of a channel first the tokens with
    bit 2 clear, then the others; scale of half h and channel c at [h, c % 32, c / 32]."""
    c, s = _to4(x.transpose(-1, -2).unflatten(-1, (8, 2, 4)).transpose(-2, -3).flatten(-2))       # [..., c, h, 32]
    return _pack(c).flatten(-2).contiguous(), s.unflatten(-2, (4, 32)).movedim(-1, -3).transpose(-1, -2).contiguous()


def _blocks4(gen, n, H, gain):
    """n blocks of a pool in 4 bits."""
    k4, v4 = (torch.empty(x, dtype=torch.uint8, device=DEV) for x in ((n, H, 2, T, 32), (n, H, 128, 32)))
    ks, vs = (torch.empty((n, H, 2, 32, 4), dtype=torch.uint8, device=DEV) for _ in range(2))
    for a in range(0, n, 1024):
        b = min(n, a + 1024)
        k4[a:b], ks[a:b] = _pack_keys(_normal(gen, (b - a, H, T, 128), gain))
        v4[a:b], vs[a:b] = _pack_values(_normal(gen, (b - a, H, T, 128)))
    return k4, v4, ks, vs


def _tree(branches, chain):
    """Which draft rows a row sees: bit j of entry i."""
    return [((1 << (i + 1)) - 1) << (a * chain) for a in range(branches) for i in range(chain)]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(20260405 + int(seed))
    kind = case["kind"]
    s = {"case": case}
    if kind == "rotary":
        n, D, dt = case["rows"], case["D"], TYPES[case["dtype"]]
        s["q"] = _normal(gen, (n, case["Hq"], D), dtype=dt)
        s["k"] = _normal(gen, (n, case["Hkv"], D), _gain(gen, D), dtype=dt) if case["Hkv"] else None
        s["pos"] = _grid(gen, n, case["axes"], case["far"])
    elif kind == "attn":
        B, H, g = case["B"], case["Hkv"], case["gamma"]
        lens = _shift(_spread(B, case["kv_lo"], case["kv_hi"]), seed)
        cols = max(lens) // T + 1
        need = [n // T for n in lens]
        pool = sum(need) + 3                                  # pages of a pool that holds others too
        gain = _gain(gen)
        s["cache"] = (*_blocks4(gen, pool, H, gain), _normal(gen, (B, H, RING, 128), gain), _normal(gen, (B, H, RING, 128)))
        order = torch.randperm(pool, generator=gen, device=DEV).to(torch.int32)
        s["table"] = torch.full((B, cols), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b, n in enumerate(need):
            s["table"][b, :n] = order[at:at + n]
            at += n
        s["kv_len"] = _i32(lens)
        s["q"] = _normal(gen, (B, g, case["Hq"], 128))
        s["vis"] = (torch.full_like(s["kv_len"], 16), torch.clamp(16 + s["kv_len"] * 7 // 8, max=max(lens)))
        s["mask"] = _tree(case["branches"], g // case["branches"])
        return s
    else:
        B, H, Hq = case["B"], case["Hkv"], case["Hq"]
        news = _shift(_spread(B, case["n_lo"], case["n_hi"]), seed)
        n, start = sum(news), case["start"]
        base = start // T
        done = [0 if case["draft"] else (start + x) // T for x in news]
        pool = sum(max(0, d - base) for d in done) + 1
        gain = _gain(gen)
        s["k"], s["v"] = _normal(gen, (n, H, 128), gain), _normal(gen, (n, H, 128))
        s["q"] = _normal(gen, (n, Hq, 128)) if Hq else None
        tails = [_normal(gen, (B, H, RING, 128), g) for g in (gain, None)]
        if kind == "append":
            shapes = ((pool, H, T, 128), F8), ((pool, H, 128, T), F8), ((pool, H), torch.float32), ((pool, H), torch.float32)
        else:
            u8 = torch.uint8
            shapes = ((pool, H, 2, T, 32), u8), ((pool, H, 128, 32), u8), ((pool, H, 2, 32, 4), u8), ((pool, H, 2, 32, 4), u8)
        s["cache"] = (*(torch.zeros(x, dtype=d, device=DEV) for x, d in shapes), *tails)
        # the maps of a plan: rows of blocks that become complete name their place in the pool
        blocks = torch.randperm(pool, generator=gen, device=DEV)
        slots, back, at, cu = [], [], 0, [0]
        for b, x in enumerate(news):
            p = torch.arange(base * T, start + x, device=DEV)
            ids = blocks[(at + p // T - base).clamp(max=pool - 1)] * T + p % T
            place = torch.where(p < done[b] * T, ids, -2 - (b * RING + p % RING))
            slots.append(place[start - base * T:])
            back.append(place)
            at += max(0, done[b] - base)
            cu.append(cu[-1] + x)
        s["cu_rows"], s["slots"], s["back"] = _i32(cu), torch.cat(slots).to(torch.int32), torch.cat(back).to(torch.int32)
        s["row_seq"] = torch.repeat_interleave(torch.arange(B, device=DEV), _i32(news)).to(torch.int32)
        s["row_pos"] = torch.cat([torch.arange(start, start + x, device=DEV) for x in news]).to(torch.int32)
        # one position a token is its place in the cache; a video's tokens have three, others than their places
        s["pos"] = None if case["axes"] == 1 else _grid(gen, n, case["axes"], start + n)
    s["inv_freq"], s["axis"] = _frequencies(case["dim"]), _axis(case["dim"], case["axes"])
    return s


# ------------------------------------------------------------------------------ plain forms
def _angles(s):
    """float64 [rows, dim / 2]"""
    pos = s["row_pos"][None] if s.get("pos") is None else s["pos"]
    pos = pos.double().T
    return (pos if s["axis"] is None else pos[:, s["axis"].long()]) * s["inv_freq"].double()


def _turn(x, cos, sin, interleaved):
    """x [rows, H, D] in the type of cos and sin [rows, dim / 2]."""
    half = cos.shape[1]
    c, n = cos[:, None], sin[:, None]
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    y = (a * c - b * n, b * c + a * n)
    turned = torch.stack(y, -1).flatten(-2) if interleaved else torch.cat(y, -1)
    return torch.cat([turned, x[..., 2 * half:]], -1)


def _plain_rotary(s):
    c = s["case"]
    angles = _angles(s)
    cos, sin = (angles.cos() * c["factor"]).float(), (angles.sin() * (-c["factor"] if c["back"] else c["factor"])).float()
    return {x: _turn(s[x].float(), cos, sin, c["interleaved"]).to(s[x].dtype) for x in ("q", "k") if s[x] is not None}


def _plain_rows(s):
    """Rotated keys and queries, rounded to bf16.  In 64 bits: the codes behind have borders."""
    angles = _angles(s)
    cos, sin = angles.cos(), angles.sin()
    return [None if s[x] is None else _turn(s[x].double(), cos, sin, s["case"]["interleaved"]).to(torch.bfloat16) for x in ("k", "q")]


def _plain_store(s, k, four):
    """Rows into the cache: the ring and, where a block becomes complete, the pool."""
    kp, vp, ks, vs, kt, vt = s["cache"]
    slots, seq, pos, cu = (s[x].long() for x in ("slots", "row_seq", "row_pos", "cu_rows"))
    last = torch.nonzero((slots >= 0) & (slots % T == T - 1))[:, 0]
    row = last[:, None] + torch.arange(1 - T, 1, device=DEV)                # [blocks, T] packed rows of a block
    there = (row < cu[seq[last]][:, None])[..., None, None]                 # or rows of the ring
    ring = ((pos[last][:, None] + torch.arange(1 - T, 1, device=DEV)) % RING).clamp(min=0)
    open_ = torch.nonzero(slots <= -2)[:, 0]
    to = -2 - slots[open_]
    for x, tail, pool, scale, values in ((k, kt, kp, ks, False), (s["v"], vt, vp, vs, True)):
        old = tail.transpose(1, 2)[seq[last][:, None], ring]                # [blocks, T, Hkv, D]
        rows = torch.where(there, old, x[row.clamp(min=0)]).transpose(1, 2)
        if four:
            q, sc = (_pack_values if values else _pack_keys)(rows)
        else:
            q, sc = _to8(rows)
            q = q.transpose(-1, -2) if values else q
        pool[slots[last] // T] = q
        scale[slots[last] // T] = sc
        tail[to // RING, :, to % RING] = x[open_]


def _cache_out(s):
    """Codes of 8 bits are the values they stand for; those of 4 bits are read back instead."""
    names = ("k8", "v8", "k_scale", "v_scale", "k_tail", "v_tail")
    return {n: x for n, x in zip(names, s["cache"]) if x.dtype != torch.uint8 or "scale" in n}


def _plain_append(s):
    k, q = _plain_rows(s)
    _plain_store(s, k, False)
    return dict(_cache_out(s), **({} if q is None else {"q": q}))


def _values4(x):
    """bytes [..., n] of two codes -> float32 [..., 2 n]"""
    both = torch.stack([x & 15, x >> 4], -1).flatten(-2).to(torch.int32)
    m = both & 7
    a = torch.where(m < 4, m * 0.5, torch.where(m < 6, m - 2.0, 2.0 * m - 8.0))
    return torch.where(both >= 8, -a, a)


def _power(e):
    """Values of scale bytes."""
    return torch.ldexp(torch.ones_like(e, dtype=torch.float32), e.to(torch.int32) - 127)


def _keys4(k4, ks):
    """bytes [..., 2, 64, 32], scales [..., 2, 32, 4] -> float32 [..., 64 tokens, 128]"""
    x = _values4(k4).unflatten(-1, (2, 32)).movedim(-4, -3)                   # [..., t, a, g, 32]
    e = _power(ks).unflatten(-1, (2, 2)).movedim(-4, -1).transpose(-4, -3)    # [..., t / 32, t % 32, a, g]
    return (x * e.flatten(-4, -3)[..., None]).flatten(-3)


def _vals4(v4, vs):
    """bytes [..., 128, 32], scales [..., 2, 32, 4] -> float32 [..., 64 tokens, 128]"""
    x = _values4(v4).unflatten(-1, (2, 32))                                   # [..., c, h, 32]
    e = _power(vs).transpose(-1, -2).movedim(-3, -1).flatten(-3, -2)          # [..., c, h]
    x = (x * e[..., None]).unflatten(-1, (8, 4)).transpose(-2, -3)            # [..., c, t / 8, h, 4]
    return x.flatten(-3).transpose(-1, -2)


def _plain_store4(s):
    k, q = _plain_rows(s)
    _plain_store(s, k, True)
    kp, vp, ks, vs, kt, vt = s["cache"]
    at = s["back"].long()
    whole = (at >= 0)[:, None, None]
    ring = (-2 - at).clamp(min=0)
    r = {}
    for name, pool, tail in (("k_back", _keys4(kp, ks), kt), ("v_back", _vals4(vp, vs), vt)):
        rows = pool.to(torch.bfloat16).transpose(1, 2).flatten(0, 1)          # [places, Hkv, D]
        r[name] = torch.where(whole, rows[at.clamp(min=0)], tail.transpose(1, 2).flatten(0, 1)[ring])
    return dict(_cache_out(s), **r, **({} if q is None else {"q": q}))


def _plain_attn(s):
    c = s["case"]
    B, g, H, G, D = c["B"], c["gamma"], c["Hkv"], c["Hq"] // c["Hkv"], 128
    k4, v4, ks, vs, kt, vt = s["cache"]
    n = s["kv_len"].long()
    blocks = s["table"].shape[1]
    ids = s["table"][:, :blocks].long().clamp(min=0)
    base = n // T * T
    ring = (base[:, None] + torch.arange(T + g - 1, device=DEV)) % RING

    def rows(x, tail):
        x = x[ids].transpose(1, 2).reshape(B, H, blocks * T, D)               # [B, blocks, Hkv, T, D]
        return torch.cat([x, torch.gather(tail, 2, ring[:, None, :, None].expand(B, H, -1, D)).float()], 2)

    key = torch.cat([torch.arange(blocks * T, device=DEV).expand(B, -1), base[:, None] + torch.arange(T + g - 1, device=DEV)], 1)
    pooled = torch.arange(key.shape[1], device=DEV) < blocks * T
    j = key - n[:, None]                                                    # draft row of a key, or a committed key
    sees = torch.tensor([[m >> i & 1 for i in range(32)] for m in s["mask"]], dtype=torch.bool, device=DEV)
    drafts = sees[:, j.clamp(0, 31)].transpose(0, 1) & ((j >= 0) & (j < g))[:, None]
    visible = torch.where(pooled, (key < base[:, None])[:, None], (j < 0)[:, None] | drafts)   # [B, g, keys]
    q = s["q"].float().view(B, g, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, g * G, D)
    z = torch.matmul(q, rows(_keys4(k4, ks), kt).transpose(-1, -2).contiguous()) * D ** -0.5
    z = z.view(B, H, g, G, -1).masked_fill_(~visible[:, None, :, None], float("-inf"))
    top = z.amax(-1, keepdim=True)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True, dtype=torch.float64)
    video = ((key >= s["vis"][0][:, None]) & (key < s["vis"][1][:, None]))[:, None, None, None]
    mass = torch.where(video, p, 0.0).sum(-1, dtype=torch.float64) / total[..., 0] if c["extras"] else None
    o = torch.matmul(p.view(B, H, g * G, -1), rows(_vals4(v4, vs), vt)).view(B, H, g, G, D) / total
    r = {"out": o.permute(0, 2, 1, 3, 4).reshape(B, g, H * G, D).to(torch.bfloat16)}
    if c["extras"]:
        rows_of = lambda x: x.permute(0, 1, 3, 2).reshape(B, H * G, g).float()  # noqa: E731
        r["lse"] = rows_of((top.double() + total.log())[..., 0])
        r["vis_mass"] = rows_of(mass)
    return r


# ------------------------------------------------------------------------------ the framework's calls
def _calls(s):
    """What a serving loop lays out once for these buffers: argument structures, outputs, workspace."""
    from paper_2604_05650_amd import binding as L
    c, lib = s["case"], L.raw()
    if c["kind"] == "attn":
        B, out, more, opt = c["B"], torch.empty_like(s["q"]), {}, {}
        if c["extras"]:
            more = {x: torch.empty((B, c["Hq"], c["gamma"]), device=DEV) for x in ("lse", "vis_mass")}
            opt = dict(vis_begin=s["vis"][0], vis_end=s["vis"][1])
        if c["branches"] > 1:
            opt["draft_mask"] = s["mask"]
        a = L.verify_attn_paged_mx_args(s["q"], L.PagedMxCache(*s["cache"]), s["table"], s["kv_len"], out=out, **opt, **more)
        space = torch.empty((lib.lvspec_verify_attn_paged_mx_workspace(C.byref(a)),), dtype=torch.uint8, device=DEV)
        a.workspace, a.workspace_bytes = space.data_ptr(), space.numel()
        return [(lib.lvspec_verify_attn_paged_mx, a)], dict(more, out=out), space
    rot = L.Rotary(s["inv_freq"], axis=s["axis"], interleaved=c["interleaved"], factor=c.get("factor", 1.0))
    q = None if s["q"] is None else torch.empty_like(s["q"])
    if c["kind"] == "rotary":
        k = None if s["k"] is None else torch.empty_like(s["k"])
        a = L.rotary_args(s["q"], s["pos"], rot, out=q, k=s["k"], k_out=k, transpose=c["back"])
        return [(lib.lvspec_rotary, a)], {n: x for n, x in (("q", q), ("k", k)) if x is not None}, None
    outs = dict(_cache_out(s), **({} if q is None else {"q": q}))
    if c["kind"] == "append":
        a = L.paged_append_rotary_args(L.PagedCache(*s["cache"]), s["k"], s["v"], s, rot, pos=s["pos"], q=s["q"], q_out=q)
        return [(lib.lvspec_paged_append_rotary, a)], outs, None
    cache = L.PagedMxCache(*s["cache"])
    back = {x: torch.empty((len(s["back"]), c["Hkv"], 128), dtype=torch.bfloat16, device=DEV) for x in ("k_back", "v_back")}
    a = L.paged_mx_append_args(cache, s["k"], s["v"], s, rot=rot, pos=s["pos"], q=s["q"], q_out=q)
    b = L.paged_mx_read_args(cache, s["back"], k=back["k_back"], v=back["v_back"])
    return [(lib.lvspec_paged_mx_append, a), (lib.lvspec_paged_mx_read, b)], dict(outs, **back), None


def run(s):
    if own:
        if "calls" not in s:
            s["calls"] = _calls(s)
        calls, outs, _ = s["calls"]
        stream = torch.cuda.current_stream().cuda_stream
        for fn, a in calls:
            rc = fn(C.byref(a), stream)
            if rc != 0:
                raise RuntimeError(f"status {rc}")
        return outs
    return {"rotary": _plain_rotary, "append": _plain_append, "store": _plain_store4, "attn": _plain_attn}[s["case"]["kind"]](s)


# ------------------------------------------------------------------------------ from the definitions, in 64 bits
def _exact_turn(x, pos, inv_freq, axis, interleaved, factor, back):
    """Every pair a complex number, turned by multiplication."""
    z = x.double()
    half = inv_freq.numel()
    p = torch.stack([pos[0 if axis is None else int(axis[i])].double() for i in range(half)], 1)
    w = torch.polar(torch.full_like(p, factor), (-1.0 if back else 1.0) * p * inv_freq.double())[:, None]
    i = torch.arange(half, device=z.device)
    re, im = (2 * i, 2 * i + 1) if interleaved else (i, half + i)
    t = torch.complex(z[..., re], z[..., im]) * w
    y = z.clone()
    y[..., re], y[..., im] = t.real, t.imag
    return y


def _nearest(y, bits, least):
    """To the nearest number of `bits` fraction bits, ties to even, steps no finer than those at 2^least."""
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(y.abs().clamp(min=1e-300))), min=least) - bits)
    return torch.round(y / step) * step


def _exact8(x):
    """[..., T, D] float64 -> (the values of the codes, scale)."""
    s = torch.exp2(torch.clamp(torch.ceil(torch.log2(x.abs().amax(dim=(-2, -1)) / 448.0)), min=-60.0))
    return _nearest(x / s[..., None, None], 3.0, -6.0), s


def _exact4(x):
    """[..., 32] float64 -> (the values that the codes stand for, scale)."""
    s = torch.exp2(torch.clamp(torch.ceil(torch.log2(x.abs().amax(dim=-1) / 7.0)), min=-60.0))[..., None]
    return torch.clamp(_nearest(x / s, 1.0, 0.0), -6.0, 6.0) * s, s


def _decode(k4, ks, v4, vs):
    """Values of a head's blocks, from the layout's definition: float64 [blocks * 64, 128] keys and values."""
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device=k4.device)
    t, ch = torch.arange(T, device=k4.device)[:, None], torch.arange(128, device=k4.device)[None]
    byte = k4[:, ch // 64, t, ch % 64 // 2]
    K = grid[(torch.where(ch % 2 == 1, byte >> 4, byte) & 15).long()]
    K = K * torch.exp2(ks[:, ch // 32 % 2, t % 32, 2 * (t // 32) + ch // 64].double() - 127.0)
    h = t // 4 % 2
    e = t // 8 * 4 + t % 4
    byte = v4[:, ch, (32 * h + e) // 2]
    V = grid[(torch.where(e % 2 == 1, byte >> 4, byte) & 15).long()]
    V = V * torch.exp2(vs[:, h, ch % 32, ch // 32].double() - 127.0)
    return K.reshape(-1, 128), V.reshape(-1, 128)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotary":
        args = (s["pos"], s["inv_freq"], s["axis"], case["interleaved"], case["factor"], case["back"])
        return {x: _exact_turn(s[x], *args) for x in ("q", "k") if s[x] is not None}
    B, H = case["B"], case["Hkv"]
    if kind == "attn":
        g, G = case["gamma"], case["Hq"] // H
        k4, v4, ks, vs, kt, vt = s["cache"]
        out = torch.empty((B, g, case["Hq"], 128), dtype=torch.float64, device=DEV)
        lse, mass = (torch.empty((B, case["Hq"], g), dtype=torch.float64, device=DEV) for _ in range(2))
        for b, n in enumerate(s["kv_len"].tolist()):
            ids = s["table"][b, :n // T].long()
            tail = [p % RING for p in range(n // T * T, n + g)]
            ok = torch.zeros((g, n + g), dtype=torch.bool, device=DEV)
            ok[:, :n] = True
            for i, m in enumerate(s["mask"]):
                for j in range(g):
                    ok[i, n + j] = bool(m >> j & 1)
            for h in range(H):
                K, V = _decode(k4[ids, h], ks[ids, h], v4[ids, h], vs[ids, h])
                K, V = torch.cat([K, kt[b, h, tail].double()]), torch.cat([V, vt[b, h, tail].double()])
                z = (s["q"][b, :, h * G:(h + 1) * G].double().reshape(g * G, 128) @ K.T).view(g, G, -1) / math.sqrt(128)
                z = torch.where(ok[:, None], z, float("-inf"))
                w = torch.softmax(z, -1)
                out[b, :, h * G:(h + 1) * G] = (w.view(g * G, -1) @ V).view(g, G, 128)
                lse[b, h * G:(h + 1) * G] = torch.logsumexp(z, -1).T
                mass[b, h * G:(h + 1) * G] = w[..., int(s["vis"][0][b]):int(s["vis"][1][b])].sum(-1).T
        return dict(out=out, **(dict(lse=lse, vis_mass=mass) if case["extras"] else {}))
    pos = s["row_pos"][None] if s["pos"] is None else s["pos"]
    turn = lambda x: _exact_turn(x, pos, s["inv_freq"], s["axis"], case["interleaved"], 1.0, False)  # noqa: E731
    q = {} if s["q"] is None else {"q": turn(s["q"])}
    slots, cu, start = s["slots"].tolist(), s["cu_rows"].tolist(), case["start"]
    tails = {"k": s["cache"][4].double(), "v": s["cache"][5].double()}
    new = {"k": turn(s["k"]).to(torch.bfloat16).double(), "v": s["v"].double()}      # (the cache's rows are bf16)
    r = dict(zip(("k8", "v8", "k_scale", "v_scale"), (x.double() for x in s["cache"][:4]))) if kind == "append" else {}
    back = {"k": [], "v": []}
    for x in ("k", "v"):
        for b in range(B):
            n, old = cu[b + 1] - cu[b], start % T
            ring = [(start - old + i) % RING for i in range(old + n)]
            line = torch.cat([tails[x][b][:, ring[:old]].transpose(0, 1), new[x][cu[b]:cu[b + 1]]])
            whole = 0 if case["draft"] else (old + n) // T
            held = line[:whole * T].view(whole, T, H, 128).transpose(1, 2)              # [blocks, H, T, 128]
            if kind == "append" and whole:
                at = torch.tensor([slots[cu[b] + (i + 1) * T - 1 - old] // T for i in range(whole)], device=DEV)
                codes, r[x + "_scale"][at] = _exact8(held)
                r[x + "8"][at] = codes.transpose(-1, -2) if x == "v" else codes
            elif whole:
                if x == "k":
                    held = _exact4(held.unflatten(-1, (4, 32)))[0].flatten(-2)
                else:
                    half = [[t for t in range(T) if t // 4 % 2 == h] for h in (0, 1)]
                    both = held.clone()
                    for tokens in half:
                        both[:, :, tokens] = _exact4(held[:, :, tokens].transpose(-1, -2))[0].transpose(-1, -2)
                    held = both
            back[x].append(torch.cat([held.transpose(1, 2).reshape(-1, H, 128), line[whole * T:]]))
            for j in range(max(whole * T, old), old + n):
                tails[x][b][:, ring[j]] = line[j]
    r.update(k_tail=tails["k"], v_tail=tails["v"])
    if kind == "store":
        # (scales are whole numbers)
        r.update(k_scale=None, v_scale=None, **{x + "_back": torch.cat(back[x]) for x in ("k", "v")})
    return dict(r, **q)
