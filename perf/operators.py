"""Cases of the operators on the paged cache in 8 bits, and their plain forms.

The cache of one layer holds blocks of 64 tokens.  A complete block is in e4m3 with one scale per
kv head for its keys and one for its values, both powers of two; the values lie transposed in their
block.  The block that is still open, and the draft rows behind it, are bf16 rows of a ring of 128
per sequence and kv head (position p at row p % 128).  A table names the blocks of a sequence.

kind      one pass is
plan      block tables, row offsets and slot maps from request lengths
append    packed new rows of one layer into the cache: complete blocks to 8 bits, the others to the ring
attn      attention of the draft rows of one layer over the cache
commit    a verified step joins the caches of all layers

Sizes: the benchmark's configurations (2048 to 65536 cached keys, 8 / 2 to 64 / 8 heads, one to four
sequences), and batches of up to 64 sequences of unequal lengths as a server holds them.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

own = False

D, T, RING = 128, 64, 128          # head dimension, tokens of a block, rows of the ring
DEV = "cuda:0"
F8 = torch.float8_e4m3fn
MOST_BYTES = 6.0e8                 # a drawn case moves no more than this

ATTN = dict(kind="attn", B=1, gamma=5, branches=1, Hq=40, Hkv=8, kv_lo=16384, kv_hi=16384, extras=False)
APPEND = dict(kind="append", B=1, Hkv=8, n_lo=16384, n_hi=16384, start=0, draft=False)
PLAN = dict(kind="plan", B=16, n_lo=5, n_hi=5, start=16384, draft=True, drop=0)
COMMIT = dict(kind="commit", B=4, Hkv=8, layers=64, branches=1, chain=5, kv=16384, full=1)


def listed():
    return [
        # plain decoding of one token over a short, odd context: the smallest call
        dict(ATTN, name="decode-short", gamma=1, Hq=8, Hkv=2, kv_lo=777, kv_hi=777),
        # one layer of the 32B shape, five drafts, one user with a video of 16384 tokens
        dict(ATTN, name="verify-16k"),
        # the same with a draft tree of two chains of ten tokens
        dict(ATTN, name="tree-16k", gamma=20, branches=2),
        # a server's batch: sequences between a short clip and a long one, with log-sum-exp and video mass
        dict(ATTN, name="serve-ragged", B=16, kv_lo=2048, kv_hi=32768, extras=True),
        # long videos, four sequences, eight drafts at the 72B shape
        dict(ATTN, name="long-video", B=4, gamma=8, Hq=64, kv_lo=65536, kv_hi=65536),
        # the draft rows of a batch, every step and layer
        dict(APPEND, name="append-drafts", B=16, n_lo=5, n_hi=5, start=16384, draft=True),
        # the prompt of one long video
        dict(APPEND, name="append-prompt"),
        # pieces of prompts of unequal lengths behind rows that are there already
        dict(APPEND, name="append-ragged", B=12, n_lo=300, n_hi=9000, start=1100),
        # every step: places of the draft rows, blocks for what may be accepted
        dict(PLAN, name="plan-step"),
        # a wave of new prompts: tables and slots of half a million rows, blocks of finished requests come back
        dict(PLAN, name="plan-prompts", B=64, n_lo=1000, n_hi=16384, start=0, draft=False, drop=4),
        # a verified step of one user: one block of every layer and head becomes complete
        dict(COMMIT, name="commit-chain", B=1),
        # a batch of draft trees, a quarter of the sequences complete a block
        dict(COMMIT, name="commit-tree", B=16, branches=2, chain=10, full=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["attn"] * 6 + ["append"] * 3 + ["plan", "commit"])
        heads = rng.choice([(8, 2), (28, 4), (40, 8), (64, 8)])
        B = _log(rng, 1, 32)
        if kind == "attn":
            branches = rng.choice([1, 1, 1, 2, 3])
            hi = _log(rng, 1, 65536)
            c = dict(ATTN, B=B, Hq=heads[0], Hkv=heads[1], kv_hi=hi, branches=branches,
                     kv_lo=hi if rng.random() < 0.4 else max(1, int(hi * rng.uniform(0.02, 1))),
                     gamma=branches * rng.randint(2, 10) if branches > 1 else rng.choice([1, 1, rng.randint(2, 16)]),
                     extras=rng.random() < 0.3)
        elif kind == "append":
            draft = rng.random() < 0.3
            hi = rng.randint(1, 32) if draft else _log(rng, 1, 40000)
            c = dict(APPEND, B=B, Hkv=heads[1], n_hi=hi, draft=draft, start=rng.choice([0, _log(rng, 1, 20000)]),
                     n_lo=hi if rng.random() < 0.4 else max(1, int(hi * rng.uniform(0.02, 1))))
        elif kind == "plan":
            draft = rng.random() < 0.5
            hi = rng.randint(1, 32) if draft else _log(rng, 1, 40000)
            c = dict(PLAN, B=_log(rng, 1, 256), n_hi=hi, draft=draft, start=rng.choice([0, _log(rng, 1, 40000)]),
                     n_lo=hi if rng.random() < 0.4 else max(1, int(hi * rng.uniform(0.02, 1))), drop=rng.randint(0, 8))
            if c["B"] * hi > 1000000:
                continue
        else:
            branches = rng.choice([1, 1, 2, 3])
            c = dict(COMMIT, B=B, Hkv=heads[1], layers=rng.choice([1, 4, 28, 64]), branches=branches,
                     chain=rng.randint(2, 10) if branches > 1 else rng.randint(1, 16), kv=_log(rng, 100, 20000),
                     full=rng.randint(0, B))
            if c["layers"] * B * c["Hkv"] > 16 * 8 * 64:
                continue
        if work(c)["bytes"] <= MOST_BYTES:
            return c


def _spread(n, lo, hi):
    """n lengths evenly over the logarithm between the two ends."""
    return [int(round(lo * (hi / lo) ** ((i + 0.5) / n))) for i in range(n)]


def _shift(v, seed):
    """The same lengths in another order for another seed."""
    return [v[(i * 7 + seed) % len(v) if len(v) % 7 else (i + seed) % len(v)] for i in range(len(v))]


def work(case):
    k, B = case["kind"], case["B"]
    if k == "plan":
        rows = sum(_spread(B, case["n_lo"], case["n_hi"]))
        return {"bytes": 12.0 * rows + 32.0 * B, "flops": 0.0}
    H = case["Hkv"]
    if k == "attn":
        g, nbytes, keys = case["gamma"], 0.0, 0
        for n in _spread(B, case["kv_lo"], case["kv_hi"]):
            full = n // T * T
            nbytes += H * (full * 2.0 * D + full // T * 8 + (n - full + g) * 4.0 * D) + full // T * 4
            keys += n + g
        nbytes += 4.0 * B * g * case["Hq"] * D + (8.0 * B * g * case["Hq"] if case["extras"] else 0)
        return {"bytes": nbytes, "flops": 4.0 * keys * g * case["Hq"] * D}
    if k == "append":
        nbytes = 0.0
        for n in _spread(B, case["n_lo"], case["n_hi"]):
            start = case["start"]
            done = 0 if case["draft"] else (start + n) // T - start // T
            old = start % T if done else 0                   # rows of the open block, read back
            nbytes += H * (4.0 * D * (n + old) + done * (T * 2.0 * D + 8) + (n + old - done * T) * 4.0 * D)
        return {"bytes": nbytes, "flops": 0.0}
    rows = case["layers"] * H * D * 4.0
    moved = B * case["chain"] / 2 if case["branches"] > 1 else 0
    return {"bytes": rows * (case["full"] * T * 1.5 + 2 * moved) + 12.0 * B, "flops": 0.0}


# ------------------------------------------------------------------------------ inputs
def _normal(gen, shape, gain=None):
    """bf16 normal rows; `gain` per channel (keys of real models have a few large channels)."""
    x = torch.randn(shape, generator=gen, device=DEV)
    return (x if gain is None else x * gain).to(torch.bfloat16)


def _gain(gen):
    return torch.exp(torch.randn((D,), generator=gen, device=DEV) * 0.5)


def _to8(x):
    """[..., T, D] -> (e4m3 of x / s, s): s the smallest power of two with max |x| <= 448 s."""
    x = x.float()
    top = x.abs().amax(dim=(-2, -1))
    m, e = torch.frexp(top)
    s = torch.ldexp(torch.ones_like(top), torch.clamp(torch.where(m <= 0.875, e - 9, e - 8), min=-60))
    return (x / s[..., None, None]).to(F8), s


def _blocks(gen, n, H, gain):
    """n blocks of a pool in 8 bits."""
    k8 = torch.empty((n, H, T, D), dtype=F8, device=DEV)
    v8 = torch.empty((n, H, D, T), dtype=F8, device=DEV)
    ks, vs = (torch.empty((n, H), device=DEV) for _ in range(2))
    for a in range(0, n, 512):
        b = min(n, a + 512)
        k8[a:b], ks[a:b] = _to8(_normal(gen, (b - a, H, T, D), gain))
        q, vs[a:b] = _to8(_normal(gen, (b - a, H, T, D)))
        v8[a:b] = q.transpose(-1, -2)
    return k8, v8, ks, vs


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _tree(branches, chain):
    """Which draft rows a row sees: bit j of entry i."""
    return [((1 << (i + 1)) - 1) << (a * chain) for a in range(branches) for i in range(chain)]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(20260405 + int(seed))
    kind, B = case["kind"], case["B"]
    s = {"case": case}
    if kind == "attn":
        H, g = case["Hkv"], case["gamma"]
        lens = _shift(_spread(B, case["kv_lo"], case["kv_hi"]), seed)
        cols = max(lens) // T + 1
        need = [n // T for n in lens]
        pool = sum(need) + 3                                  # pages of a pool that holds others too
        gain = _gain(gen)
        s["cache"] = (*_blocks(gen, pool, H, gain), _normal(gen, (B, H, RING, D), gain), _normal(gen, (B, H, RING, D)))
        order = torch.randperm(pool, generator=gen, device=DEV).to(torch.int32)
        s["table"] = torch.full((B, cols), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b, n in enumerate(need):
            s["table"][b, :n] = order[at:at + n]
            at += n
        s["kv_len"] = _i32(lens)
        s["q"] = _normal(gen, (B, g, case["Hq"], D))
        s["vis"] = (torch.full_like(s["kv_len"], 16), torch.clamp(16 + s["kv_len"] * 7 // 8, max=max(lens)))
        s["mask"] = _tree(case["branches"], g // case["branches"])
    elif kind == "append":
        H = case["Hkv"]
        news = _shift(_spread(B, case["n_lo"], case["n_hi"]), seed)
        n, start = sum(news), case["start"]
        old, base = start % T, start // T
        done = [0 if case["draft"] else (start + x) // T for x in news]
        pool = sum(max(0, d - base) for d in done) + 1
        gain = _gain(gen)
        s["k"], s["v"] = _normal(gen, (n, H, D), gain), _normal(gen, (n, H, D))
        zero = [torch.zeros(x, dtype=F8, device=DEV) for x in ((pool, H, T, D), (pool, H, D, T))]
        s["cache"] = (*zero, *(torch.zeros((pool, H), device=DEV) for _ in range(2)),
                      _normal(gen, (B, H, RING, D), gain), _normal(gen, (B, H, RING, D)))
        # the maps of a plan: rows of blocks that become complete name their place in the pool
        blocks = torch.randperm(pool, generator=gen, device=DEV)
        slots, at, cu = [], 0, [0]
        for b, x in enumerate(news):
            p = torch.arange(start, start + x, device=DEV)
            ring = -2 - (b * RING + p % RING)
            ids = blocks[(at + p // T - base).clamp(max=pool - 1)] * T + p % T
            slots.append(torch.where(p < done[b] * T, ids, ring))
            at += max(0, done[b] - base)
            cu.append(cu[-1] + x)
        s["cu_rows"], s["slots"] = _i32(cu), torch.cat(slots).to(torch.int32)
        s["row_seq"] = torch.repeat_interleave(torch.arange(B, device=DEV), _i32(news)).to(torch.int32)
        s["row_pos"] = torch.cat([torch.arange(start, start + x, device=DEV) for x in news]).to(torch.int32)
    elif kind == "plan":
        news = _shift(_spread(B, case["n_lo"], case["n_hi"]), seed)
        lens = [case["start"] + (7 * b + int(seed)) % T for b in range(B)] if case["start"] else [0] * B
        held = [n // T for n in lens]
        for i in range(min(case["drop"], B)):                 # finished requests: nothing left, nothing new
            b = (i * 5 + int(seed)) % B
            held[b], lens[b], news[b] = (lens[b] + news[b]) // T + 3, 0, 0
        cols = (case["start"] + T + case["n_hi"] + 32) // T + 4
        pool = sum((case["start"] + T + x + 32) // T + 4 for x in _spread(B, case["n_lo"], case["n_hi"]))
        free = pool - sum(held)
        ids = torch.randperm(pool, generator=gen, device=DEV).to(torch.int32)
        s["table"] = torch.full((B, cols), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b, n in enumerate(held):
            s["table"][b, :n] = ids[at:at + n]
            at += n
        head = (int(seed) * 977) % pool
        s["queue"] = torch.roll(torch.cat([ids[at:], torch.full((at,), -1, dtype=torch.int32, device=DEV)]), head)
        s["state"] = _i32([head, free])
        s["kv_len"], s["n_new"], s["held"] = _i32(lens), _i32(news), _i32(held)
        s["max_rows"] = sum(_spread(B, case["n_lo"], case["n_hi"]))
        s["reserve"] = 32 if case["draft"] else 0
    else:
        H, lay, chain, br = case["Hkv"], case["layers"], case["chain"], case["branches"]
        pool = B + 2
        gain = _gain(gen)
        zero = [torch.zeros(x, dtype=F8, device=DEV) for x in ((lay, pool, H, T, D), (lay, pool, H, D, T))]
        s["cache"] = (*zero, *(torch.zeros((lay, pool, H), device=DEV) for _ in range(2)),
                      _normal(gen, (lay, B, H, RING, D), gain), _normal(gen, (lay, B, H, RING, D)))
        # of a batch's sequences `full` stand right before the end of a block, the others in its first half
        kv = case["kv"] // T * T
        lens = _shift([kv + (T - 1 if b < case["full"] else (5 * b) % 32) for b in range(B)], seed)
        s["table"] = torch.full((B, kv // T + 1), -1, dtype=torch.int32, device=DEV)
        s["table"][:, kv // T] = torch.randperm(pool, generator=gen, device=DEV)[:B]
        s["kv_len"] = _i32(lens)
        s["accept_len"] = torch.randint(1, chain + 1, (B * br,), generator=gen, device=DEV, dtype=torch.int32)
        s["best"] = torch.randint(br, (B,), generator=gen, device=DEV, dtype=torch.int32)
    return s


# ------------------------------------------------------------------------------ plain forms
def _plain_plan(s):
    c, B = s["case"], s["case"]["B"]
    table, queue, n_blocks, rows = s["table"], s["queue"], s["queue"].numel(), s["max_rows"]
    n, new, held = s["kv_len"].long(), s["n_new"].long(), s["held"].long()
    head, count = s["state"][0].long(), s["state"][1].long()
    end = n + new
    done = (n if c["draft"] else end) // T
    need = (end + s["reserve"]) // T
    cu = torch.cat([torch.zeros_like(new[:1]), new.cumsum(0)])
    may = (need <= table.shape[1]) & (cu[1:] <= rows) & (end - done * T <= RING)
    grow, drop = (need - held).clamp(min=0) * may, (held - need).clamp(min=0) * may
    upto = grow.cumsum(0)
    granted = may & ((grow == 0) | (upto <= count))
    grow, drop = grow * granted, drop * granted
    first, behind = upto - grow, drop.cumsum(0) - drop
    col = torch.arange(table.shape[1], device=DEV)
    at = col[None] - held[:, None]
    fresh = queue[((head + first[:, None] + at) % n_blocks).clamp(min=0)]
    keep = table.clone()
    table.copy_(torch.where((at >= 0) & (at < grow[:, None]), fresh, table))
    back = (col[None] >= need[:, None]) & (col[None] < (need + drop)[:, None])
    to = (head + count + behind[:, None] + col[None] - need[:, None]) % n_blocks
    queue[to[back]] = keep[back]
    t = torch.arange(rows, device=DEV)
    b = torch.searchsorted(cu[1:], t, right=True).clamp(max=B - 1)
    real = t < cu[-1]
    pos = n[b] + t - cu[b]
    ids = table[b, (pos // T).clamp(max=table.shape[1] - 1)]
    slot = torch.where(pos < done[b] * T, ids.long() * T + pos % T, -2 - (b * RING + pos % RING))
    slot = torch.where(real & granted[b], slot, -1)
    to32 = lambda x: x.to(torch.int32)  # noqa: E731
    return {"table": table, "queue": queue, "granted": to32(granted), "new_held": to32(held + grow - drop),
            "new_state": to32(torch.stack([(head + grow.sum()) % n_blocks, count - grow.sum() + drop.sum()])),
            "cu_rows": to32(cu), "slots": to32(slot), "row_seq": to32(torch.where(real, b, -1)),
            "row_pos": to32(torch.where(real, pos, -1))}


def _plain_append(s):
    k8, v8, ks, vs, kt, vt = s["cache"]
    slots, seq, pos, cu = (s[x].long() for x in ("slots", "row_seq", "row_pos", "cu_rows"))
    last = torch.nonzero((slots >= 0) & (slots % T == T - 1))[:, 0]
    row = last[:, None] + torch.arange(1 - T, 1, device=DEV)                # [blocks, T] packed rows of a block
    there = (row < cu[seq[last]][:, None])[..., None, None]                 # or rows of the ring
    ring = ((pos[last][:, None] + torch.arange(1 - T, 1, device=DEV)) % RING).clamp(min=0)
    for x, tail, pool, scale, turn in ((s["k"], kt, k8, ks, False), (s["v"], vt, v8, vs, True)):
        old = tail.transpose(1, 2)[seq[last][:, None], ring]                # [blocks, T, Hkv, D]
        q, sc = _to8(torch.where(there, old, x[row.clamp(min=0)]).transpose(1, 2))
        pool[slots[last] // T] = q.transpose(-1, -2) if turn else q
        scale[slots[last] // T] = sc
        open_ = torch.nonzero(slots <= -2)[:, 0]
        to = -2 - slots[open_]
        tail[to // RING, :, to % RING] = x[open_]
    return _cache_out(s)


def _cache_out(s):
    return dict(zip(("k8", "v8", "k_scale", "v_scale", "k_tail", "v_tail"), s["cache"]))


def _plain_attn(s):
    c = s["case"]
    B, g, H, G = c["B"], c["gamma"], c["Hkv"], c["Hq"] // c["Hkv"]
    k8, v8, ks, vs, kt, vt = s["cache"]
    n = s["kv_len"].long()
    blocks = s["table"].shape[1]
    ids = s["table"][:, :blocks].long().clamp(min=0)
    base = n // T * T
    ring = (base[:, None] + torch.arange(T + g - 1, device=DEV)) % RING

    def rows(pool, scale, tail, turned):
        x = pool[ids].float() * scale[ids][..., None, None]                 # [B, blocks, Hkv, T, D] or D, T
        x = (x.permute(0, 2, 1, 4, 3) if turned else x.transpose(1, 2)).reshape(B, H, blocks * T, D)
        t = torch.gather(tail, 2, ring[:, None, :, None].expand(B, H, -1, D)).float()
        return torch.cat([x, t], 2)

    key = torch.cat([torch.arange(blocks * T, device=DEV).expand(B, -1), base[:, None] + torch.arange(T + g - 1, device=DEV)], 1)
    pooled = torch.arange(key.shape[1], device=DEV) < blocks * T
    j = key - n[:, None]                                                    # draft row of a key, or a committed key
    sees = torch.tensor([[m >> i & 1 for i in range(32)] for m in s["mask"]], dtype=torch.bool, device=DEV)
    drafts = sees[:, j.clamp(0, 31)].transpose(0, 1) & ((j >= 0) & (j < g))[:, None]
    visible = torch.where(pooled, (key < base[:, None])[:, None], (j < 0)[:, None] | drafts)   # [B, g, keys]
    q = s["q"].float().view(B, g, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, g * G, D)
    z = torch.matmul(q, rows(k8, ks, kt, False).transpose(-1, -2).contiguous()) * D ** -0.5
    z = z.view(B, H, g, G, -1).masked_fill_(~visible[:, None, :, None], float("-inf"))
    top = z.amax(-1, keepdim=True)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True, dtype=torch.float64)
    video = ((key >= s["vis"][0][:, None]) & (key < s["vis"][1][:, None]))[:, None, None, None]
    mass = torch.where(video, p, 0.0).sum(-1, dtype=torch.float64) / total[..., 0] if c["extras"] else None
    o = torch.matmul(p.view(B, H, g * G, -1), rows(v8, vs, vt, True)).view(B, H, g, G, D) / total
    r = {"out": o.permute(0, 2, 1, 3, 4).reshape(B, g, H * G, D).to(torch.bfloat16)}
    if c["extras"]:
        rows_of = lambda x: x.permute(0, 1, 3, 2).reshape(B, H * G, g).float()  # noqa: E731
        r["lse"] = rows_of((top.double() + total.log())[..., 0])
        r["vis_mass"] = rows_of(mass)
    return r


def _plain_commit(s):
    c, B = s["case"], s["case"]["B"]
    k8, v8, ks, vs, kt, vt = s["cache"]
    n, lanes = s["kv_len"].long(), torch.arange(B, device=DEV)
    best = s["best"].long()
    tau = s["accept_len"].long().view(B, -1)[lanes, best]
    i = torch.arange(c["chain"], device=DEV)
    b, k = torch.nonzero(i[None] < tau[:, None], as_tuple=True)
    full = torch.nonzero((n + tau) // T > n // T)[:, 0]
    ids = s["table"][full, n[full] // T].long()
    ring = ((n[full] // T * T)[:, None] + torch.arange(T, device=DEV)) % RING
    for tail, pool, scale, turn in ((kt, k8, ks, False), (vt, v8, vs, True)):
        tail[:, b, :, (n[b] + k) % RING] = tail[:, b, :, (n[b] + best[b] * c["chain"] + k) % RING]
        rows = tail.transpose(2, 3)[:, full[:, None], ring].transpose(2, 3)     # [layers, blocks, Hkv, T, D]
        q, sc = _to8(rows)
        pool[:, ids] = q.transpose(-1, -2) if turn else q
        scale[:, ids] = sc
    return dict(_cache_out(s), new_len=(n + tau).to(torch.int32))


# ------------------------------------------------------------------------------ the framework's calls
def _call(s):
    """What a serving loop lays out once for these buffers: argument structure, outputs, workspace."""
    from paper_2604_05650_amd import binding as L
    c, B, lib = s["case"], s["case"]["B"], L.raw()
    if c["kind"] == "plan":
        outs = L.alloc_paged_plan(B, s["max_rows"], DEV)
        a = L.paged_plan_args(s["kv_len"], s["n_new"], s["held"], s["queue"], s["state"], s["table"], outs=outs,
                              max_rows=s["max_rows"], reserve=s["reserve"], draft=c["draft"])
        return lib.lvspec_paged_plan, a, dict(outs, table=s["table"], queue=s["queue"]), None
    cache = L.PagedCache(*s["cache"])
    if c["kind"] == "append":
        a = L.paged_append_args(cache, s["k"], s["v"], s)
        return lib.lvspec_paged_append, a, _cache_out(s), None
    if c["kind"] == "attn":
        out, more, opt = torch.empty_like(s["q"]), {}, {}
        if c["extras"]:
            more = {x: torch.empty((B, c["Hq"], c["gamma"]), device=DEV) for x in ("lse", "vis_mass")}
            opt = dict(vis_begin=s["vis"][0], vis_end=s["vis"][1])
        if c["branches"] > 1:
            opt["draft_mask"] = s["mask"]
        a = L.verify_attn_paged_args(s["q"], cache, s["table"], s["kv_len"], out=out, **opt, **more)
        space = torch.empty((lib.lvspec_verify_attn_paged_workspace(C.byref(a)),), dtype=torch.uint8, device=DEV)
        a.workspace, a.workspace_bytes = space.data_ptr(), space.numel()
        return lib.lvspec_verify_attn_paged, a, dict(more, out=out), space
    new_len = torch.empty_like(s["kv_len"])
    a = L.paged_commit_args(cache, s["table"], s["kv_len"], s["accept_len"], c["chain"], best_branch=s["best"],
                            n_branches=c["branches"], new_len=new_len)
    return lib.lvspec_paged_commit, a, dict(_cache_out(s), new_len=new_len), None


def run(s):
    if own:
        if "call" not in s:
            s["call"] = _call(s)
        fn, a, outs, _ = s["call"]
        rc = fn(C.byref(a), torch.cuda.current_stream().cuda_stream)
        if rc != 0:
            raise RuntimeError(f"status {rc}")
        return outs
    return {"plan": _plain_plan, "append": _plain_append, "attn": _plain_attn, "commit": _plain_commit}[s["case"]["kind"]](s)


# ------------------------------------------------------------------------------ from the definitions, in 64 bits
def _exact8(x):
    """[..., T, D] float64 -> (the values of the codes, scale), rounding written out."""
    top = x.abs().amax(dim=(-2, -1))
    s = torch.exp2(torch.clamp(torch.ceil(torch.log2(top / 448.0)), min=-60.0))
    y = x / s[..., None, None]
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(y.abs().clamp(min=1e-300))), min=-6.0) - 3.0)
    return torch.round(y / step) * step, s


def exact(case, seed):
    s = prepare(case, seed)
    kind, B = case["kind"], case["B"]
    if kind == "plan":
        return None                                           # whole numbers
    host = [x.double() if kind != "attn" else x for x in s["cache"]]
    if kind == "attn":
        g, H = case["gamma"], case["Hkv"]
        G = case["Hq"] // H
        k8, v8, ks, vs, kt, vt = host
        out = torch.empty((B, g, case["Hq"], D), dtype=torch.float64, device=DEV)
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
                K = torch.cat([(k8[ids, h].double() * ks[ids, h].double()[:, None, None]).reshape(-1, D), kt[b, h, tail].double()])
                V = torch.cat([(v8[ids, h].double() * vs[ids, h].double()[:, None, None]).transpose(1, 2).reshape(-1, D), vt[b, h, tail].double()])
                z = torch.einsum("igd,kd->igk", s["q"][b, :, h * G:(h + 1) * G].double(), K) / math.sqrt(D)
                z = torch.where(ok[:, None], z, float("-inf"))
                w = torch.softmax(z, -1)
                out[b, :, h * G:(h + 1) * G] = torch.einsum("igk,kd->igd", w, V)
                lse[b, h * G:(h + 1) * G] = torch.logsumexp(z, -1).T
                mass[b, h * G:(h + 1) * G] = w[..., int(s["vis"][0][b]):int(s["vis"][1][b])].sum(-1).T
        return dict(out=out, **(dict(lse=lse, vis_mass=mass) if case["extras"] else {}))
    r = dict(zip(("k8", "v8", "k_scale", "v_scale", "k_tail", "v_tail"), host))
    if kind == "append":
        slots, cu = s["slots"].tolist(), s["cu_rows"].tolist()
        start = case["start"]
        for x, pool, scale, tail in (("k", "k8", "k_scale", "k_tail"), ("v", "v8", "v_scale", "v_tail")):
            rows = s[x].double()
            for b in range(B):
                n, old = cu[b + 1] - cu[b], start % T
                line = torch.cat([r[tail][b][:, [(start - old + i) % RING for i in range(old)]].transpose(0, 1), rows[cu[b]:cu[b + 1]]])
                i = 0
                while i + T <= old + n and slots[cu[b] + i + T - 1 - old] >= 0:
                    q, sc = _exact8(line[i:i + T].transpose(0, 1))
                    at = slots[cu[b] + i + T - 1 - old] // T
                    r[pool][at] = q.transpose(1, 2) if x == "v" else q
                    r[scale][at] = sc
                    i += T
                for j in range(max(i, old), old + n):
                    r[tail][b][:, (start - old + j) % RING] = line[j]
        return r
    for b, n in enumerate(s["kv_len"].tolist()):
        kept = int(s["best"][b])
        tau = int(s["accept_len"][b * case["branches"] + kept])
        for x in ("k", "v"):
            tail = r[x + "_tail"]
            for i in range(tau):
                tail[:, b, :, (n + i) % RING] = tail[:, b, :, (n + kept * case["chain"] + i) % RING]
            if (n + tau) // T > n // T:
                q, sc = _exact8(tail[:, b][:, :, [p % RING for p in range(n // T * T, n // T * T + T)]])
                at = int(s["table"][b, n // T])
                r[x + "8"][:, at] = q.transpose(-1, -2) if x == "v" else q
                r[x + "_scale"][:, at] = sc
    return dict(r, new_len=None)
