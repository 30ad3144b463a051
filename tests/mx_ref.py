"""Plain forms of rotary positions and of the paged cache in 4 bits on the host, in 64 bits, from their definitions."""
import numpy as np
import torch

import paged_ref as R

T, RING, D = R.T, R.RING, R.D
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


# ------------------------------------------------------------------------------ rotation
def rotate(x, pos, inv_freq, *, interleaved=False, axis=None, factor=1.0, transpose=False):
    """x float64 [n, H, D], pos [n] or [n_axes, n], inv_freq binary32 [dim / 2] -> float64.  Pair by pair."""
    pos = np.atleast_2d(np.asarray(pos, np.int64))
    inv = np.asarray(inv_freq, np.float32).astype(np.float64)
    half, y = len(inv), x.copy()
    for i in range(half):
        a = pos[0 if axis is None else int(axis[i])].astype(np.float64) * inv[i]
        c, s = factor * np.cos(a)[:, None], (-factor if transpose else factor) * np.sin(a)[:, None]
        u, v = (2 * i, 2 * i + 1) if interleaved else (i, half + i)
        y[:, :, u], y[:, :, v] = x[:, :, u] * c - x[:, :, v] * s, x[:, :, v] * c + x[:, :, u] * s
    return y


def frequencies(dim, base, scaling=0, scale=1.0, original_len=0.0, beta_fast=32.0, beta_slow=1.0):
    f = np.array([base ** (-2.0 * i / dim) for i in range(dim // 2)])
    if scaling == 1:
        return f / scale, 1.0
    if scaling == 2:
        wide = base * scale ** (dim / (dim - 2.0))
        return np.array([wide ** (-2.0 * i / dim) for i in range(dim // 2)]), 1.0
    if scaling == 3:
        at = lambda n: dim * np.log(original_len / (n * 2 * np.pi)) / (2 * np.log(base))  # noqa: E731
        low, high = max(np.floor(at(beta_fast)), 0.0), min(np.ceil(at(beta_slow)), dim - 1.0)
        r = np.array([min(max((i - low) / (high - low), 0.0), 1.0) if high > low else float(i > low) for i in range(dim // 2)])
        return f * (1 - r) + f / scale * r, 0.1 * np.log(scale) + 1.0 if scale > 1 else 1.0
    return f, 1.0


def to_bf16(x):
    """float64 -> the nearest bf16 (by way of binary32), as float64."""
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


# ------------------------------------------------------------------------------ codes
def nearest4(y):
    """|y| <= 7 -> codes 0 .. 15 of the nearest values, ties to the even code."""
    a = np.abs(y)
    hi = np.clip(np.searchsorted(GRID, a, side="left"), 1, 7)
    up, down = GRID[hi] - a, a - GRID[hi - 1]
    code = np.where(up < down, hi, np.where(up > down, hi - 1, np.where(hi % 2 == 0, hi, hi - 1)))
    return (code | np.where(np.signbit(y), 8, 0)).astype(np.uint8)


def group4(x):
    """float64 [..., 32] -> (codes uint8 [..., 32], scale byte uint8 [...])."""
    bad = ~np.all(np.isfinite(x), axis=-1)
    x = np.where(bad[..., None], 0.0, x)
    top = np.max(np.abs(x), axis=-1)
    e = np.full(top.shape, -60)
    while np.any(top > 7.0 * 2.0 ** e):
        e = e + (top > 7.0 * 2.0 ** e)
    y = x / 2.0 ** e[..., None].astype(np.float64)
    y = np.where(e[..., None] == 126, np.clip(y, -3.0, 3.0), y)
    return np.where(bad[..., None], 0, nearest4(y)).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def value4(codes, byte):
    v = GRID[codes & 7] * np.where(byte == 255, np.nan, 2.0 ** (np.where(byte == 255, 0, byte).astype(np.float64) - 127.0))
    return np.where(codes & 8, -v, v)


def keys_block(x):
    """[64, 128] -> (codes [64, 128], scale bytes [64, 4])."""
    c, s = group4(x.reshape(T, 4, 32))
    return c.reshape(T, D), s


EVEN = [t for t in range(T) if t // 4 % 2 == 0]
ODD = [t for t in range(T) if t // 4 % 2 == 1]


def values_block(x):
    """[64, 128] -> (codes [64, 128], scale bytes [2, 128])."""
    codes, scale = np.zeros((T, D), np.uint8), np.zeros((2, D), np.uint8)
    for g, tokens in enumerate((EVEN, ODD)):
        c, scale[g] = group4(x[tokens].T)
        codes[tokens] = c.T
    return codes, scale


# ------------------------------------------------------------------------------ the cache
def as_numpy(cache):
    """A layer's cache: codes [n, H, 64, 128] and scale bytes by token and group, by half and channel, from the layout's
    definition; rings in float64."""
    k, v, ks, vs, kt, vt = [x.cpu() for x in cache]
    k, v, ks, vs = (x.numpy() for x in (k, v, ks, vs))
    n, H = k.shape[:2]
    kc, vc = (np.zeros((n, H, T, D), np.uint8) for _ in range(2))
    kb, vb = np.zeros((n, H, T, 4), np.uint8), np.zeros((n, H, 2, D), np.uint8)
    for ch in range(D):
        byte = k[:, :, ch // 64, :, ch % 64 // 2]
        kc[:, :, :, ch] = byte >> 4 if ch % 2 else byte & 15
    for t in range(T):
        order, g = (EVEN, 0) if t in EVEN else (ODD, 1)
        e = 32 * g + order.index(t)
        byte = v[:, :, :, e // 2]
        vc[:, :, t] = byte >> 4 if e % 2 else byte & 15
        for c in range(4):                                     # channels 64 a + 32 g ..
            kb[:, :, t, c] = ks[:, :, c % 2, t % 32, 2 * (t // 32) + c // 2]
    for ch in range(D):
        for g in range(2):
            vb[:, :, g, ch] = vs[:, :, g, ch % 32, ch // 32]
    return [kc, vc, kb, vb, kt.double().numpy().copy(), vt.double().numpy().copy()]


def values_of(arr):
    """K and V float64 [n, H, 64, 128] of the pool."""
    kc, vc, kb, vb = arr[:4]
    half = np.array([0 if t in EVEN else 1 for t in range(T)])
    return value4(kc, np.repeat(kb, 32, axis=-1)), value4(vc, vb[:, :, half])


def same_cache(got, ref, what=""):
    for name, x, y in zip(("keys", "values", "key scales", "value scales", "k_tail", "v_tail"), as_numpy(got), ref):
        assert np.array_equal(x, y, equal_nan=x.dtype.kind == "f"), f"{what} {name} {np.argwhere(x != y)[:3].tolist()}"


def append(arr, k, v, plan_, kv_len):
    """arr: as_numpy(), changed; k, v float64 [n, Hkv, D]."""
    cu, slots = plan_["cu_rows"], plan_["slots"]
    for b in range(len(cu) - 1):
        n = max(int(kv_len[b]), 0)
        for x, pool, scale, tail, block in ((k, arr[0], arr[2], arr[4], keys_block), (v, arr[1], arr[3], arr[5], values_block)):
            rows = {p: tail[b, :, p % RING].copy() for p in range(n // T * T, n)}
            for t in range(cu[b], cu[b + 1]):
                rows[n + t - cu[b]] = x[t]
            for t in range(cu[b], cu[b + 1]):
                p, s = n + t - cu[b], int(slots[t])
                if s <= -2:
                    tail[b, :, p % RING] = x[t]
                elif s >= 0 and s % T == T - 1:
                    for h in range(x.shape[1]):
                        pool[s // T, h], scale[s // T, h] = block(np.stack([rows[i][h] for i in range(p - T + 1, p + 1)]))


def attention(q, arr, table, kv_len, mask=None, scale=None, vis=None):
    """As paged_ref.attention, over this cache."""
    B, g, Hq, _ = q.shape
    K4, V4 = values_of(arr)
    kt, vt = arr[4:]
    Hkv, n_blocks, cols = K4.shape[1], len(K4), table.shape[1]
    scale = D ** -0.5 if scale is None else scale
    mask = [(1 << (i + 1)) - 1 for i in range(g)] if mask is None else mask
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    lse, mass = np.zeros((B, Hq, g)), np.zeros((B, Hq, g))
    for b in range(B):
        n = min(max(int(kv_len[b]), 0), cols * T + T - 1)
        ids = [int(table[b, j]) for j in range(n // T)]
        ring = [p % RING for p in range(n // T * T, n + g)]
        there = np.array([ok for i in ids for ok in [0 <= i < n_blocks] * T] + [True] * len(ring))
        for h in range(Hkv):
            K = np.concatenate([K4[i, h] if 0 <= i < n_blocks else np.zeros((T, D)) for i in ids] + [kt[b, h, ring]])
            V = np.concatenate([V4[i, h] if 0 <= i < n_blocks else np.zeros((T, D)) for i in ids] + [vt[b, h, ring]])
            for i in range(g):
                see = there.copy()
                see[n:] = [bool(int(mask[i]) >> j & 1) for j in range(n // T * T - n + len(ring))]
                pos = np.flatnonzero(see)
                for hq in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                    z = K[pos] @ q[b, i, hq] * scale
                    top = z.max()
                    w = np.exp(z - top)
                    s = w.sum()
                    out[b, i, hq], size[b, i, hq] = w @ V[pos] / s, w @ np.abs(V[pos]) / s
                    lse[b, hq, i] = top + np.log(s)
                    if vis is not None:
                        mass[b, hq, i] = w[(pos >= vis[0][b]) & (pos < vis[1][b])].sum() / s
    return out, lse, mass, size


def commit(arr, table, kv_len, accept_len, chain, best=None, n_branches=1):
    """arr: as_numpy() of one layer, changed.  Returns new_len."""
    n_blocks, new = len(arr[0]), []
    for b, n in enumerate(int(x) for x in kv_len):
        kept = int(best[b]) if best is not None and n_branches > 1 else 0
        tau = int(accept_len[b * n_branches + kept])
        j = n // T
        fills = (n + tau) // T > j
        i = int(table[b, j]) if 0 <= j < table.shape[1] else -1
        if n < 0 or n > table.shape[1] * T + T - 1 or (fills and not 0 <= i < n_blocks):
            new.append(n)
            continue
        for tail, pool, scale, block in ((arr[4], arr[0], arr[2], keys_block), (arr[5], arr[1], arr[3], values_block)):
            for r in range(tau):
                tail[b, :, (n + r) % RING] = tail[b, :, (n + kept * chain + r) % RING]
            if fills:
                for h in range(tail.shape[1]):
                    pool[i, h], scale[i, h] = block(tail[b, h, [p % RING for p in range(j * T, j * T + T)]])
        new.append(n + tau)
    return np.array(new, np.int32)


def read(arr, slots):
    """float64 [n, H, 128] keys and values; NaN-filled None rows where a slot names none (returned mask False)."""
    K4, V4 = values_of(arr)
    n_blocks, H, B = len(K4), K4.shape[1], len(arr[4])
    k, v, ok = np.zeros((len(slots), H, D)), np.zeros((len(slots), H, D)), np.zeros(len(slots), bool)
    for t, s in enumerate(int(x) for x in slots):
        if 0 <= s < n_blocks * T:
            k[t], v[t], ok[t] = K4[s // T, :, s % T], V4[s // T, :, s % T], True
        elif s <= -2 and -2 - s < B * RING:
            b, r = divmod(-2 - s, RING)
            k[t], v[t], ok[t] = arr[4][b, :, r], arr[5][b, :, r], True
    return k, v, ok
