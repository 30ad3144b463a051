"""Plain forms of the paged cache's operators on the host, in 64 bits, from their definitions."""
import numpy as np
import torch

T, RING, D = 64, 128, 128

# every e4m3 value by its code; what is nearest is looked up, ties to the even code
_CODE = np.arange(128)
_E, _M = _CODE >> 3, _CODE & 7
VALUES = np.where(_E == 0, _M * 2.0 ** -9, (8 + _M) * 2.0 ** (_E - 10.0))[:127]      # code 127 is NaN


def nearest8(x):
    """float64 -> codes (uint8) of the nearest e4m3 values; |x| <= 448 or not finite (NaN)."""
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(VALUES, a, side="left"), 1, 126)
    lo = hi - 1
    up, down = VALUES[hi] - a, a - VALUES[lo]
    code = np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))
    return np.where(np.isfinite(x), code | np.where(np.signbit(x), 128, 0), 127).astype(np.uint8)


def value_of(codes):
    v = np.append(VALUES, np.nan)[codes & 127]
    return np.where(codes & 128, -v, v)


def block8(x):
    """One block [64, 128] float64 -> (codes, scale)."""
    top = np.max(np.abs(x[np.isfinite(x)]), initial=0.0)
    e = -60
    while top > 448.0 * 2.0 ** e:
        e += 1
    return nearest8(x / 2.0 ** e), 2.0 ** e


def plan(kv_len, n_new, held, queue, state, table, max_rows, reserve, draft):
    """One request after the other.  Changes queue and table; returns the outputs by name."""
    B, cols = table.shape
    n_blocks = len(queue)
    head, count = int(state[0]), int(state[1])
    before = table.copy()
    r = {k: [] for k in ("granted", "new_held")}
    cu, at, taken, back, wanted = [0], 0, 0, [], 0
    slots, seqs, poss = ([-1] * max_rows for _ in range(3))
    for b in range(B):
        n, new, h = max(int(kv_len[b]), 0), max(int(n_new[b]), 0), int(held[b])
        done = (n if draft else n + new) // T
        need = (n + new + reserve) // T
        ok = need <= cols and cu[-1] + new <= max_rows and n + new - done * T <= RING
        if ok:
            wanted += max(need - h, 0)
            ok = need <= h or wanted <= count
        if ok:
            for j in range(h, need):
                table[b, j] = queue[(head + taken) % n_blocks]
                taken += 1
            back += [before[b, j] for j in range(need, h)]
        r["granted"].append(int(ok))
        r["new_held"].append(need if ok else h)
        for i in range(new):
            t, p = cu[-1] + i, n + i
            if t >= max_rows:
                break
            seqs[t], poss[t] = b, p
            if ok:
                slots[t] = int(table[b, p // T]) * T + p % T if p < done * T else -2 - (b * RING + p % RING)
        cu.append(min(cu[-1] + new, max_rows))
    for i, x in enumerate(back):
        queue[(head + count + i) % n_blocks] = x
    r.update(new_state=[(head + taken) % n_blocks, count - taken + len(back)], cu_rows=cu, slots=slots,
             row_seq=seqs, row_pos=poss)
    return {k: np.array(v, np.int32) for k, v in r.items()}


def as_numpy(cache):
    """A layer's cache as float64 arrays and uint8 codes."""
    k8, v8, ks, vs, kt, vt = [x.cpu() for x in cache]
    return [k8.view(torch.uint8).numpy().copy(), v8.view(torch.uint8).numpy().copy(), ks.double().numpy().copy(),
            vs.double().numpy().copy(), kt.double().numpy().copy(), vt.double().numpy().copy()]


def append(cache, k, v, plan_, kv_len):
    """cache: as_numpy(); k, v float64 [n, Hkv, D].  Rows of each request in order."""
    k8, v8, ks, vs, kt, vt = cache
    cu, slots = plan_["cu_rows"], plan_["slots"]
    for b in range(len(cu) - 1):
        n = max(int(kv_len[b]), 0)
        for x, pool, scale, tail, turned in ((k, k8, ks, kt, False), (v, v8, vs, vt, True)):
            rows = {p: tail[b, :, p % RING].copy() for p in range(n // T * T, n)}
            for t in range(cu[b], cu[b + 1]):
                p = n + t - cu[b]
                rows[p] = x[t]
            for t in range(cu[b], cu[b + 1]):
                p, s = n + t - cu[b], int(slots[t])
                if s <= -2:
                    tail[b, :, p % RING] = x[t]
                elif s >= 0 and s % T == T - 1:
                    for h in range(x.shape[1]):
                        codes, sc = block8(np.stack([rows[i][h] for i in range(p - T + 1, p + 1)]))
                        pool[s // T, h] = codes.T if turned else codes
                        scale[s // T, h] = sc


def keys_values(cache, table, n, b, h, gamma):
    """The keys and values a sequence's rows attend over, in 64 bits, and which positions exist."""
    k8, v8, ks, vs, kt, vt = cache
    K, V, there = [], [], []
    for j in range(n // T):
        i = int(table[b, j])
        ok = 0 <= i < len(k8)
        K.append(value_of(k8[i, h]) * ks[i, h] if ok else np.zeros((T, D)))
        V.append(value_of(v8[i, h]).T * vs[i, h] if ok else np.zeros((T, D)))
        there += [ok] * T
    ring = [p % RING for p in range(n // T * T, n + gamma)]
    there += [True] * len(ring)
    return np.concatenate(K + [kt[b, h, ring]]), np.concatenate(V + [vt[b, h, ring]]), np.array(there)


def attention(q, cache, table, kv_len, mask=None, scale=None, vis=None):
    """q float64 [B, gamma, Hq, D].  Returns out, lse, vis_mass and sum p |v| (what the rounding of
    probabilities goes by)."""
    B, g, Hq, _ = q.shape
    Hkv = cache[0].shape[1]
    scale = D ** -0.5 if scale is None else scale
    mask = [(1 << (i + 1)) - 1 for i in range(g)] if mask is None else mask
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    lse, mass = np.zeros((B, Hq, g)), np.zeros((B, Hq, g))
    cols = table.shape[1]
    for b in range(B):
        n = min(max(int(kv_len[b]), 0), cols * T + T - 1)
        for h in range(Hkv):
            K, V, there = keys_values(cache, table, n, b, h, g)
            for i in range(g):
                see = there.copy()
                see[n:] = [bool(int(mask[i]) >> j & 1) for j in range(g)]
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


def commit(cache, table, kv_len, accept_len, chain, best=None, n_branches=1):
    """cache: as_numpy() of one layer, changed.  Returns new_len."""
    k8, v8, ks, vs, kt, vt = cache
    new = []
    for b, n in enumerate(int(x) for x in kv_len):
        kept = int(best[b]) if best is not None and n_branches > 1 else 0
        tau = int(accept_len[b * n_branches + kept])
        j = n // T
        fills = (n + tau) // T > j
        i = int(table[b, j]) if j < table.shape[1] else -1
        if n < 0 or n > table.shape[1] * T + T - 1 or (fills and not 0 <= i < len(k8)):
            new.append(n)
            continue
        for tail, pool, scale, turned in ((kt, k8, ks, False), (vt, v8, vs, True)):
            for r in range(tau):
                tail[b, :, (n + r) % RING] = tail[b, :, (n + kept * chain + r) % RING]
            if fills:
                for h in range(tail.shape[1]):
                    codes, sc = block8(tail[b, h, [p % RING for p in range(j * T, j * T + T)]])
                    pool[i, h] = codes.T if turned else codes
                    scale[i, h] = sc
        new.append(n + tau)
    return np.array(new, np.int32)
