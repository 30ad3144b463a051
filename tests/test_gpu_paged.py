"""The paged cache in 8 bits on the GPU, against the plain forms of paged_ref.

Tolerances.  Codes, scales, ring rows, tables and maps: equal.  Attention: the keys, the queries and
the values are exact, scores and sums are binary32 (errors near 1e-6), and two roundings to bf16 are left
(half a step is 2^-8 of the value): every probability, which moves an output by at most 2^-8 sum p |v|, and
the output itself.  So |out - ref| <= 2^-8 (sum p |v| + |ref|), with 2 % for the binary32 part.  The
log-sum-exp and the mass come from unrounded probabilities: binary32 scores of size |z| are off by about
|z| 128 2^-24, so 2e-5 (1 + |z|) holds both."""
import numpy as np
import pytest
import torch

import paged_ref as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
T, RING, D = 64, 128, 128


@pytest.fixture(scope="module")
def L():
    from paper_2604_05650_amd import binding
    return binding


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def normal(seed, shape, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * gain).to(torch.bfloat16).to(DEV)


def same_cache(got, ref, what=""):
    for name, x, y in zip(("k_pool", "v_pool", "k_scale", "v_scale", "k_tail", "v_tail"), R.as_numpy(got), ref):
        nan = np.isnan(x) & np.isnan(y) if x.dtype.kind == "f" else (x & 127 == 127) & (y & 127 == 127)
        assert np.array_equal(np.where(nan, 0, x), np.where(nan, 0, y)), f"{what} {name}"


def check_plan(L, kv_len, n_new, held, queue, state, table, **kw):
    """One plan on both sides; returns the GPU's answer and the changed queue and table."""
    q, t = i32(queue), i32(table)
    got = L.paged_plan(i32(kv_len), i32(n_new), i32(held), q, i32(state), t, **kw)
    rq, rt = np.array(queue, np.int32), np.array(table, np.int32)
    ref = R.plan(kv_len, n_new, held, rq, state, rt, kw["max_rows"], kw.get("reserve", 0), kw.get("draft", False))
    for name, x in ref.items():
        assert np.array_equal(got[name].cpu().numpy(), x), name
    assert np.array_equal(t.cpu().numpy(), rt)
    assert np.array_equal(q.cpu().numpy(), rq)
    return got, q, t


PLANS = [
    dict(kv=[0], new=[0]), dict(kv=[0], new=[1]), dict(kv=[63], new=[1]), dict(kv=[64], new=[64]),
    dict(kv=[0, 5, 64, 200], new=[63, 59, 0, 1000]),
    dict(kv=[60, 127, 640], new=[5, 5, 5], draft=True, reserve=5),
    dict(kv=[-7, 10], new=[3, -2]),
    dict(kv=[0, 0, 0], new=[640, 64, 0], free=9),                     # the first does not fit, nor who is behind
    dict(kv=[0, 0, 0], new=[256, 640, 63], free=9),                   # the third needs none
    dict(kv=[0, 100, 0], new=[0, 70, 0], held=[5, 3, 2]),             # finished requests, and one that shrinks
    dict(kv=[0, 0], new=[6400, 30], cols=10),                         # a table too narrow
    dict(kv=[0, 0, 10], new=[100, 50, 0], max_rows=120),              # rows that do not fit the maps
    dict(kv=[60, 0], new=[100, 2], draft=True),                       # drafts that do not fit the ring
    dict(kv=[0] * 300, new=list(range(300)), pad=77),
    dict(kv=list(range(700)), new=[5] * 700, draft=True, reserve=5),
    dict(kv=[64 * (i % 9) for i in range(4096)], new=[i % 3 for i in range(4096)], free=1000),
]


@pytest.mark.parametrize("i", range(len(PLANS)))
def test_plan(L, i):
    c = PLANS[i]
    kv, new = c["kv"], c["new"]
    held = c.get("held", [max(n, 0) // T for n in kv])
    cols = c.get("cols", max(max(n, 0) + max(x, 0) + 64 for n, x in zip(kv, new)) // T + 6)
    total = sum(max(x, 0) for x in new)
    free = c.get("free", 4096 + total // T)
    n_blocks = sum(held) + free
    ids = np.random.default_rng(i).permutation(n_blocks)
    table = np.full((len(kv), cols), -1)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = ids[at:at + n]
        at += n
    head = (17 * i + 5) % n_blocks
    queue = np.roll(np.concatenate([ids[at:], np.full(at, -1)]), head)
    kw = dict(max_rows=c.get("max_rows", total + c.get("pad", 0)), reserve=c.get("reserve", 0), draft=c.get("draft", False))
    got, q, t = check_plan(L, kv, new, held, queue, [head, free], table, **kw)
    # nothing it reads has changed: the same call gives the same answer
    again, _, _ = check_plan(L, kv, new, held, q.cpu().numpy(), [head, free], t.cpu().numpy(), **kw)
    assert all(torch.equal(got[k], again[k]) for k in got)


def test_plan_over_time(L):
    """Requests come, grow, are refused and finish; no block has two owners."""
    rng = np.random.default_rng(3)
    B, n_blocks, cols = 9, 60, 20
    st = {k: v.cpu().numpy() for k, v in L.alloc_paged_state(B, n_blocks, cols, DEV).items()}
    kv = np.zeros(B, np.int64)
    refused = 0
    for step in range(40):
        new = rng.integers(0, 200, B)
        gone = rng.random(B) < 0.15
        kv[gone], new[gone] = 0, 0
        got, q, t = check_plan(L, kv, new, st["held"], st["queue"], st["state"], st["table"],
                               max_rows=int(new.sum()) + 3, reserve=int(step % 3) * 40)
        st = dict(held=got["new_held"].cpu().numpy(), state=got["new_state"].cpu().numpy(),
                  queue=q.cpu().numpy(), table=t.cpu().numpy())
        ok = got["granted"].cpu().numpy()
        refused += int((ok == 0).sum())
        kv = np.where(ok, kv + new, kv)
        own = [x for b in range(B) for x in st["table"][b, :st["held"][b]]]
        free = [st["queue"][(st["state"][0] + i) % n_blocks] for i in range(st["state"][1])]
        assert sorted(own + free) == list(range(n_blocks))
    assert refused > 0


def ready(L, seed, B, Hkv, lens, extra=3, spare_cols=1):
    """A cache with `lens` committed rows in blocks of random places, ring rows everywhere."""
    need = [n // T for n in lens]
    n_blocks = sum(need) + extra
    cache = L.alloc_paged_cache(B, Hkv, n_blocks, DEV)
    rng = np.random.default_rng(seed)
    ids = rng.permutation(n_blocks)
    table = np.full((B, max(need) + spare_cols), -1)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    for x in (cache.k_pool, cache.v_pool):
        codes = rng.integers(0, 256, tuple(x.shape)).astype(np.uint8)
        codes = np.where(codes & 127 >= 0x70, codes & 0x8f, codes)          # up to 224: no NaN, few large ones
        x.copy_(torch.from_numpy(codes).view(torch.float8_e4m3fn))
    for x in (cache.k_scale, cache.v_scale):
        x.copy_(torch.from_numpy(2.0 ** rng.integers(-9, -5, tuple(x.shape))).float())
    cache.k_tail.copy_(normal(seed + 1, tuple(cache.k_tail.shape)))
    cache.v_tail.copy_(normal(seed + 2, tuple(cache.v_tail.shape)))
    return cache, table


APPENDS = [
    dict(kv=[0], new=[1]), dict(kv=[0], new=[64]), dict(kv=[63], new=[1]), dict(kv=[40], new=[23]),
    dict(kv=[40], new=[300]),                       # open rows, several blocks, the new tail in the old half
    dict(kv=[40], new=[64]), dict(kv=[100, 0, 17], new=[100, 128, 255]),
    dict(kv=[1] * 20, new=list(range(1, 41, 2))),   # many sequences in a tile of rows
    dict(kv=[63] * 70, new=[1] * 70),               # a block per packed row
    dict(kv=[0, 60, 127, 500], new=[5, 5, 5, 32], draft=True),
    dict(kv=[130, 250], new=[40, 0], Hkv=1), dict(kv=[9, 70], new=[777, 1], Hkv=8),
]


@pytest.mark.parametrize("i", range(len(APPENDS)))
def test_append(L, i):
    c = APPENDS[i]
    kv, new, Hkv = c["kv"], c["new"], c.get("Hkv", 2)
    B, n = len(kv), sum(new)
    need = [(a + b) // T for a, b in zip(kv, new)]
    cache, _ = ready(L, i, B, Hkv, [T * x for x in need])
    n_blocks = cache.k_pool.shape[0]
    st = L.alloc_paged_state(B, n_blocks, max(need) + 1, DEV)
    pad = 3 if i % 2 else 0                         # rows behind the last sequence
    plan = L.paged_plan(i32(kv), i32(new), st["held"], st["queue"], st["state"], st["table"],
                        max_rows=n + pad, draft=c.get("draft", False))
    assert plan["granted"].all()
    # a row of the projection's output: keys and values of all heads side by side
    both = normal(100 + i, (n + pad, 2, Hkv, D), 3.0)
    both[:, :, :, 7] *= 40
    both[n:] = float("nan")
    k, v = both[:, 0], both[:, 1]
    ref = R.as_numpy(cache)
    R.append(ref, k.double().cpu().numpy(), v.double().cpu().numpy(), {x: y.cpu().numpy() for x, y in plan.items()}, kv)
    L.paged_append(cache, k, v, plan)
    same_cache(cache, ref)


def test_append_values(L):
    """Scales at their borders, every rounding, zeros, small blocks, infinities and NaN."""
    kv, new = [0], [8 * T]
    cache, _ = ready(L, 5, 1, 1, [8 * T])
    st = L.alloc_paged_state(1, cache.k_pool.shape[0], 9, DEV)
    plan = L.paged_plan(i32(kv), i32(new), st["held"], st["queue"], st["state"], st["table"], max_rows=8 * T)
    x = torch.zeros(8, T, D)
    x[0] = torch.linspace(-448, 448, T * D).view(T, D)                   # exactly 448
    x[1] = torch.linspace(-450, 449, T * D).view(T, D)                   # one step more
    x[2] = torch.randn(T, D, generator=torch.Generator().manual_seed(1)) * torch.logspace(-12, 3, D)
    x[4] = 1e-30
    x[4, 0, 0] = 2.0 ** -52
    x[5] = torch.randn(T, D, generator=torch.Generator().manual_seed(2)) * 1e36
    x[6] = torch.randn(T, D, generator=torch.Generator().manual_seed(3))
    x[6, 3, 5], x[6, 9, 100], x[6, 60, 2] = float("inf"), float("-inf"), float("nan")
    x[7] = float("nan")
    k = x.view(8 * T, 1, D).to(torch.bfloat16).to(DEV)
    v = k.flip(0).contiguous()
    ref = R.as_numpy(cache)
    R.append(ref, k.double().cpu().numpy(), v.double().cpu().numpy(), {a: b.cpu().numpy() for a, b in plan.items()}, kv)
    L.paged_append(cache, k, v, plan)
    same_cache(cache, ref)


def test_append_leaves_rows_without_a_place(L):
    """Maps that name no block of the pool and no row of the ring store nothing."""
    cache, _ = ready(L, 6, 2, 2, [64, 64])
    n_blocks = cache.k_pool.shape[0]
    before = R.as_numpy(cache)
    k, v = normal(1, (64, 2, D)), normal(2, (64, 2, D))
    for slots in ([n_blocks * T + i for i in range(T)], [-1] * T, [-2 - 2 * RING - i for i in range(T)]):
        plan = dict(slots=i32(slots), row_seq=i32([0] * T), row_pos=i32(range(T)), cu_rows=i32([0, T, T]))
        L.paged_append(cache, k, v, plan)
        same_cache(cache, before)
    for seq, cu in ((5, [0, T, T]), (-1, [0, T, T]), (0, [-3, T, T]), (0, [T, T, T])):
        plan = dict(slots=i32(range(T)), row_seq=i32([seq] * T), row_pos=i32(range(T)), cu_rows=i32(cu))
        L.paged_append(cache, k, v, plan)
        same_cache(cache, before)
    L.paged_append(cache, k[:0], v[:0], dict(slots=i32([]), row_seq=i32([]), row_pos=i32([]), cu_rows=i32([0, 0, 0])))
    same_cache(cache, before)


def tree(branches, chain):
    return [((1 << (i + 1)) - 1) << (a * chain) for a in range(branches) for i in range(chain)]


def check_attention(L, q, cache, table, kv, vis=None, mask=None, scale=0.0, **kw):
    t = i32(table)
    opt = dict(vis_begin=i32(vis[0]), vis_end=i32(vis[1])) if vis is not None else {}
    out, lse, mass = L.verify_attn_paged(q, cache, t, i32(kv), draft_mask=mask, scale=scale, return_lse=True,
                                         return_vis_mass=vis is not None, **opt, **kw)
    ro, rl, rm, size = R.attention(q.double().cpu().numpy(), R.as_numpy(cache), np.asarray(table), kv, mask,
                                   scale if scale > 0 else None, vis)
    o = out.double().cpu().numpy()
    assert np.all(np.isfinite(o))
    assert np.all(np.abs(o - ro) <= 1.02 * 2.0 ** -8 * (size + np.abs(ro)) + 1e-30), float(
        np.max(np.abs(o - ro) / (size + np.abs(ro)))) * 256
    assert np.all(np.abs(lse.cpu().numpy() - rl) <= 2e-5 * (1 + np.abs(rl)))
    if vis is not None:
        assert np.all(np.abs(mass.cpu().numpy() - rm) <= 2e-5 * (1 + np.abs(rl)))
    return out


ATTNS = [
    dict(kv=[0], g=1), dict(kv=[0], g=7), dict(kv=[1], g=1), dict(kv=[63], g=1), dict(kv=[64], g=1),
    dict(kv=[65], g=3), dict(kv=[127], g=32, Hq=2, Hkv=2), dict(kv=[300], g=5, Hq=10, Hkv=2),
    dict(kv=[1000], g=5, Hq=40, Hkv=8), dict(kv=[64 * 9 + 40], g=9, Hq=28, Hkv=4),          # 63 rows
    dict(kv=[500, 0, 63, 64, 1, 2000], g=4, Hq=8, Hkv=2),
    dict(kv=[700, 90], g=20, Hq=10, Hkv=2, branches=2),                                     # 100 rows: two chunks
    dict(kv=[257, 600], g=32, Hq=16, Hkv=2, branches=4),                                    # 256 rows
    dict(kv=[(37 * i) % 700 for i in range(70)], g=1, Hq=4, Hkv=2),                         # more than a wave of sequences
    dict(kv=[9000], g=3, Hq=3, Hkv=1), dict(kv=[6000, 10, 3000], g=16, Hq=4, Hkv=4),
    dict(kv=[800], g=2, Hq=64, Hkv=2), dict(kv=[450], g=33 // 3, Hq=3, Hkv=1, scale=0.3),
    # units of very different lengths, fewer and more than compute units
    dict(kv=[1200, 300] + [17] * 60, g=1, Hq=8, Hkv=8), dict(kv=[9600] * 10 + [20] * 50, g=1, Hq=8, Hkv=8),
    dict(kv=[25000, 24000, 26000], g=1, Hq=16, Hkv=16), dict(kv=[(53 * i) % 300 for i in range(70)], g=2, Hq=8, Hkv=8),
    dict(kv=[(53 * i) % 300 for i in range(131)] + [5000, 0, 64, 9000], g=3, Hq=2, Hkv=1),
    dict(kv=[7000, 0] + [(71 * i) % 200 for i in range(252)] + [64, 6000], g=1, Hq=2, Hkv=1),       # as many as are cut
    dict(kv=[(71 * i) % 200 for i in range(256)] + [6500], g=1, Hq=2, Hkv=1),                       # and one more
    dict(kv=[6000, 300], g=24, Hq=20, Hkv=4), dict(kv=[3000, 9000, 64, 0, 5], g=15, Hq=14, Hkv=2),  # 120 and 105 rows
]


@pytest.mark.parametrize("spare_cols", [1, 70])        # a unit in one workgroup where it is short, or cut into parts
@pytest.mark.parametrize("i", range(len(ATTNS)))
def test_attention(L, i, spare_cols):
    c = ATTNS[i]
    kv, g, Hq, Hkv = c["kv"], c["g"], c.get("Hq", 4), c.get("Hkv", 2)
    B = len(kv)
    cache, table = ready(L, 50 + i, B, Hkv, kv, spare_cols=spare_cols)
    q = normal(200 + i, (B, g, Hq, D))
    mask = tree(c["branches"], g // c["branches"]) if "branches" in c else None
    vis = ([5] * B, [max(5, n * 2 // 3) for n in kv]) if i % 2 else None
    check_attention(L, q, cache, table, kv, vis, mask, c.get("scale", 0.0))


def test_attention_strides_and_span(L):
    """q and out as slices of wider buffers; spans that are empty, cut tiles, or reach the drafts."""
    kv, g, Hq, Hkv = [400, 65, 7], 6, 12, 4
    cache, table = ready(L, 90, 3, Hkv, kv, spare_cols=4)
    wide = normal(91, (g, 3, Hq + 3, D + 64))
    q = wide.permute(1, 0, 2, 3)[:, :, 1:Hq + 1, 64:]
    out = torch.full((3, g, 2, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    check_attention(L, q, cache, table, kv, ([0, 60, 3], [0, 66, 100]), out=out[:, :, 1])
    assert bool((out[:, :, 0] == 7.0).all())
    check_attention(L, q, cache, table, kv, ([13, -5, 0], [333, 64, 1]))


@pytest.mark.parametrize("spare_cols", [3, 70])
def test_attention_reads_declared_rows_only(L, spare_cols):
    """Unused blocks, table entries behind the length and ring rows of nobody hold NaN."""
    kv, g = [200, 64, 30, 0], 5
    cache, table = ready(L, 92, 4, 2, kv, extra=4, spare_cols=spare_cols)
    q = normal(93, (4, g, 8, D))
    want = check_attention(L, q, cache, table, kv).clone()
    used = {int(table[b, j]) for b in range(4) for j in range(kv[b] // T)}
    for i in range(cache.k_pool.shape[0]):
        if i not in used:
            for x in (cache.k_pool, cache.v_pool):
                x.view(torch.uint8)[i] = 0x7f
            cache.k_scale[i] = cache.v_scale[i] = float("nan")
    free = next(i for i in range(cache.k_pool.shape[0]) if i not in used)
    for b, n in enumerate(kv):
        mine = {p % RING for p in range(n // T * T, n + g)}
        for r in range(RING):
            if r not in mine:
                cache.k_tail[b, :, r] = float("nan")
                cache.v_tail[b, :, r] = float("inf")
        table[b, n // T:] = [free, 1 << 30, -9][b % 3]
    got = L.verify_attn_paged(q, cache, i32(table), i32(kv))
    assert torch.equal(got, want)


@pytest.mark.parametrize("spare_cols", [1, 70])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_attention_masked_draft_rows_do_not_reach_others(L, value, spare_cols):
    """A draft row that is not finite changes the rows that see it and no other."""
    kv, g = [100, 64], 6
    cache, table = ready(L, 94, 2, 2, kv, spare_cols=spare_cols)
    q = normal(95, (2, g, 8, D))
    want = L.verify_attn_paged(q, cache, i32(table), i32(kv)).clone()
    for b, n in enumerate(kv):
        cache.v_tail[b, :, (n + 3) % RING, 17] = value
    got = L.verify_attn_paged(q, cache, i32(table), i32(kv))
    assert torch.equal(got[:, :3], want[:, :3])
    rest = torch.arange(D, device=DEV) != 17
    assert torch.equal(got[:, 3:, :, rest], want[:, 3:, :, rest])
    hit = got[:, 3:, :, 17].float()
    assert bool((torch.isnan(hit) if value != value else hit == value).all())
    for b, n in enumerate(kv):
        cache.v_tail[b, :, (n + 3) % RING, 17] = 0
        cache.k_tail[b, :, (n + 3) % RING, 17] = value
    got = L.verify_attn_paged(q, cache, i32(table), i32(kv))
    assert torch.equal(got[:, :3], want[:, :3])


@pytest.mark.parametrize("spare_cols", [0, 70])
def test_attention_lengths_and_blocks_out_of_range(L, spare_cols):
    """Lengths are clamped to what the table names; entries that name no block hold no key."""
    kv, g = [300, 300, 300], 3
    cache, table = ready(L, 96, 3, 2, kv, spare_cols=spare_cols)
    q = normal(97, (3, g, 4, D))
    table[1, 2], table[2, 0] = -1, cache.k_pool.shape[0]
    assert table.shape[1] == 4 + spare_cols
    check_attention(L, q, cache, table, kv)
    most = table.shape[1] * T + T - 1
    a = L.verify_attn_paged(q, cache, i32(table), i32([-5, 10 ** 9, most]))
    b = L.verify_attn_paged(q, cache, i32(table), i32([0, most, most]))
    assert torch.equal(a, b)
    # nobody holds a block: a table without columns
    check_attention(L, q, cache, np.zeros((3, 0), np.int32), [20, 0, 63])


def test_attention_is_the_same_every_time(L):
    kv = [1500, 3000, 10, 640]
    cache, table = ready(L, 98, 4, 4, kv)
    q = normal(99, (4, 5, 20, D))
    first = L.verify_attn_paged(q, cache, i32(table), i32(kv))
    for _ in range(5):
        assert torch.equal(first, L.verify_attn_paged(q, cache, i32(table), i32(kv)))


COMMITS = [
    dict(kv=[0], tau=[1], chain=5), dict(kv=[63], tau=[1], chain=1), dict(kv=[60], tau=[16], chain=16),
    dict(kv=[127, 128, 190, 3], tau=[0, 5, 2, 4], chain=5),
    dict(kv=[62, 125, 20, 255], tau=[9, 10, 1, 3, 0, 7, 10, 2], chain=10, branches=2, best=[1, 1, 0, 1]),
    dict(kv=[60, 60, 118], tau=[4] * 24, chain=4, branches=8, best=[7, 0, 3]),
    dict(kv=[124, 60], tau=[9, 9], chain=5),                            # more than the chain: clamped
]


@pytest.mark.parametrize("i", range(len(COMMITS)))
@pytest.mark.parametrize("layers", [1, 3])
def test_commit(L, i, layers):
    c = COMMITS[i]
    kv, br, chain = c["kv"], c.get("branches", 1), c["chain"]
    B = len(kv)
    parts = [ready(L, 300 + 10 * i + y, B, 2, [T * (n // T + 1) for n in kv]) for y in range(layers)]
    table = parts[0][1]
    cache = L.PagedCache(*[torch.stack([p[0][x] for p in parts]) for x in range(6)])
    best = c.get("best")
    refs = [R.as_numpy(p[0]) for p in parts]
    want = [R.commit(r, table, kv, np.minimum(c["tau"], chain), chain, best, br) for r in refs][0]
    got = L.paged_commit(cache, i32(table), i32(kv), i32(c["tau"]), chain, n_branches=br,
                         best_branch=None if best is None else i32(best))
    assert np.array_equal(got.cpu().numpy(), want)
    for y in range(layers):
        same_cache(cache.layer(y), refs[y], f"layer {y}")
    if layers == 1:
        one = parts[0][0]
        L.paged_commit(one, i32(table), i32(kv), i32(c["tau"]), chain, n_branches=br,
                       best_branch=None if best is None else i32(best))
        same_cache(one, refs[0])


def test_commit_without_a_place(L):
    """A block that was not granted, a table without its column, a length out of range: left as they are."""
    kv = [62, 62, -4, 10 ** 8, 62, 191]
    cache, _ = ready(L, 400, 6, 2, [0] * 6, extra=5)
    n_blocks = cache.k_pool.shape[0]
    table = np.array([[-1, 0, 0], [n_blocks, 0, 0], [0, 0, 0], [1, 1, 1], [4, 0, 0], [0, 0, 3]])
    tau, best = [5] * 12, [1] * 6
    ref = R.as_numpy(cache)
    want = R.commit(ref, table, kv, tau, 5, best, 2)
    got = L.paged_commit(cache, i32(table), i32(kv), i32(tau), 5, n_branches=2, best_branch=i32(best))
    assert got.tolist() == want.tolist() == [62, 62, -4, 10 ** 8, 67, 196]
    same_cache(cache, ref)
    got = L.paged_commit(cache, i32(np.full((6, 1), 4)), i32([127] * 6), i32([1] * 6), 5)
    assert got.tolist() == [127] * 6


def test_decode_loop(L):
    """Prompts, then verified steps with trees and refused drafts, against one contiguous list of rows."""
    rng = np.random.default_rng(8)
    B, Hkv, Hq, layers, br, chain = 3, 2, 8, 2, 2, 5
    g = br * chain
    prompt = [130, 63, 1]
    st = L.alloc_paged_state(B, 40, 12, DEV)
    held, state = st["held"], st["state"]
    cache = L.alloc_paged_cache(B, Hkv, 40, DEV, layers=layers)
    plan = L.paged_plan(i32([0] * B), i32(prompt), held, st["queue"], state, st["table"], max_rows=sum(prompt))
    held, state = plan["new_held"], plan["new_state"]
    rows = [[[] for _ in range(B)] for _ in range(layers)]      # committed (k, v) rows
    for y in range(layers):
        k, v = normal(1 + y, (sum(prompt), Hkv, D)), normal(11 + y, (sum(prompt), Hkv, D))
        L.paged_append(cache.layer(y), k, v, plan)
        for b in range(B):
            for t in range(sum(prompt[:b]), sum(prompt[:b + 1])):
                rows[y][b].append((k[t], v[t]))
    kv_len = i32(prompt)
    mask = tree(br, chain)
    for step in range(25):
        n = kv_len.tolist()
        plan = L.paged_plan(kv_len, i32([g] * B), held, st["queue"], state, st["table"], max_rows=B * g, reserve=g,
                            draft=True)
        assert plan["granted"].all()
        held, state = plan["new_held"], plan["new_state"]
        tau, best = rng.integers(0, chain + 1, B * br), rng.integers(0, br, B)
        for y in range(layers):
            k, v = normal(100 * step + y, (B * g, Hkv, D)), normal(100 * step + 50 + y, (B * g, Hkv, D))
            one = cache.layer(y)
            L.paged_append(one, k, v, plan)
            q = normal(5000 + step, (B, g, Hq, D))
            if step % 6 == 0:
                check_attention(L, q, one, st["table"].cpu().numpy(), n, mask=mask)
            for b in range(B):
                at = b * g + int(best[b]) * chain
                rows[y][b] += [(k[at + i], v[at + i]) for i in range(int(tau[b * br + best[b]]))]
        kv_len = L.paged_commit(cache, st["table"], kv_len, i32(tau), chain, n_branches=br, best_branch=i32(best))
    lens = kv_len.tolist()
    assert lens == [len(r) for r in rows[0]]
    table = st["table"].cpu().numpy()
    for y in range(layers):
        arr = R.as_numpy(cache.layer(y))
        for b, n in enumerate(lens):
            for which, pool, scale, tail in ((0, 0, 2, 4), (1, 1, 3, 5)):
                x = torch.stack([r[which] for r in rows[y][b]]).double().cpu().numpy()     # [n, Hkv, D]
                for h in range(Hkv):
                    for j in range(n // T):
                        codes, sc = R.block8(x[j * T:j * T + T, h])
                        got = arr[pool][table[b, j], h]
                        assert np.array_equal(got.T if which else got, codes) and arr[scale][table[b, j], h] == sc
                    for p in range(n // T * T, n):
                        assert np.array_equal(arr[tail][b, h, p % RING], x[p, h])


def test_decode_steps_in_a_graph(L):
    """A captured step (plan, append, attention, commit), replayed between eager work."""
    B, Hkv, Hq, g = 2, 2, 8, 4
    st = L.alloc_paged_state(B, 30, 10, DEV)
    cache = L.alloc_paged_cache(B, Hkv, 30, DEV, layers=1)
    kv_len, new = i32([61, 126]), i32([g] * B)
    prompt = L.paged_plan(i32([0, 0]), kv_len, st["held"], st["queue"], st["state"], st["table"], max_rows=187)
    L.paged_append(cache.layer(0), normal(1, (187, Hkv, D)), normal(2, (187, Hkv, D)), prompt)
    held, state = prompt["new_held"].clone(), prompt["new_state"].clone()
    twin = [x.clone() for x in (*cache, st["queue"], st["table"], kv_len, held, state)]
    k, v, q = (torch.zeros(s, dtype=torch.bfloat16, device=DEV)
               for s in ((B * g, Hkv, D), (B * g, Hkv, D), (B, g, Hq, D)))
    tau = i32([0] * B)

    def step(cache, queue, table, kv_len, held, state):
        plan = L.paged_plan(kv_len, new, held, queue, state, table, max_rows=B * g, reserve=g, draft=True)
        held.copy_(plan["new_held"])
        state.copy_(plan["new_state"])
        L.paged_append(cache.layer(0), k, v, plan)
        out = L.verify_attn_paged(q, cache.layer(0), table, kv_len)
        kv_len.copy_(L.paged_commit(cache, table, kv_len, tau, g))
        return out

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache, st["queue"], st["table"], kv_len, held, state)      # (tau = 0: nothing moves on)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(cache, st["queue"], st["table"], kv_len, held, state)
    for i in range(8):
        k.copy_(normal(10 + i, tuple(k.shape)))
        v.copy_(normal(30 + i, tuple(v.shape)))
        q.copy_(normal(50 + i, tuple(q.shape)))
        tau.copy_(i32([i % 5, (3 * i) % 5]))
        graph.replay()
        want = step(L.PagedCache(*twin[:6]), *twin[6:])
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        for x, y in zip((*cache, st["queue"], st["table"], kv_len, held, state), twin):
            assert torch.equal(x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x,
                               y.view(torch.uint8) if y.dtype == torch.float8_e4m3fn else y), i
    assert kv_len.tolist()[0] > 64


def test_two_streams(L):
    """Two batches with workspaces of their own at the same time."""
    kv = [900, 40]
    made = [ready(L, 500 + i, 2, 2, kv) for i in range(2)]
    qs = [normal(510 + i, (2, 4, 8, D)) for i in range(2)]
    want = [L.verify_attn_paged(q, c, i32(t), i32(kv)) for q, (c, t) in zip(qs, made)]
    args = [(i32(t), i32(kv)) for _, t in made]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for i in range(2):
        with torch.cuda.stream(streams[i]):
            for _ in range(4):
                last = L.verify_attn_paged(qs[i], made[i][0], *args[i])
            got.append(last)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_pool_of_more_than_4_gib(L):
    """The last blocks of a large pool hold and give what the blocks of a small one do."""
    B, Hkv, Hq, g, prompt, chain = 2, 4, 8, 5, [200, 70], 5
    small, far = 8, (1 << 17) + 64                      # 4 GiB and 2 MiB of keys, as much of values
    k, v = normal(1, (sum(prompt), Hkv, D)), normal(2, (sum(prompt), Hkv, D))
    dk, dv, q = normal(3, (B * g, Hkv, D)), normal(4, (B * g, Hkv, D)), normal(5, (B, g, Hq, D))
    outs, ends = [], []
    for n_blocks in (small, far):
        st = L.alloc_paged_state(B, n_blocks, 6, DEV)
        cache = L.alloc_paged_cache(B, Hkv, n_blocks, DEV)
        state = i32([n_blocks - small, small])          # the last blocks are what is free
        plan = L.paged_plan(i32([0] * B), i32(prompt), st["held"], st["queue"], state, st["table"], max_rows=sum(prompt))
        L.paged_append(cache, k, v, plan)
        kv_len = i32([190, 67])                         # the first's drafts complete a block
        step = L.paged_plan(kv_len, i32([g] * B), plan["new_held"], st["queue"], plan["new_state"], st["table"],
                            max_rows=B * g, reserve=g, draft=True)
        L.paged_append(cache, dk, dv, step)
        outs.append(L.verify_attn_paged(q, cache, st["table"], kv_len))
        new_len = L.paged_commit(cache, st["table"], kv_len, i32([5, 2]), chain)
        assert new_len.tolist() == [195, 69]
        assert int(st["table"].max()) < n_blocks and int(st["table"][0, 0]) == n_blocks - small
        ends.append([x[n_blocks - small:].clone().view(torch.uint8) for x in (cache.k_pool, cache.v_pool)] +
                    [x[n_blocks - small:].clone() for x in (cache.k_scale, cache.v_scale)])
    assert torch.equal(outs[0], outs[1])
    assert all(torch.equal(x, y) for x, y in zip(*ends))
