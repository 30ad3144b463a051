"""The paged cache in 4 bits on the GPU, against the plain forms of mx_ref.

Tolerances.  Codes, scales, ring rows and rows read back: equal.  Attention: as over the cache in 8 bits.  Keys, queries
and values are exact, scores and sums are binary32, and two roundings to bf16 are left (half a step, 2^-8 of the value):
every probability, which moves an output by at most 2^-8 sum p |v|, and the output: |out - ref| <= 2^-8 (sum p |v| +
|ref|), with 2 % for the binary32 part.  The log-sum-exp and the mass come from unrounded probabilities: 2e-5 (1 + |z|)."""
import numpy as np
import pytest
import torch

import mx_ref as M
from test_gpu_paged import APPENDS, ATTNS, COMMITS, D, DEV, L, RING, T, i32, normal, tree  # noqa: F401

pytestmark = pytest.mark.gpu


def ready_mx(L, seed, B, Hkv, lens, extra=3, spare_cols=1):  # noqa: F811
    """A cache with `lens` committed rows in blocks of random places, ring rows everywhere."""
    need = [n // T for n in lens]
    n_blocks = sum(need) + extra
    cache = L.alloc_paged_mx_cache(B, Hkv, n_blocks, DEV)
    rng = np.random.default_rng(seed)
    ids = rng.permutation(n_blocks)
    table = np.full((B, max(need) + spare_cols), -1)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    for x in (cache.k_pool, cache.v_pool):
        x.copy_(torch.from_numpy(rng.integers(0, 256, tuple(x.shape)).astype(np.uint8)))
    for x in (cache.k_scale, cache.v_scale):
        x.copy_(torch.from_numpy(rng.integers(124, 128, tuple(x.shape)).astype(np.uint8)))
    cache.k_tail.copy_(normal(seed + 1, tuple(cache.k_tail.shape)))
    cache.v_tail.copy_(normal(seed + 2, tuple(cache.v_tail.shape)))
    return cache, table


def planned(L, kv, new, n_blocks, cols, pad=0, draft=False):  # noqa: F811
    st = L.alloc_paged_state(len(kv), n_blocks, cols, DEV)
    return L.paged_plan(i32(kv), i32(new), st["held"], st["queue"], st["state"], st["table"], max_rows=sum(new) + pad, draft=draft)


def on_host(plan):
    return {x: y.cpu().numpy() for x, y in plan.items()}


@pytest.mark.parametrize("i", range(len(APPENDS)))
def test_append_and_read(L, i):  # noqa: F811
    c = APPENDS[i]
    kv, new, Hkv = c["kv"], c["new"], c.get("Hkv", 2)
    n = sum(new)
    need = [(a + b) // T for a, b in zip(kv, new)]
    cache, _ = ready_mx(L, i, len(kv), Hkv, [T * x for x in need])
    pad = 3 if i % 2 else 0                         # rows behind the last sequence
    plan = planned(L, kv, new, cache.k_pool.shape[0], max(need) + 1, pad, c.get("draft", False))
    both = normal(100 + i, (n + pad, 2, Hkv, D), 3.0)
    both[:, :, :, 7] *= 40
    both[n:] = float("nan")
    k, v = both[:, 0], both[:, 1]
    ref = M.as_numpy(cache)
    M.append(ref, k.double().cpu().numpy(), v.double().cpu().numpy(), on_host(plan), kv)
    L.paged_mx_append(cache, k, v, plan)
    M.same_cache(cache, ref)
    # the new rows come back as the cache holds them, those of nobody are left
    wide = torch.full((n + pad, 2, Hkv, D), 5.0, dtype=torch.bfloat16, device=DEV)
    got = L.paged_mx_read(cache, plan["slots"], k=wide[:, 0], v=wide[:, 1])
    rk, rv, ok = M.read(ref, plan["slots"].cpu().numpy())
    for x, y in zip(got, (rk, rv)):
        x = x.double().cpu().numpy()
        assert np.array_equal(x[ok], y[ok]) and np.all(x[~ok] == 5.0)
    assert ok.sum() == n


def test_values(L):  # noqa: F811
    """Scales at their borders, every rounding and tie, zeros, small groups, infinities and NaN, the largest numbers."""
    cache, _ = ready_mx(L, 5, 1, 1, [12 * T])
    plan = planned(L, [0], [12 * T], cache.k_pool.shape[0], 13)
    gen = lambda s: torch.randn(T, D, generator=torch.Generator().manual_seed(s))  # noqa: E731
    most = float(torch.finfo(torch.bfloat16).max)
    x = torch.zeros(12, T, D)
    x[0] = torch.linspace(-7, 7, T * D).view(T, D)
    x[0, ::2, ::32], x[0, :8] = 7.0, 7.0                                     # exactly 7
    x[1] = (torch.arange(T * D) % 57 - 28).view(T, D) / 4.0                  # every tie
    x[2] = gen(1) * torch.logspace(-12, 3, D)
    x[3] = x[1] * 1.0078125                                                  # one step more
    x[4] = 1e-30
    x[4, 0, 0], x[4, 9, 70] = 2.0 ** -60, 2.0 ** -62
    x[5] = gen(2) * 1e36
    x[6] = gen(3)
    x[6, 3, 5], x[6, 9, 100], x[6, 60, 2] = float("inf"), float("-inf"), float("nan")
    x[7] = float("nan")
    x[8] = most
    x[8, 1::3] = -most
    x[9] = gen(4) * 2.0 ** 118
    x[9, 2, 3], x[9, 2, 40], x[9, 9, 9] = 3.5 * 2.0 ** 126, -3.25 * 2.0 ** 126, 2.5 * 2.0 ** 126
    x[10] = -0.0
    x[11] = gen(5) * 2.0 ** -126                                             # subnormal products and numbers
    k = x.view(12 * T, 1, D).to(torch.bfloat16).to(DEV)
    v = k.flip(0).contiguous()
    ref = M.as_numpy(cache)
    M.append(ref, k.double().cpu().numpy(), v.double().cpu().numpy(), on_host(plan), [0])
    L.paged_mx_append(cache, k, v, plan)
    M.same_cache(cache, ref)
    back = L.paged_mx_read(cache, plan["slots"])
    for got, want in zip(back, M.read(ref, plan["slots"].cpu().numpy())):
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
    finite = torch.isfinite(k)
    seen = torch.isfinite(back[0])
    assert bool((seen <= finite).all()) and int((finite & ~seen).sum()) == 3 * 31
    # half a step of the group's scale, which is at most a third of its largest value (a half where codes end at 3)
    top = k.double().abs().nan_to_num(posinf=0).view(-1, 4, 32).amax(-1, keepdim=True).expand(-1, 4, 32).reshape(k.shape)
    off = (back[0].double() - k.double()).abs()
    assert bool((off[seen] <= torch.maximum(top / 3, torch.tensor(2.0 ** -62, device=DEV).double())[seen]).all())


def test_read_any_slots(L):  # noqa: F811
    """Slots in any order, twice, out of range, of many blocks, of the ring."""
    cache, _ = ready_mx(L, 8, 3, 2, [T * 5, 0, T])
    rng = np.random.default_rng(1)
    n_blocks = cache.k_pool.shape[0]
    slots = np.concatenate([rng.integers(0, n_blocks * T, 300), -2 - rng.integers(0, 3 * RING, 100), [-1, n_blocks * T, -2 - 3 * RING, 2 ** 31 - 1,
                            -2 ** 31], [7] * 70])
    slots = rng.permutation(slots)
    k = torch.full((len(slots), 2, D), 5.0, dtype=torch.bfloat16, device=DEV)
    v = k.clone()
    L.paged_mx_read(cache, i32(slots), k=k, v=v)
    rk, rv, ok = M.read(M.as_numpy(cache), slots)
    for x, y in ((k, rk), (v, rv)):
        x = x.double().cpu().numpy()
        assert np.array_equal(x[ok], y[ok]) and np.all(x[~ok] == 5.0)
    assert (~ok).sum() == 5
    zeros = L.paged_mx_read(cache, i32([-1] * 3))
    assert not bool(zeros[0].any()) and not bool(zeros[1].any())
    assert L.paged_mx_read(cache, i32([]))[0].shape == (0, 2, D)


def check_attention(L, q, cache, table, kv, vis=None, mask=None, scale=0.0, **kw):  # noqa: F811
    opt = dict(vis_begin=i32(vis[0]), vis_end=i32(vis[1])) if vis is not None else {}
    out, lse, mass = L.verify_attn_paged_mx(q, cache, i32(table), i32(kv), draft_mask=mask, scale=scale, return_lse=True,
                                            return_vis_mass=vis is not None, **opt, **kw)
    ro, rl, rm, size = M.attention(q.double().cpu().numpy(), M.as_numpy(cache), np.asarray(table), kv, mask,
                                   scale if scale > 0 else None, vis)
    o = out.double().cpu().numpy()
    assert np.all(np.isfinite(o))
    assert np.all(np.abs(o - ro) <= 1.02 * 2.0 ** -8 * (size + np.abs(ro)) + 1e-30), float(
        np.max(np.abs(o - ro) / (size + np.abs(ro)))) * 256
    assert np.all(np.abs(lse.cpu().numpy() - rl) <= 2e-5 * (1 + np.abs(rl))), float(np.max(np.abs(lse.cpu().numpy() - rl)))
    if vis is not None:
        assert np.all(np.abs(mass.cpu().numpy() - rm) <= 2e-5 * (1 + np.abs(rl)))
    return out


@pytest.mark.parametrize("spare_cols", [1, 70])        # a unit in one workgroup where it is short, or cut into parts
@pytest.mark.parametrize("i", range(len(ATTNS)))
def test_attention(L, i, spare_cols):  # noqa: F811
    c = ATTNS[i]
    kv, g, Hq, Hkv = c["kv"], c["g"], c.get("Hq", 4), c.get("Hkv", 2)
    B = len(kv)
    cache, table = ready_mx(L, 50 + i, B, Hkv, kv, spare_cols=spare_cols)
    q = normal(200 + i, (B, g, Hq, D))
    mask = tree(c["branches"], g // c["branches"]) if "branches" in c else None
    vis = ([5] * B, [max(5, n * 2 // 3) for n in kv]) if i % 2 else None
    check_attention(L, q, cache, table, kv, vis, mask, c.get("scale", 0.0))


def test_attention_strides_and_span(L):  # noqa: F811
    """q and out as slices of wider buffers; spans that are empty, cut tiles, or reach the drafts."""
    kv, g, Hq, Hkv = [400, 65, 7], 6, 12, 4
    cache, table = ready_mx(L, 90, 3, Hkv, kv, spare_cols=4)
    q = normal(91, (g, 3, Hq + 3, D + 64)).permute(1, 0, 2, 3)[:, :, 1:Hq + 1, 64:]
    out = torch.full((3, g, 2, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    check_attention(L, q, cache, table, kv, ([0, 60, 3], [0, 66, 100]), out=out[:, :, 1])
    assert bool((out[:, :, 0] == 7.0).all())
    check_attention(L, q, cache, table, kv, ([13, -5, 0], [333, 64, 1]))


@pytest.mark.parametrize("spare_cols", [3, 70])
def test_attention_reads_declared_rows_only(L, spare_cols):  # noqa: F811
    """Unused blocks, table entries behind the length and ring rows of nobody hold NaN."""
    kv, g = [200, 64, 30, 0], 5
    cache, table = ready_mx(L, 92, 4, 2, kv, extra=4, spare_cols=spare_cols)
    q = normal(93, (4, g, 8, D))
    want = check_attention(L, q, cache, table, kv).clone()
    used = {int(table[b, j]) for b in range(4) for j in range(kv[b] // T)}
    free = [i for i in range(cache.k_pool.shape[0]) if i not in used]
    for i in free:
        cache.k_scale[i] = cache.v_scale[i] = 255
    for b, n in enumerate(kv):
        mine = {p % RING for p in range(n // T * T, n + g)}
        for r in range(RING):
            if r not in mine:
                cache.k_tail[b, :, r] = float("nan")
                cache.v_tail[b, :, r] = float("inf")
        table[b, n // T:] = [free[0], 1 << 30, -9][b % 3]
    assert torch.equal(L.verify_attn_paged_mx(q, cache, i32(table), i32(kv)), want)


@pytest.mark.parametrize("spare_cols", [1, 70])
def test_groups_that_are_not_finite(L, spare_cols):  # noqa: F811
    """A key group of NaN makes every row of its sequence and head NaN, one of values their channel; nobody else's."""
    kv, g = [200, 300], 3
    cache, table = ready_mx(L, 94, 2, 2, kv, spare_cols=spare_cols)
    q = normal(95, (2, g, 8, D))
    want, lse, _ = L.verify_attn_paged_mx(q, cache, i32(table), i32(kv), return_lse=True)
    v = cache.v_scale.clone()
    cache.v_scale[table[0, 1], 1, 1, 17 % 32, 17 // 32] = 255                  # head 1, channel 17
    cache.v_pool[table[0, 1], 1, 17, 16:] = 0
    got, same, _ = L.verify_attn_paged_mx(q, cache, i32(table), i32(kv), return_lse=True)
    hit = torch.zeros(want.shape, dtype=torch.bool, device=DEV)
    hit[0, :, 4:, 17] = True
    assert bool(torch.isnan(got[hit]).all()) and torch.equal(got[~hit], want[~hit]) and torch.equal(same, lse)
    cache.v_scale.copy_(v)
    cache.k_scale[table[1, 2], 0, 1, 5, 2] = 255                               # head 0, token 37, channels 32 .. 63
    cache.k_pool[table[1, 2], 0, 0, 37, 16:] = 0
    got, lse2, _ = L.verify_attn_paged_mx(q, cache, i32(table), i32(kv), return_lse=True)
    hit[:] = False
    hit[1, :, :4] = True
    assert bool(torch.isnan(got[hit]).all()) and bool(torch.isnan(lse2[1, :4]).all()) and torch.equal(lse2[0], lse[0])
    assert torch.equal(lse2[1, 4:], lse[1, 4:])
    ok = ~hit
    ok[0, :, 4:, 17] = False                                                  # (its codes are 0 now)
    assert torch.equal(got[ok], want[ok])


@pytest.mark.parametrize("spare_cols", [1, 70])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_masked_draft_rows_do_not_reach_others(L, value, spare_cols):  # noqa: F811
    kv, g = [100, 64], 6
    cache, table = ready_mx(L, 96, 2, 2, kv, spare_cols=spare_cols)
    q = normal(95, (2, g, 8, D))
    want = L.verify_attn_paged_mx(q, cache, i32(table), i32(kv)).clone()
    for b, n in enumerate(kv):
        cache.v_tail[b, :, (n + 3) % RING, 17] = value
        cache.k_tail[b, :, (n + 5) % RING, 3] = value
    got = L.verify_attn_paged_mx(q, cache, i32(table), i32(kv))
    assert torch.equal(got[:, :3], want[:, :3])
    rest = torch.arange(D, device=DEV) != 17
    assert torch.equal(got[:, 3:5, :, rest], want[:, 3:5, :, rest])
    hit = got[:, 3:5, :, 17].float()
    assert bool((torch.isnan(hit) if value != value else hit == value).all())


@pytest.mark.parametrize("spare_cols", [0, 70])
def test_attention_lengths_and_blocks_out_of_range(L, spare_cols):  # noqa: F811
    kv, g = [300, 300, 300], 3
    cache, table = ready_mx(L, 96, 3, 2, kv, spare_cols=spare_cols)
    q = normal(97, (3, g, 4, D))
    table[1, 2], table[2, 0] = -1, cache.k_pool.shape[0]
    check_attention(L, q, cache, table, kv)
    most = table.shape[1] * T + T - 1
    a = L.verify_attn_paged_mx(q, cache, i32(table), i32([-5, 10 ** 9, most]))
    assert torch.equal(a, L.verify_attn_paged_mx(q, cache, i32(table), i32([0, most, most])))
    check_attention(L, q, cache, np.zeros((3, 0), np.int32), [20, 0, 63])
    table[:] = -1                                                             # nobody has a block
    check_attention(L, q, cache, table, kv)


@pytest.mark.parametrize("spare_cols", [1, 70])
@pytest.mark.parametrize("n", [0, 3, 64, 1500])
def test_scores_far_below_any_usual_one(L, n, spare_cols):  # noqa: F811
    """All scores of a row near -2^110: exact powers of two that differ by far more than any softmax resolves, so the row
    is the value of its largest score, equal ones share it, and lse is that score."""
    H, rows = 2, 3
    cache, table = ready_mx(L, 900 + n, 1, H, [n], spare_cols=spare_cols)
    rng = np.random.default_rng(n)
    size = torch.from_numpy(2.0 ** -rng.integers(0, 2, (H, n + 1))).float()   # codes of 1 and 0.5
    value = torch.from_numpy(rng.integers(-6, 7, (H, n + 1, D)) / 4.0).float()
    plan = planned(L, [0], [n], cache.k_pool.shape[0], table.shape[1])
    k = torch.zeros((n, H, D))
    k[..., 3] = size[:, :n].T
    if n:
        L.paged_mx_append(cache, k.to(DEV, torch.bfloat16), value[:, :n].transpose(0, 1).contiguous().to(DEV, torch.bfloat16), plan)
        table = np.concatenate([np.arange(n // T), [-1] * (table.shape[1] - n // T)])[None]
        held = M.values_of(M.as_numpy(cache))
        for j in range(n // T):                                               # (values are rounded: take what is there)
            for h in range(H):
                size[h, j * T:j * T + T] = torch.from_numpy(held[0][j, h, :, 3])
                value[h, j * T:j * T + T] = torch.from_numpy(held[1][j, h])
    cache.k_tail[0, :, n % RING] = 0
    cache.k_tail[0, :, n % RING, 3] = size[:, n].to(DEV, torch.bfloat16)
    cache.v_tail[0, :, n % RING] = value[:, n].to(DEV, torch.bfloat16)
    q = torch.zeros((1, 1, rows * H, D))
    q[..., 3] = -2.0 ** 113
    out, lse, _ = L.verify_attn_paged_mx(q.to(DEV, torch.bfloat16), cache, i32(table), i32([n]), scale=1.0, return_lse=True)
    for h in range(H):
        least = float(size[h].min())
        want = value[h][size[h] == least].double().mean(0)
        got = out[0, 0, h * rows:(h + 1) * rows].double().cpu()
        assert bool(((got - want).abs() <= (2.0 ** -8 + 2.0 ** -22) * want.abs() + 1e-30).all())
        s = lse[0, h * rows:(h + 1) * rows].double().cpu()
        assert bool(((s + 2.0 ** 113 * least).abs() <= 2.0 ** 113 * least * 2.0 ** -21).all())


@pytest.mark.parametrize("spare_cols", [1, 70])
@pytest.mark.parametrize("power", [23, 30, 45, 113])
def test_scores_far_from_usual_ones(L, power, spare_cols):  # noqa: F811
    """Scores of all sizes up to 2^power, times a scale that binary32 does not hold, so that no maximum is exact: the row is the
    mean of the values of its largest score (equal scores have equal weights, the others are far below)."""
    n, H, rows = 64 * 21 + 5, 2, 3
    cache, table = ready_mx(L, 940 + power, 1, H, [n], spare_cols=spare_cols)
    rng = np.random.default_rng(power)
    for x in (cache.k_pool, cache.k_tail):
        x.zero_()
    cache.k_scale.fill_(127)
    code = torch.from_numpy(rng.integers(0, 8, (cache.k_pool.shape[0], H, T)).astype(np.uint8)).to(DEV)
    cache.k_pool[:, :, 0, :, 1] = code << 4                                    # channel 3
    cache.k_tail[..., 3] = torch.from_numpy(rng.integers(0, 7, (1, H, RING)).astype(np.float32)).to(DEV)
    q = torch.zeros((1, 1, rows * H, D))
    q[..., 3] = torch.tensor([1.0, -1.0, 1.375] * H) * 2.0 ** (power - 3)
    out, lse, _ = L.verify_attn_paged_mx(q.to(DEV, torch.bfloat16), cache, i32(table), i32([n]), scale=0.7, return_lse=True)
    ro, rl, _, size = M.attention(q.double().numpy(), M.as_numpy(cache), table, [n], None, float(np.float32(0.7)))
    assert np.all(np.abs(out.double().cpu().numpy() - ro) <= 1.02 * 2.0 ** -8 * (size + np.abs(ro)))
    assert np.all(np.abs(lse.double().cpu().numpy() - rl) <= 2e-5 * (1 + np.abs(rl)))


@pytest.mark.parametrize("spare_cols", [1, 70])
def test_queries_of_any_size(L, spare_cols):  # noqa: F811
    """Rows from bf16's smallest to its largest numbers, with channels of every size beside each other, where the score
    scale brings them back; and a row that is not finite is NaN, the others are what they are without it.

    Keys here are powers of two on one channel a token, so that a score is one product: queries within 2^-7 of their 32's
    largest go into it exactly, smaller ones with 2^-15 of that largest at most, which is below 2^-12 for scores up to 8."""
    kv, g, H = [130, 700], 4, 2
    cache, table = ready_mx(L, 970, 2, H, kv, spare_cols=spare_cols)
    cache.k_pool.zero_()
    cache.k_scale.fill_(127)
    one = torch.arange(64, device=DEV)
    cache.k_pool[:, :, 0, one, one % 32] = 0x02                                # code of 1 on channel 2 (t % 32), first half
    cache.k_tail.zero_()
    for p in range(RING):
        cache.k_tail[:, :, p, 2 * (p % 64 % 32)] = 1.0
    base = normal(971, (2, g, 4, D))
    base = base.clamp(-4, 4)
    base[:, :, 1] *= torch.logspace(-6, 0, D, device=DEV).to(torch.bfloat16)   # channels of very different sizes
    for e, scale, keys in ((0, 1.0, 0), (100, 2.0 ** -100, 0), (-100, 0.0, 0), (-100, 1.0, 100), (-115, 1.0, 115), (125, 2.0 ** -125, 0)):
        cache.k_scale.fill_(127 + keys)
        cache.k_tail.copy_(torch.where(cache.k_tail != 0, 2.0 ** keys, 0.0))
        q = (base.float() * 2.0 ** e).to(torch.bfloat16) if e != 125 else (base.float().clamp(-3.98, 3.98) * 2.0 ** 126).to(torch.bfloat16)
        q = torch.where(q.abs() < 2.0 ** -126, torch.zeros_like(q), q)         # (numbers with all their bits only)
        out, lse, _ = L.verify_attn_paged_mx(q, cache, i32(table), i32(kv), scale=scale, return_lse=True)
        ro, rl, _, size = M.attention(q.double().cpu().numpy(), M.as_numpy(cache), table, kv, None, scale if scale > 0 else None)
        o = out.double().cpu().numpy()
        assert np.all(np.isfinite(o))
        # a score off by d moves a probability by its d-th part: 2^-12, beside the two roundings to bf16
        assert np.all(np.abs(o - ro) <= (1.02 * 2.0 ** -8 + 2.0 ** -11) * (size + np.abs(ro)) + 1e-30), e
        assert np.all(np.abs(lse.cpu().numpy() - rl) <= 2.0 ** -12 + 2e-5 * (1 + np.abs(rl))), e
    cache.k_scale.fill_(127)
    cache.k_tail.copy_((cache.k_tail != 0).to(torch.bfloat16))
    want, wl, _ = L.verify_attn_paged_mx(base, cache, i32(table), i32(kv), return_lse=True)
    for value in (float("nan"), float("inf"), float("-inf")):
        q = base.clone()
        q[1, 2, 3, 77] = value
        got, gl, _ = L.verify_attn_paged_mx(q, cache, i32(table), i32(kv), return_lse=True)
        hit = torch.zeros(got.shape, dtype=torch.bool, device=DEV)
        hit[1, 2, 3] = True
        assert bool(torch.isnan(got[hit]).all()) and torch.equal(got[~hit], want[~hit])
        assert bool(torch.isnan(gl[1, 3, 2])) and torch.equal(gl[0], wl[0])


def test_attention_over_the_largest_values(L):  # noqa: F811
    """Equal weights over one block of the largest numbers: their mean is finite."""
    cache = L.alloc_paged_mx_cache(1, 1, 1, DEV)
    rows = torch.full((T, 1, D), float(torch.finfo(torch.bfloat16).max), dtype=torch.bfloat16, device=DEV)
    rows[1::2] *= -1
    plan = planned(L, [0], [T], 1, 1)
    L.paged_mx_append(cache, torch.zeros_like(rows), rows, plan)
    out = L.verify_attn_paged_mx(torch.ones((1, 1, 1, D), dtype=torch.bfloat16, device=DEV), cache, i32([[0]]), i32([T]))
    assert bool((out.abs() <= 2.0 ** 128 * 1e-6).all())


@pytest.mark.parametrize("spare_cols", [1, 70])
@pytest.mark.parametrize("step", [1, 2, 7, 9])
def test_large_values_where_scores_rise(L, step, spare_cols):  # noqa: F811
    """One key of every tile has a score, from eight tiles to the next `step` (in base 2) higher, and the value 2^121; the
    others are 2^300 below.  No weight is above 1 at any time, so sums of 41 are finite, and the output is 2^121."""
    H, tiles = 128, 40
    cache, table = ready_mx(L, 990, 1, H, [T * tiles], spare_cols=spare_cols)
    for x in (cache.k_pool, cache.v_pool, cache.k_tail, cache.v_tail):
        x.zero_()
    cache.k_scale.fill_(127)
    cache.v_scale.fill_(127 + 121)
    cache.k_pool[:, :, 0, 1:, 0] = 0x0F                                        # channel 0: -6, of token 0: 0
    cache.k_tail[..., 0] = -6.0
    for j, block in enumerate(table[0][:tiles].tolist()):
        cache.k_pool[block, :, 0, 0, 1] = (0, 2, 4, 5, 6)[j // 8]              # channel 2: 0 1 2 3 4
        cache.v_pool[block, :, :, 0] = 0x02                                    # token 0: 1
    q = torch.zeros((1, 1, 2 * H, D))
    q[..., 0], q[..., 2] = 64.0, step
    out = L.verify_attn_paged_mx(q.to(DEV, torch.bfloat16), cache, i32(table), i32([T * tiles]), scale=float(np.log(2.0)))
    # probabilities and the output rounded to bf16
    assert bool(((out.double() - 2.0 ** 121).abs() <= 2.0 ** 121 * 1.02 * 2.0 ** -7).all())


def test_attention_is_the_same_every_time_and_on_streams(L):  # noqa: F811
    kv = [1500, 3000, 10, 640]
    cache, table = ready_mx(L, 98, 4, 4, kv, spare_cols=70)
    q, t, n = normal(99, (4, 5, 20, D)), i32(table), i32(kv)
    first = L.verify_attn_paged_mx(q, cache, t, n)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [L.verify_attn_paged_mx(q, cache, t, n, stream=s) for _ in range(4) for s in (streams[0], streams[1].cuda_stream)]
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(first, x) for x in got) and torch.equal(first, L.verify_attn_paged_mx(q, cache, t, n))


@pytest.mark.parametrize("i", range(len(COMMITS)))
@pytest.mark.parametrize("layers", [1, 3])
def test_commit(L, i, layers):  # noqa: F811
    c = COMMITS[i]
    kv, br, chain = c["kv"], c.get("branches", 1), c["chain"]
    B = len(kv)
    parts = [ready_mx(L, 300 + 10 * i + y, B, 2, [T * (n // T + 1) for n in kv]) for y in range(layers)]
    table, best = parts[0][1], c.get("best")
    cache = L.PagedMxCache(*[torch.stack([p[0][x] for p in parts]) for x in range(6)])
    kw = dict(n_branches=br, best_branch=None if best is None else i32(best))
    refs = [M.as_numpy(p[0]) for p in parts]
    want = [M.commit(r, table, kv, np.minimum(c["tau"], chain), chain, best, br) for r in refs][0]
    assert np.array_equal(L.paged_mx_commit(cache, i32(table), i32(kv), i32(c["tau"]), chain, **kw).cpu().numpy(), want)
    for y in range(layers):
        M.same_cache(cache.layer(y), refs[y], f"layer {y}")
    if layers == 1:
        L.paged_mx_commit(parts[0][0], i32(table), i32(kv), i32(c["tau"]), chain, **kw)
        M.same_cache(parts[0][0], refs[0])


def test_commit_without_a_place_and_by_a_plan(L):  # noqa: F811
    kv = [62, 62, -4, 10 ** 8, 62, 191]
    cache, _ = ready_mx(L, 400, 6, 2, [0] * 6, extra=5)
    n_blocks = cache.k_pool.shape[0]
    table = np.array([[-1, 0, 0], [n_blocks, 0, 0], [0, 0, 0], [1, 1, 1], [4, 0, 0], [0, 0, 3]])
    ref = M.as_numpy(cache)
    want = M.commit(ref, table, kv, [5] * 12, 5, [1] * 6, 2)
    got = L.paged_mx_commit(cache, i32(table), i32(kv), i32([5] * 12), 5, n_branches=2, best_branch=i32([1] * 6))
    assert got.tolist() == want.tolist() == [62, 62, -4, 10 ** 8, 67, 196]
    M.same_cache(cache, ref)
    # refused, granted, nothing brought, fewer rows than accepted, and a block that is not held
    kv, br, chain = [62, 62, 62, 62, 62, 62, 20], 2, 5
    cache, table = ready_mx(L, 700, 7, 2, [T] * 7)
    plan = dict(granted=i32([0, 1, 1, 1, 1, 0, 1]), new_held=i32([1, 1, 1, 1, 0, 0, 0]), cu_rows=i32(np.cumsum([0, 10, 10, 0, 8, 10, 10, 6])))
    best, came = [1, 1, 1, 1, 0, 0, 1], [10, 10, 0, 8, 10, 10, 6]
    tau = [min(4, max(came[b] - a * chain, 0)) if b not in (0, 5) else 0 for b in range(7) for a in range(br)]
    ref, lent = M.as_numpy(cache), table.copy()
    lent[4] = -1
    want = M.commit(ref, lent, kv, tau, chain, best, br)
    got = L.paged_mx_commit(cache, i32(table), i32(kv), i32([4] * 14), chain, n_branches=br, best_branch=i32(best), plan=plan)
    assert got.tolist() == want.tolist() == [62, 66, 62, 65, 62, 62, 21]
    M.same_cache(cache, ref)


def test_serving_loop(L):  # noqa: F811
    """The operators together: prompts in pieces and verified steps with trees, keys and queries rotated on the way, on a
    pool that runs dry, against lists of rotated rows; the rows read back are those that attention goes over."""
    rng = np.random.default_rng(8)
    B, Hkv, Hq, br, chain, n_blocks, cols = 4, 2, 8, 2, 4, 5, 7
    g = br * chain
    inv, factor = L.rotary_frequencies(64, scaling=L.SCALING_YARN, scale=4.0, original_len=64, device=DEV)
    rot = L.Rotary(inv, factor)
    st = L.alloc_paged_state(B, n_blocks, cols, DEV)
    cache = L.alloc_paged_mx_cache(B, Hkv, n_blocks, DEV)
    rows = [[] for _ in range(B)]
    kv, refused, mask = np.zeros(B, np.int64), 0, tree(br, chain)
    turn = lambda k, pos: M.to_bf16(M.rotate(k.double().cpu().numpy(), pos, inv.cpu().numpy(), factor=float(np.float32(factor))))  # noqa: E731

    def plan(new, max_rows, **kw):
        p = L.paged_plan(i32(kv), i32(new), st["held"], st["queue"], st["state"], st["table"], max_rows=max_rows, **kw)
        st["held"], st["state"] = p["new_held"], p["new_state"]
        return p, p["granted"].cpu().numpy(), p["cu_rows"].cpu().numpy()

    for step in range(30):
        new = np.where(rng.random(B) < 0.35, rng.integers(1, 90, B), 0)         # prompts and further pieces
        new = np.where(kv + new + 2 * g < cols * T, new, 0)
        p, ok, cu = plan(new, int(new.sum()))
        k, v = normal(1000 + step, (int(new.sum()), Hkv, D)), normal(2000 + step, (int(new.sum()), Hkv, D))
        if new.sum():
            L.paged_mx_append(cache, k, v, p, rot=rot)
            tk, tv = turn(k, p["row_pos"].cpu().numpy()), v.double().cpu().numpy()
            for b in np.flatnonzero((new > 0) & (ok != 0)):
                rows[b] += [(tk[t], tv[t]) for t in range(cu[b], cu[b + 1])]
                kv[b] += new[b]
        p, ok, cu = plan(np.where(kv > 0, g, -1), B * g, reserve=g, draft=True)
        k, v, q = (normal(s + step, (B * g, h, D)) for s, h in ((3000, Hkv), (4000, Hkv), (5000, Hq)))
        turned = L.paged_mx_append(cache, k, v, p, rot=rot, q=q)
        tk, tv = turn(k, p["row_pos"].cpu().numpy()), v.double().cpu().numpy()
        if step % 5 == 0:
            full = torch.zeros((B, g, Hq, D), dtype=torch.bfloat16, device=DEV)
            for b in range(B):
                if cu[b + 1] > cu[b]:
                    full[b] = turned[cu[b]:cu[b + 1]]
            check_attention(L, full, cache, st["table"].cpu().numpy(), kv.tolist(), mask=mask)
        tau, best = rng.integers(1, chain + 1, B * br), rng.integers(0, br, B)
        got = L.paged_mx_commit(cache, st["table"], i32(kv), i32(tau), chain, n_branches=br, best_branch=i32(best), plan=p)
        for b in range(B):
            if cu[b + 1] > cu[b] and ok[b]:
                n, at = int(tau[b * br + best[b]]), cu[b] + int(best[b]) * chain
                rows[b] += [(tk[at + i], tv[at + i]) for i in range(n)]
                kv[b] += n
            refused += int(cu[b + 1] > cu[b] and not ok[b])
        assert got.tolist() == kv.tolist()
        arr, table = M.as_numpy(cache), st["table"].cpu().numpy()
        for b in range(B):
            if not rows[b]:
                continue
            n = len(rows[b])
            pos = np.arange(n)
            slots = np.where(pos < n // T * T, table[b, np.minimum(pos // T, cols - 1)] * T + pos % T, -2 - (b * RING + pos % RING))
            back = [x.double().cpu().numpy() for x in L.paged_mx_read(cache, i32(slots))]
            for which, block in ((0, M.keys_block), (1, M.values_block)):
                x = np.stack([r[which] for r in rows[b]])
                assert np.array_equal(back[which][n // T * T:], x[n // T * T:])
                for j in range(n // T):
                    for h in range(Hkv):
                        codes, sc = block(x[j * T:j * T + T, h])
                        at = table[b, j]
                        assert np.array_equal(arr[which][at, h], codes) and np.array_equal(arr[2 + which][at, h], sc), (b, j)
            if kv[b] > 200 and rng.random() < 0.5 or kv[b] + 3 * g >= cols * T:
                kv[b], rows[b] = 0, []
    assert refused > 0


def test_steps_in_a_graph(L):  # noqa: F811
    """A captured step (plan, append with rotation, attention, commit, read), replayed between eager work."""
    B, Hkv, Hq, g = 2, 2, 8, 4
    st = L.alloc_paged_state(B, 30, 10, DEV)
    cache = L.alloc_paged_mx_cache(B, Hkv, 30, DEV, layers=1)
    rot = L.Rotary(L.rotary_frequencies(128, device=DEV)[0])
    kv_len, new = i32([61, 126]), i32([g] * B)
    prompt = L.paged_plan(i32([0, 0]), kv_len, st["held"], st["queue"], st["state"], st["table"], max_rows=187)
    L.paged_mx_append(cache.layer(0), normal(1, (187, Hkv, D)), normal(2, (187, Hkv, D)), prompt, rot=rot)
    held, state = prompt["new_held"].clone(), prompt["new_state"].clone()
    twin = [x.clone() for x in (*cache, st["queue"], st["table"], kv_len, held, state)]
    k, v, q = (torch.zeros((B * g, h, D), dtype=torch.bfloat16, device=DEV) for h in (Hkv, Hkv, Hq))
    tau = i32([0] * B)

    def step(cache, queue, table, kv_len, held, state):
        plan = L.paged_plan(kv_len, new, held, queue, state, table, max_rows=B * g, reserve=g, draft=True)
        held.copy_(plan["new_held"])
        state.copy_(plan["new_state"])
        turned = L.paged_mx_append(cache.layer(0), k, v, plan, rot=rot, q=q)
        out = L.verify_attn_paged_mx(turned.view(B, g, Hq, D), cache.layer(0), table, kv_len)
        kv_len.copy_(L.paged_mx_commit(cache, table, kv_len, tau, g, plan=plan))
        return out, *L.paged_mx_read(cache.layer(0), plan["slots"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache, st["queue"], st["table"], kv_len, held, state)      # (tau = 0: nothing moves on)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(cache, st["queue"], st["table"], kv_len, held, state)
    step(L.PagedMxCache(*twin[:6]), *twin[6:])
    for i in range(8):
        for x, s in ((k, 10), (v, 30), (q, 50)):
            x.copy_(normal(s + i, tuple(x.shape)))
        tau.copy_(i32([i % 5, (3 * i) % 5]))
        graph.replay()
        want = step(L.PagedMxCache(*twin[:6]), *twin[6:])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want)), i
        assert all(torch.equal(x, y) for x, y in zip((*cache, st["queue"], st["table"], kv_len, held, state), twin)), i
    assert kv_len.tolist()[0] > 64


def test_pool_of_more_than_4_gib(L):  # noqa: F811
    """The last blocks of a large pool hold and give what the blocks of a small one do."""
    B, Hkv, Hq, g, prompt = 2, 4, 8, 5, [200, 70]
    small, far = 8, (1 << 18) + 64                      # 4 GiB and some of keys, as much of values
    k, v = normal(1, (sum(prompt), Hkv, D)), normal(2, (sum(prompt), Hkv, D))
    dk, dv, q = normal(3, (B * g, Hkv, D)), normal(4, (B * g, Hkv, D)), normal(5, (B, g, Hq, D))
    rot = L.Rotary(L.rotary_frequencies(128, device=DEV)[0])
    outs, ends = [], []
    for n_blocks in (small, far):
        st = L.alloc_paged_state(B, n_blocks, 6, DEV)
        cache = L.alloc_paged_mx_cache(B, Hkv, n_blocks, DEV)
        state = i32([n_blocks - small, small])          # the last blocks are what is free
        plan = L.paged_plan(i32([0] * B), i32(prompt), st["held"], st["queue"], state, st["table"], max_rows=sum(prompt))
        L.paged_mx_append(cache, k, v, plan, rot=rot)
        kv_len = i32([190, 67])                         # the first's drafts complete a block
        step = L.paged_plan(kv_len, i32([g] * B), plan["new_held"], st["queue"], plan["new_state"], st["table"],
                            max_rows=B * g, reserve=g, draft=True)
        L.paged_mx_append(cache, dk, dv, step)
        back = L.paged_mx_read(cache, plan["slots"])
        outs.append([L.verify_attn_paged_mx(q, cache, st["table"], kv_len), *back])
        assert L.paged_mx_commit(cache, st["table"], kv_len, i32([5, 2]), 5).tolist() == [195, 69]
        assert int(st["table"].max()) < n_blocks and int(st["table"][0, 0]) == n_blocks - small
        ends.append([x[n_blocks - small:].clone() for x in cache[:4]])
        del cache
    assert all(torch.equal(x, y) for x, y in zip(*outs))
    assert all(torch.equal(x, y) for x, y in zip(*ends))
