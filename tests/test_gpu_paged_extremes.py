"""The paged cache at the ends of bf16's range.  Codes and scales are equal to the plain form's."""
import numpy as np
import pytest
import torch

import paged_ref as R
from test_gpu_paged import D, DEV, L, RING, T, i32, normal, ready, same_cache  # noqa: F401

pytestmark = pytest.mark.gpu

MOST = float(torch.finfo(torch.bfloat16).max)


def finite_block(x):
    """block8 with codes of finite values that have finite values: 240 at most at the scale 2^120."""
    _, s = R.block8(x)
    top = 240.0 if s == 2.0 ** 120 else 448.0
    return R.nearest8(np.where(np.isfinite(x), np.clip(x / s, -top, top), x)), s


def extreme_rows(seed):
    """Three blocks: the largest values, ones around 248 * 2^120 with others of every size, and 247 * 2^120."""
    x = torch.randn(3, T, D, generator=torch.Generator().manual_seed(seed)) * 2.0 ** 118
    x[0, ::3] = MOST
    x[0, 1::3] = -MOST
    x[0, 5, 7], x[0, 6, 7], x[0, 7, 7] = float("inf"), float("-inf"), float("nan")
    x[1, 2, 3], x[1, 2, 4], x[1, 9, 9] = 248.0 * 2.0 ** 120, -247.0 * 2.0 ** 120, 225.0 * 2.0 ** 120
    x[1, 20:] = torch.randn(T - 20, D, generator=torch.Generator().manual_seed(seed + 1))
    x[2, 4, 4] = -247.0 * 2.0 ** 120
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("by", ["append", "commit"])
def test_largest_values_stay_finite(L, by):  # noqa: F811
    H, rows = 2, torch.stack([extreme_rows(1), extreme_rows(5)], 2)           # [3, T, H, D]
    if by == "append":
        cache = L.alloc_paged_cache(1, H, 3, DEV)
        st = L.alloc_paged_state(1, 3, 3, DEV)
        k = rows.reshape(3 * T, H, D).to(DEV)
        v = rows.flip(1).reshape(3 * T, H, D).contiguous().to(DEV)
        plan = L.paged_plan(i32([0]), i32([3 * T]), st["held"], st["queue"], st["state"], st["table"], max_rows=3 * T)
        L.paged_append(cache, k, v, plan)
        ids = st["table"][0].tolist()
    else:                                                                    # the last row of three sequences' blocks
        cache, ids = L.alloc_paged_cache(3, H, 3, DEV), [2, 0, 1]
        cache.k_tail[:, :, :T] = rows.transpose(1, 2).to(DEV)
        cache.v_tail[:, :, :T] = rows.flip(1).transpose(1, 2).to(DEV)
        assert L.paged_commit(cache, i32([[i] for i in ids]), i32([T - 1] * 3), i32([1] * 3), 1).tolist() == [T] * 3
    k8, v8, ks, vs = R.as_numpy(cache)[:4]
    for j, i in enumerate(ids):
        for h in range(H):
            for pool, scale, x in ((k8, ks, rows[j, :, h]), (v8, vs, rows[j].flip(0)[:, h])):
                x = x.double().numpy()
                got = pool[i, h] if pool is k8 else pool[i, h].T
                codes, s = finite_block(x)
                nan = ~np.isfinite(x)
                assert scale[i, h] == s and np.array_equal(got[~nan], codes[~nan]) and np.all(got[nan] & 127 == 127)
                value = (R.value_of(got[~nan]) * s).astype(np.float32)
                assert np.all(np.isfinite(value)) and np.all(np.abs(value - x[~nan]) <= np.abs(x[~nan]) * 2.0 ** -4 + s * 2.0 ** -10)
    assert ks.max() == 2.0 ** 120


def test_attention_over_the_largest_values(L):  # noqa: F811
    """Equal weights over one block of the largest values: their mean is finite, where one infinite value would
    not be."""
    cache = L.alloc_paged_cache(1, 1, 1, DEV)
    rows = torch.full((T, 1, D), MOST, dtype=torch.bfloat16, device=DEV)
    rows[1::2] = -MOST
    st = L.alloc_paged_state(1, 1, 1, DEV)
    plan = L.paged_plan(i32([0]), i32([T]), st["held"], st["queue"], st["state"], st["table"], max_rows=T)
    L.paged_append(cache, torch.zeros_like(rows), rows, plan)
    out = L.verify_attn_paged(torch.ones((1, 1, 1, D), dtype=torch.bfloat16, device=DEV), cache, st["table"], i32([T]))
    # 65 keys of score 0, the draft row's value 0
    assert bool((out.abs() <= 2.0 ** 128 * 1e-6).all())


@pytest.mark.parametrize("spare_cols", [1, 70])        # a unit in one workgroup, or cut into parts
@pytest.mark.parametrize("rows", [1, 40])              # query rows of a kv head: 16x16 and 32x32 cores
@pytest.mark.parametrize("n", [0, 3, 64, 1500])
def test_scores_far_below_any_usual_one(L, n, rows, spare_cols):  # noqa: F811
    """All scores of a row near -2^110 (-1.3e33), exact powers of two that differ by far more than any softmax
    resolves: the row is the value of its largest score, equal ones share it, and lse is that score."""
    H, g = 2, 1
    cache, table = ready(L, 900 + n, 1, H, [n], spare_cols=spare_cols)
    # keys: channel 3 alone is not zero, code 2^-6 .. 2^0 with scale 2^0 in blocks, the same in the ring
    rng = np.random.default_rng(n)
    size = torch.from_numpy(2.0 ** -rng.integers(0, 4, (H, n + g))).float()
    value = torch.from_numpy(rng.integers(-8, 9, (H, n + g, D)) / 4.0).float()
    k8, v8 = torch.zeros(cache.k_pool.shape), torch.zeros(cache.v_pool.shape)
    for j in range(n // T):
        for h in range(H):
            k8[table[0, j], h, :, 3] = size[h, j * T:j * T + T]
            v8[table[0, j], h] = value[h, j * T:j * T + T].T
    cache.k_pool.copy_(k8.to(torch.float8_e4m3fn))
    cache.v_pool.copy_(v8.to(torch.float8_e4m3fn))
    cache.k_scale.fill_(1.0)
    cache.v_scale.fill_(1.0)
    cache.k_tail.zero_()
    for p in range(n // T * T, n + g):
        cache.k_tail[0, :, p % RING, 3] = size[:, p].to(DEV, torch.bfloat16)
        cache.v_tail[0, :, p % RING] = value[:, p].to(DEV, torch.bfloat16)
    q = torch.zeros((1, g, rows * H, D))
    q[..., 3] = -2.0 ** 113
    out, lse, _ = L.verify_attn_paged(q.to(DEV, torch.bfloat16), cache, i32(table), i32([n]), scale=1.0, return_lse=True)
    for h in range(H):
        least = float(size[h].min())
        equal = size[h] == least
        want = value[h][equal].double().mean(0)
        got = out[0, 0, h * rows:(h + 1) * rows].double().cpu()
        # the weights are 1 and 0; values are multiples of 1/4: the sum is exact, 1/l and the product 2^-23, out 2^-8
        assert bool(((got - want).abs() <= (2.0 ** -8 + 2.0 ** -22) * want.abs() + 1e-30).all())
        s = lse[0, h * rows:(h + 1) * rows].double().cpu()
        assert bool(((s + 2.0 ** 113 * least).abs() <= 2.0 ** 113 * least * 2.0 ** -21).all())


def test_strides_of_dimensions_of_one(L):  # noqa: F811
    """torch gives a dimension of one any stride, as a view with a swapped dimension has: no call goes by it."""
    cache, table = ready(L, 950, 1, 1, [100])
    q, t, n = normal(951, (1, 1, 1, D)), i32(table), i32([100])
    want = L.verify_attn_paged(q, cache, t, n)
    for strides in ((1, 1, 1, 1), (0, 0, 0, 1), (4, 2, 7, 1), (D, D, 1, 1)):
        odd = q.as_strided((1, 1, 1, D), strides)
        out = torch.zeros_like(want).as_strided((1, 1, 1, D), strides)
        assert torch.equal(L.verify_attn_paged(odd, cache, t, n, out=out), want) and torch.equal(out, want)
    rows = normal(952, (1, 1, D))
    maps = dict(slots=i32([-2 - 100]), row_seq=i32([0]), row_pos=i32([100]), cu_rows=i32([0, 1]))
    for strides in ((1, 1, 1), (0, 0, 1), (129, 131, 1)):
        cache.k_tail.zero_()
        L.paged_append(cache, rows.as_strided((1, 1, D), strides), rows, maps)
        assert torch.equal(cache.k_tail[0, 0, 100], rows[0, 0])
