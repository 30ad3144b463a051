"""Queries of attention over the cache in 4 bits whose channels are of very different sizes: one large channel beside 31 others
in each group of 32, which meet keys that have nothing in the large ones, so that the scores are sums over the small ones.

Tolerances.  A query goes into the product as the sum of three numbers of 6 bits (test_query_split_host.py): numbers of 1/64
of their 32's largest and above as they are, smaller ones with 2^-14.9 of that largest at most.  With those sums in the
query's place the reference leaves binary32: 2^-18 of the sum of |q k| (six additions of 64 products each a row of them,
2^-24 apiece, with room) and 2e-5 (1 + |z|) of the softmax.  With the query as it is, a score may be off by B, the bound times
the sum of |k| over the channels that may lose: the log-sum-exp by B, a weight by a factor of e^(2 B)."""
import numpy as np
import pytest
import torch

import mx_ref as M
from test_gpu_paged import D, DEV, L, i32, normal  # noqa: F401
from test_gpu_paged_mx import ready_mx
from test_query_split_host import EXACT, LOST, split

pytestmark = pytest.mark.gpu

LARGE = [5, 40, 70, 101]                                       # a channel of each group of 32


@pytest.mark.parametrize("spare_cols", [1, 70])
@pytest.mark.parametrize("ratio", [1, 6, 7, 10, 14, 20])
def test_one_large_channel(L, ratio, spare_cols):  # noqa: F811
    kv, g, Hq, H = [128, 64 * 23], 4, 12, 2
    cache, table = ready_mx(L, 990 + ratio, 2, H, kv, spare_cols=spare_cols)
    pool = cache.k_pool.cpu()
    for ch in LARGE:
        pool[:, :, ch // 64, :, ch % 64 // 2] &= 0x0f if ch % 2 else 0xf0
    cache.k_pool.copy_(pool)
    cache.k_tail.zero_()                                       # (open rows meet queries as they are)
    q = normal(991 + ratio, (2, g, Hq, D))
    q = torch.where(q.abs() < 1, torch.copysign(torch.ones_like(q), q), q.clamp(-1.9921875, 1.9921875))      # 1 to 2
    mantissa = torch.tensor([1.0, 1.8828125, 1.875, 1.9921875, 1.3984375, 1.125], device=DEV).to(torch.bfloat16)
    for i, ch in enumerate(LARGE):
        q[..., ch] = mantissa[(torch.arange(Hq, device=DEV) + i) % 6] * 2.0 ** ratio
    out, lse, _ = L.verify_attn_paged_mx(q, cache, i32(table), i32(kv), return_lse=True)
    o, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    arr, scale = M.as_numpy(cache), D ** -0.5
    q64 = q.double().cpu().numpy()
    groups = q64.reshape(2, g, Hq, 4, 32)
    sums = split(groups)
    largest = np.max(np.abs(groups), -1, keepdims=True)
    may = np.abs(groups) < EXACT * largest
    assert np.all((sums == groups) | may) and np.all(np.abs(sums - groups) <= LOST * largest)
    assert may.any() == (ratio > 5) and (sums != groups).any() == (ratio > 6)
    size_k = np.abs(M.values_of(arr)[0]).max(axis=(0, 2))      # [H, D]: of any key
    size_k = np.repeat(size_k, Hq // H, 0)                     # by query head
    binary32 = 2.0 ** -18 * scale * np.sum(np.abs(q64) * size_k, -1)
    lost = scale * np.sum((may * LOST * largest).reshape(q64.shape) * size_k, -1)
    for query, by in ((sums.reshape(q64.shape), binary32), (q64, binary32 + lost)):
        ro, rl, _, size = M.attention(query, arr, table, kv)
        assert np.all(np.abs(lse - rl) <= np.transpose(by, (0, 2, 1)) + 2e-5 * (1 + np.abs(rl))), ratio
        tol = (1.02 * 2.0 ** -8 + np.expm1(np.minimum(2 * by, 100))[..., None]) * (size + np.abs(ro))
        assert np.all(np.abs(o - ro) <= tol), ratio
