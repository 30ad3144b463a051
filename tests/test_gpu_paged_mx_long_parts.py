"""Attention over the cache in 4 bits where one workgroup has more than 512 tiles, so that each of its eight waves asks for
the numbers of more than 64 blocks, of which it holds 64 at a time: one workgroup per unit (more than 256 sequences are never
cut), and parts (as many units as compute units, none of them shorter than the others).  Tables name few blocks many times, in
any order.  Tolerances are those of test_gpu_paged_mx."""
import numpy as np
import pytest
import torch

import mx_ref as M
from test_gpu_paged import D, DEV, L, T, i32, normal  # noqa: F401
from test_gpu_paged_mx import ready_mx

pytestmark = pytest.mark.gpu


def check(L, q, cache, table, kv, seqs, heads):  # noqa: F811
    """Those sequences and kv heads against the plain form."""
    B, g, Hq, _ = q.shape
    out, lse, _ = L.verify_attn_paged_mx(q, cache, i32(table), i32(kv), return_lse=True)
    H = cache.k_pool.shape[1]
    G = Hq // H
    rows = [h * G + i for h in heads for i in range(G)]
    some = [x[:, heads].contiguous() for x in cache[:4]] + [x[seqs][:, heads].contiguous() for x in cache[4:]]
    ro, rl, _, size = M.attention(q[seqs][:, :, rows].double().cpu().numpy(), M.as_numpy(some), table[seqs], [kv[b] for b in seqs])
    o, z = out[seqs][:, :, rows].double().cpu().numpy(), lse[seqs][:, rows].double().cpu().numpy()
    assert np.all(np.abs(o - ro) <= 1.02 * 2.0 ** -8 * (size + np.abs(ro)) + 1e-30)
    assert np.all(np.abs(z - rl) <= 2e-5 * (1 + np.abs(rl)))


@pytest.mark.parametrize("g,G", [(1, 1), (8, 5)])
def test_more_than_256_sequences(L, g, G):  # noqa: F811
    B, blocks = 257, 37
    kv = [(i * 37) % 65 for i in range(B)]
    kv[100], kv[256] = 64 * 600 + 33, 64 * 513
    cache, _ = ready_mx(L, 1200 + g, B, 1, [0] * B, extra=blocks)
    table = np.random.default_rng(g).integers(0, blocks, (B, 601)).astype(np.int32)
    table[100, [3, 511, 512, 520, 599]] = [-1, blocks, -7, 1 << 30, -1]       # no blocks: no keys
    check(L, normal(1201, (B, g, G, D)), cache, table, kv, [0, 1, 99, 100, 101, 256], [0])


@pytest.mark.parametrize("g,G,H", [(1, 1, 128), (8, 5, 64)])
def test_parts(L, g, G, H):  # noqa: F811
    blocks, kv = 19, [64 * 620 + 5, 64 * 601]
    cache, _ = ready_mx(L, 1210 + g, 2, H, [0, 0], extra=blocks)
    table = np.random.default_rng(g).integers(0, blocks, (2, 622)).astype(np.int32)
    table[0, 515], table[1, 600] = -1, blocks
    check(L, normal(1211, (2, g, H * G, D)), cache, table, kv, [0, 1], [0, H // 2 + 1, H - 1])
