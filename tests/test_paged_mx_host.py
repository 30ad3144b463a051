"""The C ABI of the paged cache in 4 bits on the host: refusals with the documented codes before anything touches a
device, and workspace sizes."""
import ctypes as C

import pytest
import torch

from test_paged_host import ATTN, BAD_CACHE, CACHE, L, fill, refused  # noqa: F401


def test_attention_refusals(L):  # noqa: F811
    one, blind, beyond = ((C.c_uint32 * 5)(1, 3, 7, 15, x) for x in (31, 15, 63))
    bad = BAD_CACHE + [({n: 0}, -1) for n in ("q", "out", "kv_len", "table")]
    bad += [(dict(gamma=0), -1), (dict(gamma=33), -1), (dict(Hq=6), -1), (dict(Hq=0), -1), (dict(Hq=65540), -2),
            (dict(table_cols=-1), -1), (dict(table_cols=(1 << 24) + 1), -2), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1),
            (dict(q=0x1008), -1), (dict(out=0x1008), -1), (dict(q_sh=120), -1), (dict(o_sg=1028), -1), (dict(vis_begin=0x1000), -1),
            (dict(vis_mass=0x1000), -1), (dict(draft_mask=blind), -1), (dict(draft_mask=beyond), -1), (dict(workspace=0), L.EWORKSPACE),
            (dict(workspace=0x10010), L.EWORKSPACE), (dict(workspace_bytes=100), L.EWORKSPACE),
            ({"cache.B": 4096, "table_cols": 1 << 20}, -2), ({"cache.B": 4096, "cache.Hkv": 1024, "Hq": 1024}, -2)]
    refused(L, "lvspec_verify_attn_paged_mx", L.PagedMxAttnArgs, dict(ATTN, draft_mask=one), bad)


def test_attention_workspace(L):  # noqa: F811
    need = lambda **kw: L.raw().lvspec_verify_attn_paged_mx_workspace(C.byref(fill(L.PagedMxAttnArgs(), {**ATTN, **kw})))  # noqa: E731
    assert need() > 0 and need(gamma=0) == 0 and need(**{"cache.D": 64}) == 0 and need(**{"cache.B": 64}) > need()
    for gamma, Hq in ((1, 4), (5, 20), (32, 64)):
        assert need(gamma=gamma, Hq=Hq) >= 2 * 4 * (gamma * Hq // 4) * 131 * 4
    a = fill(L.PagedMxAttnArgs(), {**ATTN, "workspace_bytes": need() - 1})
    assert L.raw().lvspec_verify_attn_paged_mx(C.byref(a), None) == L.EWORKSPACE


def test_commit_refusals(L):  # noqa: F811
    good = dict(CACHE, n_layers=2, n_branches=2, chain_len=10, table=0x1000, table_cols=3, kv_len=0x1000, accept_len=0x1000,
                best_branch=0x1000, new_len=0x2000)
    bad = BAD_CACHE + [({n: 0}, -1) for n in ("table", "kv_len", "accept_len", "new_len")]
    bad += [(dict(n_layers=0), -1), (dict(n_layers=65536), -1), (dict(n_branches=-1), -1), (dict(n_branches=9), -1),
            (dict(chain_len=0), -1), (dict(chain_len=17), -1), (dict(n_branches=4), -1), (dict(table_cols=0), -1),
            (dict(table_cols=(1 << 24) + 1), -2), (dict(new_len=0x1000), -1), (dict(granted=0x1000), -1),
            (dict(held=0x1000, cu_rows=0x1000), -1)]
    refused(L, "lvspec_paged_mx_commit", L.PagedMxCommitArgs, good, bad)


def test_read_refusals(L):  # noqa: F811
    good = dict(CACHE, n_rows=10, slots=0x1000, k=0x1000, v=0x2000, k_sr=1024, k_sh=128, v_sr=1024, v_sh=128)
    bad = BAD_CACHE + [({n: 0}, -1) for n in ("slots", "k", "v")]
    bad += [(dict(n_rows=-1), -1), (dict(n_rows=(1 << 28) + 1), -2), (dict(k=0x1008), -1), (dict(k_sr=100), -1), (dict(v_sr=132), -1),
            (dict(k_sh=-128), -1), (dict(v_sh=64), -1)]
    refused(L, "lvspec_paged_mx_read", L.PagedMxReadArgs, good, bad)
    none = fill(L.PagedMxReadArgs(), {**good, "n_rows": 0, "k": 0, "slots": 0})
    assert L.raw().lvspec_paged_mx_read(C.byref(none), None) == L.OK


def test_python_calls_refuse_what_the_kernels_cannot_take(L):  # noqa: F811
    cache = L.alloc_paged_mx_cache(2, 2, 4, "cpu")
    table, n = torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    k = torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    for call in (lambda: L.verify_attn_paged_mx(torch.zeros((2, 1, 4, 128), dtype=torch.bfloat16), cache, table, n),
                 lambda: L.paged_mx_append(cache, k, k, L.alloc_paged_plan(2, 3, "cpu")),
                 lambda: L.paged_mx_commit(cache, table, n, n, 5), lambda: L.paged_mx_read(cache, n)):
        with pytest.raises(AssertionError):
            call()
    assert L.alloc_paged_mx_cache(2, 2, 4, "cpu", layers=3).layer(1).k_pool.shape == (4, 2, 2, 64, 32)
