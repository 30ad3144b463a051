"""Refusals of the paged cache's calls that go by several arguments together, on the host."""
import ctypes as C

import pytest

CACHE = {"B": 2, "Hkv": 4, "D": 128, "n_blocks": 9,
         **{x: 0x1000 for x in ("k_pool", "v_pool", "k_scale", "v_scale", "k_tail", "v_tail")}}


@pytest.fixture(scope="module")
def L():
    from paper_2604_05650_amd import binding
    return binding


def commit_args(L, cache=None, **fields):
    a = L.PagedCommitArgs()
    for k, v in {**CACHE, **(cache or {})}.items():
        setattr(a.cache, k, v)
    for k, v in dict(dict(n_layers=2, n_branches=2, chain_len=10, table=0x1000, table_cols=3, kv_len=0x1000,
                          accept_len=0x1000, best_branch=0x1000, new_len=0x2000), **fields).items():
        setattr(a, k, v)
    return a


def test_commit_takes_a_plan_whole_or_not_at_all(L):
    names = ("granted", "held", "cu_rows")
    for some in range(1, 7):
        a = commit_args(L, **{n: 0x1000 for i, n in enumerate(names) if some >> i & 1})
        assert L.raw().lvspec_paged_commit(C.byref(a), None) == L.EINVAL, some
