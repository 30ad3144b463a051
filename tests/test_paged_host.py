"""The paged cache's C ABI on the host: refusals with the documented codes before anything touches a
device, workspace sizes, and the plain forms' rounding against torch's."""
import ctypes as C

import numpy as np
import pytest
import torch

import paged_ref as R


@pytest.fixture(scope="module")
def L():
    from paper_2604_05650_amd import binding
    return binding


def fill(a, fields):
    for k, v in fields.items():
        at = a
        for part in k.split(".")[:-1]:
            at = getattr(at, part)
        setattr(at, k.split(".")[-1], v)
    return a


CACHE = {"cache.B": 2, "cache.Hkv": 4, "cache.D": 128, "cache.n_blocks": 9,
         **{f"cache.{x}": 0x1000 for x in ("k_pool", "v_pool", "k_scale", "v_scale", "k_tail", "v_tail")}}
BAD_CACHE = [({"cache.B": 0}, -1), ({"cache.B": 4097}, -2), ({"cache.Hkv": 0}, -1), ({"cache.D": 64}, -2),
             ({"cache.D": 0}, -1), ({"cache.n_blocks": 0}, -1), ({"cache.n_blocks": (1 << 24) + 1}, -2),
             ({"cache.k_pool": 0}, -1), ({"cache.v_pool": 0x1008}, -1), ({"cache.k_scale": 0}, -1),
             ({"cache.v_scale": 0x1002}, -1), ({"cache.k_tail": 0}, -1), ({"cache.v_tail": 0x1004}, -1)]


def refused(L, fn, args_type, good, bad):
    assert getattr(L.raw(), fn)(None, None) == L.EINVAL
    for change, want in bad:
        assert getattr(L.raw(), fn)(C.byref(fill(args_type(), {**good, **change})), None) == want, change


def test_plan_refusals(L):
    names = ("kv_len", "n_new", "held", "state", "queue", "table", "granted", "new_held", "new_state", "cu_rows",
             "slots", "row_seq", "row_pos")
    good = dict(B=3, table_cols=4, n_blocks=5, max_rows=6, reserve=0, draft=0,
                **{n: 0x1000 + 0x100 * i for i, n in enumerate(names)})
    bad = [({n: 0}, -1) for n in names]
    bad += [(dict(B=0), -1), (dict(B=4097), -2), (dict(table_cols=0), -1), (dict(table_cols=(1 << 24) + 1), -2),
            (dict(n_blocks=0), -1), (dict(n_blocks=(1 << 24) + 1), -2), (dict(max_rows=-1), -1),
            (dict(max_rows=(1 << 28) + 1), -2), (dict(reserve=-1), -1), (dict(reserve=(1 << 20) + 1), -2),
            (dict(draft=2), -1), (dict(draft=-1), -1), (dict(new_held=good["held"]), -1),
            (dict(new_state=good["state"]), -1)]
    refused(L, "lvspec_paged_plan", L.PagedPlanArgs, good, bad)


def test_append_refusals(L):
    good = dict(CACHE, n_rows=10, k=0x1000, v=0x2000, k_sr=1024, k_sh=128, v_sr=1024, v_sh=128, slots=0x1000,
                row_seq=0x1000, row_pos=0x1000, cu_rows=0x1000)
    bad = BAD_CACHE + [({n: 0}, -1) for n in ("k", "v", "slots", "row_seq", "row_pos", "cu_rows")]
    bad += [(dict(n_rows=-1), -1), (dict(n_rows=(1 << 28) + 1), -2), (dict(k=0x1008), -1), (dict(k_sr=100), -1),
            (dict(v_sr=120), -1), (dict(k_sh=-128), -1), (dict(v_sh=64), -1), (dict(v_sh=132), -1)]
    refused(L, "lvspec_paged_append", L.PagedAppendArgs, good, bad)
    nothing = fill(L.PagedAppendArgs(), {**good, "n_rows": 0, "k": 0, "v": 0, "slots": 0})
    assert L.raw().lvspec_paged_append(C.byref(nothing), None) == L.OK


ATTN = dict(CACHE, gamma=5, Hq=8, q=0x1000, q_sb=5120, q_sg=1024, q_sh=128, table=0x1000, table_cols=7, kv_len=0x1000,
            out=0x1000, o_sb=5120, o_sg=1024, o_sh=128, workspace=0x10000, workspace_bytes=1 << 40)


def test_attention_refusals(L):
    one = (C.c_uint32 * 5)(1, 3, 7, 15, 31)
    blind = (C.c_uint32 * 5)(1, 3, 7, 15, 15)
    beyond = (C.c_uint32 * 5)(1, 3, 7, 15, 63)
    good = dict(ATTN, draft_mask=one)
    bad = BAD_CACHE + [({n: 0}, -1) for n in ("q", "out", "kv_len", "table")]
    bad += [(dict(gamma=0), -1), (dict(gamma=33), -1), (dict(Hq=6), -1), (dict(Hq=0), -1), (dict(Hq=65540), -2),
            (dict(table_cols=-1), -1), (dict(table_cols=(1 << 24) + 1), -2), (dict(scale=-1.0), -1),
            (dict(scale=float("nan")), -1), (dict(q=0x1008), -1), (dict(out=0x1008), -1), (dict(q_sh=120), -1),
            (dict(o_sg=1028), -1), (dict(vis_begin=0x1000), -1), (dict(vis_mass=0x1000), -1),
            (dict(draft_mask=blind), -1), (dict(draft_mask=beyond), -1), (dict(workspace=0), L.EWORKSPACE),
            (dict(workspace=0x10010), L.EWORKSPACE), (dict(workspace_bytes=100), L.EWORKSPACE),
            ({"cache.B": 4096, "table_cols": 1 << 20}, -2),
            ({"cache.B": 4096, "cache.Hkv": 1024, "Hq": 1024}, -2)]
    refused(L, "lvspec_verify_attn_paged", L.PagedAttnArgs, good, bad)


def test_attention_workspace(L):
    def need(**kw):
        return L.raw().lvspec_verify_attn_paged_workspace(C.byref(fill(L.PagedAttnArgs(), {**ATTN, **kw})))

    assert need() > 0 and need(gamma=0) == 0 and need(**{"cache.D": 64}) == 0
    assert need(**{"cache.B": 64}) > need()
    # rows of a kv head, with sums and maximum: never less than a record per sequence and head
    for gamma, Hq in ((1, 4), (5, 20), (32, 64)):
        rows = gamma * Hq // 4
        assert need(gamma=gamma, Hq=Hq) >= 2 * 4 * rows * 131 * 4
    exact = need()
    a = fill(L.PagedAttnArgs(), {**ATTN, "workspace_bytes": exact - 1})
    assert L.raw().lvspec_verify_attn_paged(C.byref(a), None) == L.EWORKSPACE


def test_tensors_of_a_call_are_on_one_device(L):
    here, there = torch.empty(1), torch.empty(1, device="meta")
    L._one_device(here, None, here)
    with pytest.raises(AssertionError):
        L._one_device(here, there)


def test_commit_refusals(L):
    good = dict(CACHE, n_layers=2, n_branches=2, chain_len=10, table=0x1000, table_cols=3, kv_len=0x1000,
                accept_len=0x1000, best_branch=0x1000, new_len=0x2000)
    bad = BAD_CACHE + [({n: 0}, -1) for n in ("table", "kv_len", "accept_len", "new_len")]
    bad += [(dict(n_layers=0), -1), (dict(n_layers=65536), -1), (dict(n_branches=-1), -1), (dict(n_branches=9), -1),
            (dict(chain_len=0), -1), (dict(chain_len=17), -1), (dict(n_branches=4), -1), (dict(table_cols=0), -1),
            (dict(table_cols=(1 << 24) + 1), -2), (dict(new_len=0x1000), -1)]
    refused(L, "lvspec_paged_commit", L.PagedCommitArgs, good, bad)


def test_python_calls_refuse_what_the_kernels_cannot_take(L):
    """Host tensors, other types and shapes never reach a kernel."""
    cache = L.alloc_paged_cache(2, 2, 4, "cpu")
    table, n = torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    q = torch.zeros((2, 1, 4, 128), dtype=torch.bfloat16)
    k = torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    st = L.alloc_paged_state(2, 4, 3, "cpu")
    assert st["state"].tolist() == [0, 4] and st["queue"].tolist() == [0, 1, 2, 3] and int(st["table"].max()) == -1
    with pytest.raises(AssertionError):
        L.verify_attn_paged(q, cache, table, n)
    with pytest.raises(AssertionError):
        L.paged_append(cache, k, k, L.alloc_paged_plan(2, 3, "cpu"))
    with pytest.raises(AssertionError):
        L.paged_commit(cache, table, n, n, 5)
    with pytest.raises(AssertionError):
        L.paged_plan(n, n, st["held"], st["queue"], st["state"], st["table"], max_rows=3)


def test_plain_rounding_is_e4m3(L):
    """The plain forms' lookup against torch's conversion, at every value, midpoint and between."""
    mid = (R.VALUES[1:] + R.VALUES[:-1]) / 2
    x = np.concatenate([R.VALUES, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9)])
    x = np.concatenate([x, -x, np.random.default_rng(0).uniform(-448, 448, 5000)]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(R.nearest8(x.astype(np.float64)), want)
    assert np.array_equal(R.value_of(want), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("top,exponent", [(448.0, 0), (449.0, 1), (224.0, -1), (225.0, 0), (1.0, -8), (1.75, -8),
                                          (1.7578125, -7), (0.0, -60), (2.0 ** -52, -60), (2.0 ** -51, -59), (3e38, 120)])
def test_plain_scale(top, exponent):
    x = np.zeros((64, 128))
    x[5, 9], x[0, 0], x[1, 1] = -top, np.inf, np.nan
    codes, s = R.block8(x)
    assert s == 2.0 ** exponent and codes[0, 0] == codes[1, 1] == 127
    assert abs(R.value_of(codes[5, 9]) * s + top) <= top * 2.0 ** -4
