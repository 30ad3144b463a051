"""Rotary positions on the host: frequencies against their formulas, refusals before anything touches a device, and the
plain forms of mx_ref against others."""
import ctypes as C

import numpy as np
import pytest
import torch

import mx_ref as M
from test_paged_host import CACHE, BAD_CACHE, L, fill, refused  # noqa: F401


@pytest.mark.parametrize("kw", [
    dict(dim=2, base=10000.0), dict(dim=64, base=1e6), dict(dim=128, base=10000.0, scaling=1, scale=4.0),
    dict(dim=128, base=10000.0, scaling=2, scale=8.0), dict(dim=4, base=500.0, scaling=2, scale=2.0),
    dict(dim=128, base=1e6, scaling=3, scale=4.0, original_len=32768), dict(dim=64, base=10000.0, scaling=3, scale=16.0, original_len=4096),
    dict(dim=96, base=10000.0, scaling=3, scale=0.5, original_len=2048), dict(dim=128, base=10000.0, scaling=3, scale=40.0, original_len=4096,
                                                                              beta_fast=16.0, beta_slow=2.0),
    dict(dim=8, base=10000.0, scaling=3, scale=2.0, original_len=3.0),
    dict(dim=128, base=10000.0, scaling=3, scale=2.0, original_len=4096, beta_fast=7.0, beta_slow=7.0)])
def test_frequencies(L, kw):  # noqa: F811
    got, factor = L.rotary_frequencies(**kw)
    want, f = M.frequencies(**kw)
    # two evaluations in 64 bits (a power: 2^-50 of it), rounded to 32 once
    assert got.shape == (kw["dim"] // 2,) and got.dtype == torch.float32
    assert np.all(np.abs(got.double().numpy() - want) <= want * (2.0 ** -24 + 2.0 ** -45))
    assert abs(factor - f) <= f * (2.0 ** -24 + 2.0 ** -45)


def test_frequencies_refused(L):  # noqa: F811
    good = dict(dim=64, scaling=3, base=10000.0, scale=4.0, original_len=4096.0, beta_fast=0.0, beta_slow=0.0)
    out, f = (C.c_float * 256)(), C.c_float()
    call = lambda a, o=out, g=f: L.raw().lvspec_rotary_frequencies(a, o, C.byref(g) if g is not None else None)  # noqa: E731
    assert call(C.byref(fill(L.RotaryFreqArgs(), good))) == L.OK
    inf, nan = float("inf"), float("nan")
    for bad in (dict(dim=0), dict(dim=3), dict(dim=514), dict(dim=-2), dict(scaling=4), dict(scaling=-1), dict(base=1.0), dict(base=inf),
                dict(base=nan), dict(scale=0.0), dict(scale=-1.0), dict(scale=nan), dict(scale=inf), dict(original_len=0.0),
                dict(original_len=nan), dict(beta_fast=0.5), dict(beta_slow=-1.0), dict(beta_slow=40.0), dict(scaling=2, dim=2)):
        assert call(C.byref(fill(L.RotaryFreqArgs(), {**good, **bad}))) == L.EINVAL, bad
    assert call(None) == call(C.byref(fill(L.RotaryFreqArgs(), good)), None) == L.EINVAL
    assert call(C.byref(fill(L.RotaryFreqArgs(), good)), out, None) == L.EINVAL


ROT = {"rot.dim": 64, "rot.n_axes": 1, "rot.inv_freq": 0x1000, "rot.pos": 0x1000}
BAD_ROT = [({"rot.dim": 0}, -1), ({"rot.dim": 63}, -1), ({"rot.dim": 130}, -1), ({"rot.interleaved": 2}, -1), ({"rot.transpose": -1}, -1),
           ({"rot.n_axes": 0}, -1), ({"rot.n_axes": 5}, -1), ({"rot.inv_freq": 0}, -1), ({"rot.inv_freq": 0x1002}, -1),
           ({"rot.pos": 0x1001}, -1), ({"rot.pos_sa": -4}, -1), ({"rot.factor": -1.0}, -1), ({"rot.factor": float("nan")}, -1),
           ({"rot.factor": 1e7}, -1)]


def test_rotary_refusals(L):  # noqa: F811
    good = dict(ROT, n_rows=7, Hq=8, Hkv=2, D=128, dtype=0, q=0x1000, q_sr=1024, q_sh=128, q_out=0x2000, qo_sr=1024, qo_sh=128,
                k=0x1000, k_sr=256, k_sh=128, k_out=0x2000, ko_sr=256, ko_sh=128)
    bad = BAD_ROT + [({n: 0}, -1) for n in ("q", "q_out", "k", "k_out", "rot.pos")]
    bad += [(dict(n_rows=-1), -1), (dict(Hq=0), -1), (dict(Hkv=-1), -1), (dict(D=0), -1), (dict(D=60), -1), (dict(D=520), -2),
            (dict(dtype=3), -1), (dict(dtype=-1), -1), (dict(q=0x1008), -1), (dict(k_out=0x2004), -1), (dict(q_sh=120), -1),
            (dict(q_sr=1028), -1), (dict(qo_sr=64), -1), (dict(ko_sh=-128), -1), (dict(q_out=0x1000, qo_sr=2048), -1),
            (dict(k_out=0x1000, ko_sh=256), -1), (dict(Hq=65530, Hkv=6), -2), (dict(n_rows=(1 << 25) + 1), -2),
            (dict(dtype=2, q_sr=1026), -1)]
    refused(L, "lvspec_rotary", L.RotaryArgs, good, bad)
    none = fill(L.RotaryArgs(), {**good, "n_rows": 0, "q": 0, "rot.pos": 0})
    assert L.raw().lvspec_rotary(C.byref(none), None) == L.OK


QUERIES = dict(Hq=8, q=0x1000, q_sr=1024, q_sh=128, q_out=0x2000, qo_sr=1024, qo_sh=128)
ROWS = dict(n_rows=10, k=0x1000, v=0x2000, k_sr=1024, k_sh=128, v_sr=1024, v_sh=128, slots=0x1000, row_seq=0x1000, row_pos=0x1000,
            cu_rows=0x1000)
BAD_ROWS = [({n: 0}, -1) for n in ("k", "v", "slots", "row_seq", "row_pos", "cu_rows")] + [
    (dict(n_rows=-1), -1), (dict(n_rows=(1 << 28) + 1), -2), (dict(k=0x1008), -1), (dict(k_sr=100), -1), (dict(v_sr=120), -1),
    (dict(k_sh=-128), -1), (dict(v_sh=64), -1), (dict(v_sh=132), -1)]
BAD_QUERIES = [(dict(Hq=-1), -1), (dict(Hq=65536), -2), (dict(q=0), -1), (dict(q_out=0), -1), (dict(q=0x1008), -1), (dict(q_sr=1020), -1),
               (dict(qo_sh=64), -1), (dict(q_out=0x1000, qo_sr=2048), -1), ({"rot.transpose": 1}, -1), ({"rot.dim": 24}, -2),
               ({"rot.pos": 0, "rot.n_axes": 3}, -1)]


def under(prefix, cases):
    return [({f"{prefix}.{k}": v for k, v in change.items()}, want) for change, want in cases]


def test_append_refusals(L):  # noqa: F811
    good = {**{f"rows.{k}": v for k, v in {**CACHE, **ROWS}.items()}, **ROT, **QUERIES}
    bad = under("rows", BAD_CACHE + BAD_ROWS) + BAD_ROT + BAD_QUERIES
    bad += [({"rows.n_rows": 1 << 28, "rows.cache.Hkv": 4}, -2)]
    refused(L, "lvspec_paged_append_rotary", L.PagedAppendRotaryArgs, good, bad)
    none = fill(L.PagedAppendRotaryArgs(), {**good, "rows.n_rows": 0, "Hq": 0, "q": 0, "rot.pos": 0})
    assert L.raw().lvspec_paged_append_rotary(C.byref(none), None) == L.OK


def test_mx_append_refusals(L):  # noqa: F811
    good = {**CACHE, **ROWS, **ROT, **QUERIES}
    refused(L, "lvspec_paged_mx_append", L.PagedMxAppendArgs, good, BAD_CACHE + BAD_ROWS + [x for x in BAD_ROT if x[0] != {"rot.dim": 0}] +
            BAD_QUERIES + [({"rot.dim": 0}, -1), ({"rot.dim": -16}, -1)])       # queries without a rotation
    none = fill(L.PagedMxAppendArgs(), {**CACHE, **ROWS, "n_rows": 0, "k": 0, "v": 0})
    assert L.raw().lvspec_paged_mx_append(C.byref(none), None) == L.OK


def test_python_calls_refuse_what_the_kernels_cannot_take(L):  # noqa: F811
    q, pos = torch.zeros((3, 2, 128)), torch.zeros(3, dtype=torch.int32)
    inv, _ = L.rotary_frequencies(64)
    with pytest.raises(AssertionError):
        L.rotary(q, pos, L.Rotary(inv))                        # host tensors
    with pytest.raises(L.LvspecError):
        L.rotary_frequencies(63)


# ------------------------------------------------------------------------------ the plain forms themselves
@pytest.mark.parametrize("interleaved", [False, True])
def test_plain_rotation_is_a_complex_product(interleaved):
    rng = np.random.default_rng(1)
    x, pos = rng.standard_normal((5, 3, 20)), np.array([[0, 3, -7, 10 ** 6, 12], [5, 0, 1, 2, 99]])
    inv = M.frequencies(12, 10000.0)[0].astype(np.float32)
    axis = [0, 1, 0, 1, 1, 0]
    y = M.rotate(x, pos, inv, interleaved=interleaved, axis=axis, factor=1.5)
    i = np.arange(6)
    u, v = (2 * i, 2 * i + 1) if interleaved else (i, 6 + i)
    z = (x[..., u] + 1j * x[..., v]) * 1.5 * np.exp(1j * pos[axis].T * inv.astype(np.float64))[:, None]
    assert np.allclose(y[..., u], z.real, atol=1e-9) and np.allclose(y[..., v], z.imag, atol=1e-9)
    assert np.array_equal(y[..., 12:], x[..., 12:])
    back = M.rotate(y, pos, inv, interleaved=interleaved, axis=axis, transpose=True)
    assert np.allclose(back[..., :12], 1.5 * x[..., :12], atol=1e-9)


def test_plain_codes():
    """Every bf16 magnitude of a group against the definition, by search over all codes and scales."""
    rng = np.random.default_rng(2)
    x = (rng.standard_normal((200, 32)) * 2.0 ** rng.integers(-70, 120, (200, 1)))
    x = M.to_bf16(x)
    x[0], x[1, 3] = 0.0, -0.0
    codes, byte = M.group4(x)
    for r in range(200):
        top, s = np.abs(x[r]).max(), 2.0 ** -60
        while top > 7 * s:
            s *= 2
        assert byte[r] == int(np.log2(s)) + 127
        err = np.abs(M.value4(codes[r], np.full(32, byte[r])) - x[r])
        best = np.abs(np.concatenate([M.GRID, -M.GRID])[:, None] * s - x[r]).min(0)
        assert np.all(err == best) and np.all(err <= s)
    one = np.zeros((3, 32))
    one[0, 5], one[1, 6], one[2, :2] = np.nan, -np.inf, [float(torch.finfo(torch.bfloat16).max), 2.0 ** 127]
    codes, byte = M.group4(one)
    assert byte[:2].tolist() == [255, 255] and not codes[:2].any()
    assert byte[2] == 253 and codes[2, :2].tolist() == [5, 4]          # 3 s and 2 s, s = 2^126
