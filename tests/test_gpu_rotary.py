"""Rotary positions on the GPU, against the plain forms of mx_ref.

Tolerances.  The kernel's angles, cosines, sines and sums are in 64 bits: 2^-40 (|x1| + |x2|) of factor holds what is
off by then (Taylor's remainder 2e-14, angles to 10^9 in 53 bits).  Left are the rounding to binary32 and the one to the
rows' type, half a step each: (2^-24 + eps / 2) of the value, and half of the smallest subnormal of fp16, 2^-25."""
import numpy as np
import pytest
import torch

import mx_ref as M
from test_gpu_paged import DEV, L, i32, normal  # noqa: F401

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def rows(seed, shape, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype).to(DEV)


def check(y, x, pos, rot, transpose=False):
    x64 = x.double().cpu().numpy()
    inv = rot.inv_freq.cpu().numpy()
    kw = dict(interleaved=rot.interleaved, axis=None if rot.axis is None else rot.axis.tolist(), factor=float(np.float32(rot.factor)),
              transpose=transpose)
    want = M.rotate(x64, pos, inv, **kw)
    dim = 2 * len(inv)
    size = rot.factor * np.max(np.abs(x64), axis=-1, keepdims=True) * 2
    d = np.abs(y.double().cpu().numpy() - want)
    tol = (2.0 ** -24 + torch.finfo(x.dtype).eps / 2) * np.abs(want) + 2.0 ** -40 * size + (2.0 ** -25 if x.dtype == torch.float16 else 0.0)
    assert y.dtype == x.dtype and np.all(d <= tol), float(np.max(d - tol))
    assert torch.equal(y[..., dim:], x[..., dim:])


CASES = [
    dict(n=1, Hq=1, Hkv=0, D=128, dim=128), dict(n=1, Hq=40, Hkv=8, D=128, dim=128, interleaved=True), dict(n=80, Hq=40, Hkv=8, D=128, dim=128),
    dict(n=3, Hq=7, Hkv=3, D=64, dim=64), dict(n=33, Hq=4, Hkv=4, D=80, dim=40, interleaved=True), dict(n=33, Hq=4, Hkv=4, D=80, dim=40),
    dict(n=5, Hq=2, Hkv=1, D=96, dim=24, axes=2), dict(n=300, Hq=3, Hkv=2, D=256, dim=64, axes=3), dict(n=17, Hq=2, Hkv=2, D=128, dim=2),
    dict(n=17, Hq=2, Hkv=2, D=128, dim=126), dict(n=9, Hq=3, Hkv=1, D=72, dim=46, interleaved=True), dict(n=2, Hq=1, Hkv=1, D=512, dim=512, axes=4),
    dict(n=70000, Hq=1, Hkv=1, D=64, dim=32), dict(n=1000, Hq=64, Hkv=8, D=128, dim=96, axes=3, interleaved=True), dict(n=4, Hq=5, Hkv=2, D=8, dim=8),
    dict(n=40, Hq=2, Hkv=2, D=48, dim=16), dict(n=40, Hq=2, Hkv=2, D=24, dim=8), dict(n=11, Hq=3, Hkv=0, D=16, dim=6), dict(n=6, Hq=1, Hkv=2, D=2, dim=2),
    dict(n=6, Hq=1, Hkv=2, D=37, dim=8), dict(n=6, Hq=1, Hkv=2, D=37, dim=36, interleaved=True), dict(n=20000, Hq=28, Hkv=4, D=128, dim=128)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("i", range(len(CASES)))
def test_rotary(L, i, dtype):  # noqa: F811
    c, t = CASES[i], TYPES[dtype]
    n, axes, dim, D = c["n"], c.get("axes", 1), c["dim"], c["D"]
    if n > 5000 and dtype == "fp16":
        n = 5000
    wide = -(-D // 8) * 8                                     # rows start every 16 bytes
    q = rows(i, (n, c["Hq"], wide), t)[..., :D]
    k = rows(100 + i, (n, c["Hkv"], wide), t)[..., :D] if c["Hkv"] else None
    rng = np.random.default_rng(i)
    pos = rng.integers(0, 40000, (axes, n))
    rot = L.Rotary(L.rotary_frequencies(dim, device=DEV)[0], factor=[1.0, 1.25][i % 2], interleaved=c.get("interleaved", False),
                   axis=torch.from_numpy(rng.integers(0, axes, dim // 2)).to(torch.uint8).to(DEV) if axes > 1 else None)
    p = i32(pos if axes > 1 else pos[0])
    new = lambda x: None if x is None else torch.full((*x.shape[:2], wide), 9.0, dtype=t, device=DEV)  # noqa: E731
    qw, kw = new(q), new(k)
    cut = lambda x: None if x is None else x[..., :D]         # noqa: E731
    got = L.rotary(q, p, rot, k=k, out=cut(qw), k_out=cut(kw), transpose=i % 3 == 2)
    for x, y, w in [(q, got if k is None else got[0], qw)] + ([(k, got[1], kw)] if k is not None else []):
        check(y, x, pos, rot, i % 3 == 2)
        assert bool((w[..., D:] == 9.0).all())                 # between the rows: as it was
    # in place, and with outputs allocated by the call where rows start every 16 bytes
    if wide == D:
        fresh = L.rotary(q, p, rot, k=k, transpose=i % 3 == 2)
        assert torch.equal(fresh if k is None else fresh[0], cut(qw)) and (k is None or torch.equal(fresh[1], cut(kw)))
    q2, k2 = q.clone(memory_format=torch.preserve_format), None if k is None else k.clone(memory_format=torch.preserve_format)
    if wide == D:
        L.rotary(q2, p, rot, k=k2, out=q2, k_out=k2, transpose=i % 3 == 2)
        assert torch.equal(q2, cut(qw)) and (k is None or torch.equal(k2, cut(kw)))


def test_strides_and_heads_side_by_side(L):  # noqa: F811
    """Queries and keys as slices of one projection's output, rotated in place; the values between are left."""
    n, Hq, Hkv, D = 50, 12, 4, 128
    qkv = normal(1, (n, Hq + 2 * Hkv, D))
    was = qkv.clone()
    pos = np.arange(n) * 7
    rot = L.Rotary(L.rotary_frequencies(64, device=DEV)[0])
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]
    L.rotary(q, i32(pos), rot, k=k, out=q, k_out=k)
    check(q, was[:, :Hq], pos, rot)
    check(k, was[:, Hq:Hq + Hkv], pos, rot)
    assert torch.equal(qkv[:, Hq + Hkv:], was[:, Hq + Hkv:])
    # heads outermost, positions of every second row of a wider map, one in place and one not
    x = normal(2, (Hq, n, D)).transpose(0, 1)
    wide = i32(np.arange(3 * 2 * n).reshape(3, 2 * n))[:, :n]
    rot = L.Rotary(rot.inv_freq, axis=torch.arange(32, device=DEV).to(torch.uint8) % 3, interleaved=True)
    out, same = L.rotary(x, wide, rot, k=k, k_out=k)
    check(out, x, wide.cpu().numpy(), rot)
    assert same.data_ptr() == k.data_ptr()
    # a head, a row: any stride
    one = normal(3, (1, 1, D))
    want = L.rotary(one, i32([5]), rot._replace(axis=None))
    for strides in ((1, 1, 1), (0, 0, 1), (131, 129, 1)):
        assert torch.equal(L.rotary(one.as_strided((1, 1, D), strides), i32([5]), rot._replace(axis=None)), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_far_and_negative_positions(L, dtype):  # noqa: F811
    """Positions to the ends of 32 bits: products with a frequency of one have 31 bits, others up to 55, of which 53 are
    kept: an angle of 2^31 is off by 2^-23 at most, one below 2^29 not at all."""
    pos = np.array([0, 1, -1, 65535, -65536, 10 ** 6, 2 ** 24 + 1, 2 ** 29 - 1, -2 ** 29, 3 * 10 ** 8])
    x = rows(7, (len(pos), 3, 128), TYPES[dtype])
    rot = L.Rotary(L.rotary_frequencies(128, device=DEV)[0])
    check(L.rotary(x, i32(pos), rot), x, pos, rot)
    one = L.Rotary(torch.ones(64, device=DEV))
    pos = np.array([2 ** 31 - 1, -2 ** 31] * 5)
    check(L.rotary(x, i32(pos), one), x, pos, one)


def test_quarters_and_values_that_are_not_finite(L):  # noqa: F811
    """Angles at and around the borders of the quarter turns; inf and NaN reach their pair and no other channel."""
    around = np.array([k * np.pi / 4 + d for k in range(-9, 10) for d in (-1e-7, 0, 1e-7)], np.float32)
    rot = L.Rotary(torch.from_numpy(np.resize(around, 64)).to(DEV))
    x = rows(8, (3, 2, 128), torch.float32)
    pos = np.array([1, 2, 1000])
    check(L.rotary(x, i32(pos), rot), x, pos, rot)
    rot = L.Rotary(L.rotary_frequencies(64, device=DEV)[0])
    want = L.rotary(x, i32(pos), rot)
    for ch, v in ((5, float("nan")), (40, float("inf")), (100, float("-inf"))):
        y = x.clone()
        y[1, 1, ch] = v
        got = L.rotary(y, i32(pos), rot)
        pair = [ch] if ch >= 64 else [ch % 32, ch % 32 + 32]
        rest = torch.ones(x.shape, dtype=torch.bool, device=DEV)
        rest[1, 1, pair] = False
        assert torch.equal(got[rest], want[rest]) and not bool(torch.isfinite(got[1, 1, pair]).any())


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(L, interleaved):  # noqa: F811
    """transpose is the gradient: of the plain form by torch's own differentiation, and against differences.  The call is
    linear, so a difference quotient is exact but for the rounding of both results, 2^-24 of each value."""
    n, H, D, dim = 19, 3, 64, 40
    inv = L.rotary_frequencies(dim, device=DEV)[0]
    rot = L.Rotary(inv, factor=1.5, interleaved=interleaved)
    pos = i32(np.arange(n) * 11)
    x, g, d = (rows(s, (n, H, D), torch.float32) for s in (1, 2, 3))
    got = L.rotary(g, pos, rot, transpose=True)
    z = x.double().requires_grad_()
    a = (pos.double()[:, None] * inv.double())[:, None]
    half = dim // 2
    u, v = (z[..., 0:dim:2], z[..., 1:dim:2]) if interleaved else (z[..., :half], z[..., half:dim])
    p, q = 1.5 * (u * a.cos() - v * a.sin()), 1.5 * (v * a.cos() + u * a.sin())
    gu, gv = (g[..., 0:dim:2], g[..., 1:dim:2]) if interleaved else (g[..., :half], g[..., half:dim])
    ((p * gu).sum() + (q * gv).sum() + (z[..., dim:] * g[..., dim:]).sum()).backward()
    assert bool(((got.double() - z.grad).abs() <= 2.0 ** -23 * z.grad.abs() + 2.0 ** -36).all())
    one, two = L.rotary(x, pos, rot).double(), L.rotary((x + d), pos, rot).double()
    moved = ((x + d).double() - x.double())                    # (the step that binary32 took)
    quotient, want = ((two - one) * g.double()).sum(), (got.double() * moved).sum()
    size = ((two.abs() + one.abs()) * g.double().abs()).sum() + (got.double().abs() * moved.abs()).sum()
    assert float((quotient - want).abs()) <= 2.0 ** -24 * float(size)


def test_streams_graphs_and_no_rows(L):  # noqa: F811
    q, k, pos = normal(1, (70, 8, 128)), normal(2, (70, 2, 128)), i32(range(70))
    rot = L.Rotary(L.rotary_frequencies(128, device=DEV)[0])
    want = L.rotary(q, pos, rot, k=k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for s in (side, side.cuda_stream):
        got = L.rotary(q, pos, rot, k=k, stream=s)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = L.rotary(q, pos, rot, k=k)
    for i in range(4):
        q.copy_(normal(10 + i, (70, 8, 128)))
        pos.add_(1)
        graph.replay()
        want = L.rotary(q, pos, rot, k=k)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), i
    assert L.rotary(q[:0], pos[:0], rot).shape == (0, 8, 128)


def test_rows_past_4_gib(L):  # noqa: F811
    """Rows of a buffer longer than 32-bit offsets reach."""
    n, D = (1 << 23) + 300, 256                                # 4 GiB and some in bf16
    x = torch.zeros((n, 1, D), dtype=torch.bfloat16, device=DEV)
    tail = normal(1, (300, 1, D))
    x[-300:] = tail
    pos = torch.arange(n, device=DEV, dtype=torch.int32)
    rot = L.Rotary(L.rotary_frequencies(D, device=DEV)[0])
    L.rotary(x, pos, rot, out=x)
    assert torch.equal(x[-300:], L.rotary(tail, pos[-300:].contiguous(), rot)) and not bool(x[:1000].any())
