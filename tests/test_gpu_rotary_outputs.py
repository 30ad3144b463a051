"""Outputs that rotary allocates, for heads of any size: each head from one 16-byte border to the next, as the C call wants
its rows.  Equal to what the same call writes into outputs that the caller has."""
import pytest
import torch

from test_gpu_paged import DEV, L, i32  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("n,Hq,Hkv,D,dim", [(7, 3, 2, 37, 36), (7, 3, 2, 37, 8), (5, 2, 0, 20, 20), (6, 1, 1, 2, 2), (6, 4, 1, 2, 2), (1, 1, 1, 37, 36),
                                            (9, 2, 2, 36, 16), (3, 2, 2, 6, 4), (40, 3, 2, 128, 128), (0, 3, 2, 37, 36), (1, 5, 2, 13, 10)])
def test_allocated_outputs(L, n, Hq, Hkv, D, dim, dtype):  # noqa: F811
    wide = -(-D // 8) * 8
    gen = torch.Generator().manual_seed(D)
    q, k = (torch.randn((n, h, wide), generator=gen).to(dtype).to(DEV)[..., :D] for h in (Hq, max(Hkv, 1)))
    k = k if Hkv else None
    rot = L.Rotary(L.rotary_frequencies(dim, device=DEV)[0], 1.25)
    pos = i32(range(n))
    qo, ko = (torch.full((n, h, wide), 9.0, dtype=dtype, device=DEV)[..., :D] for h in (Hq, max(Hkv, 1)))
    L.rotary(q, pos, rot, k=k, out=qo, k_out=ko if Hkv else None)
    got = L.rotary(q, pos, rot, k=k)
    for x, y, z in zip(got if Hkv else (got,), (qo, ko), (q, k)):
        assert x.shape == z.shape and x.dtype == dtype and torch.equal(x, y)
        if D * q.element_size() % 16 == 0:
            assert x.is_contiguous()
    # turned back from outputs that a call allocated, into others
    back = L.rotary(got[0] if Hkv else got, pos, rot, transpose=True)
    # Pairs no longer than r = 2^0.5 max |x|.  The first result is off by h = eps / 2 + 2^-24 of 1.25 r a channel, a pair by 2^0.5 of
    # that, which the second call makes 1.25 times as long and rounds by h of 1.25^2 r: h 1.25^2 (2 + 2^0.5) max |x| in all, and
    # half of fp16's smallest number twice.
    h, f = torch.finfo(dtype).eps / 2 + 2.0 ** -24, 1.25 ** 2
    most = q.double().abs().amax(-1, keepdim=True)
    want = torch.cat([f * q.double()[..., :dim], q.double()[..., dim:]], -1)
    assert bool(((back.double() - want).abs() <= h * f * (2 + 2 ** 0.5) * most + 2.0 ** -23).all())
