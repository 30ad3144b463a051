"""How rotated rows are rounded: from 64 bits to binary32, and that to the rows' type, in every channel and every call.

At position 0 a number is multiplied by the factor and nothing else, exactly in 64 bits (8 or 11 bits by 24).  The numbers here
are those at which the two roundings end on another neighbour than one rounding would: the product lies beside the middle of
two neighbours, and binary32 puts it on the middle.  So a channel in which the two were taken as one shows.  Outputs are
equal, without a tolerance."""
import numpy as np
import pytest
import torch

from test_gpu_paged import D, DEV, L, RING, T, i32  # noqa: F401

pytestmark = pytest.mark.gpu

TYPES = {"bf16": (torch.bfloat16, 7), "fp16": (torch.float16, 10)}


def nearest(y, bits):
    """float64 in [1, 4) to `bits` fraction bits, ties to even."""
    step = 2.0 ** -bits * np.where(y < 2, 1.0, 2.0)
    return np.round(y / step) * step


def pairs(bits):
    """(x, factor, twice rounded): four where rounding once gives more, four where it gives less."""
    rng = np.random.default_rng(bits)
    x = 1 + np.arange(2 ** bits) / 2.0 ** bits
    more, less = [], []
    while min(len(more), len(less)) < 4:
        f = (1 + rng.random(4096)).astype(np.float32).astype(np.float64)
        y = f[:, None] * x
        once, twice = nearest(y, bits), nearest(nearest(y, 23), bits)
        for r, c in np.argwhere(once != twice):
            (more if once[r, c] > twice[r, c] else less).append((x[c], f[r], twice[r, c]))
    return more[:4] + less[:4]


@pytest.mark.parametrize("dtype", TYPES)
def test_the_numbers_are_what_they_should_be(dtype):
    """torch's own conversions give the same two roundings; the example 1.0234375 * 1.0572519302368164 among bf16's kind."""
    t, bits = TYPES[dtype]
    for x, f, twice in pairs(bits):
        y = torch.tensor(x * f, dtype=torch.float64)
        assert float(y.float().to(t)) == twice != nearest(x * f, bits) and float(torch.tensor(x).to(t)) == x
    y = np.float64(1.0234375) * np.float64(np.float32(1.0572519302368164))
    assert nearest(y, 7) == 1.0859375 and nearest(nearest(y, 23), 7) == 1.078125


# four pairs of channels a thread and one; halves and neighbours; a part of a head; an odd head
SHAPES = [(128, 128, False), (128, 128, True), (128, 64, False), (80, 40, True), (128, 126, False), (72, 46, True), (37, 36, False)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("transpose", [False, True])
def test_rotary(L, shape, dtype, transpose):  # noqa: F811
    (head, dim, interleaved), (t, bits) = shape, TYPES[dtype]
    inv = L.rotary_frequencies(dim, device=DEV)[0]
    pos = i32([0] * 9)
    wide = -(-head // 8) * 8
    for x, f, want in pairs(bits):
        rot = L.Rotary(inv, f, interleaved)
        q, k, qo, ko = (torch.full((9, h, wide), x, dtype=t, device=DEV)[..., :head] for h in (6, 3, 6, 3))
        for out in ((qo, ko), (q, k)):                         # and in place
            L.rotary(q, pos, rot, k=k, out=out[0], k_out=out[1], transpose=transpose)
            for y in out:
                assert bool((y[..., :dim] == want).all()) and bool((y[..., dim:] == x).all()), (x, f)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dim,interleaved", [(128, False), (128, True), (96, False), (32, True)])
def test_appends(L, bits, dim, interleaved):  # noqa: F811
    """Rows to the ring, queries, rows through LDS into a block, and a block that the ring's rows become part of: the same
    numbers, so the block of one call is that of two."""
    H, n = 3, T + 40
    inv = L.rotary_frequencies(dim, device=DEV)[0]
    for x, f, want in pairs(7):
        rot = L.Rotary(inv, f, interleaved)
        caches = []
        for cuts in ([n], [30, n - 30]):
            cache = (L.alloc_paged_cache if bits == 8 else L.alloc_paged_mx_cache)(1, H, 4, DEV)
            st = L.alloc_paged_state(1, 4, 4, DEV)
            held, state, at = st["held"], st["state"], 0
            for c in cuts:
                plan = L.paged_plan(i32([at]), i32([c]), held, st["queue"], state, st["table"], max_rows=c)
                held, state = plan["new_held"], plan["new_state"]
                k, q = (torch.full((c, h, D), x, dtype=torch.bfloat16, device=DEV) for h in (H, 5))
                pos = i32([0] * c)
                if bits == 8:
                    got = L.paged_append_rotary(cache, k, k, plan, rot, pos=pos, q=q)
                else:
                    got = L.paged_mx_append(cache, k, k, plan, rot=rot, pos=pos, q=q)
                assert bool((got[..., :dim] == want).all()) and bool((got[..., dim:] == x).all()), (x, f)
                at += c
            ring = cache.k_tail[0, :, [p % RING for p in range(T, n)]]
            assert bool((ring[..., :dim] == want).all()) and bool((ring[..., dim:] == x).all()), (x, f)
            caches.append(cache)
        for one, two in zip(caches[0][:4], caches[1][:4]):
            assert torch.equal(one.view(torch.uint8), two.view(torch.uint8))
        # the block's codes are those of an append of the rows as they should be
        as_is = torch.full((T, H, D), x, dtype=torch.bfloat16, device=DEV)
        as_is[..., :dim] = want
        cache = (L.alloc_paged_cache if bits == 8 else L.alloc_paged_mx_cache)(1, H, 4, DEV)
        st = L.alloc_paged_state(1, 4, 4, DEV)
        plan = L.paged_plan(i32([0]), i32([T]), st["held"], st["queue"], st["state"], st["table"], max_rows=T)
        (L.paged_append if bits == 8 else L.paged_mx_append)(cache, as_is, as_is, plan)
        for got, ref in ((caches[0].k_pool, cache.k_pool), (caches[0].k_scale, cache.k_scale)):
            assert torch.equal(got.view(torch.uint8), ref.view(torch.uint8))
