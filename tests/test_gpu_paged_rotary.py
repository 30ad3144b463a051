"""Appends that rotate, into the paged caches in 8 and in 4 bits, against the plain forms of paged_ref and mx_ref.
Rotated rows are rounded to bf16 from 64 bits on both sides (a sum within 2^-40 of a border between two bf16 numbers,
which could fall either way, is one in 2^31), so ring rows, codes and scales are equal; rotated queries have the
tolerance of rotary positions, half a step of bf16."""
import numpy as np
import pytest
import torch

import mx_ref as M
import paged_ref as R
import test_gpu_paged as P
from test_gpu_paged import APPENDS, D, DEV, L, RING, T, i32, normal, ready  # noqa: F401
from test_gpu_paged_mx import ready_mx
from test_gpu_rotary import check

pytestmark = pytest.mark.gpu

ROTS = [dict(dim=128), dict(dim=64, interleaved=True), dict(dim=96, axes=3), dict(dim=16, factor=1.25), dict(dim=32, axes=2, interleaved=True),
        dict(dim=128, axes=3)]


def rotation(L, i):  # noqa: F811
    c = ROTS[i % len(ROTS)]
    axes = c.get("axes", 1)
    axis = torch.from_numpy(np.arange(c["dim"] // 2) % axes).to(torch.uint8).to(DEV) if axes > 1 else None
    return L.Rotary(L.rotary_frequencies(c["dim"], device=DEV)[0], c.get("factor", 1.0), c.get("interleaved", False), axis), axes


def rotated(k, pos, rot):
    return M.to_bf16(M.rotate(k.double().cpu().numpy(), pos, rot.inv_freq.cpu().numpy(), interleaved=rot.interleaved,
                              axis=None if rot.axis is None else rot.axis.tolist(), factor=float(np.float32(rot.factor))))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("i", range(len(APPENDS)))
def test_append(L, i, bits):  # noqa: F811
    c = APPENDS[i]
    kv, new, Hkv = c["kv"], c["new"], c.get("Hkv", 2)
    B, n = len(kv), sum(new)
    need = [(a + b) // T for a, b in zip(kv, new)]
    lens = [T * x for x in need]
    cache, _ = (ready if bits == 8 else ready_mx)(L, i, B, Hkv, lens)
    st = L.alloc_paged_state(B, cache.k_pool.shape[0], max(need) + 1, DEV)
    pad = 3 if i % 2 else 0                         # rows behind the last sequence
    plan = L.paged_plan(i32(kv), i32(new), st["held"], st["queue"], st["state"], st["table"], max_rows=n + pad,
                        draft=c.get("draft", False))
    both = normal(100 + i, (n + pad, 2, Hkv, D), 3.0)
    both[:, :, :, 7] *= 40
    both[n:] = float("nan")
    k, v = both[:, 0], both[:, 1]
    q = normal(200 + i, (n + pad, 3, D)) if i % 3 else None
    rot, axes = rotation(L, i)
    places = plan["row_pos"].cpu().numpy().astype(np.int64)
    pos = None if axes == 1 and i % 2 == 0 else np.random.default_rng(i).integers(0, 30000, (axes, n + pad))
    turned = np.nan_to_num(rotated(k, places if pos is None else pos, rot))
    host = {x: y.cpu().numpy() for x, y in plan.items()}
    ref = (R if bits == 8 else M).as_numpy(cache)
    (R if bits == 8 else M).append(ref, turned, np.nan_to_num(v.double().cpu().numpy()), host, kv)
    p = None if pos is None else i32(pos if axes > 1 else pos[0])
    out = None if q is None else torch.full_like(q, 7.0)
    if bits == 8:
        got = L.paged_append_rotary(cache, k, v, plan, rot, pos=p, q=q, q_out=out)
        P.same_cache(cache, ref)
    else:
        got = L.paged_mx_append(cache, k, v, plan, rot=rot, pos=p, q=q, q_out=out)
        M.same_cache(cache, ref)
    assert got is out
    if q is not None:
        check(out[:n], q[:n], (places if pos is None else pos)[..., :n], rot)
        assert bool((out[n:] == 7.0).all())                     # no row: left as it was
        again = L.rotary(q[:n], i32(places[:n]) if p is None else p[..., :n], rot)
        assert torch.equal(again, out[:n])                     # the same numbers as by themselves
        del again


@pytest.mark.parametrize("bits", [8, 4])
def test_pieces_or_at_once(L, bits):  # noqa: F811
    """A prompt in one call and in pieces leaves the same cache."""
    Hkv, n, B = 2, 700, 2
    k, v, q = normal(1, (n, Hkv, D)), normal(2, (n, Hkv, D)), normal(3, (n, 4, D))
    rot, _ = rotation(L, 0)
    ends = []
    for cuts in ([n], [1, 62, 1, 64, 130, 3, 439]):
        cache = (L.alloc_paged_cache if bits == 8 else L.alloc_paged_mx_cache)(B, Hkv, 24, DEV)
        st = L.alloc_paged_state(B, 24, 12, DEV)
        at, held, state, outs = 0, st["held"], st["state"], []
        for c in cuts:
            plan = L.paged_plan(i32([at, 0]), i32([c, 0]), held, st["queue"], state, st["table"], max_rows=c)
            held, state = plan["new_held"], plan["new_state"]
            one = slice(at, at + c)
            outs.append((L.paged_append_rotary(cache, k[one], v[one], plan, rot, q=q[one]) if bits == 8 else
                         L.paged_mx_append(cache, k[one], v[one], plan, rot=rot, q=q[one])))
            at += c
        used = st["table"][0, :n // T].long()
        ring = torch.arange(n // T * T, n, device=DEV) % RING
        ends.append([x[used].view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x[used] for x in cache[:4]] +
                    [x[0][:, ring] for x in cache[4:]] + [torch.cat(outs)])
    assert all(torch.equal(x, y) for x, y in zip(*ends))


@pytest.mark.parametrize("bits", [8, 4])
def test_maps_that_name_nothing(L, bits):  # noqa: F811
    cache, _ = (ready if bits == 8 else ready_mx)(L, 6, 2, 2, [64, 64])
    ref = R if bits == 8 else M
    same = P.same_cache if bits == 8 else M.same_cache
    n_blocks = cache.k_pool.shape[0]
    before = ref.as_numpy(cache)
    k, v = normal(1, (64, 2, D)), normal(2, (64, 2, D))
    rot, _ = rotation(L, 0)
    call = L.paged_append_rotary if bits == 8 else lambda c, k, v, p, r: L.paged_mx_append(c, k, v, p, rot=r)
    for slots in ([n_blocks * T + i for i in range(T)], [-1] * T, [-2 - 2 * RING - i for i in range(T)], [-2 ** 31] * T):
        call(cache, k, v, dict(slots=i32(slots), row_seq=i32([0] * T), row_pos=i32(range(T)), cu_rows=i32([0, T, T])), rot)
        same(cache, before)
    for seq, cu in ((5, [0, T, T]), (-1, [0, T, T]), (0, [-3, T, T]), (0, [T, T, T])):
        call(cache, k, v, dict(slots=i32(range(T)), row_seq=i32([seq] * T), row_pos=i32(range(T)), cu_rows=i32(cu)), rot)
        same(cache, before)
    none = dict(slots=i32([]), row_seq=i32([]), row_pos=i32([]), cu_rows=i32([0, 0, 0]))
    call(cache, k[:0], v[:0], none, rot)
    same(cache, before)


@pytest.mark.parametrize("bits", [8, 4])
def test_queries_in_place_streams_and_graphs(L, bits):  # noqa: F811
    """Rows of one projection, queries turned where they are; on a stream, and captured and replayed."""
    B, g, Hq, H = 3, 5, 4, 2
    kv = i32([61, 200, 3])
    new = L.alloc_paged_cache if bits == 8 else L.alloc_paged_mx_cache
    cache, twin = new(B, H, 20, DEV), new(B, H, 20, DEV)
    rot, _ = rotation(L, 1)
    st = L.alloc_paged_state(B, 20, 8, DEV)
    plan = L.paged_plan(kv, i32([g] * B), st["held"], st["queue"], st["state"], st["table"], max_rows=B * g + 2, reserve=g, draft=True)
    qkv = normal(5, (B * g + 2, Hq + 2 * H, D))

    def call(cache, x, **kw):
        q, k, v = x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]
        if bits == 8:
            return L.paged_append_rotary(cache, k, v, plan, rot, q=q, q_out=q, **kw)
        return L.paged_mx_append(cache, k, v, plan, rot=rot, q=q, q_out=q, **kw)

    one, two = qkv.clone(), qkv.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(cache, one, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    call(twin, two)
    check(one[:B * g, :Hq], qkv[:B * g, :Hq], plan["row_pos"][:B * g].cpu().numpy(), rot)
    assert torch.equal(one[:, Hq:], qkv[:, Hq:]) and torch.equal(one[B * g:], qkv[B * g:])
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip((*cache, one), (*twin, two)))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(cache, one)
    for i in range(4):
        x = normal(20 + i, tuple(qkv.shape))
        one.copy_(x)
        two.copy_(x)
        graph.replay()
        call(twin, two)
        torch.cuda.synchronize()
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip((*cache, one), (*twin, two))), i


def test_without_a_rotation_nothing_changes(L):  # noqa: F811
    """Positions 0 everywhere: the rotating append is the plain one, in both caches."""
    kv, new = [40, 0], [100, 70]
    rot, _ = rotation(L, 0)
    k, v = normal(1, (170, 2, D)), normal(2, (170, 2, D))
    for bits in (8, 4):
        made = [(ready if bits == 8 else ready_mx)(L, 3, 2, 2, [128, 64])[0] for _ in range(2)]
        st = L.alloc_paged_state(2, made[0].k_pool.shape[0], 4, DEV)
        plan = L.paged_plan(i32(kv), i32(new), st["held"], st["queue"], st["state"], st["table"], max_rows=170)
        pos = torch.zeros(170, dtype=torch.int32, device=DEV)
        if bits == 8:
            L.paged_append(made[0], k, v, plan)
            L.paged_append_rotary(made[1], k, v, plan, rot, pos=pos)
        else:
            L.paged_mx_append(made[0], k, v, plan)
            L.paged_mx_append(made[1], k, v, plan, rot=rot, pos=pos)
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(*made))


def test_calls_that_are_refused(L):  # noqa: F811
    """No frequencies, queries of other heads than the cache's, rows short of positions: before any launch."""
    k, q = normal(1, (6, 2, D)), normal(2, (6, 4, D))
    st = L.alloc_paged_state(1, 4, 4, DEV)
    plan = L.paged_plan(i32([0]), i32([6]), st["held"], st["queue"], st["state"], st["table"], max_rows=6)
    rot, _ = rotation(L, 0)
    none = L.Rotary(torch.empty(0, device=DEV))
    for bits in (8, 4):
        cache = (L.alloc_paged_cache if bits == 8 else L.alloc_paged_mx_cache)(1, 2, 4, DEV)
        for r, pos, queries, out in ((none, None, None, None), (rot, None, q[..., :64], q[..., :64]),
                                     (rot, None, q[:5], torch.zeros_like(q[:5])), (rot, i32([0] * 5), None, None),
                                     (rot, i32([[0] * 6] * 2), None, None), (rot, None, q.float(), q.float())):
            with pytest.raises(AssertionError):
                if bits == 8:
                    L.paged_append_rotary(cache, k, k, plan, r, pos=pos, q=queries, q_out=out)
                else:
                    L.paged_mx_append(cache, k, k, plan, rot=r, pos=pos, q=queries, q_out=out)
        torch.cuda.synchronize()
        assert all(not bool(x.view(torch.uint8).any()) for x in cache)
