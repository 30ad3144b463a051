"""Serving on the paged cache where the pool runs dry: requests that are refused, finish and come back in
another's place.  The plain forms are those of paged_ref; codes, scales, ring rows and lengths are equal."""
import numpy as np
import pytest
import torch

import paged_ref as R
from test_gpu_paged import D, DEV, L, RING, T, check_attention, i32, normal, ready, same_cache, tree  # noqa: F401

pytestmark = pytest.mark.gpu


def planned(L, st, kv_len, n_new, max_rows, **kw):
    """One plan that moves the state on."""
    p = L.paged_plan(i32(kv_len), i32(n_new), st["held"], st["queue"], st["state"], st["table"], max_rows=max_rows, **kw)
    st["held"], st["state"] = p["new_held"], p["new_state"]
    return p


def commit_of_granted(ref, table, kv_len, accept_len, chain, plan, best=None, n_branches=1):
    """The plain commit with what the plan says: who was refused accepts nothing, nobody more than came."""
    tau = np.array(accept_len).copy()
    granted, cu = plan["granted"].cpu().numpy(), plan["cu_rows"].cpu().numpy()
    for b in range(len(kv_len)):
        for a in range(n_branches):
            came = max(int(cu[b + 1] - cu[b]) - a * chain, 0)
            tau[b * n_branches + a] = min(tau[b * n_branches + a], came) if granted[b] else 0
    return R.commit(ref, table, kv_len, tau, chain, best, n_branches)


@pytest.mark.parametrize("rows,tau", [(63, 2), (63, 5), (61, 2), (10, 5)])     # with and without a block to complete
def test_commit_of_a_refused_request_in_a_used_place(L, rows, tau):
    """Place 0 held blocks 0 and 1, which belong to request 1 when a new request in place 0 is refused."""
    layers, H, g = 3, 2, 5
    st = L.alloc_paged_state(2, 4, 6, DEV)
    cache = L.alloc_paged_cache(2, H, 4, DEV, layers=layers)

    def step(kv, new, seed, **kw):
        p = planned(L, st, kv, new, sum(new), **kw)
        for y in range(layers):
            L.paged_append(cache.layer(y), normal(seed + y, (sum(new), H, D)), normal(seed + 50 + y, (sum(new), H, D)), p)
        return p

    assert step([0, 0], [128, 0], 1)["granted"].tolist() == [1, 1]
    planned(L, st, [0, 0], [0, 0], 0)                                        # the first has finished
    assert step([0, 0], [0, 256], 200)["granted"].tolist() == [1, 1]
    assert step([0, 256], [rows, 0], 400)["granted"].tolist() == [1, 1]
    drafts = step([rows, 256], [g, g], 600, reserve=64, draft=True)
    assert drafts["granted"].tolist() == [0, 0]
    table = st["table"].cpu().numpy()
    assert set(table[1, :4]) == {0, 1, 2, 3} and table[0, 0] in table[1, :4]
    before = [R.as_numpy(cache.layer(y)) for y in range(layers)]
    got = L.paged_commit(cache, st["table"], i32([rows, 256]), i32([tau, 0]), g, plan=drafts)
    assert got.tolist() == [rows, 256]
    for y in range(layers):
        same_cache(cache.layer(y), before[y], f"layer {y}")


def test_commit_goes_by_the_plan(L):
    """Refused, granted, nothing brought, fewer rows than accepted, and a block that is not held."""
    kv, br, chain = [62, 62, 62, 62, 62, 62, 20], 2, 5
    B = len(kv)
    cache, table = ready(L, 700, B, 2, [T] * B)
    plan = dict(granted=i32([0, 1, 1, 1, 1, 0, 1]), new_held=i32([1, 1, 1, 1, 0, 0, 0]),
                cu_rows=i32(np.cumsum([0, 10, 10, 0, 8, 10, 10, 6])))
    tau, best = [4] * (B * br), [1, 1, 1, 1, 0, 0, 1]
    ref = R.as_numpy(cache)
    lent = table.copy()
    lent[4] = -1                                                             # (its entry is not its own)
    want = commit_of_granted(ref, lent, kv, tau, chain, plan, best, br)
    got = L.paged_commit(cache, i32(table), i32(kv), i32(tau), chain, n_branches=br, best_branch=i32(best), plan=plan)
    assert got.tolist() == want.tolist() == [62, 66, 62, 65, 62, 62, 21]
    same_cache(cache, ref)


@pytest.mark.parametrize("branches,chain", [(1, 5), (2, 4)])
def test_loop_on_a_pool_that_runs_dry(L, branches, chain):
    """Requests come, are refused, go on, finish and leave their place to others; every granted one's cache is
    that of a list of its rows, and attention over it too."""
    rng = np.random.default_rng(branches)
    B, H, Hq, n_blocks, cols, g = 6, 2, 4, 7, 6, branches * chain
    st = L.alloc_paged_state(B, n_blocks, cols, DEV)
    cache = L.alloc_paged_cache(B, H, n_blocks, DEV)
    mask = tree(branches, chain)
    rows = [[] for _ in range(B)]                                            # committed (k, v) rows
    kv, alive = np.zeros(B, np.int64), np.zeros(B, bool)
    refused_steps = finished = 0

    def holds_its_rows():
        table, arr = st["table"].cpu().numpy(), R.as_numpy(cache)
        for b in range(B):
            if not rows[b]:
                continue
            for which, pool, scale, tail in ((0, 0, 2, 4), (1, 1, 3, 5)):
                x = torch.stack([r[which] for r in rows[b]]).double().cpu().numpy()
                n = len(x)
                for h in range(H):
                    for j in range(n // T):
                        codes, sc = R.block8(x[j * T:j * T + T, h])
                        got = arr[pool][table[b, j], h]
                        assert np.array_equal(got.T if which else got, codes) and arr[scale][table[b, j], h] == sc, (b, j)
                    open_ = np.arange(n // T * T, n)
                    assert np.array_equal(arr[tail][b, h, open_ % RING], x[open_, h]), b

    for step in range(50):
        # new requests in places that are free
        new = np.zeros(B, np.int64)
        for b in range(B):
            if not alive[b] and rng.random() < 0.4:
                new[b] = rng.integers(1, 200)
        p = planned(L, st, kv, new, int(new.sum()))
        k, v = normal(1000 + step, (int(new.sum()), H, D)), normal(2000 + step, (int(new.sum()), H, D))
        L.paged_append(cache, k, v, p)
        ok, cu = p["granted"].cpu().numpy(), p["cu_rows"].cpu().numpy()
        for b in np.flatnonzero((new > 0) & (ok != 0)):
            rows[b] = [(k[t], v[t]) for t in range(cu[b], cu[b + 1])]
            kv[b], alive[b] = new[b], True
        # a verified step of all places, the empty ones among them: they bring no rows
        drafts = np.where(alive, g, 0)
        p = planned(L, st, kv, drafts, B * g, reserve=g, draft=True)
        k, v = normal(3000 + step, (B * g, H, D)), normal(4000 + step, (B * g, H, D))
        L.paged_append(cache, k, v, p)
        ok, cu = p["granted"].cpu().numpy(), p["cu_rows"].cpu().numpy()
        tau, best = rng.integers(1, chain + 1, B * branches), rng.integers(0, branches, B)
        if step % 8 == 0:
            check_attention(L, normal(5000 + step, (B, g, Hq, D)), cache, st["table"].cpu().numpy(), kv.tolist(), mask=mask)
        got = L.paged_commit(cache, st["table"], i32(kv), i32(tau), chain, n_branches=branches, best_branch=i32(best), plan=p)
        for b in range(B):
            if alive[b] and ok[b]:
                at = cu[b] + int(best[b]) * chain
                n = int(tau[b * branches + best[b]])
                rows[b] += [(k[at + i], v[at + i]) for i in range(n)]
                kv[b] += n
            refused_steps += int(alive[b] and not ok[b])
        assert got.tolist() == kv.tolist()
        holds_its_rows()
        for b in range(B):                                                   # some are done
            if alive[b] and (rng.random() < 0.08 or kv[b] + 2 * g >= cols * T):
                kv[b], alive[b], rows[b] = 0, False, []
                finished += 1
    assert refused_steps > 10 and finished > 5


def test_captured_steps_with_refusals(L):
    """Plan, append and commit of a step in a graph, replayed past the pool's last block: refused sequences
    stay where they are and go on once another one's blocks come back, as eager steps do."""
    B, H, g, n_blocks = 3, 2, 8, 4
    st = L.alloc_paged_state(B, n_blocks, 6, DEV)
    cache = L.alloc_paged_cache(B, H, n_blocks, DEV, layers=2)
    kv_len, new = i32([50, 120, 40]), i32([g] * B)
    prompt = L.paged_plan(i32([0] * B), kv_len, st["held"], st["queue"], st["state"], st["table"], max_rows=210)
    for y in range(2):
        L.paged_append(cache.layer(y), normal(1 + y, (210, H, D)), normal(5 + y, (210, H, D)), prompt)
    k, v = (torch.zeros((2, B * g, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    tau = i32([0] * B)
    one = (cache, st["queue"], st["table"], kv_len, prompt["new_held"].clone(), prompt["new_state"].clone())
    twin = (L.PagedCache(*[x.clone() for x in cache]), *[x.clone() for x in one[1:]])

    def step(cache, queue, table, kv_len, held, state):
        p = L.paged_plan(kv_len, new, held, queue, state, table, max_rows=B * g, reserve=g, draft=True)
        held.copy_(p["new_held"])
        state.copy_(p["new_state"])
        for y in range(2):
            L.paged_append(cache.layer(y), k[y], v[y], p)
        kv_len.copy_(L.paged_commit(cache, table, kv_len, tau, g, plan=p))
        return p["granted"]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*one)                                                           # (tau = 0: nothing moves on)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        granted = step(*one)
    step(*twin)
    seen = []
    for i in range(20):
        k.copy_(normal(100 + i, tuple(k.shape)))
        v.copy_(normal(200 + i, tuple(v.shape)))
        tau.copy_(i32([i % (g + 1), (3 * i) % (g + 1), g]))
        if i == 13:                                                          # the second has finished
            for x in (one, twin):
                x[3][1] = 0
            new[1] = 0
        graph.replay()
        want = step(*twin)
        torch.cuda.synchronize()
        assert torch.equal(granted, want), i
        seen.append(want.tolist())
        for x, y in zip((*one[0], *one[1:]), (*twin[0], *twin[1:])):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), i
    refused = [i for i, x in enumerate(seen) if 0 in x]
    assert refused and refused[-1] < 19 and min(seen[-1]) == 1
    assert kv_len.tolist()[1] == 0


@pytest.mark.parametrize("reserve", [0, 63, 64, 80, 640])
def test_finished_requests_hold_nothing_whatever_the_reserve(L, reserve):
    """kv_len = 0 and n_new < 0: no block, in a place that had some and in one that had none."""
    B, n_blocks, cols = 5, 40, 20
    st = L.alloc_paged_state(B, n_blocks, cols, DEV)
    planned(L, st, [0] * B, [300, 100, -1, 200, -1], 600)
    assert st["held"].tolist() == [4, 1, 0, 3, 0]
    table = st["table"].tolist()
    p = planned(L, st, [0, 100, 0, -5, 0], [-1, 5, -1, -2, 0], 5, reserve=reserve)
    assert p["granted"].tolist() == [1] * B and p["cu_rows"].tolist() == [0, 0, 5, 5, 5, 5]
    live, empty = (105 + reserve) // T, reserve // T
    assert st["held"].tolist() == [0, live, 0, 0, empty]
    assert st["state"].tolist()[1] == n_blocks - live - empty
    head, n = st["state"].tolist()
    free = [int(st["queue"][(head + i) % n_blocks]) for i in range(n)]
    assert free[-7:] == table[0][:4] + table[3][:3]
    own = [x for b in range(B) for x in st["table"][b, :st["held"][b]].tolist()]
    assert sorted(own + free) == list(range(n_blocks))


def test_places_without_a_request_take_nothing_from_live_ones(L):
    """First come, first served: twenty places without a request before one that needs the whole pool."""
    B, n_blocks = 21, 10
    st = L.alloc_paged_state(B, n_blocks, 12, DEV)
    p = planned(L, st, [0] * B, [-1] * 20 + [64 * 8], 64 * 8, reserve=128)
    assert p["granted"].tolist() == [1] * B and st["held"].tolist() == [0] * 20 + [10]
    p = planned(L, st, [0] * B, [300] + [-1] * 20, 300, reserve=128)          # the first is served once it is back
    assert p["granted"].tolist() == [0] + [1] * 20 and st["held"].tolist() == [0] * B
    assert planned(L, st, [0] * B, [300] + [-1] * 20, 300, reserve=128)["granted"].tolist() == [1] * B
