"""`stream=` of the Python calls: what a call allocates belongs to the stream that it runs on."""
import pytest
import torch

from test_gpu_paged import DEV, L, i32, normal, ready  # noqa: F401

pytestmark = pytest.mark.gpu

KV = [3000, 700]


@pytest.fixture(scope="module")
def inputs(L):  # noqa: F811
    """Two batches, with a table wide enough for the path of two kernels, and a bf16 cache of the same sizes."""
    made = []
    for i in range(2):
        cache, table = ready(L, 800 + i, 2, 2, KV, spare_cols=70)
        made.append(dict(q=normal(810 + i, (2, 4, 8, 128)), cache=cache, table=i32(table), kv=i32(KV),
                         k=normal(820 + i, (2, 2, 3100, 128)), v=normal(830 + i, (2, 2, 3100, 128))))
    return made


def paged(L, x, **kw):  # noqa: F811
    return L.verify_attn_paged(x["q"], x["cache"], x["table"], x["kv"], **kw)


def contiguous(L, x, **kw):  # noqa: F811
    return L.verify_attn(x["q"], x["k"], x["v"], x["kv"], **kw)


CALLS = [paged, contiguous]


@pytest.mark.parametrize("call", CALLS)
def test_streams_do_not_share_a_workspace(L, inputs, call, monkeypatch):  # noqa: F811
    """Calls on two streams from one current stream: scratch is not given out again to the second."""
    spaces, allocate = [], L._workspace

    def noted(*args):
        ws = allocate(*args)
        spaces.append((ws.data_ptr(), ws.data_ptr() + ws.numel()))
        return ws

    monkeypatch.setattr(L, "_workspace", noted)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for s in streams:
        call(L, inputs[0], stream=s)
    torch.cuda.synchronize()
    (a0, a1), (b0, b1) = spaces
    assert a1 <= b0 or b1 <= a0


@pytest.mark.parametrize("call", CALLS)
def test_memory_of_the_callers_stream_is_left_alone(L, inputs, call):  # noqa: F811
    """Neither is memory that the current stream has just freed taken for the output, nor is an output that is
    dropped while its stream may still write it given to the current stream."""
    want = call(L, inputs[0])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    x = torch.empty_like(want)
    was = x.data_ptr()
    del x
    out = call(L, inputs[0], stream=s)
    assert out.data_ptr() != was
    at = out.data_ptr()
    del out
    assert torch.empty_like(want).data_ptr() != at
    torch.cuda.synchronize()


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("call", CALLS)
def test_calls_on_two_streams(L, inputs, call, handle):  # noqa: F811
    want = [call(L, x) for x in inputs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(6):
        for i, s in enumerate(streams):
            got[i].append(call(L, inputs[i], stream=s.cuda_stream if handle else s))
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])
    # the current stream, the default stream by its handle, and from within another stream
    for s in (torch.cuda.current_stream(), 0):
        assert torch.equal(call(L, inputs[0], stream=s), want[0])
    with torch.cuda.stream(streams[0]):
        out = call(L, inputs[0], stream=streams[1])
    torch.cuda.synchronize()
    assert torch.equal(out, want[0])


def test_every_call_that_allocates(L, inputs):  # noqa: F811
    """The other calls on a stream of their own, against the same on the current one."""
    s = torch.cuda.Stream()
    x = inputs[0]
    h_d, h_v, w = normal(1, (2, 5, 256)), normal(2, (2, 300, 256)), normal(3, (1000, 256))
    l_v, ids = i32([300, 77]), i32([[1, 2, 3, 4, 5], [6, 7, 8, 9, 10]])
    n, one = i32([40, 60]), i32([2, 3])

    def all_of_them(**kw):
        st = L.alloc_paged_state(2, 8, 4, DEV)
        cache = L.alloc_paged_cache(2, 2, 8, DEV)
        k = x["k"].clone()
        torch.cuda.synchronize()
        norms = L.hv_prepare(h_v, **kw)
        rel = L.visual_relevance(h_d, h_v, l_v, hv_inv_norm=norms, **kw)
        acc = L.loose_accept(h_d, w, ids, rel, 2, 4, **kw)
        plan = L.paged_plan(n, n, st["held"], st["queue"], st["state"], st["table"], max_rows=100, **kw)
        L.paged_append(cache, x["k"][0, :, :100].transpose(0, 1), x["v"][0, :, :100].transpose(0, 1), plan, **kw)
        new = L.paged_commit(cache, st["table"], n, one, 5, plan=plan, **kw)
        both = L.kv_commit(k, x["v"].clone(), n, one, 5, **kw)
        torch.cuda.synchronize()
        return [norms, rel, *acc.values(), *plan.values(), *[y.view(torch.uint8) for y in cache], new, both, k]

    for got, want in zip(all_of_them(stream=s), all_of_them()):
        assert torch.equal(got, want)


def test_captured_on_a_forked_stream(L, inputs):  # noqa: F811
    """A call that names a side stream within a capture, replayed."""
    x = inputs[1]
    want = paged(L, x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    paged(L, x, stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        out = paged(L, x, stream=side)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(4):
        out.zero_()
        graph.replay()
        assert torch.equal(out, want)
        paged(L, x)
        torch.cuda.synchronize()
