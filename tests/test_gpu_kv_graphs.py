"""GPU: graphs and streams of the paged 8-bit cache, where other calls come between."""
import pytest
import torch

import _kv_ref as ref
from paper_2608_07971_amd import kv

pytestmark = pytest.mark.gpu


def _say(msg):
    print(f"[gpu-case] {msg}", flush=True)


def _randn(seed, *shape, dtype=torch.float16):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _junk(*sizes):
    """Tensors that would take the place of memory given back."""
    return [torch.full((n,), 0x7f7f7f7f, dtype=torch.int32, device="cuda") for n in sizes for _ in range(8)]


def test_a_captured_step_goes_on_after_a_compaction():
    lengths, rope, offs = [100, 30, 77, 5], kv.Rope(64), ref.offsets([1] * 4)
    caches = [ref.make(kv, lengths, heads=2, dim=64, pages=60, width=12, seed=2) for _ in range(2)]
    now = _dev(lengths)
    k, v, q = (torch.zeros(4, n, 64, dtype=torch.float16, device="cuda") for n in (2, 2, 8))

    def step(cache):
        cache.resize(now)
        turned = cache.append(0, k, v, offs, rope=rope, q=q)
        return cache.attend(0, turned, offs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(caches[0])
    for i in range(8):
        _say(f"replay {i}")
        now += 1
        for j, t in enumerate((k, v, q)):
            t.copy_(_randn(10 * i + j, *t.shape))
        graph.replay()
        torch.cuda.synchronize()
        want = step(caches[1])
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        if i % 3 == 1:
            table, refs, live = caches[0].compact()
            caches[0].install(table, refs)
            del table, refs
            junk = _junk(4 * 12, 60)
            assert int(caches[0].table.max()) == int(live) - 1
    assert all(bool((x == 0x7f7f7f7f).all()) for x in junk)
    assert caches[0].device_status() == 0 and torch.equal(caches[0].lengths, caches[1].lengths)
    assert torch.equal(caches[0].refs.sort().values, caches[1].refs.sort().values)


def test_a_reader_on_another_stream_goes_on_during_an_installation():
    cache = ref.make(kv, [900, 30, 477, 5], heads=2, dim=64, pages=200, seed=3)
    q, offs, side = _randn(1, 4, 8, 64), ref.offsets([1] * 4), torch.cuda.Stream()
    want = cache.attend(0, q, offs)
    a = torch.randn(4096, 4096, device="cuda", dtype=torch.bfloat16)
    torch.cuda.synchronize()
    _say("reader queued behind other work")
    with torch.cuda.stream(side):
        for _ in range(20):
            a = a @ a
    got = cache.attend(0, q, offs, stream=side)
    table, refs, _ = cache.compact()
    cache.install(table, refs)
    del table, refs
    junk = _junk(cache.table.numel(), 200)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert all(torch.equal(x, y) for x, y in zip(cache.attend(0, q, offs), want))
    assert all(bool((x == 0x7f7f7f7f).all()) for x in junk) and cache.device_status() == 0


@pytest.mark.parametrize("new", [[1, 1], [700, 900]])
def test_graphs_of_one_stream_replay_beside_each_other_and_eager_calls(new):
    """Captured on a stream that has scratch, replayed on two others while that one runs calls of its own; units of
    several parts throughout."""
    cache = ref.make(kv, [9000, 7000], heads=4, dim=64, seed=5)
    offs, streams = ref.offsets(new), [torch.cuda.Stream() for _ in range(3)]
    qs = [torch.zeros(sum(new), 16, 64, dtype=torch.float16, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    cache.attend(0, qs[2], offs, stream=streams[2])               # the capturing stream has scratch of its own
    graphs, out = [], []
    for q in qs[:2]:
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=streams[2]):
            out.append([cache.attend(0, q, offs) for _ in range(3)])
    for i in range(6):
        _say(f"new {new}, replays {i}")
        for j, q in enumerate(qs):
            q.copy_(_randn(10 * i + j, *q.shape))
        want = [cache.attend(0, q, offs) for q in qs]
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        eager = [cache.attend(0, qs[2], offs, stream=streams[2]) for _ in range(3)]
        torch.cuda.synchronize()
        for w, got in zip(want, out + [eager]):
            assert all(torch.equal(a, b) for g in got for a, b in zip(g, w))
    assert cache.device_status() == 0


def test_an_error_taken_leaves_good_scratch():
    """A call whose lengths changed under it may leave tickets behind: they are put there by hand."""
    cache = ref.make(kv, [9000, 7000], heads=4, dim=64, seed=6)
    q, offs = _randn(1, 2, 16, 64), ref.offsets([1, 1])
    want = cache.attend(0, q, offs)
    for (kind, _), w in cache._work.items():
        if kind == "attend":
            w[:4 * 768].view(torch.int32).fill_(1)
    cache.status.fill_(2)                                         # what the call records
    assert cache.device_status() == 2 and cache.device_status() == 0
    got = cache.attend(0, q, offs)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and cache.device_status() == 0
