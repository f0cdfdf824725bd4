"""GPU: beams that go on as each other, all at once, against the form on host integers."""
import numpy as np
import pytest
import torch

import _kv_forms as forms
import _kv_ref as ref
import paper_2608_07971_amd as esp
from paper_2608_07971_amd import kv

pytestmark = pytest.mark.gpu


def _say(msg):
    print(f"[gpu-case] {msg}", flush=True)


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _state(cache):
    return [t.view(torch.uint8).clone() for t in (cache.k, cache.v)] + [cache.scale.view(torch.int32).clone()]


def _same(cache, pages, first):
    """Table, lengths, references and every owned page's contents."""
    assert np.array_equal(cache.table.cpu().numpy(), pages.table) and np.array_equal(cache.refs.cpu().numpy(), pages.refs)
    assert np.array_equal(cache.lengths.cpu().numpy(), pages.lengths)
    live = np.nonzero(pages.refs > 0)[0]
    assert np.array_equal(pages.refs, np.bincount(pages.table[pages.table >= 0], minlength=len(pages.refs)))
    for t, f in zip(_state(cache), first):
        assert torch.equal(t[torch.from_numpy(live).cuda()], f[torch.from_numpy(pages.names[live]).cuda()])


@pytest.mark.parametrize("page,heads,dim,layers,sequences,width", [(16, 1, 64, 1, 1, 3), (16, 2, 64, 1, 7, 5), (32, 3, 128, 2, 40, 9), (64, 2, 64, 3, 300, 20)])
def test_reorder_in_a_row(page, heads, dim, layers, sequences, width):
    _say(f"reorder, pages of {page}, {sequences} sequences of at most {width} pages")
    g = np.random.default_rng(sequences)
    lengths = [int(g.integers(0, width * page + 1)) if g.random() < 0.8 else int(g.integers(0, width + 1)) * page for _ in range(sequences)]
    cache = ref.make(kv, lengths, page=page, heads=heads, dim=dim, layers=layers, width=width, spare=sequences // 2 + 2)
    pages, first = forms.Pages(cache), _state(cache)

    for step in range(10):
        near = [int(np.clip(i + g.integers(-2, 3), 0, sequences - 1)) for i in range(sequences)]
        parents = [near, list(range(sequences)), [int(x) for x in g.permutation(sequences)], [0] * sequences,
                   [int(x) for x in g.integers(-1, sequences, sequences)]][step % 5]
        if step == 9:
            parents = [-1] * sequences
        ok = pages.reorder(parents)
        cache.reorder(_dev(parents))
        assert cache.device_status() == (0 if ok else esp.ESP_ERR_RANGE), step
        _same(cache, pages, first)
        if step % 2 == 0:                                         # lengths change in between, partly filled pages with them
            want = [int(min(width * page, max(0, x + g.integers(-page, 2)))) for x in pages.lengths]
            if pages.resize(want):
                cache.resize(_dev(want))
                _same(cache, pages, first)
    assert not cache.refs.any() and not cache.lengths.any() and bool((cache.table == -1).all())


@pytest.mark.parametrize("layers,heads,dim,page,sequences", [(9, 2, 64, 64, 6), (32, 2, 64, 32, 40), (17, 8, 128, 16, 5)])
def test_pages_that_are_copied_by_a_launch_of_their_own(layers, heads, dim, page, sequences):
    _say(f"reorder, pages of {2 * layers * heads * dim * page >> 10} KB, {sequences} sequences")
    assert 2 * layers * heads * dim * page > 128 << 10
    g = np.random.default_rng(layers)
    lengths = [int(g.integers(0, 4 * page + 1)) for _ in range(sequences)]
    cache = ref.make(kv, lengths, page=page, heads=heads, dim=dim, layers=layers, width=4, spare=sequences)
    pages, first = forms.Pages(cache), _state(cache)
    for parents in ([0] * sequences, list(range(sequences)), [int(x) for x in g.integers(-1, sequences, sequences)], [sequences - 1] * sequences, [sequences] * sequences):
        ok = max(parents) < sequences and pages.reorder(parents)
        cache.reorder(_dev(parents))
        assert cache.device_status() == (0 if ok else esp.ESP_ERR_INVALID_ARG)
        _same(cache, pages, first)


def test_beams_write_apart_after_a_reordering():
    cache = ref.make(kv, [40, 40, 33, 5], heads=1, dim=64, pages=20, width=4)
    before = [cache.gather(0, _dev([0]), ref.offsets([n]), n, seqs=_dev([s]))[0] for s, n in enumerate((40, 40, 33, 5))]
    cache.reorder(_dev([1, 1, 0, -1]))                            # 0 was replaced by 1 and goes on as 2
    assert cache.lengths.tolist() == [40, 40, 40, 0] and len(set(cache.table[:3, 2].tolist())) == 3
    cache.resize(_dev([41, 41, 41, 0]))
    k = torch.randn(3, 1, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    cache.append(0, k, k, ref.offsets([1, 1, 1]), seqs=_dev([0, 1, 2]))
    for s, was in enumerate((1, 1, 0)):
        assert torch.equal(cache.gather(0, _dev([0]), ref.offsets([32]), 32, seqs=_dev([s]))[0], before[was][:32])
        new = cache.gather(0, _dev([40]), ref.offsets([1]), 1, seqs=_dev([s]))[0]
        assert ((new - k[s:s + 1]).abs().double() <= 2.0 ** -4 * k[s:s + 1].abs().double() + 2.0 ** -9).all()
    assert cache.device_status() == 0


def test_bad_reorderings_change_nothing():
    cache = ref.make(kv, [40, 10, 0], heads=1, dim=64, pages=4, width=4)
    state = [t.clone() for t in (cache.table, cache.lengths, cache.refs)]

    def unchanged(code):
        assert cache.device_status() == code
        assert all(torch.equal(a, b) for a, b in zip(state, (cache.table, cache.lengths, cache.refs)))
    for parents in ([0, 1, 3], [0, -2, 0], [2 ** 31 - 1, 0, 0]):
        cache.reorder(_dev(parents))
        unchanged(esp.ESP_ERR_INVALID_ARG)
    cache.reorder(_dev([0, 0, 0]))                                # two copies of a page, the other sequence's only one goes
    unchanged(esp.ESP_ERR_RANGE)
    cache.table[1, 0], state[0][1, 0] = 4, 4
    cache.reorder(_dev([0, 1, 2]))
    unchanged(esp.ESP_ERR_SHAPE)
    cache.table[1, 0], state[0][1, 0] = -1, -1                    # its partly filled page is missing
    cache.reorder(_dev([0, 1, 2]))
    unchanged(esp.ESP_ERR_SHAPE)
    for bad in (_dev([0, 1]), _dev([0, 1, 2]).long(), torch.tensor([0, 1, 2], dtype=torch.int32)):
        with pytest.raises(ValueError):
            cache.reorder(bad)


def test_a_decoding_step_of_beams_in_a_graph():
    """Selection, reordering and room for the next token, captured and replayed with eager work between."""
    G, B, V = 3, 4, 999
    caches = [ref.make(kv, [37, 0, 0, 0] * G, heads=2, dim=64, pages=120, width=8, seed=4) for _ in range(2)]
    logits, scores = torch.zeros(G, B, V, dtype=torch.bfloat16, device="cuda"), torch.full((G, B), -float("inf"), device="cuda")
    scores[:, 0] = 0.0                                            # the first step: one beam of each

    def step(cache, scores):
        out, parents, tokens = kv.select_beams(logits, scores, B)
        cache.reorder(parents.view(-1))
        cache.resize(cache.lengths + 1)
        scores.copy_(out)
        return parents, tokens
    mine = [scores.clone() for _ in range(2)]
    warm = ref.make(kv, [37, 0, 0, 0] * G, heads=2, dim=64, pages=120, width=8, seed=4)
    step(warm, scores.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(caches[0], mine[0])
    for i in range(6):
        _say(f"replay {i}")
        logits.copy_(torch.randn(G, B, V, generator=torch.Generator().manual_seed(i)))
        graph.replay()
        torch.cuda.synchronize()
        want = step(caches[1], mine[1])
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(*mine)
        for a, b in ((caches[0].table, caches[1].table), (caches[0].lengths, caches[1].lengths), (caches[0].refs, caches[1].refs)):
            assert torch.equal(a, b)
    assert bool((caches[0].lengths == 43).all()) and caches[0].device_status() == 0 and caches[1].device_status() == 0
