"""GPU: a graph that saved what a call then wrote says so in backward(), as after torch's own writes in place."""
import pytest
import torch

import _kv_ref as ref
from paper_2608_07971_amd import kv

pytestmark = pytest.mark.gpu


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _saved(*tensors):
    """What goes on from a product with each of the tensors, which it saves."""
    return [(torch.ones(t.shape, device="cuda", requires_grad=True) * t.detach()).sum() for t in tensors]


def _all_raise(graphs):
    for y in graphs:
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()


def test_what_calls_write_is_counted():
    cache, rope = ref.make(kv, [40, 17], heads=2, dim=64, layers=1, width=8, spare=9), kv.Rope(64)
    q = torch.randn(2, 4, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    offs, pos, mass = ref.offsets([1, 1]), _dev([5, 6]), torch.zeros(cache.mass_shape, device="cuda")
    out = torch.zeros_like(q)
    graphs = _saved(out)
    _, lse = cache.attend(0, q, offs, out=out)
    _all_raise(graphs)
    graphs = _saved(mass)
    cache.weigh(0, q, lse, offs, mass)
    _all_raise(graphs)
    for into in (out, q):
        graphs = _saved(into)
        kv.rotate(rope, q, pos, out=into)
        _all_raise(graphs)
    graphs = _saved(cache.scale)
    cache.append(0, q[:, :2], q[:, 2:], offs)
    _all_raise(graphs)
    graphs = _saved(mass, cache.scale)
    cache.evict(_dev([20, 9]), mass)
    _all_raise(graphs)
    assert cache.device_status() == 0


@pytest.mark.parametrize("name", ["resize", "fork", "reorder", "evict"])
def test_lengths_that_were_positions(name):
    """The next token's position is its sequence's length, which the gradient of the turning asks for again."""
    rope, q = kv.Rope(64), torch.randn(2, 4, 64, generator=torch.Generator().manual_seed(1)).cuda().requires_grad_()
    for graph in (lambda at: kv.norm_rotate(rope, q, q.detach(), None, None, at)[0], lambda at: kv.rotate(rope, q, at)):
        cache = ref.make(kv, [40, 0], heads=2, dim=64, width=4, spare=9)
        y = graph(cache.lengths)
        {"resize": lambda: cache.resize(cache.lengths + 1), "fork": lambda: cache.fork(_dev([0]), _dev([1])), "reorder": lambda: cache.reorder(_dev([1, 0])),
         "evict": lambda: cache.evict(_dev([20, 0]), torch.zeros(cache.mass_shape, device="cuda"))}[name]()
        assert cache.device_status() == 0
        _all_raise([y.sum()])


def test_a_compaction_copies_pages():
    cache = ref.make(kv, [40, 17], heads=1, dim=64, width=4, spare=9)
    graphs = _saved(cache.scale)
    table, refs, _ = cache.compact()
    _all_raise(graphs)
    cache.install(table, refs)
    assert cache.device_status() == 0
