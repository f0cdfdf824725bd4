"""Without a GPU: leaves whose accumulators a graph from before a capture holds are found."""
import types

import pytest
import torch

from paper_2608_07971_amd import kv


def test_leaves_of_an_older_graph_are_found():
    x, y = torch.ones(3, requires_grad=True), torch.ones(3, requires_grad=True)
    assert kv._accumulators((x, None, torch.ones(3), y * 2), 7)[1] is False     # no other graph, no leaf
    older = x * 2                                                 # not marked with the capture's stream
    assert kv._accumulators((y, x), 7)[1] is True
    del older
    nodes, found = kv._accumulators((x,), 7)
    assert found is False and len(nodes) == 1
    mine = x * 3                                                  # a graph captured on the stream, this capture's or an earlier one
    del nodes
    assert kv._accumulators((x,), 7)[1] is False
    assert kv._accumulators((x,), 8)[1] is True                   # another stream's
    del mine
    assert kv._accumulators((x,), 8)[1] is False


def test_the_stream_of_an_accumulator_decides(monkeypatch):
    """Whichever call made it: a product recorded on the stream before is no older graph."""
    x, asked = torch.ones(3, requires_grad=True), []
    for told, older in ((7, False), (0, True), (9, True), (None, True)):
        monkeypatch.setattr(kv, "_stream_of", lambda node, leaf: (asked.append(leaf), told)[1])
        first = (x * x).sum()
        nodes, found = kv._accumulators((x,), 7)
        assert found is older and asked and asked[-1] is x
        asked.clear()
        assert kv._accumulators((x,), 7)[1] is older and bool(asked) is (told is None)      # once is enough
        del first, nodes


def test_asking_for_the_stream_leaves_the_leaf_alone():
    x = torch.ones(3, requires_grad=True)
    kept = x * 2
    node = torch.autograd.graph.get_gradient_edge(x).node
    assert kv._stream_of(node, x) is None and x.grad is None      # a leaf on the CPU has none
    kept.sum().backward()
    assert x.grad.tolist() == [2.0] * 3


def test_a_captured_rotation_of_an_older_graphs_leaf_has_no_backward(monkeypatch):
    rope = types.SimpleNamespace(index=0)
    monkeypatch.setattr(kv, "_turn", lambda rope, x, positions, inverse, out, s: x * 1)
    x, pos = torch.ones(2, 1, 4, requires_grad=True), torch.zeros(2, dtype=torch.int32)
    older = x * 2
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    y = kv.rotate.__wrapped__(rope, x, pos, s=7)
    with pytest.raises(RuntimeError, match="before the capture"):
        y.backward(torch.ones_like(y))
    del older


def test_asking_does_not_end_another_threads_pass(monkeypatch):
    """The question is told from a pass that has a gradient to add."""
    node, leaf = types.SimpleNamespace(hooks=[]), torch.ones(3, requires_grad=True)
    node.register_prehook = lambda hook: (node.hooks.append(hook), types.SimpleNamespace(remove=lambda: node.hooks.remove(hook)))[1]
    fake = types.SimpleNamespace(is_cuda=True, _backward_hooks=None, device=types.SimpleNamespace(index=0), detach=leaf.detach)
    monkeypatch.setattr(kv, "_raw_stream", lambda index: 7)
    monkeypatch.setattr(kv._Ask, "apply", lambda x: leaf)

    def backward(root, grad):
        try:
            assert node.hooks[0]((torch.ones(3),)) is None
        except kv._Told:
            pytest.fail("a pass with a gradient was ended")
        node.hooks[0]((None,))
    monkeypatch.setattr(torch.autograd, "backward", backward)
    assert kv._stream_of(node, fake) == 7 and node.hooks == []
