"""Without a GPU: leaves whose accumulators a graph from before a capture holds are found."""
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
