"""The paged cache's binding without a GPU: what it does around the C calls."""

import pytest
import torch

from paper_2608_07971_amd import kv


@pytest.fixture
def on_the_host(monkeypatch):
    """A cache's object over tensors on the host: nothing here reaches a C call."""
    monkeypatch.setattr(kv, "_current_device", lambda: None)
    monkeypatch.setattr(kv, "_raw_stream", lambda index: 0)
    cache = object.__new__(kv.PagedCache)
    cache.device, cache.index = torch.device("cpu"), None
    cache.pages, cache.sequences, cache.table_width, cache.page_tokens = 6, 2, 3, 16
    cache.table = torch.full((2, 3), -1, dtype=torch.int32)
    cache.refs = torch.zeros(6, dtype=torch.int32)
    cache.lengths = torch.zeros(2, dtype=torch.int32)
    return cache


def test_install_keeps_the_addresses_that_calls_were_given(on_the_host):
    cache = on_the_host
    table, refs = cache.table, cache.refs
    places = table.data_ptr(), refs.data_ptr()
    new = torch.tensor([[0, 2, -1], [1, -1, -1]], dtype=torch.int32), torch.tensor([1, 1, 1, 0, 0, 0], dtype=torch.int32)
    cache.install(*new)
    assert cache.table is table and cache.refs is refs and places == (table.data_ptr(), refs.data_ptr())
    assert torch.equal(table, new[0]) and torch.equal(refs, new[1])
    for bad in ((new[0].view(3, 2), new[1]), (new[0], new[1][:5]), (new[0].long(), new[1])):
        with pytest.raises(ValueError):
            cache.install(*bad)
    assert torch.equal(table, new[0]) and torch.equal(refs, new[1])
