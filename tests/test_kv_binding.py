"""The paged cache's binding without a GPU: what it does around the C calls."""

import ctypes as C
import types

import pytest
import torch

import paper_2608_07971_amd as esp
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


def test_captured_calls_take_scratch_of_their_graph(on_the_host, monkeypatch):
    cache, now = on_the_host, [None]
    cache._work, cache._graph_work, cache._outgrown, cache.kv_heads = {}, (None, {}), [], 2
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: now[0] is not None)
    monkeypatch.setattr(kv, "_capture", lambda stream: now[0], raising=False)
    for kind in ("attend", "pages"):
        now[0] = None
        eager = cache._workspace(kind, 5000, 7)
        seen = [eager]
        for now[0] in (1, 2):                                     # two captures on a stream that has scratch
            w = cache._workspace(kind, 5000, 7)
            assert w.numel() >= 5000 and all(w.data_ptr() != x.data_ptr() for x in seen)
            assert cache._workspace(kind, 4000, 7) is w           # the graph's calls share it
            assert cache._workspace(kind, 5000, 8) is not w       # but not those on another stream of the capture
            more = cache._workspace(kind, 9000, 7)
            assert more.numel() >= 9000 and more is not w
            seen += [w, more]
        now[0] = None
        assert cache._workspace(kind, 5000, 7) is eager
        if kind == "attend":                                      # the counters are clear
            assert not any(bool(x[:4 * (768 + 2)].any()) for x in seen)


def test_scratch_is_not_kept_past_an_error(on_the_host, monkeypatch):
    cache, code = on_the_host, [0]
    cache._work, cache._graph_work, cache._outgrown, cache.kv_heads, cache.ptr = {}, (None, {}), [], 2, 0
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(kv, "lib", lambda: types.SimpleNamespace(esp_kv_device_status=lambda ptr, stream: code[0]))
    w = cache._workspace("attend", 5000, 7)
    w[40] = 3                                                     # a ticket that was drawn and not given back
    assert cache.device_status() == 0 and cache._workspace("attend", 5000, 7) is w
    code[0] = 2
    assert cache.device_status() == 2
    again = cache._workspace("attend", 5000, 7)
    assert again is not w and not bool(again[:4 * (768 + 2)].any())


def test_attention_beyond_32_bits_of_threads_is_refused():
    at = 0x10000                                                  # stands for a device address: never read
    c = kv.esp_kv_cache(8, 1, 2, 16, 64, 4, 4, at, at, at, at, at, at, at)
    p, n, view = C.addressof(c), C.c_size_t(0), kv.esp_kv_view(at, 0, 0)
    ask = lambda tokens: kv.lib().esp_kv_attend_workspace(p, 1, tokens, 8, 1000, 64, C.byref(n))  # noqa: E731
    most = (2 ** 24 - 16) // 2 * 128 // 4                         # tokens of 2 heads' units of 128 rows, 4 a token
    assert ask(most - 128) == esp.ESP_OK and n.value < 1 << 20
    assert ask(most + 128) == ask(2 ** 31 - 1) == esp.ESP_ERR_SHAPE
    assert kv.lib().esp_kv_attend(p, 0, 0, 1, 2 ** 31 - 1, at, None, 8, view, 0.1, 0, 1000, 64, view, None, at, 1 << 20, None) == esp.ESP_ERR_SHAPE
