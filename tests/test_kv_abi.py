"""The paged cache's C-ABI without a GPU: exports, rotary frequencies, refusals on the host."""
import ctypes as C
import os
import re

import numpy as np
import pytest

import paper_2608_07971_amd as esp
from paper_2608_07971_amd import kv
from _kv_ref import frequencies

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000                                                # stands for a device address: never read here


def _cache(**change):
    c = dict(pages=8, layers=1, kv_heads=2, page_tokens=16, head_dim=64, sequences=4, table_width=4, k=A, v=A, scale=A, table=A,
             lengths=A, refs=A, status=A)
    c.update(change)
    return kv.esp_kv_cache(*c.values())


def _view(data=A, token=128, head=64):
    return kv.esp_kv_view(data, token, head)


def _rope(turns=A, magnitude=1.0, rotary=64, interleaved=0):
    return kv.esp_kv_rope(turns, magnitude, rotary, interleaved)


def test_header_and_binding_agree():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "esp_kv.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(esp_kv_[a-z_]+)\s*\(", text))
    assert names == set(kv._SIGS)
    for n in names:
        assert hasattr(kv.lib(), n), n


@pytest.mark.parametrize("rotary", [2, 6, 32, 128])
@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "parts"])
def test_frequencies(rotary, scaling):
    if scaling == "ntk" and rotary < 4:
        return
    turns, magnitude = kv.esp_kv_rope_turns(rotary, 5e5, kv.SCALINGS[scaling], 8.0, 2048)
    f, m = frequencies(rotary, 5e5, scaling, 8.0, 2048)
    # pow and the products: a few roundings of 2^-53 each, pow under 2^-50
    assert np.allclose(np.array(turns) * 2 * np.pi, f, rtol=1e-14, atol=0)
    assert abs(magnitude - m) <= 2.0 ** -24 * m


@pytest.mark.parametrize("args,code", [
    ((0, 1e4, 0, 1.0, 0), esp.ESP_ERR_SHAPE), ((7, 1e4, 0, 1.0, 0), esp.ESP_ERR_SHAPE), ((8, 1.0, 0, 1.0, 0), esp.ESP_ERR_INVALID_ARG),
    ((8, float("nan"), 0, 1.0, 0), esp.ESP_ERR_INVALID_ARG), ((8, 1e4, 4, 1.0, 0), esp.ESP_ERR_INVALID_ARG),
    ((8, 1e4, 1, 0.5, 0), esp.ESP_ERR_INVALID_ARG), ((8, 1e4, 1, float("inf"), 0), esp.ESP_ERR_INVALID_ARG),
    ((2, 1e4, 2, 2.0, 0), esp.ESP_ERR_SHAPE), ((8, 1e4, 3, 2.0, 0), esp.ESP_ERR_INVALID_ARG),
])
def test_frequencies_refused(args, code):
    with pytest.raises(esp.EspError) as e:
        kv.esp_kv_rope_turns(*args)
    assert e.value.code == code


BAD_CACHES = [(dict(pages=0), esp.ESP_ERR_SHAPE), (dict(page_tokens=24), esp.ESP_ERR_SHAPE), (dict(page_tokens=8), esp.ESP_ERR_SHAPE),
              (dict(head_dim=96), esp.ESP_ERR_SHAPE), (dict(kv_heads=0), esp.ESP_ERR_SHAPE), (dict(table_width=1 << 28), esp.ESP_ERR_SHAPE),
              (dict(sequences=1 << 30), esp.ESP_ERR_SHAPE), (dict(k=0), esp.ESP_ERR_INVALID_ARG), (dict(v=A + 8), esp.ESP_ERR_INVALID_ARG),
              (dict(status=0), esp.ESP_ERR_INVALID_ARG)]


@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_bad_caches_are_refused_by_every_call(change, code):
    L, c = kv.lib(), _cache(**change)
    p, n, v, r = C.addressof(c), C.c_size_t(0), _view(), _rope()
    big = 1 << 20
    assert L.esp_kv_append(p, 0, 0, 1, 1, A, None, v, v, C.addressof(r), 0, v, v, None) == code
    assert L.esp_kv_gather(p, 0, 0, 1, 1, A, None, A, A, A, None) == code
    assert L.esp_kv_attend_workspace(p, 1, 1, 2, 1, 64, C.byref(n)) == code
    assert L.esp_kv_attend(p, 0, 0, 1, 1, A, None, 2, v, 0.1, 0, 1, 64, v, A, A, big, None) == code
    assert L.esp_kv_pages_workspace(p, 1, C.byref(n)) == code
    assert L.esp_kv_resize(p, A, A, big, None) == code
    assert L.esp_kv_fork(p, 1, A, A, A, big, None) == code
    assert L.esp_kv_compact(p, -1, A, A, A, A, big, None) == code
    assert L.esp_kv_resize(None, A, A, big, None) == esp.ESP_ERR_INVALID_ARG


def test_bad_rotations_are_refused():
    L, r, v = kv.lib(), _rope(), _view()
    call = lambda rope=r, type=0, tokens=1, heads=1, dim=64, x=v, pos=A, out=v: L.esp_kv_rotate(  # noqa: E731
        None if rope is None else C.addressof(rope), type, tokens, heads, dim, x, pos, 0, out, None)
    assert call(rope=None) == call(type=3) == call(pos=None) == call(x=_view(0)) == call(out=_view(0)) == esp.ESP_ERR_INVALID_ARG
    assert call(rope=_rope(turns=0)) == call(rope=_rope(interleaved=2)) == call(rope=_rope(magnitude=float("nan"))) == esp.ESP_ERR_INVALID_ARG
    assert call(rope=_rope(rotary=0)) == call(rope=_rope(rotary=7)) == call(rope=_rope(rotary=66)) == esp.ESP_ERR_SHAPE
    assert call(tokens=-1) == call(heads=-1) == call(dim=63) == call(tokens=1 << 31) == esp.ESP_ERR_SHAPE
    assert call(tokens=0, pos=None) == call(heads=0) == esp.ESP_OK


def test_bad_appends_gathers_and_attentions_are_refused():
    L, c, r, v = kv.lib(), _cache(), _rope(), _view()
    p = C.addressof(c)
    app = lambda layer=0, type=0, rows=1, tokens=1, off=A, k=v, vv=v, rope=r, qh=0, q=v: L.esp_kv_append(  # noqa: E731
        p, layer, type, rows, tokens, off, None, k, vv, None if rope is None else C.addressof(rope), qh, q, q, None)
    assert app(type=2) == app(off=None) == app(k=_view(0)) == app(vv=_view(0)) == esp.ESP_ERR_INVALID_ARG
    assert app(qh=2, rope=None) == app(qh=2, q=_view(0)) == app(qh=2, q=_view(A + 2)) == app(qh=2, q=_view(A, 9)) == esp.ESP_ERR_INVALID_ARG
    assert app(layer=1) == app(layer=-1) == app(rows=-1) == app(tokens=-1) == app(rope=_rope(rotary=8)) == app(rope=_rope(rotary=128)) == esp.ESP_ERR_SHAPE
    assert app(rows=0) == app(tokens=0, off=None) == esp.ESP_OK
    gat = lambda layer=0, type=0, tokens=1, starts=A, k=A: L.esp_kv_gather(p, layer, type, 1, tokens, A, None, starts, k, A, None)  # noqa: E731
    assert gat(type=2) == gat(starts=None) == gat(k=None) == gat(k=A + 4) == esp.ESP_ERR_INVALID_ARG
    assert gat(layer=1) == gat(tokens=-1) == esp.ESP_ERR_SHAPE
    n = C.c_size_t(0)
    assert L.esp_kv_attend_workspace(p, 2, 2, 2, 1, 64, C.byref(n)) == esp.ESP_OK and n.value > 0
    att = lambda layer=0, type=0, heads=2, q=v, scale=0.1, window=0, new=1, length=64, out=v, w=A, size=n.value: L.esp_kv_attend(  # noqa: E731
        p, layer, type, 2, 2, A, None, heads, q, scale, window, new, length, out, None, w, size, None)
    assert att(type=2) == att(scale=float("nan")) == att(window=-1) == att(q=_view(0)) == att(out=_view(0)) == esp.ESP_ERR_INVALID_ARG
    assert att(layer=1) == att(heads=3) == att(heads=0) == att(new=-1) == att(length=-1) == esp.ESP_ERR_SHAPE
    assert att(w=None) == att(w=A + 16) == att(size=n.value - 1) == esp.ESP_ERR_WORKSPACE


def test_bad_page_operations_are_refused():
    L, c = kv.lib(), _cache()
    p, n = C.addressof(c), C.c_size_t(0)
    assert L.esp_kv_pages_workspace(p, 4, C.byref(n)) == esp.ESP_OK
    size = n.value
    assert L.esp_kv_pages_workspace(p, 5, C.byref(n)) == L.esp_kv_pages_workspace(p, -1, C.byref(n)) == esp.ESP_ERR_SHAPE
    assert L.esp_kv_pages_workspace(p, 1, None) == esp.ESP_ERR_INVALID_ARG
    assert L.esp_kv_resize(p, None, A, size, None) == L.esp_kv_fork(p, 1, None, A, A, size, None) == esp.ESP_ERR_INVALID_ARG
    assert L.esp_kv_compact(p, 1, None, A, A, A, size, None) == L.esp_kv_compact(p, 1, A, None, A, A, size, None) == esp.ESP_ERR_INVALID_ARG
    assert L.esp_kv_fork(p, 5, A, A, A, size, None) == L.esp_kv_fork(p, -1, A, A, A, size, None) == esp.ESP_ERR_SHAPE
    for w, s in ((None, size), (A + 8, size), (A, size - 1)):
        assert L.esp_kv_resize(p, A, w, s, None) == L.esp_kv_fork(p, 1, A, A, w, s, None) == esp.ESP_ERR_WORKSPACE
        assert L.esp_kv_compact(p, 1, A, A, A, w, s, None) == esp.ESP_ERR_WORKSPACE
    assert L.esp_kv_fork(p, 0, None, None, None, 0, None) == esp.ESP_OK
    assert L.esp_kv_device_status(None, None) == esp.ESP_ERR_INVALID_ARG


def test_launches_beyond_32_bits_of_threads_are_refused():
    L, c, r, v = kv.lib(), _cache(), _rope(), _view()
    p, most = C.addressof(c), 2 ** 31 - 1
    assert L.esp_kv_append(p, 0, 0, 1, most, A, None, v, v, C.addressof(r), 64, v, v, None) == esp.ESP_ERR_SHAPE
    assert L.esp_kv_gather(p, 0, 0, 1, most, A, None, A, A, A, None) == esp.ESP_ERR_SHAPE
