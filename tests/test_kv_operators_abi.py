"""Norms, selection, reordering, weights and eviction without a GPU: refusals on the host."""
import ctypes as C

import pytest

import paper_2608_07971_amd as esp
from paper_2608_07971_amd import kv
from test_kv_abi import A, BAD_CACHES, _cache, _rope, _view

BIG = 1 << 24


@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_bad_caches_are_refused_by_every_call(change, code):
    L, c = kv.lib(), _cache(**change)
    p, n, v = C.addressof(c), C.c_size_t(0), _view()
    assert L.esp_kv_reorder(p, A, A, BIG, None) == code
    assert L.esp_kv_weigh(p, 0, 0, 1, 1, A, None, 2, v, A, 0.1, 0, 1.0, 1, 64, A, None) == code
    assert L.esp_kv_evict_workspace(p, C.byref(n)) == code
    assert L.esp_kv_evict(p, A, 0, A, A, BIG, None) == code


def test_bad_norms_are_refused():
    L, r, v = kv.lib(), _rope(), _view()

    def call(rope=r, type=0, tokens=1, dim=64, qh=1, kh=1, q=v, k=v, w=A, wt=0, pos=A, eps=1e-6, qo=v, ko=v, back=False, dw=None, work=None, size=0):
        head = (None if rope is None else C.addressof(rope), type, tokens, dim, qh, kh, q, k, w, w, wt, pos, eps)
        if not back:
            return L.esp_kv_norm_rotate(*head, qo, ko, None)
        return L.esp_kv_norm_rotate_backward(*head, v, v, qo, ko, dw, dw, work, size, None)
    for back in (False, True):
        assert call(rope=None, back=back) == call(type=3, back=back) == call(type=-1, back=back) == call(wt=1, back=back) == esp.ESP_ERR_INVALID_ARG
        assert call(type=2, wt=0, back=back) == call(pos=None, back=back) == call(q=_view(0), back=back) == call(ko=_view(0), back=back) == esp.ESP_ERR_INVALID_ARG
        assert all(call(eps=e, back=back) == esp.ESP_ERR_INVALID_ARG for e in (0.0, -1.0, float("nan"), float("inf")))
        assert all(call(rope=x, back=back) == esp.ESP_ERR_INVALID_ARG for x in (_rope(turns=0), _rope(interleaved=2), _rope(magnitude=float("nan"))))
        assert all(call(rope=x, back=back) == esp.ESP_ERR_SHAPE for x in (_rope(rotary=0), _rope(rotary=7), _rope(rotary=66)))
        assert all(call(**x, back=back) == esp.ESP_ERR_SHAPE for x in (dict(tokens=-1), dict(tokens=1 << 31), dict(dim=63), dict(dim=514), dict(qh=-1), dict(kh=65537)))
        assert call(tokens=0, pos=None, q=_view(0), k=_view(0), back=back) == call(qh=0, kh=0, pos=None, back=back) == esp.ESP_OK
    n = C.c_size_t(0)
    assert L.esp_kv_norm_rotate_workspace(100, 64, 4, 2, C.byref(n)) == esp.ESP_OK and n.value > 0
    assert L.esp_kv_norm_rotate_workspace(100, 64, 4, 2, None) == esp.ESP_ERR_INVALID_ARG
    assert L.esp_kv_norm_rotate_workspace(-1, 64, 4, 2, C.byref(n)) == L.esp_kv_norm_rotate_workspace(1, 514, 4, 2, C.byref(n)) == esp.ESP_ERR_SHAPE
    assert L.esp_kv_norm_rotate_workspace(0, 64, 4, 2, C.byref(n)) == esp.ESP_OK
    assert L.esp_kv_norm_rotate_workspace(1, 64, 1, 1, C.byref(n)) == esp.ESP_OK
    for work, size in ((None, n.value), (A + 8, n.value), (A, n.value - 1)):
        assert call(back=True, dw=A, work=work, size=size) == esp.ESP_ERR_WORKSPACE


def test_bad_selections_are_refused():
    L, n = kv.lib(), C.c_size_t(0)
    size = lambda g=2, b=3, v=50, w=4: L.esp_kv_select_beams_workspace(g, b, v, w, C.byref(n))  # noqa: E731
    assert size() == esp.ESP_OK and n.value > 0
    need = n.value

    def call(type=0, g=2, b=3, v=50, w=4, x=A, s=A, e=None, pad=0, out=A, work=A, size=need):
        return L.esp_kv_select_beams(type, g, b, v, w, x, v * b, v, s, e, pad, out, A, A, work, size, None)
    assert L.esp_kv_select_beams_workspace(2, 3, 50, 4, None) == esp.ESP_ERR_INVALID_ARG
    for bad in (dict(g=-1), dict(b=0), dict(b=1025), dict(v=0), dict(w=0), dict(w=65), dict(g=1 << 23, b=2)):
        assert size(**bad) == call(**bad) == esp.ESP_ERR_SHAPE
    for bad in (dict(type=3), dict(x=None), dict(s=None), dict(out=None), dict(e=A, pad=50), dict(e=A, pad=-1)):
        assert call(**bad) == esp.ESP_ERR_INVALID_ARG
    for bad in (dict(work=None), dict(work=A + 8), dict(size=need - 1)):
        assert call(**bad) == esp.ESP_ERR_WORKSPACE
    assert call(g=0, x=None, work=None) == esp.ESP_OK


def test_bad_reorderings_weights_and_evictions_are_refused():
    L, c, v = kv.lib(), _cache(), _view()
    p, n = C.addressof(c), C.c_size_t(0)
    assert L.esp_kv_pages_workspace(p, 4, C.byref(n)) == esp.ESP_OK
    assert L.esp_kv_reorder(p, None, A, n.value, None) == esp.ESP_ERR_INVALID_ARG
    for w, size in ((None, n.value), (A + 8, n.value), (A, n.value - 1)):
        assert L.esp_kv_reorder(p, A, w, size, None) == esp.ESP_ERR_WORKSPACE
    many = _cache(sequences=1 << 24, table_width=1)
    assert L.esp_kv_reorder(C.addressof(many), A, A, 1 << 40, None) == esp.ESP_ERR_SHAPE

    def weigh(layer=0, type=0, rows=1, tokens=1, off=A, heads=2, q=v, lse=A, scale=0.1, window=0, decay=1.0, new=1, length=64, mass=A, cache=p):
        return L.esp_kv_weigh(cache, layer, type, rows, tokens, off, None, heads, q, lse, scale, window, decay, new, length, mass, None)
    for bad in (dict(type=2), dict(off=None), dict(q=_view(0)), dict(lse=None), dict(mass=None), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(decay=float("nan")), dict(window=-1)):
        assert weigh(**bad) == esp.ESP_ERR_INVALID_ARG
    for bad in (dict(layer=1), dict(layer=-1), dict(rows=-1), dict(tokens=-1), dict(tokens=1 << 31), dict(heads=0), dict(heads=3), dict(new=-1), dict(length=-1),
                dict(heads=128, tokens=1 << 27)):
        assert weigh(**bad) == esp.ESP_ERR_SHAPE
    assert weigh(rows=0) == weigh(tokens=0) == weigh(new=0) == weigh(length=0) == esp.ESP_OK

    assert L.esp_kv_evict_workspace(p, C.byref(n)) == esp.ESP_OK and n.value > 0
    assert L.esp_kv_evict_workspace(p, None) == esp.ESP_ERR_INVALID_ARG
    assert L.esp_kv_evict(p, None, 0, A, A, n.value, None) == L.esp_kv_evict(p, A, 0, None, A, n.value, None) == esp.ESP_ERR_INVALID_ARG
    assert L.esp_kv_evict(p, A, -1, A, A, n.value, None) == esp.ESP_ERR_SHAPE
    for w, size in ((None, n.value), (A + 8, n.value), (A, n.value - 1)):
        assert L.esp_kv_evict(p, A, 0, A, w, size, None) == esp.ESP_ERR_WORKSPACE
    many = _cache(sequences=1 << 25, layers=16)
    assert L.esp_kv_evict_workspace(C.addressof(many), C.byref(n)) == esp.ESP_ERR_SHAPE


def test_counts_that_would_pass_32_bits_are_refused():
    L, n, v = kv.lib(), C.c_size_t(0), _view()
    for sequences, code in (((1 << 30) - (1 << 11), esp.ESP_OK), ((1 << 30) - (1 << 11) + 1, esp.ESP_ERR_SHAPE), ((1 << 30) - 1, esp.ESP_ERR_SHAPE)):
        many = _cache(sequences=sequences, table_width=1, layers=1, kv_heads=1)       # keys and values: 2 items a sequence, 4,096 workgroups
        assert L.esp_kv_evict_workspace(C.addressof(many), C.byref(n)) == code
        if code:
            assert L.esp_kv_evict(C.addressof(many), A, 0, A, A, 1 << 60, None) == code
    for width, code in (((1 << 27) - 128 - 1, esp.ESP_OK), ((1 << 27) - 64, esp.ESP_ERR_SHAPE), ((1 << 27) - 1, esp.ESP_ERR_SHAPE)):
        wide = _cache(sequences=1, table_width=width, page_tokens=16)
        assert L.esp_kv_evict_workspace(C.addressof(wide), C.byref(n)) == code
        if code:
            for length in (16 * width, (1 << 31) - 1):
                assert L.esp_kv_weigh(C.addressof(wide), 0, 0, 1, 1, A, None, 2, v, A, 0.1, 0, 1.0, 1, length, A, None) == code
