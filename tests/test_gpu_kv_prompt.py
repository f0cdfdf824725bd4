"""GPU: attention of many new tokens over the paged 8-bit cache against the plain 64-bit form.

The launch is chosen by the call's shape, so each case says which kernel it is
for and how many parts a unit's tiles are cut into, and that is checked first.
"""
import ctypes as C

import numpy as np
import pytest
import torch

import _kv_ref as ref
import paper_2608_07971_amd as esp
from paper_2608_07971_amd import kv

EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # p significant bits: at most 2^-p of the value
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}          # half the least fp16 step


def _say(msg):
    print(f"[gpu-case] {msg}", flush=True)


def _randn(seed, *shape, dtype, gain=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * gain).to(dtype).cuda()


def _np(t):
    return t.double().cpu().numpy()


def launch_of(heads, dim, page, rows, tokens, group, max_new, max_length):
    """("many", parts) or ("few", None) from the workspace that the call asks for.  In front lie the counters of 768
    workgroups and the heads; behind them the kernel of many new tokens has 128 rows of dim + 2 numbers for each part of
    a unit, or nothing where units have one part, as in caches of length 0; the one of few new tokens always has some."""
    at = 0x10000                                                  # stands for a device address: never read
    c = kv.esp_kv_cache(8, 1, heads, page, dim, 4096, 4096, at, at, at, at, at, at, at)

    def more(length):
        n = C.c_size_t(0)
        assert kv.lib().esp_kv_attend_workspace(C.addressof(c), rows, tokens, heads * group, max_new, length, C.byref(n)) == esp.ESP_OK
        return n.value - -(-(768 + heads) * 4 // 256) * 256
    if more(0):
        return "few", None
    parts, rest = divmod(more(max_length), (tokens * group // 128 + rows) * heads * 128 * (dim + 2) * 4)
    assert rest == 0 and parts != 1
    return "many", max(1, parts)


# new tokens, lengths, heads, group, dim, page, window, type, parts of a unit
MANY = [
    ([400], [1500], 16, 1, 64, 16, 0, torch.bfloat16, 2),
    ([150, 0, 170], [700, 30, 1600], 4, 6, 128, 32, 0, torch.float16, 3),
    ([200, 130, 90], [150, 130, 5], 8, 2, 128, 64, 0, torch.bfloat16, 1),
    ([333], [1200], 8, 3, 64, 16, 100, torch.float16, 2),
    ([120], [121], 16, 5, 128, 16, 0, torch.float16, 1),
    ([150], [4100], 1, 64, 64, 64, 0, torch.bfloat16, 6),
    ([130, 257, 1], [130, 900, 77], 16, 2, 128, 16, 64, torch.bfloat16, 1),
    ([1100], [1300], 8, 4, 128, 64, 0, torch.bfloat16, 1),
    ([500, 300], [2000, 2500], 8, 2, 64, 32, 700, torch.bfloat16, 4),
    ([400], [400], 16, 1, 128, 32, 1, torch.float16, 1),
    ([700], [2100], 6, 3, 128, 16, 0, torch.float16, 4),
    ([65, 64, 63, 129, 128, 127], [65, 640, 63, 129, 1280, 127], 8, 3, 64, 64, 0, torch.float16, 2),
]


@pytest.mark.parametrize("new,lengths,heads,group,dim,page,window,dtype,parts", MANY)
def test_the_cases_take_the_launch_that_they_are_for(new, lengths, heads, group, dim, page, window, dtype, parts):
    assert launch_of(heads, dim, page, len(new), sum(new), group, max(new), max(lengths)) == ("many", parts)


def _reference(q, k, v, n, window, scale, held):
    """As _kv_ref.attend, of the tokens that are held (bool [L])."""
    L, G = k.shape[0], q.shape[1] // k.shape[1]
    out, lse = np.zeros_like(q), np.full(q.shape[:2], -np.inf)
    spread, most = np.zeros_like(q), np.zeros(q.shape[:2])
    for i in range(n):
        p = L - n + i
        at = np.nonzero(held[max(0, p - window + 1) if window else 0:max(0, p + 1)])[0] + (max(0, p - window + 1) if window else 0)
        if not len(at):
            continue
        for h in range(k.shape[1]):
            kk, vv, qq = k[at, h], v[at, h], q[i, h * G:h * G + G]
            s = scale * (qq @ kk.T)
            m = s.max(-1, keepdims=True)
            w = np.exp(s - m)
            total = w.sum(-1, keepdims=True)
            out[i, h * G:h * G + G], spread[i, h * G:h * G + G] = w @ vv / total, w @ np.abs(vv) / total
            lse[i, h * G:h * G + G] = (m + np.log(total))[:, 0]
            most[i, h * G:h * G + G] = (np.abs(qq) @ np.abs(kk).T).max(-1) * abs(scale)
    return out, lse, spread, most


def _check(cache, q, new, window=0, scale=None, foreign=False, out=None, want_status=esp.ESP_OK, layer=0):
    """The call against the reference.  Scores: dim products added in float32, one scale and one exponential; weights
    rounded to fp16, 2^-11 of each, and 2^-38 of the largest below its range; values with a scale that is no power of
    two rounded to fp16 once more."""
    D = cache.head_dim
    scale = D ** -0.5 if scale is None else scale
    lengths = cache.lengths.tolist()
    heads, group = cache.kv_heads, q.shape[1] // cache.kv_heads
    kind, parts = launch_of(heads, D, cache.page_tokens, len(new), sum(new), group, max(new), max(lengths))
    assert kind == "many"
    out, lse = cache.attend(layer, q, ref.offsets(new), window=window, scale=scale, max_new=max(new), max_length=max(lengths), out=out)
    kp, vp = ref.host(cache, layer)
    table, at, qn, on, ln = cache.table.cpu().numpy(), 0, _np(q), _np(out), _np(lse)
    for b, (n, L) in enumerate(zip(new, lengths)):
        names = np.repeat(table[b], cache.page_tokens)[:L]
        held = (names >= 0) & (names < cache.pages)
        k, v = (ref.tokens_of(x, np.clip(table[b], 0, cache.pages - 1), L) for x in (kp, vp))
        want, want_lse, spread, most = _reference(qn[at:at + n], k, v, n, window, scale, held)
        d = (D * 2.0 ** -24 * most + 2.0 ** -20 * (1 + most))[..., None]
        top = np.nanmax(np.abs(v[held])) if held.any() else 0
        bound = spread * (2.0 ** -11 * (2 if foreign else 1) + 2 * d + 2.0 ** -20) + 2.0 ** -38 * L * top + EPS[q.dtype] * np.abs(want) * 1.01 + TINY[q.dtype]
        got, got_lse, none = on[at:at + n], ln[at:at + n], np.isneginf(want_lse)
        nan = np.isnan(want)
        assert np.array_equal(np.isnan(got), nan) and np.array_equal(np.isnan(got_lse), np.isnan(want_lse))
        off = np.abs(got - want)
        assert (off <= bound)[~nan].all(), (b, n, L, np.nanmax(off - bound))
        assert np.array_equal(np.isneginf(got_lse), none) and not got[none].any()
        fine = np.isfinite(want_lse)
        assert (np.abs(got_lse[fine] - want_lse[fine]) <= 2 * d[..., 0][fine] + 2.0 ** -20 * (1 + np.abs(want_lse[fine]))).all()
        at += n
    assert cache.device_status() == want_status
    return out, lse


def _say_case(what, new, cache, dtype):
    _say(f"{what} {new} of {cache.lengths.tolist()} heads={cache.kv_heads} dim={cache.head_dim} page={cache.page_tokens} {dtype}")


@pytest.mark.gpu
@pytest.mark.parametrize("new,lengths,heads,group,dim,page,window,dtype,parts", MANY)
def test_attend_many_new_tokens(new, lengths, heads, group, dim, page, window, dtype, parts):
    cache = ref.make(kv, lengths, page=page, heads=heads, dim=dim, seed=len(lengths) + page)
    _say_case(f"attend window={window} group={group}", new, cache, dtype)
    q = _randn(11, sum(new), heads * group, dim, dtype=dtype, gain=2.0)
    a = _check(cache, q, new, window)
    b = cache.attend(0, q, ref.offsets(new), window=window, max_new=max(new), max_length=max(lengths))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dim,page,dtype,length", [(64, 16, torch.float16, 700), (128, 32, torch.bfloat16, 1700)])
def test_many_new_tokens_extreme_scores(dim, page, dtype, length):
    """One token far above the rest, equal scores, scores of the other sign."""
    cache = ref.make(kv, [length], page=page, heads=16, dim=dim, seed=page)
    for scale, gain in ((None, 60.0), (0.0, 1.0), (-0.5, 1.0)):
        _say_case(f"attend scale={scale} gain={gain}", [400], cache, dtype)
        _check(cache, _randn(3, 400, 16, dim, dtype=dtype, gain=gain), [400], scale=scale)


@pytest.mark.gpu
@pytest.mark.parametrize("dim,page,dtype,length", [(128, 16, torch.float16, 700), (64, 64, torch.bfloat16, 1700)])
def test_many_new_tokens_scales_of_any_value(dim, page, dtype, length):
    """Block scales that are no powers of two, of zero, and apart by 2^14."""
    cache = ref.make(kv, [length], page=page, heads=16, dim=dim, seed=page)
    t = cache.table[0].long()
    q = _randn(4, 400, 16, dim, dtype=dtype)
    g = np.random.default_rng(5)
    for which in (0, 1):
        cache.scale[t, 0, which] = torch.from_numpy(g.uniform(0.01, 0.03, (t.numel(), 16)).astype(np.float32)).cuda()
    _say_case("attend scales of any value", [400], cache, dtype)
    _check(cache, q, [400], foreign=True)
    cache.scale[t[2], 0] = 0.0
    _check(cache, q, [400], foreign=True)
    cache.scale[t, 0, 1] = torch.from_numpy(np.exp2(g.integers(-7, 8, (t.numel(), 16))).astype(np.float32)).cuda()
    _check(cache, q, [400])


@pytest.mark.gpu
@pytest.mark.parametrize("window", [0, 90])
@pytest.mark.parametrize("heads,group,dim,page,length", [(16, 1, 64, 16, 600), (8, 3, 128, 32, 1300), (16, 2, 64, 64, 1300)])
def test_many_new_tokens_nan_reaches_only_the_queries_that_see_it(heads, group, dim, page, length, window):
    n, dtype = 400, torch.float16
    q = _randn(5, n, heads * group, dim, dtype=dtype)
    for at in (length - n + 130, length - 1, length - n - 5):
        for which in ("k", "v"):
            cache = ref.make(kv, [length], heads=heads, dim=dim, page=page)
            name, i = int(cache.table[0, at // page]), at % page
            if which == "k":
                cache.k.view(torch.uint8)[name, 0, 1, i, 3] = 0x7f
            else:
                cache.v.view(torch.uint8)[name, 0, 1, 3, i] = 0xff
            _say_case(f"attend NaN in {which} at {at} window={window}", [n], cache, dtype)
            out, lse = _check(cache, q, [n], window)
            p = torch.arange(length - n, length, device="cuda")
            sees = (p >= at) & ((p - window < at) if window else True)
            hit = torch.isnan(out[:, group:2 * group]).any(-1).any(-1)
            assert torch.equal(hit, sees) and bool(sees.any())
            assert not torch.isnan(out[:, :group]).any() and not torch.isnan(out[:, 2 * group:]).any()


@pytest.mark.gpu
@pytest.mark.parametrize("dim,page,length", [(64, 32, 700), (128, 64, 1700)])
def test_many_new_tokens_pages_that_are_not_there(dim, page, length):
    cache = ref.make(kv, [length], page=page, heads=16, dim=dim)
    q = _randn(6, 400, 16, dim, dtype=torch.bfloat16)
    cache.table[0, 1], cache.table[0, (length - 200) // page] = -1, 99999
    _say_case("attend holes", [400], cache, torch.bfloat16)
    _check(cache, q, [400], want_status=esp.ESP_ERR_SHAPE)
    _check(cache, q, [400], window=50, want_status=esp.ESP_ERR_SHAPE)
    cache.table[0] = -1                                           # nothing at all
    out, lse = _check(cache, q, [400], want_status=esp.ESP_ERR_SHAPE)
    assert not out.any() and bool((lse == -torch.inf).all())


@pytest.mark.gpu
@pytest.mark.parametrize("length", [700, 1700])
def test_many_new_tokens_strides(length):
    cache = ref.make(kv, [length], page=16, heads=16, dim=64, layers=2)
    wide = _randn(7, 400, 35, 67, dtype=torch.bfloat16)           # rows of 67: not 16-byte aligned
    for layer, q in enumerate((wide[:, 1:33, 3:], wide.transpose(0, 1).contiguous().transpose(0, 1)[:, :32, :64])):
        _say_case(f"attend strides {q.stride()}", [400], cache, torch.bfloat16)
        out = torch.zeros(400, 34, 69, dtype=torch.bfloat16, device="cuda")
        _check(cache, q, [400], layer=layer, out=out[:, 1:33, 5:])
        assert not out[:, 0].any() and not out[:, 33].any() and not out[..., :5].any()
        again = cache.attend(layer, q.contiguous(), ref.offsets([400]), max_new=400, max_length=length)[0]
        assert torch.equal(out[:, 1:33, 5:], again)


@pytest.mark.gpu
def test_many_new_tokens_rows_over_their_bounds():
    cache = ref.make(kv, [700, 650, 600], page=32, heads=8, dim=64)
    q, new = _randn(8, 600, 16, 64, dtype=torch.float16), [200, 200, 200]
    want = cache.attend(0, q, ref.offsets(new))
    _say_case("attend bounds", new, cache, torch.float16)
    assert launch_of(8, 64, 32, 3, 600, 2, 600, 704) == ("many", 1) == launch_of(8, 64, 32, 3, 600, 2, 200, 650)
    out = torch.full_like(q, 7.0)
    cache.attend(0, q, ref.offsets(new), max_new=200, max_length=650, out=out)
    assert cache.device_status() == esp.ESP_ERR_SHAPE
    assert bool((out[:200] == 7).all()) and torch.equal(out[200:], want[0][200:])
    seqs = torch.tensor([2, 9, 0], dtype=torch.int32, device="cuda")
    got = cache.attend(0, q, ref.offsets(new), seqs=seqs)
    assert cache.device_status() == esp.ESP_ERR_SHAPE
    alone = torch.tensor([2, 1, 0], dtype=torch.int32, device="cuda")
    want = cache.attend(0, q, ref.offsets(new), seqs=alone)
    assert torch.equal(got[0][:200], want[0][:200]) and torch.equal(got[0][400:], want[0][400:]) and cache.device_status() == 0
