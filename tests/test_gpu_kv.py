"""GPU: the paged 8-bit cache against plain 64-bit forms.

Tolerances follow from the formats.  e4m3 has 4 significant bits, so a value
is within 2^-4 of itself of its code, or 2^-10 of the scale below the normal
range; bf16 has 8 and fp16 11 significant bits.
"""
import math

import numpy as np
import pytest
import torch

import _kv_ref as ref
import paper_2608_07971_amd as esp
from paper_2608_07971_amd import kv

pytestmark = pytest.mark.gpu

EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}   # p significant bits: at most 2^-p of the value
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}               # half the least fp16 step


def _say(msg):
    print(f"[gpu-case] {msg}", flush=True)


def _randn(seed, *shape, dtype=torch.float32, gain=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * gain).to(dtype).cuda()


def _np(t):
    return t.double().cpu().numpy()


# ---------------------------------------------------------------------------
# Rotation
# ---------------------------------------------------------------------------

def _rotation_bound(x, y, f, magnitude, interleaved, dtype):
    """Half a unit of the result, plus 4e-7 of the pair: cos and sin are within 2e-7 (polynomials 2.5e-8, the reduced
    angle 5e-8, magnitude and products 2^-24 each) and two products add up."""
    pair = ref.rotate(np.abs(x), np.zeros(x.shape[0]), f, magnitude, interleaved)
    n = len(f)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    both = pair.copy()
    both[..., a] = both[..., b] = pair[..., a] + pair[..., b]
    return EPS[dtype] * (np.abs(y) + 4e-7 * both) * 1.001 + 4e-7 * both + TINY[dtype]


ROTATIONS = [
    (1, 1, 64, 64, False, "none", torch.bfloat16), (257, 3, 128, 128, False, "parts", torch.bfloat16), (33, 9, 128, 32, True, "linear", torch.float16),
    (100, 5, 64, 64, True, "ntk", torch.float32), (64, 2, 80, 20, False, "none", torch.float32), (31, 3, 66, 66, True, "none", torch.float16),
    (5, 40, 256, 64, False, "parts", torch.float32), (7, 1, 128, 2, True, "none", torch.bfloat16),
]


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("tokens,heads,dim,rotary,interleaved,scaling,dtype", ROTATIONS)
def test_rotate(tokens, heads, dim, rotary, interleaved, scaling, dtype, inverse):
    _say(f"rotate {tokens}x{heads}x{dim} rotary={rotary} {scaling} {dtype} inverse={inverse}")
    rope = kv.Rope(dim, rotary, interleaved=interleaved, scaling=scaling, factor=8.0, context=4096)
    x = _randn(1, tokens, heads, dim, dtype=dtype)
    pos = torch.randint(-5, 1 << 20, (tokens,), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    pos[0] = (1 << 20) + 7
    y = kv.rotate(rope, x, pos.cuda(), inverse=inverse)
    f, m = ref.frequencies(rotary, 10000.0, scaling, 8.0, 4096)
    want = ref.rotate(_np(x), pos.numpy(), f, m, interleaved, inverse)
    assert (np.abs(_np(y) - want) <= _rotation_bound(_np(x), want, f, m, interleaved, dtype)).all()
    assert torch.equal(y[..., rotary:], x[..., rotary:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rotate_strides_and_in_place(dtype):
    rope = kv.Rope(64, 32)
    f, m = ref.frequencies(32)
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    wide = _randn(3, 50, 7, 65, dtype=dtype)                    # rows of 65: not 16-byte aligned
    for x in (wide[..., 1:], wide[:, 2:5, :64], wide.transpose(0, 1).contiguous().transpose(0, 1)[..., :64]):
        _say(f"rotate strides {x.stride()} {dtype}")
        want = ref.rotate(_np(x), pos.cpu().numpy(), f, m, False)
        bound = _rotation_bound(_np(x), want, f, m, False, dtype)
        assert (np.abs(_np(kv.rotate(rope, x, pos)) - want) <= bound).all()
        out = torch.zeros(x.shape[0], x.shape[1], 72, dtype=dtype, device="cuda")
        kv.rotate(rope, x, pos, out=out[..., 3:67])
        assert (np.abs(_np(out[..., 3:67]) - want) <= bound).all() and not out[..., :3].any() and not out[..., 67:].any()
        y = x.clone()
        assert kv.rotate(rope, y, pos, out=y) is y and (np.abs(_np(y) - want) <= bound).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_inverse_rotation_is_the_gradient(interleaved):
    rope = kv.Rope(64, 48, interleaved=interleaved, scaling="parts", factor=4.0, context=64)
    f, m = ref.frequencies(48, 10000.0, "parts", 4.0, 64)
    pos = torch.tensor([0, 1, 77, 4000], dtype=torch.int32, device="cuda")
    x, g = _randn(4, 4, 2, 64), _randn(5, 4, 2, 64)
    got = _np(kv.rotate(rope, g, pos, inverse=True))
    # by the formula: the transpose of the turning, column by column
    p = pos.cpu().numpy()
    want = np.zeros_like(got)
    for d in range(64):
        unit = np.zeros((4, 2, 64))
        unit[..., d] = 1.0
        want[..., d] = (ref.rotate(unit, p, f, m, interleaved) * _np(g)).sum(-1)
    assert np.abs(got - want).max() <= 4e-7 * 2 * m * float(g.abs().max()) + 2.0 ** -23 * np.abs(want).max()
    # by differences: the map is linear, so a step of 2^-3 is exact up to the two results' rounding
    h = 0.125
    for d in (0, 1, 23, 24, 47, 48, 63):
        up, down = x.clone(), x.clone()
        up[..., d] += h
        down[..., d] -= h
        slope = ((_np(kv.rotate(rope, up, pos)) - _np(kv.rotate(rope, down, pos))) * _np(g)).sum(-1) / (2 * h)
        size = float(x.abs().max() + h) * m
        assert np.abs(slope - got[..., d]).max() <= 64 * float(g.abs().max()) * size * 2.0 ** -22 / h


def test_rotate_nothing():
    rope = kv.Rope(64)
    none = torch.zeros(0, 3, 64, device="cuda")
    assert kv.rotate(rope, none, torch.zeros(0, dtype=torch.int32, device="cuda")).shape == (0, 3, 64)


# ---------------------------------------------------------------------------
# Append and gather
# ---------------------------------------------------------------------------

def _least(most):
    if most == 0:
        return 2.0 ** -100
    e = math.ceil(math.log2(most / 448)) - 1
    while most > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** max(-100, min(100, e))


def _check_append(cache, before, new, lengths, k, v, offs, T):
    """The cache after an append of exact new keys and values (float64, packed) against the formats."""
    table, after = cache.table.cpu().numpy(), ref.host(cache)
    scale = cache.scale[:, 0].double().cpu().numpy()
    for b, (n, L) in enumerate(zip(new, lengths)):
        for which, x in enumerate((k, v)):
            x = x[offs[b]:offs[b] + n][max(0, n - L):]
            first = max(0, L - n)
            old = ref.tokens_of(before[0][which], table[b], first) if first else None
            now = ref.tokens_of(after[which], table[b], L)
            for j in range(first // T, -(-L // T)):
                a, e = max(first, j * T), min(L, j * T + T)
                for h in range(x.shape[1]):
                    most = np.abs(x[a - first:e - first, h]).max()
                    s = scale[table[b, j], which, h]
                    was = before[1][table[b, j], which, h] if j * T < first else 0.0
                    assert s in (max(was, _least(most * (1 - 1e-6))), max(was, _least(most * (1 + 1e-6)))), (b, j, h)
                    near = np.abs(now[a:e, h] - x[a - first:e - first, h])
                    assert (near <= np.maximum(2.0 ** -4 * np.abs(x[a - first:e - first, h]), s * 2.0 ** -10) * 1.0001 + 1e-6 * most).all()
                    if j * T < first:
                        was_x = old[j * T:first, h]
                        # a grown scale moves only what leaves the normal range, by at most half its step
                        assert (np.abs(now[j * T:first, h] - was_x) <= (s * 2.0 ** -10 if s > was else 0.0)).all()


APPENDS = [
    ([1, 1, 1], [1, 16, 40], 16, 2, 64, 1, False, torch.bfloat16), ([5, 33, 1, 64], [5, 40, 17, 100], 16, 3, 128, 2, True, torch.float16),
    ([70, 3], [131, 3], 64, 1, 128, 4, False, torch.bfloat16), ([31, 32, 33], [31, 64, 96], 32, 2, 64, 3, True, torch.float16),
]


@pytest.mark.parametrize("gain", [1e-4, 1.0, 300.0])
@pytest.mark.parametrize("new,lengths,page,heads,dim,group,interleaved,dtype", APPENDS)
def test_append_and_gather(new, lengths, page, heads, dim, group, interleaved, dtype, gain):
    _say(f"append {new} of {lengths} page={page} heads={heads} dim={dim} {dtype} gain={gain}")
    cache = ref.make(kv, lengths, page=page, heads=heads, dim=dim, seed=7)
    T, offs = sum(new), np.concatenate([[0], np.cumsum(new)])
    rope = kv.Rope(dim, interleaved=interleaved, scaling="ntk", factor=2.0)
    k, v, q = (_randn(8 + i, T, n, dim, dtype=dtype, gain=gain) for i, n in enumerate((heads, heads, heads * group)))
    before = ref.host(cache), cache.scale[:, 0].double().cpu().numpy()
    turned = cache.append(0, k, v, ref.offsets(new), rope=rope, q=q)
    f, m = ref.frequencies(dim, 10000.0, "ntk", 2.0)
    pos = np.concatenate([np.arange(L - n, L) for n, L in zip(new, lengths)])
    want_q = ref.rotate(_np(q), pos, f, m, interleaved)
    assert (np.abs(_np(turned) - want_q) <= _rotation_bound(_np(q), want_q, f, m, interleaved, dtype)).all()
    _check_append(cache, before, new, lengths, ref.rotate(_np(k), pos, f, m, interleaved), _np(v), offs, page)
    starts = [max(0, L - n - 3) for n, L in zip(new, lengths)]
    back = [L - a for L, a in zip(lengths, starts)]
    kg, vg = cache.gather(0, torch.tensor(starts, dtype=torch.int32, device="cuda"), ref.offsets(back), sum(back), dtype=dtype)
    kn, vn = ref.host(cache)
    table, at = cache.table.cpu().numpy(), 0
    for b, (a, n) in enumerate(zip(starts, back)):
        for pool, got in ((kn, kg), (vn, vg)):
            want = ref.tokens_of(pool, table[b], lengths[b])[a:]
            assert torch.equal(got[at:at + n].cpu(), torch.from_numpy(want).to(dtype)) or dtype == torch.float16 and \
                (np.abs(_np(got[at:at + n]) - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -25).all()
        at += n
    assert cache.device_status() == 0


def test_append_token_by_token_keeps_old_tokens():
    """Growing values: a block's scale grows again and again, old codes stay within the sum of the halves of the steps."""
    cache = ref.make(kv, [0], pages=4, width=2, heads=1, dim=64, page=16)
    xs, T = [], 16
    for t in range(T):
        cache.resize(torch.tensor([t + 1], dtype=torch.int32, device="cuda"))
        x = _randn(t, 1, 1, 64, dtype=torch.bfloat16, gain=2.0 ** (t - 8))
        xs.append(_np(x)[0])
        cache.append(0, x, -x, ref.offsets([1]))
    k, v = cache.gather(0, torch.zeros(1, dtype=torch.int32, device="cuda"), ref.offsets([T]), T)
    s = cache.scale[int(cache.table[0, 0]), 0, 0, 0].item()
    x = np.stack(xs)
    assert s == _least(np.abs(x).max())
    bound = 2.0 ** -4 * np.abs(x) + 2 * s * 2.0 ** -10      # halves of steps that double: at most twice the last
    assert (np.abs(_np(k) - x) <= bound).all() and (np.abs(_np(v) + x) <= bound).all()
    assert cache.device_status() == 0


def test_append_takes_infinities_nan_and_zeros():
    cache = ref.make(kv, [16, 16], heads=1, dim=64)
    k = _randn(1, 32, 1, 64, dtype=torch.float16)
    k[3, 0, 5], k[4, 0, 6], k[5, 0, 7] = math.inf, -math.inf, math.nan
    k[16:] = 0
    cache.append(0, k, k, ref.offsets([16, 16]))
    for x in cache.gather(0, torch.zeros(2, dtype=torch.int32, device="cuda"), ref.offsets([16, 16]), 32, dtype=torch.float16):
        rest = torch.isfinite(k[:16, 0])
        most = 448 * _least(float(k[:16, 0][rest].abs().max()))
        assert x[3, 0, 5] == most and x[4, 0, 6] == -most and torch.isnan(x[5, 0, 7])
        assert int(torch.isnan(x).sum()) == 1 and not x[16:].any()


def test_append_strided_inputs_subset_of_sequences_and_layers():
    lengths = [20, 0, 35, 64]
    cache = ref.make(kv, lengths, heads=2, dim=64, layers=3, seed=3)
    other = [cache.k.view(torch.uint8)[:, i].clone() for i in (0, 2)]
    both = _randn(5, 9, 2, 2 * 64 + 1, dtype=torch.bfloat16)
    k, v = both[..., 1:65], both[..., 65:]
    seqs = torch.tensor([3, 0], dtype=torch.int32, device="cuda")
    cache.append(1, k, v, ref.offsets([4, 5]), seqs=seqs)
    kg, vg = cache.gather(1, torch.tensor([60, 15], dtype=torch.int32, device="cuda"), ref.offsets([4, 5]), 9, seqs=seqs)
    for x, g in ((k, kg), (v, vg)):
        assert (np.abs(_np(g) - _np(x)) <= 2.0 ** -4 * np.abs(_np(x)) + 2.0 ** -10 * 0.05).all()
    assert all(torch.equal(cache.k.view(torch.uint8)[:, i], o) for i, o in zip((0, 2), other))
    # rows with more new tokens than the sequence holds: the last ones are written, nothing before the start
    cache.append(1, _randn(6, 40, 2, 64, dtype=torch.bfloat16), _randn(7, 40, 2, 64, dtype=torch.bfloat16), ref.offsets([40]),
                 seqs=torch.tensor([0], dtype=torch.int32, device="cuda"))
    got = cache.gather(1, torch.zeros(1, dtype=torch.int32, device="cuda"), ref.offsets([20]), 20, seqs=seqs[1:])[0]
    want = _np(_randn(6, 40, 2, 64, dtype=torch.bfloat16))[20:]
    assert (np.abs(_np(got) - want) <= 2.0 ** -4 * np.abs(want) + 2.0 ** -10 * 0.05).all()
    assert cache.device_status() == 0


@pytest.mark.parametrize("page,dim", [(16, 64), (64, 128)])
def test_gather_past_the_end_and_wrong_starts(page, dim):
    cache = ref.make(kv, [70, 0, 33], heads=3, dim=dim, page=page)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    kp, vp = ref.host(cache)
    table = cache.table.cpu().numpy()
    k, v = cache.gather(0, dev([60, 5, 0]), ref.offsets([200, 3, 40]), 243, dtype=torch.float16)
    assert cache.device_status() == 0
    for pool, got in ((kp, k), (vp, v)):
        want = np.zeros((243, 3, dim))
        want[:10], want[203:236] = ref.tokens_of(pool, table[0], 70)[60:], ref.tokens_of(pool, table[2], 33)
        assert (np.abs(_np(got) - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -25).all()
    good = cache.gather(0, dev([60, 0, 0]), ref.offsets([3, 0, 2]), 5)[0]
    bad = cache.gather(0, dev([60, 0, -1]), ref.offsets([3, 0, 2]), 5)[0]
    assert torch.equal(bad[:3], good[:3]) and cache.device_status() == esp.ESP_ERR_SHAPE
    cache.table[0, 0] = -1
    assert not cache.gather(0, dev([0]), ref.offsets([16]), 16)[0].any() and cache.device_status() == esp.ESP_ERR_SHAPE


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------

def _check_attend(cache, q, new, window=0, scale=None, layer=0, seqs=None, **more):
    D = cache.head_dim
    scale = D ** -0.5 if scale is None else scale
    out, lse = cache.attend(layer, q, ref.offsets(new), window=window, scale=scale, seqs=seqs, **more)
    kp, vp = ref.host(cache, layer)
    table, lengths = cache.table.cpu().numpy(), cache.lengths.cpu().numpy()
    at, qn, on, ln = 0, _np(q), _np(out), _np(lse)
    for b, n in enumerate(new):
        s = b if seqs is None else int(seqs[b])
        L = int(lengths[s])
        k, v = ref.tokens_of(kp, table[s], L), ref.tokens_of(vp, table[s], L)
        want, want_lse, spread, most = ref.attend(qn[at:at + n], k, v, n, window, scale)
        # scores: D products added in float32, one scale and one exponential; weights: fp16, 2^-11 of each,
        # 2^-38 of the largest below its range
        d = D * 2.0 ** -24 * most + 2.0 ** -20 * (1 + most)
        bound = spread * (2.0 ** -11 + 2 * d + 2.0 ** -20) + 2.0 ** -38 * L * (np.abs(v).max() if L else 0) + EPS[q.dtype] * np.abs(want) * 1.01 + TINY[q.dtype]
        assert (np.abs(on[at:at + n] - want) <= bound).all(), (b, n, L, np.abs(on[at:at + n] - want).max())
        none = np.isinf(want_lse)
        assert (np.isneginf(ln[at:at + n]) == none).all() and not on[at:at + n][none].any()
        assert (np.abs(ln[at:at + n] - want_lse)[~none] <= 2 * d + 2.0 ** -20 * (1 + np.abs(want_lse[~none]))).all()
        at += n
    assert cache.device_status() == 0
    return out, lse


ATTENTIONS = [
    # new tokens, lengths, heads, group, dim, page, window, type
    ([1], [1], 1, 1, 64, 16, 0, torch.bfloat16), ([1], [777], 2, 4, 128, 16, 0, torch.bfloat16),
    ([1] * 5, [0, 1, 63, 64, 65], 2, 8, 64, 32, 0, torch.float16), ([1] * 3, [2049, 17, 300], 3, 5, 128, 64, 0, torch.float16),
    ([1, 1], [700, 9], 1, 16, 128, 16, 100, torch.bfloat16), ([1], [500], 1, 40, 64, 16, 1, torch.float16),
    ([3, 4, 2], [3, 400, 1], 2, 4, 64, 16, 0, torch.bfloat16), ([5, 0, 7], [2, 30, 0], 1, 3, 128, 32, 0, torch.float16),
    ([130, 1, 65], [130, 200, 500], 2, 2, 128, 16, 0, torch.bfloat16), ([200], [333], 1, 1, 64, 64, 37, torch.float16),
    ([257, 90], [300, 90], 1, 6, 128, 32, 64, torch.float16), ([64], [1200], 2, 4, 64, 16, 0, torch.bfloat16),
]


@pytest.mark.parametrize("new,lengths,heads,group,dim,page,window,dtype", ATTENTIONS)
def test_attend(new, lengths, heads, group, dim, page, window, dtype):
    _say(f"attend {new} of {lengths} heads={heads}x{group} dim={dim} page={page} window={window} {dtype}")
    cache = ref.make(kv, lengths, page=page, heads=heads, dim=dim, seed=len(lengths))
    q = _randn(11, sum(new), heads * group, dim, dtype=dtype, gain=2.0)
    a = _check_attend(cache, q, new, window)
    b = cache.attend(0, q, ref.offsets(new), window=window, max_new=max(new), max_length=max(lengths))
    for x, y in zip(a, b):                                       # bounds only shape the launch
        assert (np.abs(_np(x) - _np(y))[np.isfinite(_np(x))] <= 4 * EPS[dtype] * (1 + np.abs(_np(x)[np.isfinite(_np(x))]))).all()
    again = cache.attend(0, q, ref.offsets(new), window=window)
    assert torch.equal(a[0], again[0]) and torch.equal(a[1], again[1])


def test_attend_many_ragged_rows():
    g = np.random.default_rng(0)
    lengths = [int(x) for x in np.exp(g.uniform(0, 7, 150))]
    lengths[7] = lengths[149] = 0
    _say(f"attend ragged, 150 rows up to {max(lengths)}")
    cache = ref.make(kv, lengths, heads=2, dim=64)
    _check_attend(cache, _randn(3, 150, 6, 64, dtype=torch.float16), [1] * 150)
    seqs = torch.tensor(g.permutation(150)[:40], dtype=torch.int32, device="cuda")
    _check_attend(cache, _randn(4, 40, 6, 64, dtype=torch.float16), [1] * 40, seqs=seqs)


@pytest.mark.parametrize("n", [1, 40])
def test_attend_extreme_scores_and_scales(n):
    """One token far above the rest, scores of one sign, block scales 2^40 apart, a scale of zero."""
    cache = ref.make(kv, [300], heads=1, dim=64)
    _check_attend(cache, _randn(1, n, 4, 64, dtype=torch.bfloat16, gain=60.0), [n])
    _check_attend(cache, _randn(1, n, 4, 64, dtype=torch.bfloat16), [n], scale=0.0)
    _check_attend(cache, _randn(1, n, 4, 64, dtype=torch.bfloat16), [n], scale=-0.5)
    t = cache.table[0].long()
    cache.scale[t, 0, 1, 0] = torch.exp2(torch.linspace(-20, 20, t.numel(), device="cuda").round())
    _check_attend(cache, _randn(2, n, 4, 64, dtype=torch.bfloat16), [n])
    cache.scale[t, 0, 1, 0] = 2.0 ** -40
    cache.scale[t[3], 0, 1, 0] = 0.0
    cache.scale[t[5], 0, 1, 0] = 3.0e-9                          # not a power of two
    _check_attend(cache, _randn(2, n, 4, 64, dtype=torch.bfloat16), [n])


@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("n,group", [(8, 2), (120, 1), (100, 4)])
def test_nan_reaches_only_the_queries_that_see_it(n, group, window):
    L, at = 200, 200 - n // 2
    clean = ref.make(kv, [L], heads=1, dim=64)
    q = _randn(5, n, group, 64, dtype=torch.float16)
    want, want_lse = _check_attend(clean, q, [n], window)
    for which in ("k", "v"):
        cache = ref.make(kv, [L], heads=1, dim=64)
        page, i = int(cache.table[0, at // 16]), at % 16
        if which == "k":
            cache.k.view(torch.uint8)[page, 0, 0, i, 3] = 0x7f
        else:
            cache.v.view(torch.uint8)[page, 0, 0, 3, i] = 0xff
        out, lse = cache.attend(0, q, ref.offsets([n]), window=window)
        p = torch.arange(L - n, L, device="cuda")
        sees = (p >= at) & ((p - window < at) if window else True)
        _say(f"NaN in {which} at {at}: n={n} window={window}, {int(sees.sum())} rows see it")
        assert 0 < int(sees.sum()) < n
        assert torch.equal(out[~sees], want[~sees]) and torch.equal(lse[~sees], want_lse[~sees])
        if which == "k":
            assert torch.isnan(out[sees]).all() and torch.isnan(lse[sees]).all()
        else:
            assert torch.isnan(out[sees][..., 3]).all() and not torch.isnan(out[sees][..., 4:]).any() and torch.equal(lse, want_lse)


def test_one_workspace_serves_calls_of_any_shape():
    """Calls of few and of many workgroups in turn, single tokens and prompts: what one leaves in the workspace is
    nothing to the next."""
    g = np.random.default_rng(3)
    lengths = [5000, 9, 3000, 777] + [int(x) for x in g.integers(1, 400, 60)]
    cache = ref.make(kv, lengths, heads=2, dim=64, seed=9)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    shapes = [([0], [1]), (list(range(64)), [1] * 64), ([2], [300]), ([0, 2], [1, 1]), ([0, 1, 2, 3], [40, 9, 200, 64]), (list(range(40)), [2] * 40), ([1], [1])]
    for seqs, new in shapes * 2:
        _say(f"workspace: rows {len(seqs)}, new {max(new)}")
        q = _randn(len(seqs), sum(new), 8, 64, dtype=torch.float16)
        got = cache.attend(0, q, ref.offsets(new), seqs=dev(seqs))
        alone = kv.PagedCache.adopt(cache.k, cache.v, cache.scale, cache.table, cache.lengths, cache.refs)
        want = alone.attend(0, q, ref.offsets(new), seqs=dev(seqs))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_attend_strides():
    cache = ref.make(kv, [90, 40], heads=2, dim=128)
    wide = _randn(1, 6, 9, 131, dtype=torch.bfloat16)
    for q in (wide[:, 1:9, 3:], wide.transpose(0, 1).contiguous().transpose(0, 1)[:, :8, :128]):
        want = cache.attend(0, q.contiguous(), ref.offsets([2, 4]))
        got = cache.attend(0, q, ref.offsets([2, 4]))
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
        out = torch.zeros(6, 9, 133, dtype=torch.bfloat16, device="cuda")
        cache.attend(0, q, ref.offsets([2, 4]), out=out[:, 1:, 5:], lse=False)
        assert torch.equal(out[:, 1:, 5:], want[0]) and not out[:, 0].any() and not out[..., :5].any()


def test_attend_finds_wrong_rows_and_pages():
    cache = ref.make(kv, [100, 100, 100], heads=1, dim=64)
    q = _randn(1, 3, 2, 64, dtype=torch.float16)
    want = cache.attend(0, q, ref.offsets([1, 1, 1]))[0]
    cache.table[1, 2] = -1                                       # a hole: its tokens are left out
    cache.table[2, 2] = 9999
    got = cache.attend(0, q, ref.offsets([1, 1, 1]))[0]
    assert torch.equal(got[0], want[0]) and torch.isfinite(got).all()
    assert cache.device_status() == esp.ESP_ERR_SHAPE and cache.device_status() == 0
    cache.attend(0, q, ref.offsets([1, 1, 1]), max_length=50)
    assert cache.device_status() == esp.ESP_ERR_SHAPE
    for off in ([0, 2, 1, 3], [0, 1, 2, 9], [-1, 1, 2, 3]):
        cache.attend(0, q, torch.tensor(off, dtype=torch.int32, device="cuda"))
        assert cache.device_status() == esp.ESP_ERR_SHAPE
    cache.lengths[0] = 10000
    cache.attend(0, q, ref.offsets([1, 1, 1]))
    cache.append(0, q[:, :1], q[:, 1:], ref.offsets([1, 1, 1]))
    assert cache.device_status() == esp.ESP_ERR_SHAPE
    cache.lengths[0] = 100
    assert torch.equal(cache.attend(0, q, ref.offsets([1, 1, 1]))[0][0], want[0])


def test_far_pages_of_a_large_pool():
    """Offsets beyond 32 bits: keys and values of 5 GB each, the sequence at their end."""
    pages = 5 * (1 << 30) // (16 * 8 * 128)
    _say(f"large pool: {pages} pages")
    small = ref.make(kv, [50], heads=8, dim=128)
    big = kv.PagedCache(pages, 16, 8, 128, 1, 4)
    t = small.table[0].long()
    place = torch.tensor([pages - 1, 5, pages - 3, pages // 2 + 1], device="cuda")
    for name in ("k", "v"):
        getattr(big, name).view(torch.uint8)[place] = getattr(small, name).view(torch.uint8)[t]
    big.scale[place] = small.scale[t]
    big.table[0], big.lengths[0], big.refs[place] = place.int(), 50, 1
    q, k = _randn(1, 1, 16, 128, dtype=torch.bfloat16), _randn(2, 1, 8, 128, dtype=torch.bfloat16)
    for a, b in zip(big.attend(0, q, ref.offsets([1])), small.attend(0, q, ref.offsets([1]))):
        assert torch.equal(a, b)
    one = torch.tensor([49], dtype=torch.int32, device="cuda")
    got = []
    for c in (big, small):
        c.append(0, k, k, ref.offsets([1]))
        got.append(c.gather(0, one, ref.offsets([1]), 1))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    table, refs, live = big.compact()
    assert int(live) == 4 and sorted(table[0].tolist()) == [0, 1, 2, 3]
    big.install(table, refs)
    assert torch.equal(big.attend(0, q, ref.offsets([1]))[0], small.attend(0, q, ref.offsets([1]))[0])
    assert big.device_status() == 0


# ---------------------------------------------------------------------------
# Page operations
# ---------------------------------------------------------------------------

def _same(cache, pages, first):
    """Table, lengths, references and every owned page's contents."""
    assert np.array_equal(cache.table.cpu().numpy(), pages.table) and np.array_equal(cache.refs.cpu().numpy(), pages.refs)
    assert np.array_equal(cache.lengths.cpu().numpy(), pages.lengths)
    live = np.nonzero(pages.refs > 0)[0]
    assert np.array_equal(pages.refs, np.bincount(pages.table[pages.table >= 0], minlength=len(pages.refs)))
    for t, f in zip((cache.k, cache.v, cache.scale), first):
        t = t.view(torch.uint8) if t.dtype != torch.float32 else t.view(torch.int32)
        assert torch.equal(t[torch.from_numpy(live).cuda()], f[torch.from_numpy(pages.names[live]).cuda()])


@pytest.mark.parametrize("page,heads,dim,layers,sequences,width", [(16, 1, 64, 1, 5, 6), (32, 3, 128, 2, 40, 9), (64, 2, 64, 3, 300, 30)])
def test_page_operations_in_a_row(page, heads, dim, layers, sequences, width):
    _say(f"pages of {page}, {sequences} sequences of at most {width} pages")
    g = np.random.default_rng(sequences)
    lengths = [int(g.integers(0, width * page + 1)) if g.random() < 0.5 else 0 for _ in range(sequences)]
    cache = ref.make(kv, lengths, page=page, heads=heads, dim=dim, layers=layers, width=width, pages=int(sequences * width * 0.7) + 3)
    pages = ref.Pages(cache)
    first = [t.view(torch.uint8).clone() for t in (cache.k, cache.v)] + [cache.scale.view(torch.int32).clone()]
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    refused = 0
    for step in range(12):
        kind = step % 3
        if kind == 0:
            order = g.permutation(sequences)
            n = int(g.integers(1, max(2, sequences // 2)))
            parents = [int(x) for x in g.choice(order[n:], n)]
            children = [int(x) for x in order[:n]]
            ok = pages.fork(parents, children)
            cache.fork(dev(parents), dev(children))
        elif kind == 1:
            want = [int(min(width * page, max(0, x + g.integers(-3 * page, 2 * page)))) if g.random() < 0.6 else int(x) for x in pages.lengths]
            if step == 4:
                want = [width * page] * sequences
            ok = pages.resize(want)
            cache.resize(dev(want))
        else:
            limit = None if step % 2 else int(len(pages.refs) * 0.9)
            ok = pages.compact(limit)
            table, refs, live = cache.compact(limit)
            assert int(live) == int((pages.refs > 0).sum())
            cache.install(table, refs)
        refused += not ok
        assert cache.device_status() == (0 if ok else esp.ESP_ERR_RANGE), step
        _same(cache, pages, first)
    assert refused >= 1


def test_a_compaction_leaves_the_old_places_readable():
    cache = ref.make(kv, [100, 30, 77, 5], heads=2, dim=64, pages=60)
    q = _randn(1, 4, 4, 64, dtype=torch.bfloat16)
    want = cache.attend(0, q, ref.offsets([1] * 4))[0]
    table, refs, live = cache.compact()
    assert torch.equal(cache.attend(0, q, ref.offsets([1] * 4))[0], want)
    assert int(table.max()) == int(live) - 1 and int((refs[int(live):] != 0).sum()) == 0
    cache.install(table, refs)
    assert torch.equal(cache.attend(0, q, ref.offsets([1] * 4))[0], want)
    table, refs, _ = cache.compact(limit=int(live) - 1)          # a budget below what lives: refused, nothing moves
    assert cache.device_status() == esp.ESP_ERR_RANGE
    assert torch.equal(table, cache.table) and torch.equal(refs, cache.refs)
    assert torch.equal(cache.attend(0, q, ref.offsets([1] * 4))[0], want)


def test_a_compaction_in_place():
    cache = ref.make(kv, [100, 30, 77, 5], heads=2, dim=64, pages=60)
    q = _randn(1, 4, 4, 64, dtype=torch.bfloat16)
    want = cache.attend(0, q, ref.offsets([1] * 4))[0]
    table, refs, live = cache.compact()
    work = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    assert kv.lib().esp_kv_compact(cache.ptr, -1, cache.table.data_ptr(), cache.refs.data_ptr(), None, work.data_ptr(), work.numel(),
                                   torch.cuda.current_stream().cuda_stream) == esp.ESP_OK
    assert torch.equal(cache.table, table) and torch.equal(cache.refs, refs)
    assert torch.equal(cache.attend(0, q, ref.offsets([1] * 4))[0], want)


def test_forks_share_full_pages_and_write_apart():
    cache = ref.make(kv, [40, 0, 0], heads=1, dim=64, pages=12, width=4)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache.fork(dev([0, 0]), dev([1, 2]))
    assert cache.refs[cache.table[0, :2].long()].tolist() == [3, 3] and len(set(cache.table[:, 2].tolist())) == 3
    cache.resize(dev([41, 41, 41]))
    k = _randn(1, 3, 1, 64, dtype=torch.bfloat16)
    cache.append(0, k, k, ref.offsets([1, 1, 1]))
    got = cache.gather(0, dev([40, 40, 40]), ref.offsets([1, 1, 1]), 3)[0]
    assert (np.abs(_np(got) - _np(k)) <= 2.0 ** -4 * np.abs(_np(k)) + 2.0 ** -9).all()
    a, b, c = (cache.gather(0, dev([0]), ref.offsets([40]), 40, seqs=dev([s]))[0] for s in range(3))
    assert torch.equal(a[:32], b[:32]) and torch.equal(a[:32], c[:32])
    cache.resize(dev([41, 20, 0]))                               # into a shared page: it is copied first
    assert int(cache.table[1, 1]) != int(cache.table[0, 1]) and cache.refs[cache.table[0, 1]].item() == 1
    _check_attend(cache, _randn(2, 2, 2, 64, dtype=torch.bfloat16), [1, 1])
    assert cache.device_status() == 0


def test_bad_page_operations_change_nothing():
    cache = ref.make(kv, [40, 10, 0], heads=1, dim=64, pages=12, width=4)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    state = [t.clone() for t in (cache.table, cache.lengths, cache.refs)]

    def unchanged(code):
        assert cache.device_status() == code
        assert all(torch.equal(a, b) for a, b in zip(state, (cache.table, cache.lengths, cache.refs)))
    for lengths in ([65, 0, 0], [-1, 0, 0]):
        cache.resize(dev(lengths))
        unchanged(esp.ESP_ERR_SHAPE)
    for parents, children in (([0], [0]), ([0, 0], [1, 1]), ([0, 1], [1, 2]), ([3], [1]), ([0], [-1])):
        cache.fork(dev(parents), dev(children))
        unchanged(esp.ESP_ERR_INVALID_ARG)
    cache.table[1, 0], state[0][1, 0] = 12, 12
    cache.resize(dev([1, 1, 1]))
    unchanged(esp.ESP_ERR_SHAPE)
    cache.fork(dev([1]), dev([2]))
    unchanged(esp.ESP_ERR_SHAPE)


# ---------------------------------------------------------------------------
# Streams, graphs, refusals
# ---------------------------------------------------------------------------

def _step(cache, rope, lengths, k, v, q, offs, stream=None):
    cache.resize(lengths, stream=stream)
    turned = cache.append(0, k, v, offs, rope=rope, q=q, stream=stream)
    return cache.attend(0, turned, offs, stream=stream)


def test_side_streams():
    """Two caches on two streams at once, many steps each, against the same steps on the default stream."""
    def inputs(seed):
        cache = ref.make(kv, [200, 31, 64], heads=2, dim=64, pages=60, width=20, seed=seed)
        steps = []
        for i in range(6):
            steps.append((torch.tensor([201 + i, 32 + i, 65 + i], dtype=torch.int32, device="cuda"),
                          *(_randn(seed * 100 + i * 3 + j, 3, n, 64, dtype=torch.float16) for j, n in enumerate((2, 2, 8)))))
        return cache, steps
    rope, offs = kv.Rope(64), ref.offsets([1, 1, 1])
    want = []
    for seed in (1, 2):
        cache, steps = inputs(seed)
        want.append([_step(cache, rope, *x, offs) for x in steps])
    torch.cuda.synchronize()
    both = [(*inputs(seed), torch.cuda.Stream()) for seed in (1, 2)]
    torch.cuda.synchronize()
    got = [[], []]
    for i in range(6):
        for g, (cache, steps, stream) in zip(got, both):
            g.append(_step(cache, rope, *steps[i], offs, stream=stream))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(a, b) for x, y in zip(w, g) for a, b in zip(x, y))


def test_a_step_in_a_graph():
    rope, offs = kv.Rope(64), ref.offsets([1, 1])
    caches = [ref.make(kv, [900, 47], heads=2, dim=64, pages=90, width=70, seed=4) for _ in range(2)]
    lengths = torch.tensor([900, 47], dtype=torch.int32, device="cuda")
    k, v, q = (torch.zeros(2, n, 64, dtype=torch.bfloat16, device="cuda") for n in (2, 2, 8))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                               # the workspaces of this stream, outside the graph
        caches[0].attend(0, q, offs)
        caches[0].resize(lengths)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = _step(caches[0], rope, lengths, k, v, q, offs)
    for i in range(4):
        lengths += 1
        for j, t in enumerate((k, v, q)):
            t.copy_(_randn(i * 3 + j, *t.shape, dtype=torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        want = _step(caches[1], rope, lengths, k, v, q, offs)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert torch.equal(caches[0].table, caches[1].table)
    assert caches[0].device_status() == 0


def test_graphs_without_a_warm_up():
    """Graphs captured before their stream has scratch, replayed in another order than captured, with larger eager calls
    on the stream between."""
    offs = {n: ref.offsets([1] * n) for n in (1, 3)}
    cache = ref.make(kv, [4000, 47, 900], heads=2, dim=64, seed=6)
    q = {n: torch.zeros(n, 8, 64, dtype=torch.float16, device="cuda") for n in (1, 3)}
    side, plain = torch.cuda.Stream(), kv.PagedCache.adopt(cache.k, cache.v, cache.scale, cache.table, cache.lengths, cache.refs)
    torch.cuda.synchronize()
    graphs, out = {}, {}
    for n in (3, 1):
        graphs[n] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[n], stream=side):
            out[n] = [cache.attend(0, q[n], offs[n]) for _ in range(2)]
    for i, n in enumerate((1, 3, 1, 1, 3)):
        _say(f"graph of {n} rows, replay {i}")
        q[n].copy_(_randn(i, n, 8, 64, dtype=torch.float16))
        graphs[n].replay()
        torch.cuda.synchronize()
        want = plain.attend(0, q[n], offs[n])
        for got in out[n]:
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        many = _randn(90 + i, 300 * (i + 1), 8, 64, dtype=torch.float16)
        torch.cuda.synchronize()
        got, want = (c.attend(0, many, ref.offsets([300 * (i + 1)]), stream=s) for c, s in ((cache, side), (plain, None)))
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_graph_keeps_its_scratch_when_the_cache_takes_more():
    cache = ref.make(kv, [4000, 47], heads=2, dim=64, seed=7)
    plain = kv.PagedCache.adopt(cache.k, cache.v, cache.scale, cache.table, cache.lengths, cache.refs)
    offs, side = ref.offsets([1, 1]), torch.cuda.Stream()
    q = _randn(1, 2, 8, 64, dtype=torch.float16)
    want = plain.attend(0, q, offs)
    torch.cuda.synchronize()
    cache.attend(0, q, offs, stream=side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = cache.attend(0, q, offs)
    for i in range(3):
        many = torch.zeros(700 * (i + 1), 8, 64, dtype=torch.float16, device="cuda")
        torch.cuda.synchronize()
        cache.attend(0, many, ref.offsets([700 * (i + 1), 0]), stream=side)
        with torch.cuda.stream(side):                            # what scratch given back would hold
            junk = [torch.full((1 << n,), 255, dtype=torch.uint8, device="cuda") for n in range(12, 24)]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and all(bool((x == 255).all()) for x in junk)


def test_the_binding_refuses_what_does_not_fit():
    cache = ref.make(kv, [20, 20], heads=2, dim=64)
    rope, offs = kv.Rope(64), ref.offsets([1, 1])
    k, q = _randn(1, 2, 2, 64, dtype=torch.bfloat16), _randn(1, 2, 4, 64, dtype=torch.bfloat16)
    for call in (lambda: cache.append(0, k, k.half(), offs), lambda: cache.append(0, k, k[:1], offs), lambda: cache.append(0, k[..., :32], k, offs),
                 lambda: cache.append(0, k, k, offs.long()), lambda: cache.append(0, k, k, offs, q=q), lambda: cache.append(0, k, k, offs, rope=kv.Rope(128)),
                 lambda: cache.append(0, k.float(), k.float(), offs), lambda: cache.attend(0, q.float(), offs), lambda: cache.attend(0, q, offs.cpu()),
                 lambda: cache.attend(0, q.transpose(1, 2).contiguous().transpose(1, 2), offs), lambda: cache.attend(0, q, offs, out=q.half()),
                 lambda: cache.resize(offs), lambda: cache.fork(offs[:1], offs[:2]), lambda: cache.install(cache.refs, cache.table),
                 lambda: kv.rotate(rope, k.cpu(), offs[:2]), lambda: kv.rotate(rope, k, offs[:1]), lambda: kv.rotate(kv.Rope(128), k, offs[:2]), lambda: kv.rotate(rope, k.double(), offs[:2]),
                 lambda: kv.Rope(64, 128), lambda: kv.Rope(64, scaling="other"), lambda: kv.PagedCache.adopt(cache.v, cache.v, cache.scale, cache.table, cache.lengths, cache.refs)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: cache.attend(1, q, offs), lambda: cache.attend(0, q[:, :3], offs), lambda: cache.attend(0, q, offs, window=-1),
                 lambda: cache.attend(0, q, offs, scale=math.inf), lambda: cache.append(2, k, k, offs), lambda: kv.Rope(64, 7), lambda: kv.Rope(64, base=0.5)):
        with pytest.raises(esp.EspError):
            call()
    assert cache.device_status() == 0
