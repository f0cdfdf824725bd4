"""GPU: the attention weight that cached tokens get, against the plain 64-bit form.

A score's product over a head of D elements: D sums of float32, each off by at most 2 u of the sum of |q k| (u = 2^-24;
products of 16-bit numbers are exact); scale, difference to lse, log2 e and the exponential: 4 u of the score and of
lse, 4 u of the weight.  A token's n G weights are added up one after another.
"""
import numpy as np
import pytest
import torch

import _kv_forms as forms
import _kv_ref as ref
import paper_2608_07971_amd as esp
from paper_2608_07971_amd import kv

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _say(msg):
    print(f"[gpu-case] {msg}", flush=True)


def _randn(seed, *shape, dtype=torch.bfloat16, gain=1.4):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * gain).to(dtype).cuda()


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _np(t):
    return t.double().cpu().numpy()


def _mass(cache, seed=9):
    return torch.rand(cache.mass_shape, generator=torch.Generator().manual_seed(seed)).cuda()


def _check(cache, q, new, window=0, scale=None, decay=1.0, layer=0, seqs=None, lse=None, mass=None, **more):
    offs, T = ref.offsets(new), cache.page_tokens
    if lse is None:
        lse = cache.attend(layer, q, offs, window=window, scale=scale, seqs=None if seqs is None else _dev(seqs))[1]
    mass = _mass(cache) if mass is None else mass
    before = _np(mass)
    cache.weigh(layer, q, lse, offs, mass, window=window, scale=scale, decay=decay, seqs=None if seqs is None else _dev(seqs), **more)
    assert cache.device_status() == 0
    got, pool = _np(mass), ref.host(cache, layer)[0]
    table, lengths, q64, l64 = cache.table.cpu().numpy(), cache.lengths.cpu().numpy(), _np(q), _np(lse)
    want, bound, at = before.copy(), np.zeros_like(before), 0
    G, D = q.shape[1] // cache.kv_heads, cache.head_dim
    for b, n in enumerate(new):
        s = b if seqs is None else seqs[b]
        L = int(lengths[s])
        if n and L:
            k = ref.tokens_of(pool, table[s], L)
            w, most, top = forms.weigh(q64[at:at + n], l64[at:at + n], k, n, window, D ** -0.5 if scale is None else scale, G)
            p0 = max(0, L - n)
            old = want[layer, s, :, :p0] * float(np.float32(decay))
            want[layer, s, :, :p0] = old + w[:, :p0]
            want[layer, s, :, p0:L] = w[:, p0:]
            bound[layer, s, :, :L] = w * (2 * D * most + 4 * 2 * top + 4 + n * G) * U + 2 * U * np.abs(want[layer, s, :, :L])
        at += n
    same = bound == 0.0
    assert np.array_equal(got[same & (want == before)], before[same & (want == before)])
    assert (np.abs(got - want) <= bound * 1.01 + 1e-37).all()
    return mass


CASES = [
    ([1], [1], 1, 1, 64, 16, 0, torch.bfloat16), ([1, 1, 1], [100, 1, 0], 2, 4, 128, 16, 0, torch.bfloat16), ([1] * 9, [64, 65, 63, 128, 1000, 0, 17, 129, 2], 3, 5, 64, 32, 0, torch.float16),
    ([2, 0, 5, 3], [300, 200, 5, 2], 2, 8, 128, 64, 0, torch.bfloat16), ([1, 1], [700, 90], 1, 8, 128, 16, 50, torch.float16),
    ([40, 7, 0, 130], [400, 7, 30, 131], 2, 4, 64, 16, 0, torch.bfloat16), ([300], [900], 1, 3, 128, 32, 100, torch.bfloat16), ([33, 64], [33, 700], 2, 1, 128, 64, 1, torch.float16),
    ([3, 200], [2, 150], 2, 2, 64, 16, 0, torch.float16), ([6], [5000], 2, 6, 64, 64, 3000, torch.bfloat16), ([1, 1], [257, 258], 16, 1, 64, 16, 0, torch.bfloat16),
    ([65], [130], 4, 16, 64, 16, 0, torch.bfloat16), ([12] + [0] * 11, [300] * 12, 1, 16, 64, 16, 0, torch.float16),
    ([0] * 5 + [9, 1], [40] * 5 + [200, 70], 2, 12, 128, 32, 120, torch.bfloat16),
]


@pytest.mark.parametrize("decay", [1.0, 0.9])
@pytest.mark.parametrize("new,lengths,heads,group,dim,page,window,dtype", CASES)
def test_weigh(new, lengths, heads, group, dim, page, window, dtype, decay):
    _say(f"weigh {new} of {lengths}, {heads} x {group} x {dim}, pages of {page}, window {window}, {dtype}, decay {decay}")
    cache = ref.make(kv, lengths, page=page, heads=heads, dim=dim)
    q = _randn(1, sum(new), heads * group, dim, dtype=dtype)
    first = _check(cache, q, new, window, decay=decay)
    again = _check(cache, q, new, window, decay=decay, max_new=max(new), max_length=max(lengths))
    assert torch.equal(first, again)                              # bounds change how, not what


@pytest.mark.parametrize("heads,group,dtype", [(2, 4, torch.bfloat16), (1, 16, torch.float16)])
def test_rows_of_every_kind_among_empty_ones(heads, group, dtype):
    new = [0] * 140
    new[3], new[4], new[40], new[77], new[139] = 1, 40, 5, 70, 8
    g = np.random.default_rng(group)
    lengths = [int(n + g.integers(0, 300)) for n in new]
    cache = ref.make(kv, lengths, heads=heads, dim=64)
    q, found = _randn(11, sum(new), heads * group, 64, dtype=dtype), []
    for more in ({}, dict(max_new=70), dict(max_new=1000), dict(max_new=70, window=60)):
        _say(f"weigh rows of every kind among empty ones, {heads} x {group}, {more}")
        found.append(_check(cache, q, new, decay=0.5, **more))
    assert torch.equal(found[0], found[1]) and torch.equal(found[0], found[2])
    before = _mass(cache)
    assert all(torch.equal(found[0][:, b], before[:, b]) for b in range(140) if new[b] == 0)


@pytest.mark.parametrize("new,lengths,heads,group,dim,page,window,dtype", [
    # shares of several tiles that go on in the next row: rounds of 16 rows, of 32, and many queries (beside few of them, and alone)
    ([1] * 7, [2000, 130, 1, 0, 3001, 900, 2500], 32, 2, 64, 16, 0, torch.bfloat16), ([3, 2, 1, 3], [2222, 64, 1999, 3100], 32, 8, 64, 64, 1500, torch.float16),
    ([20, 0, 17] + [0] * 60, [3100, 40, 2900] + [5] * 60, 32, 8, 64, 32, 0, torch.bfloat16), ([3, 130], [900, 9000], 256, 1, 64, 16, 400, torch.bfloat16),
])
def test_shares_of_several_tiles(new, lengths, heads, group, dim, page, window, dtype):
    _say(f"weigh {new[:4]} of {lengths[:4]}, {heads} x {group} x {dim}, window {window}")
    cache = ref.make(kv, lengths, heads=heads, dim=dim, page=page)
    _check(cache, _randn(13, sum(new), heads * group, dim, dtype=dtype), new, window, decay=0.5, max_new=max(new), max_length=max(lengths))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("page", [16, 64])
def test_many_queries_of_any_strides(dtype, page):
    cache = ref.make(kv, [500, 190], heads=2, dim=128, page=page)
    wide = _randn(14, 110, 9, 136, dtype=dtype)
    for q in (wide[:, 1:7, :128], wide[:, 1:7, 3:131], wide[:, :6, 8:], wide.transpose(0, 1).contiguous().transpose(0, 1)[:, 2:8, 1:129], wide[:, :1, :128].expand(110, 6, 128)):
        _say(f"weigh 60 + 50 queries of strides {q.stride()}, pages of {page}, {dtype}")
        _check(cache, q, [60, 50], decay=0.5)
        _check(cache, q, [50, 60], window=70)


def test_one_long_row_among_empty_ones_takes_what_it_takes():
    """Its own kernel's time, not that of the rounds of single tokens (which is eight times as long)."""
    H, G, n, length = 8, 4, 512, 4096
    q, lse, times = _randn(12, n, H * G, 128), torch.full((n, H * G), 9.0, device="cuda"), []
    for rows in (2, 512):
        cache = ref.make(kv, [length] + [0] * (rows - 1), heads=H, dim=128)
        offs, mass = ref.offsets([n] + [0] * (rows - 1)), torch.zeros(cache.mass_shape, device="cuda")
        best = []
        for _ in range(12):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            cache.weigh(0, q, lse, offs, mass, max_new=n)
            b.record()
            torch.cuda.synchronize()
            best.append(a.elapsed_time(b))
        times.append(min(best))
    assert times[1] < 4 * times[0]


def test_weights_add_up_to_one_a_query():
    cache = ref.make(kv, [500, 77], heads=2, dim=128)
    q, offs, mass = _randn(2, 5, 8, 128), ref.offsets([4, 1]), torch.zeros(1, 2, 2, cache.table_width * 16, device="cuda")
    _, lse = cache.attend(0, q, offs)
    for _ in range(3):
        cache.weigh(0, q, lse, offs, mass)
    # three calls: the row's new tokens begin at 0 each time, the others have three times theirs
    mass[:, 0, :, :496] /= 3
    mass[:, 1, :, :76] /= 3
    total = mass.double().sum(-1)[0]
    # attend's lse and these weights: each within a few hundred u of scores of about 10
    assert (total - torch.tensor([[16.0, 16.0], [4.0, 4.0]], device="cuda")).abs().max() <= 16 * 4096 * U


def test_layers_sequences_strides_and_scales():
    cache = ref.make(kv, [90, 200, 0, 33], heads=2, dim=64, layers=3, width=20, seed=3)
    wide = _randn(3, 3, 9, 72, dtype=torch.float16)
    for q in (wide[:, 1:, 4:68], wide[:, :8, :64], wide.transpose(0, 1).contiguous().transpose(0, 1)[:, :2, 8:]):
        _check(cache, q, [2, 1], layer=2, seqs=[3, 1])
        _check(cache, q, [1, 2], layer=1, seqs=[0, 3], scale=-0.3, decay=0.0)
    _check(cache, wide[:1, :1, :64].expand(3, 4, 64), [3], layer=0, seqs=[1])


def test_many_ragged_rows():
    g = np.random.default_rng(5)
    lengths = [int(x) for x in g.integers(0, 400, 700)]
    cache = ref.make(kv, lengths, heads=1, dim=64)
    _check(cache, _randn(4, 700, 2, 64), [1] * 700)


def test_queries_that_see_nothing_and_infinities():
    cache = ref.make(kv, [100, 60], heads=1, dim=64)
    q, offs = _randn(5, 4, 2, 64), ref.offsets([3, 1])
    _, lse = cache.attend(0, q, offs)
    lse[0], lse[1, 1], lse[3] = -float("inf"), float("inf"), -float("inf")
    _check(cache, q, [3, 1], lse=lse)
    lse[2, 0] = float("nan")                                      # reaches what that query sees
    mass = _mass(cache)
    before = mass.clone()
    cache.weigh(0, q, lse, offs, mass)
    assert bool(mass[0, 0, 0, :100].isnan().all()) and torch.equal(mass[0, 1, 0, 59:], torch.cat((torch.zeros(1, device="cuda"), before[0, 1, 0, 60:])))
    # a key of NaN: its own weight only
    cache.k.view(torch.uint8)[cache.table[1, 1].long(), 0, 0, 3, 5] = 0x7f
    lse = torch.zeros(4, 2, device="cuda")
    mass = _mass(cache)
    cache.weigh(0, q, lse, offs, mass)
    assert mass[0, 1, 0].isnan().nonzero().flatten().tolist() == [19]
    mass = torch.full_like(mass, float("inf"))
    cache.weigh(0, q, torch.full((4, 2), float("inf"), device="cuda"), offs, mass, decay=0.5)
    assert bool(mass[0, 0, 0, :97].isinf().all()) and not mass[0, 0, 0, 97:100].any()


@pytest.mark.parametrize("new,lengths,group,page,window", [([1, 3], [500, 3], 4, 16, 0), ([20, 9], [800, 200], 2, 32, 150), ([300], [900], 3, 16, 0),
                                                           ([150, 200], [1100, 200], 2, 64, 400)])
def test_padded_queries_hold_anything(new, lengths, group, page, window):
    """A query whose lse is -inf adds nothing, whatever it holds itself."""
    _say(f"weigh with padded queries {new} of {lengths}, group {group}, window {window}")
    cache = ref.make(kv, lengths, heads=2, dim=64, page=page)
    q = _randn(8, sum(new), 2 * group, 64)
    _, lse = cache.attend(0, q, ref.offsets(new), window=window)
    for i, x in ((0, float("nan")), (sum(new) // 2, float("inf")), (sum(new) - 1, -float("inf"))):
        q[i, 1::2], lse[i, 1::2] = x, -float("inf")
    q[-1, 0, 5], lse[-1, 0] = float("nan"), -float("inf")
    _check(cache, q, new, window, lse=lse, decay=0.5)
    lse.fill_(-float("inf"))
    _check(cache, torch.full_like(q, float("nan")), new, window, lse=lse, decay=0.5)


def test_wrong_rows_and_pages_are_left_out():
    cache = ref.make(kv, [100, 60, 20], heads=1, dim=64, width=8)
    q, lse = _randn(6, 3, 2, 64), torch.zeros(3, 2, device="cuda")
    good = _mass(cache)
    cache.weigh(0, q, lse, ref.offsets([1, 1, 1]), good)
    assert cache.device_status() == 0
    start = _mass(cache)
    for offs, seqs, more in ((_dev([0, 1, 2, 9]), None, {}), (ref.offsets([1, 1, 1]), _dev([0, 1, 3]), {}), (ref.offsets([1, 1, 1]), _dev([0, 1, -1]), {}),
                             (_dev([0, 1, 2, 1]), None, {})):
        mass = _mass(cache)
        cache.weigh(0, q, lse, offs, mass, seqs=seqs, **more)
        assert cache.device_status() == esp.ESP_ERR_SHAPE
        assert torch.equal(mass[0, :2], good[0, :2]) and torch.equal(mass[0, 2], start[0, 2])
    for more, left in ((dict(max_length=60), [0]), (dict(max_length=10), [0, 1, 2])):
        mass = _mass(cache)
        cache.weigh(0, q, lse, ref.offsets([1, 1, 1]), mass, **more)
        assert cache.device_status() == esp.ESP_ERR_SHAPE
        assert all(torch.equal(mass[0, s], (start if s in left else good)[0, s]) for s in range(3))
    mass, two = _mass(cache), _randn(7, 3, 2, 64)
    cache.weigh(0, two, lse, ref.offsets([1, 2, 0]), mass, max_new=1)
    assert cache.device_status() == esp.ESP_ERR_SHAPE and torch.equal(mass[0, 1:], start[0, 1:])
    for page in (-1, cache.pages, 2 ** 31 - 1):                   # tokens without a page keep what they had
        mass, old = _mass(cache), cache.table[0, 2].clone()
        cache.table[0, 2] = page
        cache.weigh(0, q, lse, ref.offsets([1, 1, 1]), mass)
        cache.table[0, 2] = old
        assert cache.device_status() == esp.ESP_ERR_SHAPE
        assert torch.equal(mass[..., 32:48], torch.cat((start[:, :1, :, 32:48], good[:, 1:, :, 32:48]), 1)) and torch.equal(mass[..., :32], good[..., :32])
        assert torch.equal(mass[..., 48:], good[..., 48:])


def test_weigh_in_a_graph_and_on_another_stream():
    cache, side = ref.make(kv, [300, 41], heads=2, dim=64), torch.cuda.Stream()
    q, offs = torch.zeros(2, 4, 64, dtype=torch.float16, device="cuda"), ref.offsets([1, 1])
    mass = torch.zeros(cache.mass_shape, device="cuda")
    other = mass.clone()

    def step(mass, **more):
        out, lse = cache.attend(0, q, offs, **more)
        cache.weigh(0, q, lse, offs, mass, decay=0.5, **more)
    step(torch.zeros_like(mass))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(mass)
    for i in range(5):
        _say(f"replay {i}")
        q.copy_(_randn(i, 2, 4, 64))
        torch.cuda.synchronize()
        graph.replay()
        step(other, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(mass, other)
    assert cache.device_status() == 0


def test_what_does_not_fit_is_refused():
    cache = ref.make(kv, [20, 20], heads=2, dim=64)
    q, offs, mass = _randn(1, 2, 4, 64), ref.offsets([1, 1]), torch.zeros(cache.mass_shape, device="cuda")
    lse = torch.zeros(2, 4, device="cuda")
    call = lambda layer=0, q=q, lse=lse, offs=offs, mass=mass, **more: cache.weigh(layer, q, lse, offs, mass, **more)  # noqa: E731
    for bad in (dict(q=q.float()), dict(q=q[0]), dict(q=q[..., :32]), dict(lse=lse[:1]), dict(lse=lse.double()), dict(lse=lse.cpu()), dict(lse=lse.t().contiguous().t()),
                dict(mass=mass[0]), dict(mass=mass.double()), dict(mass=mass.cpu()), dict(mass=mass.transpose(1, 2)), dict(mass=mass.clone().requires_grad_()),
                dict(offs=offs.long()), dict(seqs=offs)):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(layer=1), dict(layer=-1), dict(q=q[:, :3], lse=lse[:, :3].contiguous()), dict(window=-1), dict(scale=float("inf")), dict(decay=float("nan")),
                dict(max_new=-1), dict(max_length=-1)):
        with pytest.raises(esp.EspError):
            call(**bad)
    assert not mass.any() and cache.device_status() == 0
