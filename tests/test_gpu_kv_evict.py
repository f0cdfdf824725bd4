"""GPU: eviction by accumulated attention weight against the form on host integers; codes bit by bit."""
import numpy as np
import pytest
import torch

import _kv_forms as forms
import _kv_ref as ref
import paper_2608_07971_amd as esp
from paper_2608_07971_amd import kv

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn


def _say(msg):
    print(f"[gpu-case] {msg}", flush=True)


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _mass(cache, seed=1):
    x = torch.exp(3.0 * torch.randn(cache.mass_shape, generator=torch.Generator().manual_seed(seed)))
    x[torch.rand(x.shape, generator=torch.Generator().manual_seed(seed + 1)) < 0.2] = 0.0       # ties
    return x.cuda()


def _codes(cache):
    """k, v [P][L][H][T][D] codes, scales [P][L][2][H], on the host."""
    return (cache.k.view(torch.uint8).cpu().numpy(), cache.v.view(torch.uint8).cpu().numpy().swapaxes(-1, -2), cache.scale.cpu().numpy().copy())


def _check(cache, keep, mass, recent):
    pages, before, scale = forms.Pages(cache), _codes(cache)[:2], _codes(cache)[2]
    table, lengths, old = pages.table.copy(), pages.lengths.copy(), mass.cpu().numpy().copy()
    cut = pages.evict(keep)
    cache.evict(_dev(keep), mass, recent=recent)
    assert cache.device_status() == 0
    assert np.array_equal(cache.table.cpu().numpy(), pages.table) and np.array_equal(cache.refs.cpu().numpy(), pages.refs)
    assert np.array_equal(cache.lengths.cpu().numpy(), pages.lengths)
    got_mass, (k, v, s) = mass.cpu().numpy(), _codes(cache)
    T, want_mass = cache.page_tokens, old.copy()
    touched = {int(p) for x in cut for p in pages.table[x] if p >= 0}
    for layer in range(cache.layers):
        for h in range(cache.kv_heads):
            for x in cut:
                stay = forms.kept(old[layer, x, h], int(lengths[x]), keep[x], recent)
                assert len(stay) == keep[x]
                want_mass[layer, x, h, :keep[x]] = old[layer, x, h, stay]
                page, at = table[x][stay // T], stay % T
                for side, (codes, now) in enumerate(((before[0], k), (before[1], v))):
                    for j in range(-(-keep[x] // T)):
                        own = slice(j * T, min(keep[x], j * T + T))
                        was = scale[page[own], layer, side, h]
                        top = np.float32(was.max())
                        to = int(pages.table[x, j])
                        assert s[to, layer, side, h] == top
                        c = codes[page[own], layer, h, at[own]]
                        by = was / top if top > 0 else np.ones_like(was)
                        num = torch.from_numpy(np.ascontiguousarray(c)).view(F8).float() * torch.from_numpy(by)[:, None]
                        exp, new = num.to(F8).float().numpy(), torch.from_numpy(np.ascontiguousarray(now[to, layer, h, :own.stop - own.start])).view(F8).float().numpy()
                        assert np.array_equal(exp, new, equal_nan=True), (layer, h, x, side, j)
                        assert np.array_equal(now[to, layer, h, own.stop - own.start:], codes[to, layer, h, own.stop - own.start:])   # past the end
    assert np.array_equal(got_mass, want_mass, equal_nan=True)
    rest = [p for p in range(cache.pages) if p not in touched]   # pages that nobody was moved to
    assert all(np.array_equal(a[rest], b[rest]) for a, b in zip((k, v), before)) and np.array_equal(s[rest], scale[rest], equal_nan=True)


CASES = [
    ([1], [0], 0, 1, 64, 16, 1), ([2, 1], [1, 1], 1, 1, 64, 16, 1), ([100, 40, 0, 17], [50, 50, 3, 17], 8, 2, 64, 16, 2), ([500, 333, 64], [1, 200, 63], 0, 2, 128, 32, 1),
    ([1000], [999], 999, 1, 128, 64, 2), ([700, 900, 65, 129], [300, 17, 64, 128], 5000, 3, 64, 64, 1), ([5000, 4097, 4096], [4096, 2049, 64], 30, 1, 64, 16, 1),
    ([9000], [4500], 0, 2, 64, 32, 1), ([300] * 20, [7 * i for i in range(20)], 16, 1, 128, 16, 3), ([257, 256], [255, 128], 100, 2, 128, 16, 1),
    ([20, 3, 19] * 34, [9] * 102, 2, 6, 64, 16, 11),
]


@pytest.mark.parametrize("lengths,keep,recent,heads,dim,page,layers", CASES)
def test_evict(lengths, keep, recent, heads, dim, page, layers):
    _say(f"evict {lengths[:4]} to {keep[:4]}, recent {recent}, {layers} x {heads} x {dim}, pages of {page}")
    cache = ref.make(kv, lengths, page=page, heads=heads, dim=dim, layers=layers, seed=len(lengths))
    mass = _mass(cache)
    _check(cache, keep, mass, recent)
    _check(cache, [x // 2 for x in keep], mass, recent // 3)      # what was moved, once more
    _check(cache, [x // 2 for x in keep], mass, recent)           # nothing to do


def test_shared_pages_are_left_to_the_others():
    cache = ref.make(kv, [200, 0, 0, 90], heads=2, dim=64, page=16, width=14, spare=40)
    cache.fork(_dev([0, 0]), _dev([1, 2]))
    mass = _mass(cache)
    others = [cache.gather(0, _dev([0]), ref.offsets([200]), 200, seqs=_dev([2]))]
    _check(cache, [60, 100, 200, 80], mass, 10)                   # two of the three that share; each has its own choice
    others.append(cache.gather(0, _dev([0]), ref.offsets([200]), 200, seqs=_dev([2])))
    assert all(torch.equal(a, b) for a, b in zip(*others))
    _check(cache, [60, 100, 30, 80], mass, 0)
    assert int(cache.refs.max()) == 1


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("gone", [16, 64, 128, 200])
def test_a_beginning_that_goes(gone, page):
    """Each stretch of new places takes its tokens, and their scales, from the places of the next."""
    cache = ref.make(kv, [1500, 700, 900], heads=8, dim=64, page=page, layers=4, seed=gone)
    mass = _mass(cache) + 1.0
    mass[..., :gone] = 0.0
    _check(cache, [1500 - gone, 700 - gone, 900 - gone], mass, 0)


def test_equal_weights_infinities_and_nan():
    cache = ref.make(kv, [300, 300, 300, 300], heads=1, dim=64)
    mass = torch.full(cache.mass_shape, 0.25, device="cuda")
    mass[0, 1] = 0.0
    mass[0, 1, 0, ::3] = -0.0                                     # equal to 0
    mass[0, 2, 0, 5:250:7], mass[0, 2, 0, 3:200:11], mass[0, 2, 0, 8] = float("nan"), float("inf"), -float("inf")
    mass[0, 3, 0, :290] = float("nan")
    _check(cache, [100, 200, 150, 40], mass, 10)


def test_scales_that_are_no_powers_of_two_zeros_and_nan_codes():
    cache = ref.make(kv, [333, 200], heads=2, dim=128, page=32)
    g = torch.Generator().manual_seed(3)
    cache.scale.copy_(torch.rand(cache.scale.shape, generator=g) * 0.01)
    cache.scale[::3] *= 1e-4                                      # most of their codes vanish beside the others
    cache.scale[cache.table[1].long()] = 0.0
    cache.k.view(torch.uint8)[cache.table[0, 2].long(), 0, 0, 3, 5] = 0x7f
    cache.v.view(torch.uint8)[cache.table[0, 4].long(), 0, 1, 7, 9] = 0xff
    _check(cache, [222, 111], _mass(cache), 111)


def test_evictions_that_cannot_be_done_change_nothing():
    cache = ref.make(kv, [100, 100, 30], heads=1, dim=64, width=8, spare=0)
    mass = _mass(cache)
    state = [t.clone() for t in (cache.table, cache.lengths, cache.refs, mass)] + [t.view(torch.uint8).clone() for t in (cache.k, cache.v)]

    def unchanged(code):
        assert cache.device_status() == code
        assert all(torch.equal(a, b) for a, b in zip(state, [cache.table, cache.lengths, cache.refs, mass] + [t.view(torch.uint8) for t in (cache.k, cache.v)]))
    cache.evict(_dev([50, -1, 30]), mass)
    unchanged(esp.ESP_ERR_SHAPE)
    for at, bad in (((0, 1), cache.pages), ((0, 2), -1), ((2, 5), -2)):
        good = int(cache.table[at])
        cache.table[at] = bad
        state[0][at] = bad
        cache.evict(_dev([50, 100, 30]), mass)
        unchanged(esp.ESP_ERR_SHAPE)
        cache.table[at] = state[0][at] = good
    cache.lengths[1] = state[1][1] = 129
    cache.evict(_dev([50, 100, 30]), mass)
    unchanged(esp.ESP_ERR_SHAPE)
    cache.lengths[1] = state[1][1] = 100
    cache.table[1, :6] = cache.table[0, :6]                       # shared by two, and no page is free
    cache.refs.fill_(1)
    cache.refs[cache.table[0, :6].long()] = 2
    state[0], state[2] = cache.table.clone(), cache.refs.clone()
    cache.evict(_dev([50, 100, 30]), mass)
    unchanged(esp.ESP_ERR_RANGE)
    cache.evict(_dev([100, 100, 10]), mass)                       # nothing shared: goes on
    assert cache.device_status() == 0 and cache.lengths.tolist() == [100, 100, 10]
    for bad in (dict(keep=_dev([1, 2])), dict(keep=_dev([1, 2, 3]).long()), dict(mass=mass[0]), dict(mass=mass.half())):
        with pytest.raises(ValueError):
            cache.evict(**{"keep": _dev([1, 2, 3]), "mass": mass, **bad})
    with pytest.raises(esp.EspError):
        cache.evict(_dev([1, 2, 3]), mass, recent=-1)


def test_far_pages_of_a_large_pool():
    """Blocks past 2^32 bytes."""
    T, H, D = 64, 8, 128
    P = (1 << 32) // (H * T * D) + 40
    cache = kv.PagedCache(P, T, H, D, sequences=1, table_width=6)
    small = kv.PagedCache(6, T, H, D, sequences=1, table_width=6)
    k = torch.randn(300, H, D, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    for c in (cache, small):
        c.table[0, :5] = torch.arange(c.pages - 5, c.pages, dtype=torch.int32)
        c.refs[-5:] = 1
        c.lengths[0] = 300
        c.append(0, k, k.flip(0), ref.offsets([300]))
    mass = _mass(small)
    masses = [mass.clone(), mass]
    got = []
    for c, m in zip((cache, small), masses):
        c.evict(_dev([130]), m, recent=20)
        got.append(c.gather(0, _dev([0]), ref.offsets([130]), 130))
        assert c.device_status() == 0
    assert torch.equal(*masses) and all(torch.equal(a, b) for a, b in zip(*got))


def test_a_whole_step_together_and_in_a_graph():
    """Norms and rotation at positions that evictions leave as they were, append, attention, weights, eviction; the same
    step captured and replayed with eager work between."""
    lengths, T, H, G, D, L, keep = [70, 33, 90], 16, 2, 2, 64, 2, 64
    rope, offs = kv.Rope(D), ref.offsets([1] * 3)
    caches = [ref.make(kv, lengths, page=T, heads=H, dim=D, layers=L, width=8, seed=6) for _ in range(3)]
    qw, kw = (1.0 + 0.1 * torch.randn(D, generator=torch.Generator().manual_seed(i)).cuda() for i in (1, 2))
    q, k, v = (torch.zeros(L, 3, n, D, dtype=torch.bfloat16, device="cuda") for n in (H * G, H, H))
    positions, limit = [_dev(lengths) for _ in caches], _dev([keep] * 3)
    masses = [_mass(c, 7) for c in caches]

    def step(i):
        cache, mass, outs = caches[i], masses[i], []
        cache.resize(cache.lengths + 1)
        for layer in range(L):
            with torch.no_grad():
                turned, keys = kv.norm_rotate(rope, q[layer], k[layer], qw, kw, positions[i])
            cache.append(layer, keys, v[layer], offs)
            out, lse = cache.attend(layer, turned, offs, max_new=1)
            cache.weigh(layer, turned, lse, offs, mass, max_new=1)
            outs += [out, lse]
        cache.evict(limit, mass, recent=8)
        positions[i] += 1
        return outs
    step(2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(0)
    for i in range(6):
        _say(f"replay {i}")
        for j, t in enumerate((q, k, v)):
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(10 * i + j)))
        graph.replay()
        torch.cuda.synchronize()
        want = step(1)
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(masses[0], masses[1])
        for a, b in ((caches[0].table, caches[1].table), (caches[0].lengths, caches[1].lengths), (caches[0].refs, caches[1].refs)):
            assert torch.equal(a, b)
    assert caches[0].lengths.tolist() == [64, 39, 64] and positions[0].tolist() == [76, 39, 96]
    assert all(c.device_status() == 0 for c in caches)
    # the last step's results against the plain form, on what the cache held
    cache, old = caches[1], [t.clone() for t in (q, k, v)]
    cache.resize(cache.lengths + 1)
    turned, keys = kv.norm_rotate(rope, old[0][0], old[1][0], qw, kw, positions[1])
    cache.append(0, keys, old[2][0], offs)
    out, lse = cache.attend(0, turned, offs)
    pool = ref.host(cache, 0)
    for b in range(3):
        n = int(cache.lengths[b])
        kk, vv = (ref.tokens_of(x, cache.table[b].cpu().numpy(), n) for x in pool)
        o, l, spread, most = ref.attend(turned[b:b + 1].double().cpu().numpy(), kk, vv, 1, 0, D ** -0.5)
        off = 2 * D * most * 2.0 ** -24 + 8 * 2.0 ** -24 * (1 + np.abs(l).max())
        assert np.abs(lse[b].double().cpu().numpy() - l[0]).max() <= off + 2.0 ** -11
        # weights rounded to fp16, the result to bf16
        assert (np.abs(out[b].double().cpu().numpy() - o[0]) <= 2.0 ** -8 * np.abs(o[0]) + (2 * off + 2.0 ** -10) * spread[0]).all()
