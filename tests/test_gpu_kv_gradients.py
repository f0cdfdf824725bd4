"""GPU: gradients of the rotation through backward(), and calls of the cache that have none."""
import numpy as np
import pytest
import torch

import _kv_ref as ref
from paper_2608_07971_amd import kv

pytestmark = pytest.mark.gpu

EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def _say(msg):
    print(f"[gpu-case] {msg}", flush=True)


def _randn(seed, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def _np(t):
    return t.detach().double().cpu().numpy()


def _near(got, g, positions, f, m, interleaved, inverse):
    """A gradient against the formula's: the pair turned the other way, each rounded once; cos, sin and the products
    are within 4e-7 of the pair."""
    want = ref.rotate(_np(g), positions, f, m, interleaved, not inverse)
    size = 2 * m * np.abs(_np(g)).max()
    assert (np.abs(_np(got) - want) <= EPS[got.dtype] * np.abs(want) * 1.01 + 4e-7 * size + 2.0 ** -25).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_backward_turns_back(dtype, interleaved, inverse):
    _say(f"backward {dtype} interleaved={interleaved} inverse={inverse}")
    rope = kv.Rope(64, 48, interleaved=interleaved, scaling="parts", factor=4.0, context=64)
    f, m = ref.frequencies(48, 10000.0, "parts", 4.0, 64)
    pos = torch.tensor([0, 1, 77, 4000, 100000], dtype=torch.int32, device="cuda")
    p = pos.cpu().numpy()
    x, g = _randn(1, 5, 3, 64, dtype=dtype).requires_grad_(), _randn(2, 5, 3, 64, dtype=dtype)
    y = kv.rotate(rope, x, pos, inverse=inverse)
    assert torch.equal(y.detach(), kv.rotate(rope, x.detach(), pos, inverse=inverse))
    y.backward(g)
    _near(x.grad, g, p, f, m, interleaved, inverse)
    # a gradient that is broadcast, and one whose last dimension is not contiguous
    x.grad = None
    kv.rotate(rope, x, pos, inverse=inverse).sum().backward()
    _near(x.grad, torch.ones_like(g), p, f, m, interleaved, inverse)
    x.grad = None
    kv.rotate(rope, x, pos, inverse=inverse).transpose(1, 2).backward(g.transpose(1, 2).contiguous())
    _near(x.grad, g, p, f, m, interleaved, inverse)
    # inputs shared by several heads: the expansion's own gradient adds them up
    shared = _randn(3, 5, 1, 64, dtype=dtype).requires_grad_()
    kv.rotate(rope, shared.expand(5, 3, 64), pos, inverse=inverse).backward(g)
    one = kv.rotate(rope, g, pos, inverse=not inverse)
    assert torch.equal(shared.grad, one.sum(1, keepdim=True))
    with torch.no_grad():
        assert not kv.rotate(rope, x, pos).requires_grad


def test_backward_by_differences():
    rope, pos = kv.Rope(64, 32), torch.tensor([3, 500], dtype=torch.int32, device="cuda")
    x, g = _randn(4, 2, 2, 64).requires_grad_(), _randn(5, 2, 2, 64)
    grad, = torch.autograd.grad((kv.rotate(rope, x, pos) * g).sum(), x)
    h = 0.125                                                     # the map is linear: exact up to the results' rounding
    for d in (0, 5, 16, 31, 32, 63):
        step = torch.zeros_like(g)
        step[..., d] = h
        with torch.no_grad():
            slope = ((_np(kv.rotate(rope, x + step, pos)) - _np(kv.rotate(rope, x - step, pos))) * _np(g)).sum(-1) / (2 * h)
        assert np.abs(slope - _np(grad)[..., d]).max() <= 64 * float(g.abs().max()) * float(x.detach().abs().max() + h) * 2.0 ** -22 / h


def test_gradients_of_outputs_in_place_and_of_gradients():
    rope, pos = kv.Rope(64), torch.arange(7, dtype=torch.int32, device="cuda")
    x, g = _randn(6, 7, 2, 64).requires_grad_(), _randn(7, 7, 2, 64)
    want = kv.rotate(rope, g, pos, inverse=True)
    y = x * 1.0
    assert kv.rotate(rope, y, pos, out=y) is y
    y.backward(g)
    assert torch.equal(x.grad, want)
    out = torch.zeros_like(g)
    got = kv.rotate(rope, x, pos, out=out)
    assert got is out and torch.equal(torch.autograd.grad(out, x, g)[0], want)
    with pytest.raises(RuntimeError):
        kv.rotate(rope, x, pos, out=x)                            # a leaf is not turned in place
    v = g.clone().requires_grad_()
    grad, = torch.autograd.grad(kv.rotate(rope, x, pos), x, v, create_graph=True)
    again, = torch.autograd.grad(grad, v, g)                      # turned back, then turned
    assert torch.equal(again, kv.rotate(rope, g, pos))


def test_a_step_on_another_stream_has_its_gradient():
    rope, pos, side = kv.Rope(64), torch.arange(50, dtype=torch.int32, device="cuda"), torch.cuda.Stream()
    x, g = _randn(8, 50, 4, 64).requires_grad_(), _randn(9, 50, 4, 64)
    torch.cuda.synchronize()
    y = kv.rotate(rope, x, pos, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    y.backward(g)
    torch.cuda.synchronize()
    assert torch.equal(x.grad, kv.rotate(rope, g, pos, inverse=True))


def test_the_cache_says_where_a_gradient_would_be_lost():
    rope, offs = kv.Rope(64), ref.offsets([1, 1])
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    k, q = _randn(1, 2, 2, 64, dtype=torch.float16), _randn(2, 2, 4, 64, dtype=torch.float16)

    def calls(cache, k, q):
        turned = cache.append(0, k, k, offs, rope=rope, q=q)
        out, lse = cache.attend(0, turned.detach(), offs)
        return turned, out, lse, *cache.gather(0, dev([19, 19]), offs, 2)
    want = calls(ref.make(kv, [20, 20], heads=2, dim=64), k, q)
    assert not any(t.requires_grad for t in want)
    for which in ("q", "k"):
        cache = ref.make(kv, [20, 20], heads=2, dim=64)
        kk, qq = (k.clone().requires_grad_(), q) if which == "k" else (k, q.clone().requires_grad_())
        got = calls(cache, kk, qq)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        if which == "q":
            attended = cache.attend(0, qq, offs)
            alone = cache.attend(0, qq, offs, lse=False)
            assert alone[1] is None
            lost = [got[0], *attended, alone[0]]
        else:
            lost = got[1:]
        for t in lost:
            with pytest.raises(RuntimeError, match="no gradient"):
                t.float().sum().backward()
        for out in (torch.zeros_like(q), torch.zeros(2, 5, 64, dtype=q.dtype, device="cuda")[:, 1:]):
            assert cache.attend(0, qq, offs, out=out)[0] is out and out.requires_grad
        with torch.no_grad():
            assert not any(t.requires_grad for t in calls(cache, kk, qq))
        assert cache.device_status() == 0
