"""GPU: norms of queries and keys with the rotation, and their gradient, against plain 64-bit forms.

u = 2^-24 is float32's half step.  The root: at most 16 terms in a row and 6 sums over lanes (the path for any
shape: 8 and 6), so the sum of squares is within 24 u of itself and its root within 12 u; the reciprocal root adds
4 u, scale and weight 2 u: 18 u of the normed element.  cos, sin and the products of a pair are within 4e-7 of the
pair's size.
"""
import numpy as np
import pytest
import torch

import _kv_forms as forms
import _kv_ref as ref
import paper_2608_07971_amd as esp
from paper_2608_07971_amd import kv

pytestmark = pytest.mark.gpu

EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}
U = 2.0 ** -24


def _say(msg):
    print(f"[gpu-case] {msg}", flush=True)


def _randn(seed, *shape, dtype=torch.float32, gain=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * gain).to(dtype).cuda()


def _np(t):
    return t.detach().double().cpu().numpy()


def _pair(x, f, magnitude, interleaved):
    """Size of the pair that each element is turned with."""
    size = ref.rotate(np.abs(x), np.zeros(x.shape[0]), f, magnitude, interleaved)
    n = len(f)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    both = size.copy()
    both[..., a] = both[..., b] = size[..., a] + size[..., b]
    return both


class Check:
    def __init__(self, dim, rotary, interleaved, scaling="none", eps=1e-6):
        self.rope = kv.Rope(dim, rotary, interleaved=interleaved, scaling=scaling, factor=8.0, context=4096)
        self.f, self.m = ref.frequencies(rotary, 10000.0, scaling, 8.0, 4096)
        self.interleaved, self.eps, self.dim = interleaved, eps, dim

    def forward(self, y, x, w, pos):
        p, x64, w64 = pos.cpu().numpy(), _np(x), np.ones(self.dim) if w is None else _np(w)
        want, n, _ = forms.norm_rotate(x64, w64, p, self.f, self.m, self.interleaved, self.eps)
        off = (18 * U + 4e-7) * _pair(n * w64, self.f, self.m, self.interleaved)
        bound = EPS[x.dtype] * (np.abs(want) + off) * 1.001 + off + TINY[x.dtype]
        assert y.dtype == x.dtype and (np.abs(_np(y) - want) <= bound).all()

    def backward(self, dx, dw, x, w, dy, pos):
        """40 u: the root's 16, the sum's 22 over a head and two products.  Over tokens and heads at most 128 sums follow
        each other at these sizes."""
        p, x64, w64 = pos.cpu().numpy(), _np(x), np.ones(self.dim) if w is None else _np(w)
        want, want_w, g, n, r, c = forms.norm_rotate_back(x64, w64, _np(dy), p, self.f, self.m, self.interleaved, self.eps)
        dg = 4e-7 * _pair(_np(dy), self.f, self.m, self.interleaved)
        gw, size = np.abs(g * w64), np.abs(g * w64 * n).mean(-1, keepdims=True)
        off = r * (dg * np.abs(w64) + np.abs(n) * ((dg * np.abs(w64 * n)).mean(-1, keepdims=True) + 40 * U * size))
        off = off + 40 * U * r * (gw + np.abs(n) * size)
        assert dx.dtype == x.dtype and (np.abs(_np(dx) - want) <= EPS[x.dtype] * (np.abs(want) + off) * 1.001 + off + TINY[x.dtype]).all()
        if w is not None:
            off = (dg * np.abs(n) + 40 * U * np.abs(g * n)).sum((0, 1)) + 128 * U * np.abs(g * n).sum((0, 1))
            assert dw.dtype == w.dtype and (np.abs(_np(dw) - want_w) <= EPS[w.dtype] * (np.abs(want_w) + off) * 1.001 + off + TINY[w.dtype]).all()

    def both(self, q, k, qw, kw, pos, gq, gk):
        leaves = [t for t in (q, k, qw, kw) if t is not None]
        for t in leaves:
            t.requires_grad_(True)
        yq, yk = kv.norm_rotate(self.rope, q, k, qw, kw, pos, eps=self.eps)
        grads = iter(torch.autograd.grad((yq, yk), leaves, (gq, gk)))
        dq, dk, dqw, dkw = (None if t is None else next(grads) for t in (q, k, qw, kw))
        for y, x, w, dx, dw, g in ((yq, q, qw, dq, dqw, gq), (yk, k, kw, dk, dkw, gk)):
            self.forward(y, x, w, pos)
            self.backward(dx, dw, x, w, g, pos)
        with torch.no_grad():
            again = kv.norm_rotate(self.rope, q, k, qw, kw, pos, eps=self.eps)
        assert torch.equal(again[0], yq) and torch.equal(again[1], yk) and not again[0].requires_grad
        return yq, yk, dq, dk, dqw, dkw


CASES = [
    (1, 1, 1, 64, 64, False, "none", torch.bfloat16, None), (257, 32, 8, 128, 128, False, "none", torch.bfloat16, torch.bfloat16),
    (1000, 4, 1, 128, 32, True, "parts", torch.bfloat16, torch.float32), (33, 5, 3, 96, 96, False, "linear", torch.float16, torch.float16),
    (70, 3, 5, 80, 80, True, "none", torch.float16, torch.float32), (41, 2, 7, 80, 40, False, "none", torch.bfloat16, torch.bfloat16),
    (90, 9, 2, 256, 64, False, "parts", torch.bfloat16, torch.float32), (19, 2, 2, 512, 512, True, "none", torch.float32, torch.float32),
    (50, 3, 4, 512, 128, False, "none", torch.float16, None), (23, 4, 4, 64, 32, False, "none", torch.float32, None),
    (31, 3, 2, 66, 66, True, "none", torch.float16, torch.float16), (29, 1, 2, 258, 130, False, "ntk", torch.float32, torch.float32),
    (12, 5, 1, 2, 2, False, "none", torch.float32, torch.float32), (64, 1, 6, 16, 16, True, "none", torch.bfloat16, torch.float32),
    (200, 9, 5, 24, 8, False, "none", torch.bfloat16, torch.float32), (60, 2, 3, 512, 508, False, "none", torch.float16, torch.float16),
    (77, 3, 2, 120, 60, True, "none", torch.float32, torch.float32), (40, 6, 1, 32, 16, False, "none", torch.float16, torch.float16), (2, 3, 3, 500, 500, False, "none", torch.bfloat16, torch.bfloat16),
]


@pytest.mark.parametrize("tokens,q_heads,k_heads,dim,rotary,interleaved,scaling,dtype,weights", CASES)
def test_norm_rotate_and_its_gradient(tokens, q_heads, k_heads, dim, rotary, interleaved, scaling, dtype, weights):
    _say(f"norm {tokens}x{q_heads}+{k_heads}x{dim} rotary={rotary} interleaved={interleaved} {scaling} {dtype} weights={weights}")
    check = Check(dim, rotary, interleaved, scaling)
    q, gq = (_randn(i, tokens, q_heads, dim, dtype=dtype, gain=3.0) for i in (1, 2))
    k, gk = (_randn(i, tokens, k_heads, dim, dtype=dtype, gain=0.3) for i in (3, 4))
    qw, kw = (None if weights is None else (1.0 + 0.2 * _randn(i, dim)).to(weights) for i in (5, 6))
    pos = torch.randint(-5, 1 << 20, (tokens,), generator=torch.Generator().manual_seed(7), dtype=torch.int32).cuda()
    first = check.both(q, k, qw, kw, pos, gq, gk)
    again = check.both(q, k, qw, kw, pos, gq, gk)
    assert all(a is None or torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides(dtype):
    check = Check(64, 32, False)
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    fused = _randn(3, 50, 12, 64, dtype=dtype)                   # queries, keys and values of one product
    wide = _randn(4, 50, 7, 65, dtype=dtype)                     # rows of 65: not 16-byte aligned
    one = _randn(5, 1, 7, 64, dtype=dtype)
    eights = _randn(7, 50, 9, 64 + 8 // one.element_size(), dtype=dtype)[..., 8 // one.element_size():]     # places at multiples of 8 bytes
    w = (1.0 + 0.1 * _randn(6, 64)).to(dtype)
    for q, k in ((fused[:, :8], fused[:, 8:10]), (wide[..., 1:], wide[:, 2:5, :64]), (one.expand(50, 7, 64), wide[:, :1, 1:].expand(50, 3, 64)),
                 (wide.transpose(0, 1).contiguous().transpose(0, 1)[..., :64], fused[:, 10:]), (eights[:, :5], fused[:, :2]), (eights[:, 5:], eights[:, :1])):
        _say(f"norm strides {q.stride()} {k.stride()} {dtype}")
        q, k = q.detach(), k.detach()
        gq, gk = (torch.randn(*x.shape[:2], 128, device="cuda").to(dtype)[..., 64:] for x in (q, k))
        check.both(q, k, w.clone(), w.clone(), pos, gq, gk)
        check.both(q, k, w.clone(), None, pos, gq[..., :1].expand(q.shape), gk[:1].expand(k.shape))


def test_gradient_by_differences():
    check = Check(64, 32, True)
    rope, pos = check.rope, torch.tensor([3, 500], dtype=torch.int32, device="cuda")
    q, k = _randn(4, 2, 2, 64).requires_grad_(), _randn(5, 2, 1, 64).requires_grad_()
    w = (1.0 + 0.2 * _randn(6, 64)).requires_grad_()
    gq, gk = _randn(7, 2, 2, 64), _randn(8, 2, 1, 64)
    dq, dk, dw = torch.autograd.grad(kv.norm_rotate(rope, q, k, w, w, pos), (q, k, w), (gq, gk))
    h = 2.0 ** -6

    def at(q, k, w):
        with torch.no_grad():
            yq, yk = kv.norm_rotate(rope, q, k, w, w, pos)
        return (_np(yq) * _np(gq)).sum() + (_np(yk) * _np(gk)).sum()

    def plain(q, k, w):
        return sum((forms.norm_rotate(_np(x), _np(w), pos.cpu().numpy(), check.f, check.m, True, 1e-6)[0] * _np(g)).sum() for x, g in ((q, gq), (k, gk)))
    y = [np.abs(_np(t)) for t in kv.norm_rotate(rope, q, k, w, w, pos)]
    # each of the two values is off by at most the forward's bound, here (18 u + 4e-7 + u) of a pair, twice the largest
    noise = 2 * (2 * (19 * U + 4e-7) * 2 * max(t.max() for t in y) * (np.abs(_np(gq)).sum() + np.abs(_np(gk)).sum())) / (2 * h)
    for name, leaf, grad in (("q", q, dq), ("k", k, dk), ("w", w, dw)):
        for i in (0, 5, 31, 32, 63):
            step = torch.zeros_like(leaf)
            step.view(-1)[i] = h
            up, down = ([t + step if n == name else t for n, t in (("q", q), ("k", k), ("w", w))], [t - step if n == name else t for n, t in (("q", q), ("k", k), ("w", w))])
            slope, exact = (at(*up) - at(*down)) / (2 * h), (plain(*up) - plain(*down)) / (2 * h)
            got = float(grad.view(-1)[i])
            assert abs(slope - got) <= abs(exact - got) + noise
            assert abs(exact - got) <= 0.02 * (1 + abs(got))     # h^2 times a third derivative of order one


def test_rows_of_zeros_large_and_small_numbers():
    check = Check(128, 128, False, eps=1e-5)
    pos = torch.arange(6, dtype=torch.int32, device="cuda")
    q = _randn(1, 6, 2, 128)
    q[0] = 0.0
    q[1] *= 1e-15
    q[2] *= 1e15
    k, g = q[:, :1].clone(), _randn(2, 6, 2, 128)
    w = torch.ones(128, device="cuda")
    yq, _, dq, *_ = check.both(q.clone(), k, w, w.clone(), pos, g, g[:, :1].contiguous())
    assert not yq[0].any() and bool(torch.isfinite(dq).all())
    q[3, 0, 5], q[4, 1, 7] = float("nan"), float("inf")          # stay with their head
    with torch.no_grad():
        yq, _ = kv.norm_rotate(check.rope, q, k, w, w, pos, eps=1e-5)
    bad = ~torch.isfinite(yq).all(-1)
    assert bad.nonzero().tolist() == [[3, 0], [4, 1]]


@pytest.mark.parametrize("dim,rotary,interleaved,off,dtype", [(64, 32, False, 0, torch.bfloat16), (64, 32, True, 0, torch.float32), (128, 8, True, 0, torch.float16),
                                                              (80, 40, False, 0, torch.bfloat16), (64, 30, False, 0, torch.float32), (64, 32, True, 1, torch.bfloat16)])
def test_infinities_in_the_part_that_passes_through(dim, rotary, interleaved, off, dtype):
    """They stay where they are: no element of that part has to do with another but through the norm."""
    _say(f"norm, infinities behind {rotary} of {dim}, interleaved={interleaved}, {dtype}")
    rope, pos = kv.Rope(dim, rotary, interleaved=interleaved), torch.arange(9, dtype=torch.int32, device="cuda")
    place = lambda seed, heads: _randn(seed, 9, heads, dim + off, dtype=dtype)[..., off:]  # noqa: E731
    q, k, gq, gk, w = place(1, 5), place(2, 1), place(3, 5), place(4, 1), torch.ones(dim, device="cuda")
    for at in sorted({rotary, rotary + 1, dim // 2 + rotary // 2, dim - 1}):
        big = w.clone()
        big[at] = float("inf")
        yq, yk = kv.norm_rotate(rope, q, k, big, big, pos)
        rest = torch.arange(dim, device="cuda") != at
        plain = kv.norm_rotate(rope, q, k, w, w, pos)
        for y, one in ((yq, plain[0]), (yk, plain[1])):
            assert bool(y[..., at].isinf().all()) and torch.equal(y[..., rest], one[..., rest])
        x, mine = q.clone().requires_grad_(), w.clone().requires_grad_()
        wide, turned = gq.clone(), kv.norm_rotate(rope, x, k, mine, None, pos)[0]
        want, = torch.autograd.grad(turned, mine, gq, retain_graph=True)
        wide[3, 2, at] = -float("inf")
        got, = torch.autograd.grad(turned, mine, wide)
        assert bool(got[at].isinf()) and torch.equal(got[rest], want[rest])


def test_no_tokens_no_heads_and_parts_of_the_gradient():
    rope, pos = kv.Rope(64), torch.arange(5, dtype=torch.int32, device="cuda")
    none, w = torch.zeros(0, 3, 64, device="cuda", requires_grad=True), torch.ones(64, device="cuda", requires_grad=True)
    y, _ = kv.norm_rotate(rope, none, none, w, w, pos[:0])
    dn, dw = torch.autograd.grad(y, (none, w), torch.zeros_like(y))
    assert y.shape == (0, 3, 64) and dn.shape == (0, 3, 64) and not dw.any()
    q, empty, g = _randn(1, 5, 2, 64).requires_grad_(), torch.zeros(5, 0, 64, device="cuda"), _randn(2, 5, 2, 64)
    yq, yk = kv.norm_rotate(rope, q, empty, w, None, pos)
    assert yk.shape == (5, 0, 64)
    Check(64, 64, False).forward(yq, q, w, pos)
    all_of = torch.autograd.grad(yq, (q, w), g)
    # only one of the two outputs, only one of the leaves
    k = _randn(3, 5, 1, 64)
    for leaves in ((q,), (w,), (q, w)):
        yq, yk = kv.norm_rotate(rope, q, k, w, None, pos)
        for leaf, got in zip(leaves, torch.autograd.grad(yq, leaves, g)):
            assert torch.equal(got, all_of[0 if leaf is q else 1])
    # a weight that queries and keys share gets the sum of both
    yq, yk = kv.norm_rotate(rope, q, q, w, w, pos)
    dq, dw = torch.autograd.grad((yq, yk), (q, w), (g, g))
    assert torch.equal(dw, all_of[1] + all_of[1]) and torch.equal(dq, all_of[0] + all_of[0])
    yq, _ = kv.norm_rotate(rope, q, k, w, None, pos)
    first, second = torch.autograd.grad(yq, (q, w), g.clone().requires_grad_(), create_graph=True)
    assert torch.equal(first, all_of[0]) and torch.equal(second, all_of[1])
    for lost in (first, second):
        with pytest.raises(RuntimeError, match="no gradient"):
            lost.sum().backward()                                 # of the gradient there is none


def test_a_training_step_in_a_graph():
    """Captured forward and backward, replayed with other work between.  While an eager graph of the same leaves lives,
    autograd would leave the capture's stream in the backward pass: it is refused."""
    rope, pos = kv.Rope(128), torch.arange(300, dtype=torch.int32, device="cuda")
    q, k = torch.zeros(300, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(300, 2, 128, dtype=torch.bfloat16, device="cuda")
    qw, kw = torch.ones(128, device="cuda"), torch.ones(128, device="cuda")
    gq, gk = torch.zeros_like(q), torch.zeros_like(k)
    leaves = [t.requires_grad_(True) for t in (q, k, qw, kw)]

    def step():
        y = kv.norm_rotate(rope, q, k, qw, kw, pos)
        return [*(t.detach() for t in y), *torch.autograd.grad(y, leaves, (gq, gk))]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
        got = step()                                              # the leaves again, in the same capture
    for i in range(5):
        _say(f"replay {i}")
        with torch.no_grad():
            for j, t in enumerate((q, k, gq, gk)):
                t.copy_(_randn(10 * i + j, *t.shape))
            qw.copy_(1.0 + 0.1 * _randn(10 * i + 5, 128))
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    _say("another capture while the first one's results live")
    second = torch.cuda.CUDAGraph()
    y = None
    with torch.cuda.graph(second):
        y = kv.norm_rotate(rope, q, k, qw, kw, pos)
    third = torch.cuda.CUDAGraph()
    with torch.cuda.graph(third):
        again = step()
    third.replay()
    torch.cuda.synchronize()
    assert y[0].grad_fn is not None and all(torch.equal(a, b) for a, b in zip(again, want))
    del y
    _say("a captured backward pass beside an eager graph of the same leaves")
    lives = kv.norm_rotate(rope, q, k, qw, kw, pos)
    torch.cuda.synchronize()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        with pytest.raises(RuntimeError, match="before the capture"):
            step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(lives, leaves, (gq, gk)), want[2:]))


def _captured(leaves, step, **more):
    """step's results from a graph and eagerly, for three sets of inputs."""
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, **more):
        got = step()
    for i in range(3):
        _say(f"replay {i}")
        with torch.no_grad():
            for j, t in enumerate(leaves):
                t.copy_(1.0 + 0.1 * _randn(20 * i + j, *t.shape))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


def test_other_users_of_the_leaves_in_a_capture():
    """A leaf that another operation of the same capture used first."""
    rope, pos = kv.Rope(64), torch.arange(30, dtype=torch.int32, device="cuda")
    q, k, w = (torch.ones(*n, device="cuda", requires_grad=True) for n in ((30, 4, 64), (30, 2, 64), (64,)))
    grads = [_randn(i, *n) for i, n in enumerate(((30, 4, 64), (30, 2, 64), (64,), (30, 4, 64)))]

    def step():
        other = w * w, q * q
        y = kv.norm_rotate(rope, q, k, w, w, pos)
        return torch.autograd.grad((*y, *other), (q, k, w), grads)
    step()
    _captured((q, k, w), step)

    def added():
        for t in (q, k, w):
            t.grad = None
        other = w * w
        y = kv.norm_rotate(rope, q, k, w, None, pos)
        torch.autograd.backward((*y, other), grads[:3])
        return [t.grad.clone() for t in (q, k, w)]
    added()
    _captured((q, k, w), added)


def test_accumulators_that_were_made_on_the_stream_that_is_captured():
    rope, pos, side = kv.Rope(64), torch.arange(9, dtype=torch.int32, device="cuda"), torch.cuda.Stream()
    q, w = (torch.ones(*n, device="cuda", requires_grad=True) for n in ((9, 2, 64), (64,)))
    g = _randn(1, 9, 2, 64)
    with torch.cuda.stream(side):
        kept = [q.view_as(q), w.view_as(w)]                       # hold them, as wrappers that keep accumulators do
    torch.cuda.synchronize()
    node = torch.autograd.graph.get_gradient_edge(w).node
    assert kv._stream_of(node, w) == side.cuda_stream and q.grad is None
    _captured((q, w), lambda: torch.autograd.grad(kv.norm_rotate(rope, q, q.detach(), w, None, pos)[0], (q, w), g), stream=side)
    assert len(kept) == 2


def test_another_stream():
    rope, pos, side = kv.Rope(64), torch.arange(50, dtype=torch.int32, device="cuda"), torch.cuda.Stream()
    q, k, w = _randn(8, 50, 4, 64).requires_grad_(), _randn(9, 50, 2, 64), torch.ones(64, device="cuda")
    g = _randn(10, 50, 4, 64)
    want = kv.norm_rotate(rope, q, k, w, w, pos)
    grad, = torch.autograd.grad(want[0], q, g)
    torch.cuda.synchronize()
    y = kv.norm_rotate(rope, q, k, w, w, pos, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    got, = torch.autograd.grad(y[0], q, g)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*y, got), (*want, grad)))


def test_what_does_not_fit_is_refused():
    rope, pos = kv.Rope(64), torch.arange(5, dtype=torch.int32, device="cuda")
    q, w = _randn(1, 5, 2, 64), torch.ones(64, device="cuda")
    call = lambda rope=rope, q=q, k=q, qw=w, kw=w, pos=pos, **more: kv.norm_rotate(rope, q, k, qw, kw, pos, **more)  # noqa: E731
    for bad in (dict(k=q.half()), dict(q=q.double(), k=q.double()), dict(q=q[0]), dict(k=q[:4]), dict(q=q[..., :32]), dict(rope=kv.Rope(128)),
                dict(qw=w[:32]), dict(qw=w.half()), dict(q=q.half(), k=q.half(), qw=w.half()), dict(kw=w.cpu()), dict(pos=pos.long()), dict(pos=pos[:4]),
                dict(qw=torch.ones(128, device="cuda")[::2]), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(k=q.cpu())):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        with pytest.raises(esp.EspError):
            call(**bad)
    wide = _randn(2, 5, 2, 514)
    with pytest.raises(esp.EspError):
        kv.norm_rotate(kv.Rope(514), wide, wide, None, None, pos)
