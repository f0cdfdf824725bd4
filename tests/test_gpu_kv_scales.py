"""GPU: attention where value blocks' scales are far apart: what a query gets depends on the tokens that it sees alone."""
import numpy as np
import pytest
import torch

import _kv_ref as ref
from paper_2608_07971_amd import kv
from test_gpu_kv_prompt import launch_of

pytestmark = pytest.mark.gpu

EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # p significant bits: at most 2^-p of the value

# new tokens, length, heads, group, dim, page, window, type, launch
SHAPES = [
    (1, 700, 2, 4, 64, 16, 0, torch.bfloat16, "few"), (40, 700, 1, 2, 128, 16, 0, torch.bfloat16, "few"),
    (33, 300, 2, 1, 64, 64, 100, torch.bfloat16, "few"), (90, 500, 1, 1, 128, 32, 0, torch.bfloat16, "few"),
    (400, 700, 16, 1, 64, 16, 0, torch.bfloat16, "many"), (400, 900, 16, 1, 128, 32, 150, torch.bfloat16, "many"),
    (400, 1700, 16, 2, 128, 16, 0, torch.bfloat16, "many"), (400, 1500, 16, 1, 64, 64, 0, torch.bfloat16, "many"),
]


def _check(cache, q, n, L, window):
    """Scores: dim products added in float32, one scale and one exponential.  Weights rounded to fp16: 2^-11 of each,
    2^-35 of the largest below its range.  Values exact.  All relative to what the row sees, none to what it does not."""
    D = cache.head_dim
    out, _ = cache.attend(0, q, ref.offsets([n]), window=window, max_new=n, max_length=L)
    assert cache.device_status() == 0
    kp, vp = ref.host(cache)
    k, v = (ref.tokens_of(x, cache.table[0].cpu().numpy(), L) for x in (kp, vp))
    on, qn, G = out.double().cpu().numpy(), q.double().cpu().numpy(), q.shape[1] // cache.kv_heads
    worst = 0.0
    for i in range(n):
        p = L - n + i
        lo = max(0, p - window + 1) if window else 0
        for h in range(q.shape[1]):
            kk, vv = k[lo:p + 1, h // G], v[lo:p + 1, h // G]
            s = D ** -0.5 * (kk @ qn[i, h])
            w = np.exp(s - s.max())
            want, spread = w @ vv / w.sum(), w @ np.abs(vv) / w.sum()
            most = D ** -0.5 * (np.abs(kk) @ np.abs(qn[i, h])).max()
            d = D * 2.0 ** -24 * most + 2.0 ** -20 * (1 + most)
            bound = spread * (2.0 ** -11 + 2 * d + 2.0 ** -20) + 2.0 ** -35 * np.abs(vv).sum(0) + EPS[q.dtype] * np.abs(want) * 1.01
            off = np.abs(on[i, h] - want)
            worst = max(worst, (off / bound).max())
    assert worst <= 1.0, worst


def _make(n, L, heads, group, dim, page, dtype, launch, kind):
    assert launch_of(heads, dim, page, 1, n, group, n, L)[0] == launch
    cache = ref.make(kv, [L], page=page, heads=heads, dim=dim, seed=page + n)
    q = (torch.randn(n, heads * group, dim, generator=torch.Generator().manual_seed(3))).to(dtype).cuda()
    t, g = cache.table[0].long(), np.random.default_rng(7)
    pages = t.numel()
    e = {"last": np.where(np.arange(pages) == pages - 1, 25, 0),                     # hidden from all but the last rows
         "last far": np.where(np.arange(pages) == pages - 1, 60, -10),
         "first": np.where(np.arange(pages) == 0, 30, 0),
         "in turn": np.where(np.arange(pages) % 2, 27, -12),
         "any": g.integers(-35, 36, pages),
         "falling": np.linspace(38, -38, pages).round()}[kind]
    cache.scale[t, 0, 1] = torch.exp2(torch.from_numpy(np.repeat(e[:, None], heads, 1).astype(np.float32))).cuda()
    return cache, q


@pytest.mark.parametrize("kind", ["last", "last far", "first", "in turn", "any", "falling"])
@pytest.mark.parametrize("n,L,heads,group,dim,page,window,dtype,launch", SHAPES)
def test_blocks_far_apart(n, L, heads, group, dim, page, window, dtype, launch, kind):
    print(f"[gpu-case] scales {kind}: {n} of {L}, heads={heads}x{group} dim={dim} page={page} window={window}, {launch}", flush=True)
    cache, q = _make(n, L, heads, group, dim, page, dtype, launch, kind)
    _check(cache, q, n, L, window)


@pytest.mark.parametrize("n,heads", [(30, 1), (400, 16)])
def test_a_later_token_changes_no_earlier_row(n, heads):
    """The last page's values 2^25 times larger: rows before it keep every bit."""
    cache, q = _make(n, 640, heads, 1, 64, 16, torch.float16, "few" if n == 30 else "many", "falling")
    cache.scale[cache.table[0].long(), 0, 1] = 2.0 ** -9
    want = cache.attend(0, q, ref.offsets([n]), max_new=n, max_length=640)[0]
    cache.scale[cache.table[0, -1].long(), 0, 1] = 2.0 ** 16
    got = cache.attend(0, q, ref.offsets([n]), max_new=n, max_length=640)[0]
    assert torch.equal(got[:n - 16], want[:n - 16]) and not torch.equal(got[n - 16:], want[n - 16:])
