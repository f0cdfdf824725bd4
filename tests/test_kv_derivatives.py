"""Derivatives that calls of the paged cache do not have are refused, not lost.  Without a GPU, as far as the refusal goes."""
import types

import pytest
import torch
from torch.autograd import forward_ad

from paper_2608_07971_amd import kv

CACHE = types.SimpleNamespace(index=0)                            # refusals come before anything is asked of it
X, POS = torch.ones(2, 3, 8), torch.zeros(2, dtype=torch.int32)
CALLS = {
    "rotate": lambda x: kv.rotate(CACHE, x, POS), "rotate into": lambda x: kv.rotate(CACHE, X, POS, out=x),
    "norm_rotate q": lambda x: kv.norm_rotate(CACHE, x, X, None, None, POS), "norm_rotate k": lambda x: kv.norm_rotate(CACHE, X, x, None, None, POS),
    "norm_rotate weight": lambda x: kv.norm_rotate(CACHE, X, X, None, x, POS), "norm_rotate's gradient": lambda x: kv._norm_back(CACHE, X, X, X, X, POS, 1e-6, x, X, (True, True)),
    "select_beams": lambda x: kv.select_beams(x, X[0], 2), "select_beams' scores": lambda x: kv.select_beams(X, x, 2),
    "append": lambda x: kv.PagedCache.append(CACHE, 0, X, x, POS), "append's queries": lambda x: kv.PagedCache.append(CACHE, 0, X, X, POS, q=x),
    "attend": lambda x: kv.PagedCache.attend(CACHE, 0, x, POS), "weigh": lambda x: kv.PagedCache.weigh(CACHE, 0, x, X, POS, X),
    "weigh's lse": lambda x: kv.PagedCache.weigh(CACHE, 0, X, x, POS, X), "evict": lambda x: kv.PagedCache.evict(CACHE, POS, x),
}


@pytest.mark.parametrize("name", CALLS)
def test_tangents_are_refused(name):
    with forward_ad.dual_level():
        with pytest.raises(RuntimeError, match="no forward-mode derivative"):
            CALLS[name](forward_ad.make_dual(torch.ones(2, 3, 8), torch.ones(2, 3, 8)))
    with pytest.raises(RuntimeError, match="no forward-mode derivative"):
        torch.func.jvp(CALLS[name], (torch.ones(2, 3, 8),), (torch.ones(2, 3, 8),))


@pytest.mark.gpu
def test_tensors_without_a_tangent_pass_where_others_have_one():
    rope, pos = kv.Rope(64), torch.arange(5, dtype=torch.int32, device="cuda")
    q = torch.randn(5, 2, 64, generator=torch.Generator().manual_seed(1)).cuda()
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(q, torch.ones_like(q))
        want = kv.norm_rotate(rope, q, q, None, None, pos)
        assert all(torch.equal(a, b) for a, b in zip(kv.norm_rotate(rope, q, forward_ad.unpack_dual(dual).primal, None, None, pos), want))
        assert torch.equal(kv.rotate(rope, q, pos), kv.rotate(rope, q.clone(), pos))
        for call in (lambda: kv.rotate(rope, dual, pos), lambda: kv.norm_rotate(rope, dual, q, None, None, pos), lambda: kv.select_beams(dual, q[..., 0].contiguous(), 2)):
            with pytest.raises(RuntimeError, match="no forward-mode derivative"):
                call()
