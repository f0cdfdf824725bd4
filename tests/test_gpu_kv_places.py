"""GPU: operands of the paged cache's calls at odd places and of odd strides that nothing depends on."""
import pytest
import torch

import _kv_ref as ref
from paper_2608_07971_amd import kv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,heads", [(3, 4), (1, 4), (1, 1), (5, 1)])
def test_append_takes_queries_at_any_place(tokens, heads):
    """Contiguous but not at a multiple of 16 bytes; one token (one head) of a tensor whose rows are not."""
    rope, offs = kv.Rope(64), ref.offsets([tokens])
    k = torch.randn(tokens, 1, 64, generator=torch.Generator().manual_seed(1)).half().cuda()
    q = torch.randn(tokens, heads, 64, generator=torch.Generator().manual_seed(2)).half().cuda()
    want = ref.make(kv, [20], heads=1, dim=64).append(0, k, k, offs, rope=rope, q=q)
    flat = torch.zeros(q.numel() + 8, dtype=q.dtype, device="cuda")
    rows = torch.zeros(tokens, heads * 64 + 3, dtype=q.dtype, device="cuda")
    places = [flat[i:i + q.numel()].view(q.shape) for i in (1, 4)] + [rows[:, :heads * 64].view(q.shape)]
    for place in places:
        print(f"[gpu-case] queries {tuple(place.shape)} strides {place.stride()} at {place.data_ptr() % 16}", flush=True)
        place.copy_(q)
        cache = ref.make(kv, [20], heads=1, dim=64)
        assert torch.equal(cache.append(0, k, k, offs, rope=rope, q=place), want)
        got, _ = cache.attend(0, place, offs)
        assert torch.equal(got, cache.attend(0, q, offs)[0])
        assert torch.equal(kv.rotate(rope, place, offs[:1].expand(tokens).contiguous()), kv.rotate(rope, q, offs[:1].expand(tokens).contiguous()))
        assert cache.device_status() == 0
