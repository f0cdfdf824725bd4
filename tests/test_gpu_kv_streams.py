"""GPU: tensors that the caller drops while a stream that was given has yet to read them."""
import math

import pytest
import torch

import _kv_ref as ref
from paper_2608_07971_amd import kv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("raw", [False, True])
def test_inputs_that_are_dropped_are_read_first(raw):
    print(f"[gpu-case] dropped inputs, stream as a {'number' if raw else 'Stream'}", flush=True)
    lengths = [300, 77]
    rope, offs = kv.Rope(64), ref.offsets([100, 60])
    k, v, q = (torch.randn(160, n, 64, generator=torch.Generator().manual_seed(n)).half().cuda() for n in (2, 3, 8))
    v = v[:, :2].contiguous()
    positions = torch.arange(160, dtype=torch.int32, device="cuda")
    cache = ref.make(kv, lengths, heads=2, dim=64)
    turned = cache.append(0, k, v, offs, rope=rope, q=q)
    want = [turned, *cache.attend(0, q, offs), kv.rotate(rope, q, positions)]
    cache, side = ref.make(kv, lengths, heads=2, dim=64), torch.cuda.Stream()
    a = torch.randn(4096, 4096, device="cuda", dtype=torch.bfloat16)
    temporary = [t.clone() for t in (k, v, q, q, q)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):                                # the stream is busy for a while
        for _ in range(40):
            a = a @ a
    stream = side.cuda_stream if raw else side
    got = [cache.append(0, temporary[0], temporary[1], offs, rope=rope, q=temporary[2], stream=stream),
           *cache.attend(0, temporary[3], offs, stream=stream), kv.rotate(rope, temporary[4], positions, stream=stream)]
    temporary += [rope.turns, *cache.tensors]
    places, shapes = {t.data_ptr() for t in temporary}, [t.shape for t in temporary]
    temporary.clear()
    del rope, cache
    junk = [torch.full(shape, math.nan, dtype=d, device="cuda") for shape in shapes for d in (torch.half, torch.double) for _ in range(3)]
    assert not places & {t.data_ptr() for t in junk}
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
