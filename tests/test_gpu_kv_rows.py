"""GPU: offsets that do not ascend, over more tokens than the pages' numbering of a call's work absorbs."""
import pytest
import torch

import _kv_ref as ref
import paper_2608_07971_amd as esp
from paper_2608_07971_amd import kv

pytestmark = pytest.mark.gpu


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("offsets", [[0, 200, 100, 600], [0, 200, 168, 600], [0, 600, 0, 600], [0, 300, -300, 600], [0, 200, 400, 700]])
def test_rows_that_go_back_are_recorded(offsets):
    print(f"[gpu-case] offsets {offsets}", flush=True)
    cache = ref.make(kv, [700, 650, 640], heads=8, dim=64)
    q = torch.randn(600, 16, 64, generator=torch.Generator().manual_seed(1)).half().cuda()
    off, starts = _dev(offsets), _dev([0, 0, 0])
    cache.attend(0, q, off)                                       # many new tokens
    assert cache.device_status() == esp.ESP_ERR_SHAPE
    cache.attend(0, q[:, :8], off, max_new=600)
    assert cache.device_status() == esp.ESP_ERR_SHAPE
    cache.gather(0, starts, off, 600)
    assert cache.device_status() == esp.ESP_ERR_SHAPE
    cache.append(0, q[:, :8], q[:, 8:], off)
    assert cache.device_status() == esp.ESP_ERR_SHAPE
    cache.append(0, q[:, :8], q[:, 8:], off, rope=kv.Rope(64), q=q)
    assert cache.device_status() == esp.ESP_ERR_SHAPE
    good = _dev([0, 200, 400, 600])
    cache.attend(0, q, good)
    cache.gather(0, starts, good, 600)
    cache.append(0, q[:, :8], q[:, 8:], good, rope=kv.Rope(64), q=q)
    assert cache.device_status() == 0
