"""Pools over tensors whose pages share memory are refused before any call could address them."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from pages_common import DEV  # noqa: E402


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float8_e4m3fn])
def test_overlapping_pages_are_refused(dtype):
    import paper_2601_13631_amd as ckv
    one = torch.zeros(1, 16, 4, 64, dtype=torch.float32, device=DEV).to(dtype)
    scales = [torch.zeros(100, 4, dtype=torch.uint8, device=DEV) for _ in "kv"] if dtype is torch.float8_e4m3fn else []
    with pytest.raises(ValueError, match="overlap"):
        ckv.PagePool(one.expand(100, 16, 4, 64), one.expand(100, 16, 4, 64), *scales)
    row = torch.zeros(99 * 256 + 4096, dtype=torch.float32, device=DEV).to(dtype)
    slid = row.as_strided((100, 16, 4, 64), (256, 256, 64, 1))
    with pytest.raises(ValueError, match="overlap"):
        ckv.PagePool(slid, slid, *scales)
    ckv.PagePool(one.expand(1, 16, 4, 64), one, *[s[:1] for s in scales])
