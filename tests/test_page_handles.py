"""What a pool's handle takes and refuses by its tensors' layout, decided on the host: no page's
address may lie past the tensor's own memory."""
import pytest
import torch

import paper_2601_13631_amd as ckv

SHAPE = (100, 16, 4, 128)  # 100 pages of 8,192 elements


class OnDevice(torch.Tensor):
    """A host tensor that says it is on device 0, for checks that read nothing."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


@pytest.fixture(autouse=True)
def device_0(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)


def pages(stride, shape=SHAPE, dtype=torch.bfloat16, numel=None):
    need = 1 + sum((n - 1) * s for n, s in zip(shape, stride))
    return torch.zeros(max(need, numel or 0), dtype=dtype).as_strided(shape, stride).as_subclass(OnDevice)


def last_byte(pool):
    """One past the last byte that the C side addresses, from k on."""
    c, row = pool._c, pool.n_kv_heads * pool.head_dim
    span = c.page_size * row
    return ((c.n_pages - 1) * (c.page_stride or span) + span) * pool.k.element_size()


@pytest.mark.parametrize("apart", [0, 8, 512, 4096, 8184])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
def test_pages_that_overlap_are_refused(apart, dtype):
    """Pages that share memory, an expanded dimension (0 apart) among them: 0 means pages without a
    gap to the C side, which would go past the end of the tensor."""
    scales = [torch.zeros(100, 4, dtype=torch.uint8).as_subclass(OnDevice) for _ in "kv"]
    scales = scales if dtype is torch.float8_e4m3fn else []
    bad, good = pages((apart, 512, 128, 1), dtype=dtype), pages((8192, 512, 128, 1), dtype=dtype)
    for k, v in ((bad, bad), (good, bad), (bad, good)):
        with pytest.raises(ValueError):
            ckv.PagePool(k, v, *scales)


def test_expanded_pages_are_refused():
    for shape in (SHAPE, (2, 8, 1, 64)):
        x = torch.zeros((1,) + shape[1:], dtype=torch.bfloat16).expand(shape).as_subclass(OnDevice)
        with pytest.raises(ValueError, match="overlap"):
            ckv.PagePool(x, x)


@pytest.mark.parametrize("stride", [(8192, 512, 128, 1), (9216, 512, 128, 1), (16384, 512, 128, 1)])
def test_addressed_bytes_lie_in_the_tensor(stride):
    k = pages(stride)
    pool = ckv.PagePool(k, pages(stride))
    assert last_byte(pool) <= k.untyped_storage().nbytes()


def test_one_page_has_no_stride():
    """A pool of one page may come from an expanded or a sliced tensor: no second page is addressed."""
    for apart in (0, 7, 1 << 40):
        k = pages((apart, 512, 128, 1), (1,) + SHAPE[1:])
        pool = ckv.PagePool(k, pages((8192, 512, 128, 1), (1,) + SHAPE[1:]))
        assert last_byte(pool) <= k.untyped_storage().nbytes()


def test_one_head():
    """Pages of one KV head that come from [n_pages, 1, page_size, head_dim]: contiguous, whatever the
    stride of the one head says; heads cut out of more are not."""
    x = torch.zeros(9, 1, 16, 64, dtype=torch.bfloat16)
    turned, plain = x.transpose(1, 2).as_subclass(OnDevice), x.view(9, 16, 1, 64).as_subclass(OnDevice)
    assert turned.stride() == (1024, 64, 1024, 1) and turned[0].is_contiguous()
    for k, v in ((turned, turned), (turned, plain), (plain, turned)):
        assert last_byte(ckv.PagePool(k, v)) <= x.untyped_storage().nbytes()
    cut = torch.zeros(9, 16, 2, 64, dtype=torch.bfloat16)[:, :, :1].as_subclass(OnDevice)
    for k, v in ((cut, cut), (plain, cut), (cut, plain)):
        with pytest.raises(ValueError):
            ckv.PagePool(k, v)
