"""The paged cache's calls refuse what they cannot do before anything is launched (host only)."""
import ctypes

import pytest
import torch

import paper_2601_13631_amd as ckv
from pages_common import nearest_e4m3, scale_byte

P = 4096  # a fake aligned address: never dereferenced


def pool(**over):
    d = dict(k=P, v=P, k_scale=None, v_scale=None, n_pages=100, page_stride=0, page_size=16,
             n_kv_heads=4, head_dim=128, dtype=ckv.DTYPE_BF16)
    d.update(over)
    return ckv._PagePool(**d)


def batch(**over):
    d = dict(table=P, lens=P, tok_off=P, table_stride=0, n_tokens=8, n_seqs=4, max_pages=10, max_tokens=0,
             max_len=0)
    d.update(over)
    return ckv._PageBatch(**d)


BAD_POOLS = [
    (dict(k=None), ckv.EINVAL), (dict(v=None), ckv.EINVAL), (dict(k=P + 8), ckv.EINVAL),
    (dict(v=P + 2), ckv.EINVAL), (dict(n_pages=0), ckv.EINVAL), (dict(n_pages=1 << 31), ckv.EINVAL),
    (dict(page_stride=16 * 4 * 128 - 8), ckv.EINVAL), (dict(page_stride=16 * 4 * 128 + 4), ckv.EINVAL),
    (dict(page_stride=-1), ckv.EINVAL), (dict(page_size=0), ckv.EINVAL), (dict(page_size=4), ckv.EUNSUPPORTED),
    (dict(page_size=24), ckv.EUNSUPPORTED), (dict(page_size=48), ckv.EUNSUPPORTED),
    (dict(page_size=1 << 30), ckv.EUNSUPPORTED), (dict(n_kv_heads=0), ckv.EINVAL),
    (dict(head_dim=0), ckv.EINVAL), (dict(head_dim=96), ckv.EUNSUPPORTED),
    (dict(dtype=ckv.DTYPE_F32), ckv.EUNSUPPORTED), (dict(dtype=3), ckv.EINVAL), (dict(dtype=-1), ckv.EINVAL),
    (dict(dtype=ckv.DTYPE_E4M3), ckv.EINVAL), (dict(dtype=ckv.DTYPE_E4M3, k_scale=P), ckv.EINVAL),
    (dict(k_scale=P, v_scale=P), ckv.EINVAL),
]
BAD_BATCHES = [
    (dict(table=None), ckv.EINVAL), (dict(lens=None), ckv.EINVAL), (dict(tok_off=None), ckv.EINVAL),
    (dict(n_seqs=-1), ckv.EINVAL), (dict(n_seqs=(1 << 20) + 1), ckv.EINVAL), (dict(n_tokens=-1), ckv.EINVAL),
    (dict(n_tokens=1 << 31), ckv.EINVAL), (dict(max_pages=0), ckv.EINVAL), (dict(table_stride=9), ckv.EINVAL),
    (dict(max_tokens=-1), ckv.EINVAL), (dict(max_len=-1), ckv.EINVAL),
]


def append(p, b, k=P, v=P):
    return ckv._lib.ckv_page_append(p, b, k, v, None)


def attn(p, b, q=P, hq=28, sm=0.0, window=0, sinks=0, out=P, ws=None, ws_bytes=0):
    return ckv._lib.ckv_page_attn(p, b, q, hq, sm, window, sinks, out, ws, ws_bytes, None)


@pytest.mark.parametrize("over,status", BAD_POOLS)
def test_bad_pools(over, status):
    p = pool(**over)
    assert append(p, batch()) == status and ckv.last_error()
    assert attn(p, batch()) == status
    assert ckv._lib.ckv_page_copy((ckv._PagePool * 2)(pool(), p), 2, P, P, 3, None) in (status, ckv.EINVAL)
    assert ckv._lib.ckv_page_copy((ckv._PagePool * 1)(p), 1, P, P, 3, None) == status


@pytest.mark.parametrize("over,status", BAD_BATCHES)
def test_bad_batches(over, status):
    assert append(pool(), batch(**over)) == status and ckv.last_error()
    assert attn(pool(), batch(**over)) == status


def test_bad_attention():
    assert attn(None, batch()) == ckv.EINVAL and attn(pool(), None) == ckv.EINVAL
    assert append(None, batch()) == ckv.EINVAL and append(pool(), None) == ckv.EINVAL
    for hq in (0, -4, 6):
        assert attn(pool(), batch(), hq=hq) == ckv.EINVAL
    for over in (dict(q=None), dict(out=None), dict(q=P + 4), dict(out=P + 8), dict(ws=P + 4)):
        assert attn(pool(), batch(), **over) == ckv.EINVAL
    for sm in (-1.0, float("nan"), float("inf")):
        assert attn(pool(), batch(), sm=sm) == ckv.EINVAL
    assert attn(pool(), batch(), window=-1) == ckv.EINVAL and attn(pool(), batch(), sinks=-1) == ckv.EINVAL
    assert attn(pool(), batch(n_tokens=1 << 27)) == ckv.EUNSUPPORTED
    assert attn(pool(), batch(max_pages=1 << 27)) == ckv.EUNSUPPORTED
    assert append(pool(), batch(), k=None) == ckv.EINVAL and append(pool(), batch(), v=P + 2) == ckv.EINVAL
    # many splits need their workspace
    long = batch(n_tokens=1, n_seqs=1, max_pages=10000)
    need = ckv._lib.ckv_page_attn_workspace_bytes(pool(), long, 28, 0, 0)
    assert need > 0
    assert attn(pool(), long) == ckv.EINVAL and "workspace" in ckv.last_error()
    assert attn(pool(), long, ws=P, ws_bytes=need - 1) == ckv.EINVAL
    assert ckv._lib.ckv_page_attn_workspace_bytes(pool(head_dim=96), long, 28, 0, 0) == 0
    assert ckv._lib.ckv_page_attn_workspace_bytes(pool(), long, 27, 0, 0) == 0


def test_nothing_to_do():
    for b in (batch(n_seqs=0), batch(n_tokens=0), batch(n_seqs=0, table=None, lens=None, tok_off=None)):
        assert append(pool(), b) == ckv.OK and attn(pool(), b) == ckv.OK
    assert ckv._lib.ckv_page_copy(None, 0, P, P, 3, None) == ckv.OK
    assert ckv._lib.ckv_page_copy((ckv._PagePool * 1)(pool()), 1, None, None, 0, None) == ckv.OK


def test_bad_moves():
    two = lambda **over: (ckv._PagePool * 2)(pool(), pool(**over))  # noqa: E731
    for over in (dict(n_pages=99), dict(page_size=32), dict(n_kv_heads=2), dict(head_dim=64),
                 dict(page_stride=1 << 20)):
        assert ckv._lib.ckv_page_copy(two(**over), 2, P, P, 3, None) == ckv.EINVAL
        assert "pool 1" in ckv.last_error()
    assert ckv._lib.ckv_page_copy(two(page_stride=16 * 4 * 128), 2, P, P, 0, None) == ckv.OK  # dense either way
    assert ckv._lib.ckv_page_copy(two(), -1, P, P, 3, None) == ckv.EINVAL
    assert ckv._lib.ckv_page_copy(None, 2, P, P, 3, None) == ckv.EINVAL
    assert ckv._lib.ckv_page_copy(two(), 2, None, P, 3, None) == ckv.EINVAL
    assert ckv._lib.ckv_page_copy(two(), 2, P, P, -1, None) == ckv.EINVAL
    need = ckv.page_compact_workspace_bytes(100)
    assert need > 0 and ckv.page_compact_workspace_bytes(0) == 0

    def compact(n=100, refs=P, out=P, table=P, table_out=P, entries=5, live=P, ws=P, ws_bytes=need):
        return ckv._lib.ckv_page_compact(two(), 2, refs, out, n, table, table_out, entries, live, ws, ws_bytes, None)

    for over in (dict(n=99), dict(n=0), dict(refs=None), dict(out=None), dict(table=None), dict(table_out=None),
                 dict(entries=-1), dict(live=None), dict(ws=None), dict(ws=P + 4), dict(ws_bytes=need - 1)):
        assert compact(**over) == ckv.EINVAL and ckv.last_error()
    assert ckv._lib.ckv_page_compact(None, 0, P, P, (1 << 26) + 1, None, None, 0, P, P, 1 << 40, None) == ckv.EUNSUPPORTED


def test_handles_refuse_host_tensors():
    k = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        ckv.PagePool(k, k)
    with pytest.raises(ValueError):
        ckv.PagePool(k.half(), k.half())
    with pytest.raises(ValueError):
        ckv.PagePool(k, k[:3])
    with pytest.raises(ValueError):
        ckv.PageBatch(torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32),
                      torch.zeros(3, dtype=torch.int32), 2)
    for bad in (-1, 1 << 31):
        with pytest.raises(ValueError):
            ckv._int32(bad, "window")


def test_model_of_e4m3():
    """The host model that the GPU tests use: every code is its own nearest value, ties go to even."""
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    x = codes[torch.isfinite(codes)].numpy()
    assert (nearest_e4m3(x) == x).all()
    assert nearest_e4m3(x * 1.0).max() == 448
    assert list(nearest_e4m3(pytest.importorskip("numpy").array([17.0, 19.0, 1e9, 2.0 ** -10, 3 * 2.0 ** -10]))) == [
        16.0, 20.0, 448.0, 0.0, 2.0 ** -8]
    assert list(scale_byte(pytest.importorskip("numpy").array([0.0, 448.0, 449.0, 224.0, 2.0 ** -130]))) == [
        10, 127, 128, 126, 10]
