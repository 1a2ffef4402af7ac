"""Workspaces of attention over shared pages: what their size says of the plan, and the calls that are given
too little (host only)."""
import pytest

import paper_2601_13631_amd as ckv
from test_pages import P, batch, pool
from test_shared_prefix import attn, groups


def need(p, b, g, hq=28):
    return ckv._lib.ckv_page_attn_shared_workspace_bytes(p, b, g, hq)


HINTS = [dict(), dict(max_tokens=1, max_len=5), dict(max_tokens=1 << 30, max_len=1 << 30)]
GROUP_HINTS = [dict(), dict(max_tokens=1, max_shared=1), dict(max_tokens=1 << 30, max_shared=1 << 30)]


@pytest.mark.parametrize("hints", HINTS)
@pytest.mark.parametrize("over", GROUP_HINTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "e4m3"])
def test_less_than_the_workspace_is_refused(hints, over, dtype):
    p = {"f32": pool(dtype=ckv.DTYPE_F32, head_dim=64), "bf16": pool(),
         "e4m3": pool(dtype=ckv.DTYPE_E4M3, k_scale=P, v_scale=P)}[dtype]
    b, g = batch(n_tokens=300, n_seqs=100, max_pages=4000, **hints), groups(**over)
    n = need(p, b, g)
    # 2 groups of 100 sequences: in parts, with a place for either part of every row, unless the hints say that
    # next to nothing is shared
    few = hints.get("max_len") == 5 or over.get("max_shared") == 1
    assert n < 1 << 32
    if not few:
        d = p.head_dim
        assert n >= 2 * 300 * 28 * (4 * d + 8)
    if n:
        for size in (0, n - 1):
            assert attn(p, b, g, ws=P, ws_bytes=size) == ckv.EINVAL and "workspace" in ckv.last_error()
        assert attn(p, b, g, ws=None, ws_bytes=n) == ckv.EINVAL and "workspace" in ckv.last_error()


@pytest.mark.parametrize("max_shared", [0, 16384, 30000, 32768])
def test_own_keys_have_places_whatever_is_shared(max_shared):
    """4 decoding sequences of up to 32,768 keys in 2 groups: one that shares nothing has several places for its
    1,024 steps of 32, beside the shared keys', one per 16 steps at most."""
    b = batch(n_tokens=4, n_seqs=4, max_pages=2048, max_tokens=1, max_len=32768)
    g = groups(n_groups=2, max_tokens=2, max_shared=max_shared)
    places = need(pool(), b, g) // (4 * 28 * (4 * 128 + 8))
    assert places - (max_shared or 32768) // 512 >= 16
