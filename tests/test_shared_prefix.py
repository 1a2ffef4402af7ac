"""The calls of a step over shared prefixes refuse what they cannot do before anything is launched (host only)."""
import pytest
import torch

import paper_2601_13631_amd as ckv
from test_pages import BAD_BATCHES, BAD_POOLS, P, batch, pool


def groups(**over):
    d = dict(grp_off=P, shared=P, n_groups=2, max_tokens=0, max_shared=0)
    d.update(over)
    return ckv._PageGroups(**d)


def tables(**over):
    d = dict(table=P, table_out=2 * P, lens=P, lens_out=2 * P, refs=P, refs_out=2 * P, table_stride=0,
             table_out_stride=0, n_pages=100, n_seqs=4, n_out=4, max_pages=10, page_size=16)
    d.update(over)
    return ckv._PageTables(**d)


def step(**over):
    d = dict(tok_off=P, slots=P, positions=P, seqs=P, copy_src=P, copy_dst=P, counts=P, n_tokens=8)
    d.update(over)
    return ckv._PageStep(**d)


def beams(**over):
    d = dict(logits=P, scores=P, done=None, row_stride=0, n_reqs=2, n_beams=4, vocab=1000, keep=4, eos=-1,
             dtype=ckv.DTYPE_BF16)
    d.update(over)
    return ckv._Beams(**d)


def share(b, g, page=16):
    return ckv._lib.ckv_page_share(page, b, g, None)


def attn(p, b, g, q=P, hq=28, sm=0.0, out=P, ws=None, ws_bytes=0):
    return ckv._lib.ckv_page_attn_shared(p, b, g, q, hq, sm, out, ws, ws_bytes, None)


BAD_GROUPS = [dict(grp_off=None), dict(shared=None), dict(n_groups=-1), dict(n_groups=(1 << 20) + 1),
              dict(max_tokens=-1), dict(max_shared=-1)]


@pytest.mark.parametrize("over,status", BAD_POOLS)
def test_bad_pools(over, status):
    assert attn(pool(**over), batch(), groups()) == status and ckv.last_error()


@pytest.mark.parametrize("over,status", BAD_BATCHES)
def test_bad_batches(over, status):
    assert attn(pool(), batch(**over), groups()) == status
    assert share(batch(**over), groups()) == status and ckv.last_error()


@pytest.mark.parametrize("over", BAD_GROUPS)
def test_bad_groups(over):
    assert attn(pool(), batch(), groups(**over)) == ckv.EINVAL
    assert share(batch(), groups(**over)) == ckv.EINVAL and ckv.last_error()


def test_bad_attention():
    assert attn(None, batch(), groups()) == attn(pool(), None, groups()) == attn(pool(), batch(), None) == ckv.EINVAL
    assert share(None, groups()) == share(batch(), None) == ckv.EINVAL
    for page, status in ((0, ckv.EINVAL), (-8, ckv.EINVAL), (24, ckv.EUNSUPPORTED)):
        assert share(batch(), groups(), page) == status
    assert share(batch(max_pages=1 << 27), groups()) == ckv.EUNSUPPORTED
    for hq in (0, -4, 6):
        assert attn(pool(), batch(), groups(), hq=hq) == ckv.EINVAL
    for over in (dict(q=None), dict(out=None), dict(q=P + 4), dict(out=P + 8), dict(ws=P + 4)):
        assert attn(pool(), batch(), groups(), **over) == ckv.EINVAL
    for sm in (-1.0, float("nan"), float("inf")):
        assert attn(pool(), batch(), groups(), sm=sm) == ckv.EINVAL
    assert attn(pool(), batch(n_tokens=1 << 27), groups()) == ckv.EUNSUPPORTED
    # parts need their workspace, a batch that shares little as much as page_attn
    long = batch(n_tokens=64, n_seqs=64, max_pages=10000, max_tokens=1)
    g = groups(max_tokens=64)
    need = ckv._lib.ckv_page_attn_shared_workspace_bytes(pool(), long, g, 28)
    assert need > 0
    assert attn(pool(), long, g) == ckv.EINVAL and "workspace" in ckv.last_error()
    assert attn(pool(), long, g, ws=P, ws_bytes=need - 1) == ckv.EINVAL
    few = batch(n_tokens=4, n_seqs=4, max_pages=10000, max_tokens=1, max_len=200)
    for b, grp in ((few, groups()), (long, groups(n_groups=0)), (long, groups(n_groups=64))):
        assert (ckv._lib.ckv_page_attn_shared_workspace_bytes(pool(), b, grp, 28)
                == ckv._lib.ckv_page_attn_workspace_bytes(pool(), b, 28, 0, 0))
    assert ckv._lib.ckv_page_attn_shared_workspace_bytes(pool(), long, groups(n_groups=-1), 28) == 0
    assert ckv._lib.ckv_page_attn_shared_workspace_bytes(pool(head_dim=96), long, g, 28) == 0


def test_workspace_bytes_hold_for_any_hints():
    """Hints choose kernels, and a batch of any size gets a workspace that fits them."""
    for hints in (dict(), dict(max_tokens=1, max_len=5), dict(max_tokens=1 << 30, max_len=1 << 30)):
        for over in (dict(), dict(max_tokens=1, max_shared=1), dict(max_tokens=1 << 30, max_shared=1 << 30)):
            b = batch(n_tokens=300, n_seqs=100, max_pages=4000, **hints)
            assert ckv._lib.ckv_page_attn_shared_workspace_bytes(pool(), b, groups(**over), 28) < 1 << 32


BAD_TABLES = [
    (dict(table=None), ckv.EINVAL), (dict(table_out=None), ckv.EINVAL), (dict(lens=None), ckv.EINVAL),
    (dict(lens_out=None), ckv.EINVAL), (dict(refs=None), ckv.EINVAL), (dict(refs_out=None), ckv.EINVAL),
    (dict(table_stride=9), ckv.EINVAL), (dict(table_out_stride=9), ckv.EINVAL), (dict(n_pages=0), ckv.EINVAL),
    (dict(n_pages=1 << 31), ckv.EINVAL), (dict(n_pages=(1 << 26) + 1), ckv.EUNSUPPORTED), (dict(n_seqs=-1), ckv.EINVAL),
    (dict(n_seqs=(1 << 20) + 1), ckv.EINVAL), (dict(n_out=-1), ckv.EINVAL), (dict(max_pages=0), ckv.EINVAL),
    (dict(max_pages=(1 << 26) + 1), ckv.EUNSUPPORTED), (dict(page_size=0), ckv.EINVAL),
    (dict(page_size=12), ckv.EUNSUPPORTED),
]


@pytest.mark.parametrize("over,status", BAD_TABLES)
def test_bad_tables(over, status):
    t = tables(**over)
    assert ckv._lib.ckv_page_fork(t, P, None, 0, None) == status and ckv.last_error()
    assert ckv._lib.ckv_page_extend(t, P, step(), P, 1 << 40, None) == status


def test_bad_forks():
    def fork(t=tables(), parents=P, rows=(), n=None):
        c = (ckv._SeqRows * max(len(rows), 1))(*rows)
        return ckv._lib.ckv_page_fork(t, parents, c if rows else None, len(rows) if n is None else n, None)

    def rows(**over):
        return ckv._SeqRows(**{**dict(src=P, dst=2 * P, row_bytes=64, src_stride=0, dst_stride=0), **over})
    assert fork(parents=None) == ckv.EINVAL and fork(n=1) == ckv.EINVAL and fork(n=-1) == ckv.EINVAL
    assert fork(rows=[rows()] * 9) == ckv.EINVAL
    for over in (dict(src=None), dict(dst=None), dict(dst=P), dict(row_bytes=0), dict(src_stride=63), dict(dst_stride=1)):
        assert fork(rows=[rows(), rows(**over)]) == ckv.EINVAL and ckv.last_error()
    assert fork(tables(table_out=P)) == ckv.EINVAL and fork(tables(lens_out=P)) == ckv.EINVAL


def test_bad_steps():
    need = ckv.page_extend_workspace_bytes(100, 4)
    assert need > 0 and ckv.page_extend_workspace_bytes(0, 4) == 0

    def extend(t=tables(), n_new=P, ws=P, ws_bytes=need, **over):
        return ckv._lib.ckv_page_extend(t, n_new, step(**over), ws, ws_bytes, None)
    for over in (dict(tok_off=None), dict(copy_src=None), dict(copy_dst=None), dict(counts=None), dict(n_tokens=-1),
                 dict(n_tokens=1 << 31), dict(n_new=None), dict(ws=None), dict(ws=P + 4), dict(ws_bytes=need - 1),
                 dict(t=tables(n_out=5)), dict(t=tables(table_out=P, table_out_stride=11))):
        assert extend(**over) == ckv.EINVAL and ckv.last_error()


BAD_BEAMS = [
    (dict(logits=None), ckv.EINVAL), (dict(scores=None), ckv.EINVAL), (dict(logits=P + 1), ckv.EINVAL),
    (dict(row_stride=999), ckv.EINVAL), (dict(n_reqs=-1), ckv.EINVAL), (dict(n_reqs=(1 << 20) + 1), ckv.EINVAL),
    (dict(n_beams=0), ckv.EINVAL), (dict(n_beams=65), ckv.EUNSUPPORTED), (dict(keep=0), ckv.EINVAL),
    (dict(keep=65), ckv.EUNSUPPORTED), (dict(vocab=0), ckv.EINVAL), (dict(vocab=(1 << 30) + 1), ckv.EUNSUPPORTED),
    (dict(eos=1000), ckv.EINVAL), (dict(eos=-2), ckv.EINVAL), (dict(done=P), ckv.EINVAL),
    (dict(dtype=ckv.DTYPE_E4M3), ckv.EINVAL), (dict(n_reqs=1 << 18, n_beams=8), ckv.EUNSUPPORTED),
]


@pytest.mark.parametrize("over,status", BAD_BEAMS)
def test_bad_beams(over, status):
    assert ckv._lib.ckv_beam_select(beams(**over), P, P, P, P, P, 1 << 40, None) == status and ckv.last_error()


def test_bad_select():
    need = ckv._lib.ckv_beam_select_workspace_bytes(beams())
    assert need > 0 and ckv._lib.ckv_beam_select_workspace_bytes(beams(keep=65)) == 0
    Q = 2 * P
    for args in ((None, P, Q, P, P, need), (P, None, Q, P, P, need), (P, P, None, P, P, need), (P, P, Q, P, None, need),
                 (P, P, Q, P, P, need - 1), (P, P, Q, P, P + 8, need)):
        parent, token, score, done, ws, nbytes = args
        assert ckv._lib.ckv_beam_select(beams(), parent, token, score, done, ws, nbytes, None) == ckv.EINVAL
    assert ckv._lib.ckv_beam_select(None, P, P, P, P, P, need, None) == ckv.EINVAL
    # outputs in the inputs' buffers
    for over, score, done in ((dict(scores=P), P, 2 * P), (dict(scores=P, done=2 * P, eos=3), 3 * P, 2 * P)):
        assert ckv._lib.ckv_beam_select(beams(**over), P, P, score, done, P, need, None) == ckv.EINVAL
        assert "buffers" in ckv.last_error()
    for eos in (-2, 1 << 31, 1 << 40):
        with pytest.raises(ValueError, match="eos"):
            ckv._beams(torch.zeros(1, 2, 30), 2, eos=eos)


def test_nothing_to_do():
    for b in (batch(n_seqs=0), batch(n_tokens=0), batch(n_seqs=0, table=None, lens=None, tok_off=None)):
        assert share(b, groups()) == ckv.OK and attn(pool(), b, groups()) == ckv.OK
    assert share(batch(), groups(n_groups=0, grp_off=None, shared=None)) == ckv.OK
    assert ckv._lib.ckv_beam_select(beams(n_reqs=0, logits=None, scores=None), None, None, None, None, None, 0, None) == ckv.OK


def test_handles_refuse_host_tensors():
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        ckv.PageGroups(i(3), i(20))
    with pytest.raises(ValueError):
        ckv.PageFork(16, i(4, 3), i(4, 3), i(4), i(4), i(9), i(9))
    with pytest.raises(ValueError):
        ckv.PageStep(16, i(4, 3), i(4, 3), i(4), i(4), i(9), i(9), i(4), i(5), i(4), i(4), i(4))
    with pytest.raises(ValueError):
        ckv.beam_select(torch.zeros(1, 2, 30), torch.zeros(1, 2), i(1, 2), i(1, 2), torch.zeros(1, 2), None)
    for bad in (torch.zeros(2, 30), torch.zeros(1, 2, 30).double(), torch.zeros(1, 30, 2).transpose(1, 2),
                torch.zeros(1, 1, 30).expand(1, 2, 30), torch.zeros(3, 2, 90)[:, :, :30].transpose(0, 1)):
        with pytest.raises(ValueError):
            ckv.beam_select_workspace_bytes(bad, 2)
