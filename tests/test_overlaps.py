"""Forks, steps and selections refuse arrays that overlap in part, and take those that lie between each
other's rows (host only: the sizes of the calls that are not refused for it are too large to launch)."""
import itertools

import numpy as np
import pytest

import paper_2601_13631_amd as ckv
from test_shared_prefix import beams, step, tables

N, WIDTH = 1 << 20, 1 << 14          # (sequences, entries: more workgroups than a launch has)
TABLE, INTS = N * WIDTH * 4, N * 4   # bytes
G = 1 << 40                          # arrays lie this far apart
PAGES = 1000


def places(**over):
    """A fork's and a step's arrays, far apart."""
    names = ["table", "table_out", "lens", "lens_out", "refs", "refs_out", "parents", "src", "dst", "n_new", "tok_off",
             "slots", "positions", "seqs", "copy_src", "copy_dst", "counts", "ws"]
    at = {n: (i + 1) * G for i, n in enumerate(names)}
    at.update(over)
    return at


def table_struct(at, **over):
    return tables(**{**dict(n_seqs=N, n_out=N, max_pages=WIDTH, n_pages=PAGES),
                     **{k: at[k] for k in ("table", "table_out", "lens", "lens_out", "refs", "refs_out")}, **over})


def fork(at, rows=None, **over):
    states = (ckv._SeqRows * 1)(ckv._SeqRows(**{**dict(src=at["src"], dst=at["dst"], row_bytes=64, src_stride=0,
                                                       dst_stride=0), **(rows or {})}))
    return ckv._lib.ckv_page_fork(table_struct(at, **over), at["parents"], states, 1, None)


def extend(at, **over):
    s = step(n_tokens=5000, **{k: at[k] for k in ("tok_off", "slots", "positions", "seqs", "copy_src", "copy_dst", "counts")})
    return ckv._lib.ckv_page_extend(table_struct(at, **over), at["n_new"], s, at["ws"], 1 << 40, None)


SIZE = dict(table=TABLE, table_out=TABLE, lens=INTS, lens_out=INTS, refs=4 * PAGES, refs_out=4 * PAGES, parents=INTS,
            src=64 * N, dst=64 * N, n_new=INTS, tok_off=INTS + 4, slots=40000, positions=20000, seqs=20000, copy_src=INTS,
            copy_dst=INTS, counts=16, ws=ckv.page_extend_workspace_bytes(PAGES, N))
FORK = (("table_out", "lens_out", "refs_out", "dst"), ("table", "lens", "refs", "parents", "src"))
EXTEND = (("table_out", "lens_out", "refs_out", "tok_off", "slots", "positions", "seqs", "copy_src", "copy_dst", "counts",
           "ws"), ("table", "lens", "refs", "n_new"))
IN_PLACE = {("table_out", "table"), ("lens_out", "lens"), ("refs_out", "refs")}


def pairs(arrays):
    writes, reads = arrays
    return list(itertools.combinations(writes, 2)) + list(itertools.product(writes, reads))


@pytest.mark.parametrize("call,a,b", [("fork", *p) for p in pairs(FORK)] + [("extend", *p) for p in pairs(EXTEND)])
def test_overlap_in_part(call, a, b):
    """The first byte of one on the last of the other, both ways; side by side is taken."""
    run = {"fork": fork, "extend": extend}[call]
    step_ = 16  # (the workspace's alignment, and more than an element)
    at = places()
    for x, y in ((a, b), (b, a)):
        at = places()
        at[y] = at[x] + -(-SIZE[x] // step_) * step_
        assert run(at) == ckv.EUNSUPPORTED and "too large" in ckv.last_error()
        at[y] -= step_
        assert run(at) == ckv.EINVAL and "overlap" in ckv.last_error()
    if a in ("ws", "counts") or b in ("ws", "counts"):
        return
    at = places()
    at[b] = at[a]
    allowed = (a, b) in IN_PLACE and (call == "extend" or a == "refs_out")
    assert run(at) == (ckv.EUNSUPPORTED if allowed else ckv.EINVAL)


def test_nothing_overlaps():
    assert fork(places()) == extend(places()) == ckv.EUNSUPPORTED and "too large" in ckv.last_error()


def test_rows_between_rows():
    """The two tables as halves of wider rows; their last and first entries on each other."""
    at = places()
    wide = dict(table_stride=2 * WIDTH, table_out_stride=2 * WIDTH)
    for run in (fork, extend):
        for other in (WIDTH, -WIDTH, 3 * WIDTH, 2 * WIDTH * (N - 1) + WIDTH):
            assert run(places(table_out=at["table"] + 4 * other), **wide) == ckv.EUNSUPPORTED, other
        for other in (WIDTH - 1, WIDTH + 1, 1 - WIDTH, 2 * WIDTH * (N - 1) + WIDTH - 1, 2 * WIDTH * (N - 1) - WIDTH - 1):
            assert run(places(table_out=at["table"] + 4 * other), **wide) == ckv.EINVAL, other
    # strides of their own: rows of 64 bytes 128 apart, and 192 apart from 64 on
    for rows, status in ((dict(src_stride=128, dst_stride=384, dst=at["src"] + 64), ckv.EUNSUPPORTED),
                         (dict(src_stride=128, dst_stride=192, dst=at["src"] + 64), ckv.EINVAL),
                         (dict(src_stride=128, dst_stride=128, dst=at["src"] + 64), ckv.EUNSUPPORTED),
                         (dict(src_stride=128, dst_stride=128, dst=at["src"] + 65), ckv.EINVAL),
                         (dict(src_stride=1 << 50, dst_stride=1 << 50, dst=at["src"] + 64), ckv.EUNSUPPORTED)):
        assert fork(at, rows) == status, rows


@pytest.mark.parametrize("stride", [1 << 60, 1 << 61, 1 << 62, (1 << 63) - 1])
def test_strides_past_the_address_space(stride):
    """Only the first rows are anywhere."""
    at = places()
    wide = dict(table_stride=stride, table_out_stride=stride)
    for run in (fork, extend):
        assert run(at, **wide) == ckv.EUNSUPPORTED
        assert run(places(table_out=at["table"] + 4), **wide) == ckv.EINVAL and "overlap" in ckv.last_error()


@pytest.mark.parametrize("seed", range(20))
def test_overlaps_by_bytes(seed):
    """Random rows of few bytes, against the bytes themselves."""
    rng = np.random.default_rng(seed)
    for _ in range(60):
        n, m = (int(x) for x in rng.integers(1, 9, 2))
        size = int(rng.integers(1, 30))
        sa, sb = (int(x) for x in size + rng.integers(0, 40, 2))
        d = int(rng.integers(-300, 300))
        taken = [{o + i * s + x for i in range(k) for x in range(size)} for o, k, s in ((0, n, sa), (d, m, sb))]
        # (rows of 2^40 bytes of another state make the call too large)
        t = table_struct(places(), n_seqs=n, n_out=m, max_pages=10)
        states = (ckv._SeqRows * 2)(ckv._SeqRows(src=50 * G, dst=50 * G + d, row_bytes=size, src_stride=sa, dst_stride=sb),
                                    ckv._SeqRows(src=60 * G, dst=80 * G, row_bytes=1 << 40, src_stride=0, dst_stride=0))
        want = ckv.EINVAL if d == 0 or taken[0] & taken[1] else ckv.EUNSUPPORTED
        assert ckv._lib.ckv_page_fork(t, 40 * G, states, 2, None) == want, (n, m, size, sa, sb, d)


@pytest.mark.parametrize("a,b", [(x, y) for x in ("parent", "token", "score", "done_out", "ws") for y in
                                 ("parent", "token", "score", "done_out", "ws", "logits", "scores", "done") if x < y or
                                 y in ("logits", "scores", "done")])
def test_selections(a, b):
    names = ["parent", "token", "score", "done_out", "ws", "logits", "scores", "done"]
    at = {n: (i + 1) * G for i, n in enumerate(names)}
    b_ = beams(n_reqs=100, keep=6, eos=3, done=G, scores=G)
    size = dict(parent=2400, token=2400, score=2400, done_out=600, logits=400 * 2000, scores=1600, done=400,
                ws=ckv._lib.ckv_beam_select_workspace_bytes(b_))
    at[b] = at[a] + size[a] // 16 * 16 - 16
    if b == "ws" or a == "ws":
        at["ws"] = at["ws"] // 16 * 16
    s = beams(n_reqs=100, keep=6, eos=3, logits=at["logits"], scores=at["scores"], done=at["done"])
    assert ckv._lib.ckv_beam_select(s, at["parent"], at["token"], at["score"], at["done_out"], at["ws"], size["ws"],
                                    None) == ckv.EINVAL
    assert "buffers" in ckv.last_error()
