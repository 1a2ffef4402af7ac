"""Steps of pages by hand-made numbers, and with some of their arrays in place."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from pages_common import DEV  # noqa: E402
from shared_common import extend_model, fork_model, select_model  # noqa: E402
from test_gpu_page_tables import dev, run_extend, tables  # noqa: E402


def test_pages_run_out_by_hand():
    """Pages of 16 tokens, 6 of them; 1 and 4 are free.  Sequence 0 is full and takes page 1; sequence 1 has
    room on its own page 2; sequences 2 and 3 hold page 3 together, half full: the first gets page 4 in its
    place, the second would need a third page and is refused, as is sequence 4, which would need two."""
    refs = np.array([1, 0, 1, 2, 0, 1])
    table = np.array([[0, -1, -1], [2, -1, -1], [3, -1, -1], [3, -1, -1], [5, -1, -1]])
    lens, n_new = np.array([16, 15, 8, 8, 16]), np.array([1, 1, 1, 1, 20])
    want = {"table": [[0, 1, -1], [2, -1, -1], [4, -1, -1], [3, -1, -1], [5, -1, -1]], "refs": [1, 1, 1, 1, 1, 1],
            "lens": [17, 16, 9, 8, 16], "tok_off": [0, 1, 2, 3, 3, 3], "copy_src": [-1, -1, 3, -1, -1],
            "copy_dst": [-1, -1, 4, -1, -1], "slots": [16, 47, 72] + [-1] * 21, "positions": [16, 15, 8] + [-1] * 21,
            "seqs": [0, 1, 2] + [-1] * 21, "counts": [3, 2, 0, 2]}
    model = extend_model(16, table, lens, refs, n_new, 24)
    for in_place in (False, True):
        got = run_extend(16, table, lens, refs, n_new, 24, in_place)
        for k in want:
            assert np.array_equal(model[k], want[k]), k
            assert np.array_equal(got[k], want[k]), k


@pytest.mark.parametrize("mix", range(8))
@pytest.mark.parametrize("kind", ["step", "more"])
def test_some_arrays_in_place(mix, kind):
    """The table, the lengths and the use counts, each in place or not."""
    import paper_2601_13631_amd as ckv
    n, width, n_pages, page = 130, 20, 5000, 16
    rng = np.random.default_rng(40 + mix)
    table, lens, refs = tables(rng, n, width, n_pages, page, over=kind == "more")
    n_new = np.ones(n, int) if kind == "step" else rng.integers(-2, width * page, n)
    n_tokens = int(np.maximum(n_new, 0).sum() * (1 if kind == "step" else 0.7))
    t, l, r = dev(table), dev(lens), dev(refs)
    out = {"table": t if mix & 1 else dev(np.full((n, width), -9)), "lens": l if mix & 2 else dev(np.full(n, -9)),
           "refs": r if mix & 4 else dev(np.full(n_pages, -9)), "tok_off": dev(np.full(n + 1, -9)),
           "copy_src": dev(np.full(n, -9)), "copy_dst": dev(np.full(n, -9)), "counts": dev(np.full(4, -9)),
           "slots": torch.full((n_tokens,), -9, dtype=torch.int64, device=DEV),
           "positions": dev(np.full(n_tokens, -9)), "seqs": dev(np.full(n_tokens, -9))}
    step = ckv.PageStep(page, t, out["table"], l, out["lens"], r, out["refs"], dev(n_new),
                        **{k: out[k] for k in ("tok_off", "copy_src", "copy_dst", "counts", "slots", "positions", "seqs")})
    ckv.page_extend(step, torch.full((ckv.page_extend_workspace_bytes(n_pages, n),), 0xFF, dtype=torch.uint8, device=DEV))
    want = extend_model(page, table, lens, refs, n_new, n_tokens)
    for k, x in out.items():
        assert (x.cpu().numpy() == np.asarray(want[k])).all(), k
    for x, before, place in ((t, table, 1), (l, lens, 2), (r, refs, 4)):
        assert mix & place or (x.cpu().numpy() == before).all()


def test_arrays_of_one_buffer():
    """Two tables in the halves of wider rows, lengths, counts, parents and a state's rows side by side: a fork
    there and back, a step on the second."""
    import paper_2601_13631_amd as ckv
    n, width, n_pages, page = 70, 33, 3000, 16
    rng = np.random.default_rng(5)
    table, lens, refs = tables(rng, n, width, n_pages, page)
    both = torch.full((n, 2 * width), -77, dtype=torch.int32, device=DEV)
    a, b = both[:, :width], both[:, width:]
    a.copy_(dev(table))
    ints = torch.zeros(3 * n + 2 * n_pages, dtype=torch.int32, device=DEV)
    la, lb, parents, ra, rb = ints.split([n, n, n, n_pages, n_pages])
    la.copy_(dev(lens))
    ra.copy_(dev(refs))
    p = rng.integers(-1, n, n)
    parents.copy_(dev(p))
    state = torch.zeros(n, 2, 50, dtype=torch.int32, device=DEV)
    state[:, 0] = torch.arange(50 * n, device=DEV).view(n, 50)
    ckv.page_fork(ckv.PageFork(page, a, b, la, lb, ra, rb, states=[(state[:, 0], state[:, 1])]), parents)
    want = fork_model(page, table, lens, refs, p)
    for x, y in zip((b, lb, rb), want):
        assert (x.cpu().numpy() == y).all()
    there = torch.from_numpy(p >= 0).to(DEV)
    assert (state[there, 1] == state[parents.long()[there], 0]).all() and (a.cpu().numpy() == table).all()
    n_new = rng.integers(0, 40, n)
    total = int(n_new.sum())
    out = torch.zeros(3 * n + 1 + 4 + 2 * total, dtype=torch.int32, device=DEV)
    off, src, dst, counts, pos, seqs = out.split([n + 1, n, n, 4, total, total])
    step = ckv.PageStep(page, b, a, lb, la, rb, rb, dev(n_new), off, src, dst, counts, positions=pos, seqs=seqs)
    ckv.page_extend(step, torch.zeros(ckv.page_extend_workspace_bytes(n_pages, n), dtype=torch.uint8, device=DEV))
    more = extend_model(page, *want, n_new, total)
    for k, x in {"table": a, "lens": la, "refs": rb, "tok_off": off, "copy_src": src, "copy_dst": dst, "counts": counts,
                 "positions": pos, "seqs": seqs}.items():
        assert (x.cpu().numpy() == np.asarray(more[k])).all(), k
    with pytest.raises(ckv.CkvError, match="overlap"):
        ckv.page_fork(ckv.PageFork(page, both[:, 1:width + 1], both[:, width:], la, lb, ra, rb), parents)
    with pytest.raises(ckv.CkvError, match="overlap"):
        ckv.page_fork(ckv.PageFork(page, a, b, la, lb, ints[3 * n:3 * n + n_pages], ints[3 * n + 1:3 * n + 1 + n_pages]), parents)


def test_a_selection_of_one_buffer():
    import paper_2601_13631_amd as ckv
    g = torch.Generator().manual_seed(8)
    logits = torch.randn(5, 3, 700, generator=g)
    scores = -torch.rand(5, 3, generator=g)
    out = torch.zeros(3 * 5 * 4 + 5 * 3, device=DEV)
    parent, token, best, given = out.split([20, 20, 20, 15])
    given.copy_(scores.reshape(-1))
    parent, token = (x.view(torch.int32).view(5, 4) for x in (parent, token))
    x = logits.to(DEV)
    ws = torch.empty(ckv.beam_select_workspace_bytes(x, 4), dtype=torch.uint8, device=DEV)
    ckv.beam_select(x, given.view(5, 3), parent, token, best.view(5, 4), ws)
    want = select_model(logits.numpy(), scores.numpy(), None, 4, -1)
    assert (parent.cpu().numpy() == want[0]).all() and (token.cpu().numpy() == want[1]).all()
    for bad in ((out[50:70], given), (out[40:60], out[59:74])):
        with pytest.raises(ckv.CkvError, match="buffers"):
            ckv.beam_select(x, bad[1].view(5, 3), parent, token, bad[0].view(5, 4), ws)
