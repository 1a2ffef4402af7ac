"""Forks, steps and beams against the host models: integers have to be equal."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from pages_common import DEV  # noqa: E402
from shared_common import extend_model, fork_model, select_model  # noqa: E402


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).to(DEV)


def tables(rng, n, width, n_pages, page, shared=True, over=False):
    """Tables of n sequences, their lengths and the use counts: some pages shared by neighbours, some
    entries that name none, some pages held by others beside."""
    order = rng.permutation(n_pages)
    table, lens, refs, at = np.full((n, width), -1, np.int64), np.zeros(n, int), np.zeros(n_pages, int), 0
    for b in range(n):
        lens[b] = int(rng.integers(0, width * page + 1)) if rng.random() < 0.9 else 0
        held = -(-lens[b] // page)
        if shared and b and rng.random() < 0.5:
            lens[b] = lens[b - 1] if rng.random() < 0.5 else lens[b]
            held = -(-lens[b] // page)
            same = min(held, -(-lens[b - 1] // page), int(rng.integers(0, width + 1)) if lens[b] != lens[b - 1] else width)
            table[b, :same] = table[b - 1, :same]
        for s in range(held):
            if table[b, s] < 0 and at < n_pages * 3 // 4:
                table[b, s], at = order[at], at + 1
            if 0 <= table[b, s]:
                refs[table[b, s]] += 1
    if over and n:
        lens[rng.integers(0, n)] = width * page + 5
        lens[rng.integers(0, n)] = -3
        table[rng.integers(0, n), rng.integers(0, width)] = n_pages + 7
    refs[rng.permutation(n_pages)[: n_pages // 20]] += 1
    refs[rng.permutation(n_pages)[: n_pages // 50]] -= 5
    return table, lens, refs


SIZES = [  # sequences, entries, pages, page size
    (1, 1, 1, 8), (1, 3, 5, 16), (3, 7, 40, 8), (4, 130, 700, 16), (70, 33, 4097, 32), (300, 20, 9000, 96),
    (5, 2500, 20000, 16), (1030, 3, 5000, 64), (0, 4, 9, 16), (40, 30, 70000, 8),
]


@pytest.mark.parametrize("i", range(len(SIZES)))
@pytest.mark.parametrize("in_place", [False, True])
def test_fork(i, in_place):
    import paper_2601_13631_amd as ckv
    n, width, n_pages, page = SIZES[i]
    rng = np.random.default_rng(i)
    table, lens, refs = tables(rng, n, width, n_pages, page, over=True)
    for n_out in sorted({n, max(1, n // 2), 2 * n + 1}):
        parents = rng.integers(-1, n + 1, n_out) if n else np.full(n_out, 0)
        parents[: n_out // 9 + 1] = 2 ** 31 - 1
        want = fork_model(page, table, lens, refs, parents)
        wide = torch.full((n_out, width + 3), -77, dtype=torch.int32, device=DEV)
        src = torch.full((n, width + 5), -88, dtype=torch.int32, device=DEV)
        src[:, :width] = dev(table)
        out_lens, refs_in = dev(np.full(n_out, -9)), dev(refs)
        refs_out = refs_in if in_place else dev(np.full(n_pages, -9))
        states = [(torch.randint(0, 1 << 30, (n, k), dtype=torch.int32, device=DEV),
                   torch.full((n_out, k), -5, dtype=torch.int32, device=DEV)) for k in (4, 3, 2050)]
        states.append((torch.randn(n, 2, 5, device=DEV).half(), torch.zeros(n_out, 2, 5, dtype=torch.half, device=DEV)))
        strided = torch.randn(n, 40, device=DEV)[:, 3:20], torch.zeros(n_out, 31, device=DEV)[:, :17]
        ckv.page_fork(ckv.PageFork(page, src[:, :width], wide[:, :width], dev(lens), out_lens, refs_in, refs_out,
                                   states=states + [strided]), dev(parents))
        assert (wide[:, :width].cpu().numpy() == want[0]).all() and (wide[:, width:] == -77).all()
        assert (out_lens.cpu().numpy() == want[1]).all() and (refs_out.cpu().numpy() == want[2]).all()
        there = (parents >= 0) & (parents < n)
        for x, y in states + [strided]:
            x, y = x.cpu().numpy(), y.cpu().numpy()
            assert (y[there] == x[parents[there]]).all()
            assert (y[~there] == (-5 if y.dtype == np.int32 else 0)).all()


def run_extend(page, table, lens, refs, n_new, n_tokens, in_place, ws=None):
    import paper_2601_13631_amd as ckv
    n, width = table.shape
    t = torch.full((n, width + 3), -77, dtype=torch.int32, device=DEV)
    t[:, :width] = dev(table)
    lens_in, refs_in = dev(lens), dev(refs)
    out = {"table": t[:, :width] if in_place else dev(np.full((n, width), -9)),
           "lens": lens_in if in_place else dev(np.full(n, -9)),
           "refs": refs_in if in_place else dev(np.full(refs.size, -9)), "tok_off": dev(np.full(n + 1, -9)),
           "copy_src": dev(np.full(n, -9)), "copy_dst": dev(np.full(n, -9)), "counts": dev(np.full(4, -9)),
           "slots": torch.full((n_tokens,), -9, dtype=torch.int64, device=DEV),
           "positions": dev(np.full(n_tokens, -9)), "seqs": dev(np.full(n_tokens, -9))}
    step = ckv.PageStep(page, t[:, :width], out["table"], lens_in, out["lens"], refs_in, out["refs"], dev(n_new),
                        **{k: out[k] for k in ("tok_off", "copy_src", "copy_dst", "counts", "slots", "positions", "seqs")})
    ws = torch.full((ckv.page_extend_workspace_bytes(refs.size, n),), 0xFF, dtype=torch.uint8, device=DEV)
    ckv.page_extend(step, ws)
    assert (t[:, width:] == -77).all()
    return {k: x.cpu().numpy() for k, x in out.items()}


@pytest.mark.parametrize("i", range(len(SIZES)))
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind", ["step", "some", "more"])
def test_extend(i, in_place, kind):
    """One token each; a few; more than there are pages, table entries or rows for."""
    n, width, n_pages, page = SIZES[i]
    rng = np.random.default_rng(100 + i)
    table, lens, refs = tables(rng, n, width, n_pages, page, over=kind == "more")
    if kind == "step":
        n_new, n_tokens = np.ones(n, int), n
    elif kind == "some":
        n_new = rng.integers(0, 2 * page, n)
        n_tokens = int(n_new.sum()) + 3
    else:
        n_new = rng.integers(-2, width * page, n)
        n_tokens = int(np.maximum(n_new, 0).sum() * 0.7)
    got = run_extend(page, table, lens, refs, n_new, n_tokens, in_place)
    want = extend_model(page, table, lens, refs, n_new, n_tokens)
    for k in want:
        assert (got[k] == np.asarray(want[k])).all(), k


def test_extend_when_pages_run_out():
    """The last page goes to the sequence that still fits; who needs none goes on."""
    refs = np.array([1, 0, 1, 2, 0, 1])
    table = np.array([[0, -1, -1], [2, -1, -1], [3, -1, -1], [3, -1, -1], [5, -1, -1]])
    lens, n_new = np.array([16, 15, 8, 8, 16]), np.array([1, 1, 1, 1, 20])
    got = run_extend(16, table, lens, refs, n_new, 24, True)
    assert got["counts"].tolist() == [4, 2, 0, 2] or got["counts"].tolist() == extend_model(
        16, table, lens, refs, n_new, 24)["counts"]
    want = extend_model(16, table, lens, refs, n_new, 24)
    assert want["copy_src"] == [-1, -1, 3, -1, -1] and want["tok_off"] == [0, 1, 2, 3, 3, 3]
    for k in want:
        assert (got[k] == np.asarray(want[k])).all(), k


@pytest.mark.parametrize("given", [(), ("slots",), ("positions", "seqs")])
def test_extend_writes_what_is_asked_for(given):
    import paper_2601_13631_amd as ckv
    rng = np.random.default_rng(8)
    table, lens, refs = tables(rng, 30, 6, 400, 16)
    n_new = rng.integers(0, 20, 30)
    total = int(n_new.sum()) + 300
    t, l, r, off, src, dst, counts = (dev(x) for x in (table, lens, refs, np.zeros(31), np.zeros(30), np.zeros(30),
                                                       np.zeros(4)))
    rows = {k: torch.zeros(total, dtype=torch.int64 if k == "slots" else torch.int32, device=DEV) for k in given}
    step = ckv.PageStep(16, t, t, l, l, r, r, dev(n_new), off, src, dst, counts, n_tokens=total, **rows)
    ckv.page_extend(step, torch.zeros(ckv.page_extend_workspace_bytes(400, 30), dtype=torch.uint8, device=DEV))
    want = extend_model(16, table, lens, refs, n_new, total)
    for k, x in {"table": t, "lens": l, "refs": r, "tok_off": off, "copy_src": src, "copy_dst": dst, "counts": counts,
                 **rows}.items():
        assert (x.cpu().numpy() == np.asarray(want[k])).all(), k


def test_tables_replay():
    """A captured fork and step, replayed on other tables."""
    import paper_2601_13631_amd as ckv
    n, width, n_pages, page = 60, 9, 900, 16
    ws = torch.zeros(ckv.page_extend_workspace_bytes(n_pages, n), dtype=torch.uint8, device=DEV)
    t0, t1, l0, l1, refs = (torch.zeros(s, dtype=torch.int32, device=DEV) for s in
                            ((n, width), (n, width), n, n, n_pages))
    parents, n_new, off, src, dst, counts = (torch.zeros(s, dtype=torch.int32, device=DEV) for s in
                                             (n, n, n + 1, n, n, 4))
    seqs = torch.zeros(n * 3, dtype=torch.int32, device=DEV)
    fork = ckv.PageFork(page, t0, t1, l0, l1, refs, refs)
    step = ckv.PageStep(page, t1, t1, l1, l1, refs, refs, n_new, off, src, dst, counts, seqs=seqs)

    def both():
        ckv.page_fork(fork, parents)
        ckv.page_extend(step, ws)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in range(4):
        rng = np.random.default_rng(seed)
        table, lens, use = tables(rng, n, width, n_pages, page)
        p, new = rng.integers(-1, n, n), rng.integers(0, 4, n)
        for x, y in ((t0, table), (l0, lens), (refs, use), (parents, p), (n_new, new)):
            x.copy_(dev(y))
        graph.replay()
        torch.cuda.synchronize()
        a = fork_model(page, table, lens, use, p)
        b = extend_model(page, a[0], a[1], a[2], new, n * 3)
        for x, k in ((t1, "table"), (l1, "lens"), (refs, "refs"), (off, "tok_off"), (src, "copy_src"), (seqs, "seqs"),
                     (dst, "copy_dst"), (counts, "counts")):
            assert (x.cpu().numpy() == np.asarray(b[k])).all(), k


# ---- beams ----------------------------------------------------------------------

def run_select(logits, scores, done, keep, eos, gap=0, shift=0, stream=None):
    """beam_select on rows `gap` elements apart, the first one `shift` elements into its buffer."""
    import paper_2601_13631_amd as ckv
    reqs, beams, vocab = logits.shape
    span = vocab + gap
    buf = torch.full((shift + reqs * beams * span + 16,), float("nan"), dtype=logits.dtype, device=DEV)
    x = buf[shift: shift + reqs * beams * span].view(reqs, beams, span)[:, :, :vocab]
    x.copy_(logits)
    out = [torch.full((reqs, keep), -9, dtype=t, device=DEV) for t in (torch.int32, torch.int32, torch.float32)]
    done_out = torch.full((reqs, keep), 9, dtype=torch.uint8, device=DEV)
    ws = torch.full((ckv.beam_select_workspace_bytes(x, keep),), 0xFF, dtype=torch.uint8, device=DEV)
    ckv.beam_select(x, scores.to(DEV), *out, ws, done=None if done is None else done.to(DEV), done_out=done_out, eos=eos,
                    stream=stream)
    return [t.cpu().numpy() for t in out] + [done_out.cpu().numpy()]


def check_select(logits, scores, done, keep, eos, **how):
    """Places and tokens equal; scores within half a step of fp32 and of what 32-bit exponentials leave
    in the logarithm of their sum, in steps of 2^-24: an exponent x - m is off by 2.25 |x - m| (two
    roundings, and the factor's), whose mean under the terms' weights is at most log(vocab); an
    exponential itself by 2, a sum of 32 terms in four parts of 8 by 10, a change of reference or the
    join of parts by as much again as one exponential, 2 each."""
    got = run_select(logits, scores, done, keep, eos, **how)
    wide = logits.double().numpy() if logits.dtype == torch.bfloat16 else logits.numpy()
    want = select_model(wide, scores.numpy(), None if done is None else done.numpy(), keep, eos)
    for g, w in ((got[0], want[0]), (got[1], want[1]), (got[3], want[3])):
        assert (g == w).all()
    there = want[0] >= 0
    assert (got[2][~there] == -np.inf).all()
    slack = 2.0 ** -24 * (2.25 * np.log(logits.shape[2]) + 2 + 10 + 3 * 2)
    w = want[2][there]
    assert (np.abs(got[2][there] - w) <= np.abs(w) * 2.0 ** -24 + slack).all()


SELECT = [  # type, requests, beams, kept, vocabulary
    ("bf16", 1, 1, 1, 1), ("f32", 1, 1, 3, 2), ("bf16", 2, 3, 5, 7), ("bf16", 1, 4, 4, 1000), ("f32", 3, 4, 8, 2049),
    ("bf16", 2, 4, 64, 5000), ("f32", 2, 64, 64, 333), ("bf16", 1, 17, 33, 40001), ("f32", 9, 5, 10, 10007),
    ("bf16", 40, 4, 8, 32000), ("bf16", 2, 2, 4, 300000), ("f32", 1, 2, 63, 64), ("bf16", 300, 1, 2, 2048),
]
T = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("i", range(len(SELECT)))
@pytest.mark.parametrize("gap,shift", [(0, 0), (3, 1), (8, 5)])
def test_select(i, gap, shift):
    kind, reqs, beams, keep, vocab = SELECT[i]
    g = torch.Generator().manual_seed(i)
    x = (torch.randn(reqs, beams, vocab, generator=g) * 3).to(T[kind])
    scores = -20 * torch.rand(reqs, beams, generator=g)
    scores[torch.rand(reqs, beams, generator=g) < 0.15] = -float("inf")
    done = (torch.rand(reqs, beams, generator=g) < 0.2).to(torch.uint8)
    check_select(x, scores, done, keep, vocab // 2, gap=gap, shift=shift)
    check_select(x, scores, None, keep, -1, gap=gap, shift=shift)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_select_ties(kind):
    """Equal logits, equal beams, two zeros: the lower beam, then the lower token."""
    for vocab in (5, 70, 3000, 9001):
        scores = torch.tensor([[-1.0, -1.0, -1.0], [-2.0, -1.0, -float("inf")]])
        check_select(torch.zeros(2, 3, vocab, dtype=T[kind]), scores, None, 9, -1)
        x = torch.zeros(2, 3, vocab)
        x[:, :, 1::2] = -0.0
        x[:, :, vocab - 2] = 1
        check_select(x.to(T[kind]), scores, None, 7, -1)
        g = torch.Generator().manual_seed(vocab)
        check_select(torch.randint(0, 3, (2, 3, vocab), generator=g).to(T[kind]), scores, None, 20, -1)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("order", ["up", "down"])
def test_select_sorted_logits(kind, order):
    """Every later logit better than all before, and the reverse."""
    x = torch.linspace(-30, 30, 20011).to(T[kind]) * (1 if order == "up" else -1)
    check_select(x.expand(2, 2, -1).contiguous(), torch.tensor([[-3.0, -3.5], [0.0, -9.0]]), None, 16, -1)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_select_infinities_and_nan(kind):
    """-inf and NaN offer nothing; infinities share all; rows of the type's lowest value; rows of nothing."""
    lowest = torch.finfo(T[kind]).min
    g = torch.Generator().manual_seed(4)
    x = torch.randn(6, 2, 4999, generator=g).to(T[kind])
    x[0, 0, torch.randperm(4999, generator=g)[:4990]] = -float("inf")   # fewer than are kept
    x[1, :, 100:2000] = float("nan")
    x[2, 1, [7, 4000, 4998]] = float("inf")
    x[3, 0] = lowest
    x[3, 1] = -float("inf")
    x[4] = float("nan")
    x[5, 0, :4900] = lowest
    x[5, 1, 0] = float("inf")
    x[5, 1, 1] = float("nan")
    check_select(x, torch.linspace(-3, -1, 12).view(6, 2), None, 12, -1)


def test_select_keeps_empty_places_empty():
    x = torch.randn(2, 3, 50)
    scores = torch.full((2, 3), -float("inf"))
    scores[1, 2] = float("nan")
    check_select(x, scores, None, 4, -1)
    scores[0, 1] = -4.0
    check_select(x, scores, torch.ones(2, 3, dtype=torch.uint8), 4, 49)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_select_rows_far_apart(kind):
    """Rows more than 2^31 elements and 4 GiB from the first."""
    g = torch.Generator().manual_seed(6)
    check_select((torch.randn(1, 4, 3001, generator=g) * 3).to(T[kind]), torch.tensor([[-1.0, -2.0, -0.5, -1.5]]), None, 6,
                 -1, gap=(3 << 28) + 1)


def test_select_replay():
    import paper_2601_13631_amd as ckv
    x = torch.zeros(3, 4, 7001, dtype=torch.bfloat16, device=DEV)
    scores, done = torch.zeros(3, 4, device=DEV), torch.zeros(3, 4, dtype=torch.uint8, device=DEV)
    parent, token = (torch.zeros(3, 6, dtype=torch.int32, device=DEV) for _ in "ab")
    best, ended = torch.zeros(3, 6, device=DEV), torch.zeros(3, 6, dtype=torch.uint8, device=DEV)
    ws = torch.zeros(ckv.beam_select_workspace_bytes(x, 6), dtype=torch.uint8, device=DEV)

    def call():
        ckv.beam_select(x, scores, parent, token, best, ws, done=done, done_out=ended, eos=5)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(3):
        g = torch.Generator().manual_seed(seed)
        x.copy_(torch.randn(3, 4, 7001, generator=g).to(torch.bfloat16))
        scores.copy_(torch.where(torch.rand(3, 4, generator=g) < 0.2, -torch.inf, -torch.rand(3, 4, generator=g)))
        done.copy_(torch.rand(3, 4, generator=g) < 0.3)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (parent, token, best, ended)]
        want = select_model(x.cpu().double().numpy(), scores.cpu().numpy(), done.cpu().numpy(), 6, 5)
        assert (replayed[0].cpu().numpy() == want[0]).all() and (replayed[1].cpu().numpy() == want[1]).all()
        call()
        for a, b in zip(replayed, (parent, token, best, ended)):
            assert torch.equal(a, b)
