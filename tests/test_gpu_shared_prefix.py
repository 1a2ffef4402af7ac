"""Attention of groups that share their first pages, against the host model in 64 bits; what a
group shares; the calls of a decoding step together."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from pages_common import DEV, attend, check_attention  # noqa: E402
from shared_common import GroupCache, attend_shared, extend_model, fork_model, select_model  # noqa: E402

H05, H7, H14, HF, H1 = (14, 2, 64), (28, 4, 128), (40, 8, 128), (4, 1, 64), (3, 3, 64)
ONE = (1, 5)

# (cache, heads, page, groups, sequences before them that are in none)
CASES = [
    ("bf16", H7, 16, [(64, [ONE] * 4)], []),
    ("bf16", H7, 32, [(4000, [(1, 1 + 37 * i) for i in range(9)])], []),         # many splits
    ("bf16", H05, 8, [(1000, [ONE] * 3), (77, [(1, 300), (1, 1)])], [(1, 40), (1, 1)]),
    ("bf16", H14, 96, [(500, [(1, 3), (1, 200)]), (96, [ONE]), (0, [(1, 10), (1, 90)])], []),
    ("bf16", H1, 64, [(640, [(3, 3), (1, 64), (2, 130)])], [(5, 5)]),
    ("bf16", H7, 64, [(700, [(37, 40), (1, 300), (0, 90), (130, 180), (5, 64)])], []),   # ragged, one idle
    ("bf16", H7, 16, [(300, [(0, 20), (0, 3)]), (300, [(0, 20), (1, 20), (1, 4)])], []),  # nobody; an idle leader
    ("bf16", H7, 32, [(320, [(1, 0)] * 3)], []),                                  # no keys of their own
    ("bf16", H7, 32, [(320, [(40, 0), (1, 0)])], []),                             # queries inside the shared pages
    ("bf16", H7, 16, [(1, [(1, 0)] * 3), (16, [(1, 0)] * 2), (31, [(1, 1)] * 2)], []),
    ("bf16", H05, 16, [(2000, [(1, 17)] * 2)], []),                               # 14 rows
    ("bf16", H7, 16, [(2000, [(1, 9)] * 4), (1500, [(1, 3)] * 5)], []),           # 28 and 35 rows
    ("bf16", H7, 16, [(900, [(1, 9)] * 8), (2500, [(1, 30)] * 9)], []),           # 56 and 63 rows
    ("bf16", H7, 16, [(1200, [(2, 9)] * 12), (60, [(1, 3)] * 2)], []),            # 168 rows
    ("bf16", (16, 1, 128), 32, [(3000, [(1, 40)] * 3)], []),                      # 48 rows of one head
    ("bf16", (20, 1, 64), 8, [(777, [(1, 40)] * 3)], []),
    ("e4m3", H7, 16, [(64, [ONE] * 4)], [(1, 900)]),
    ("e4m3", H14, 8, [(2000, [(1, 9)] * 8), (333, [(2, 77), (5, 5)])], []),       # 40 rows
    ("e4m3", H05, 32, [(1000, [(19, 30), (1, 3)])], []),
    ("e4m3", H05, 8, [(4000, [(1, 1 + i) for i in range(9)])], []),               # 63 rows
    ("e4m3", H7, 96, [(3000, [(1, 30)] * 2)], []),
    ("e4m3", H7, 64, [(500, [(140, 150), (0, 3), (70, 70)])], [(3, 70)]),
    ("e4m3", (5, 5, 64), 16, [(200, [(1, 7)] * 5)], []),
    ("f32", HF, 16, [(1024, [(1, 1), (1, 100), (1, 20)])], [(1, 3)]),
    ("f32", (4, 2, 64), 32, [(500, [(9, 9), (33, 64)]), (64, [(1, 0)] * 2)], []),
    ("f32", HF, 8, [(3000, [(1, 5)] * 9)], []),
    ("f32", (20, 1, 64), 96, [(1000, [(1, 5)] * 2)], []),
]
# a table this wide, of a length that is not known, says that shared pages may be many
WIDE = 1 << 18


@pytest.mark.parametrize("hints", ["exact", "wide", "rows", "wrong"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_attention(i, hints):
    cache, heads, page, groups, loose = CASES[i]
    c = GroupCache(cache, heads, page, groups, loose, seed=i, wide=0 if hints == "exact" else WIDE // page)
    c.poison()
    pool, batch = c.device(**{"exact": {}, "wide": dict(max_len=0), "rows": dict(max_len=0),
                             "wrong": dict(max_tokens=3, max_len=WIDE)}[hints])
    g = c.device_groups(batch, **{"exact": {}, "wide": dict(max_tokens=0, max_shared=0), "rows": dict(max_shared=0),
                                  "wrong": dict(max_tokens=20, max_shared=WIDE - 100)}[hints])
    of_group, leader, of_seq = c.shared()
    got = g.shared.cpu().numpy()
    n = len(of_group)
    assert (got[:n] == of_group).all() and (got[n:2 * n] == leader).all() and (got[2 * n:] == of_seq).all()
    check_attention(c, attend_shared(pool, batch, g, c.q.to(DEV)))


@pytest.mark.parametrize("cache,heads", [("bf16", H7), ("bf16", H05), ("e4m3", H7), ("e4m3", H05), ("f32", HF)])
@pytest.mark.parametrize("page", [8, 32])
@pytest.mark.parametrize("new", [1, 30])
def test_layouts(cache, heads, page, new):
    """Missing pages among the shared and the own ones, pages that lie apart or K and V in turn, table
    rows that lie apart, rows behind the last sequence."""
    want = None
    for how in range(3):
        c = GroupCache(cache, heads, page, [(400, [(new, 60), (1, 33), (new, new)]), (64, [(1, 40)])], [(new, new)],
                       seed=5, wide=WIDE // page, missing=[(b, s) for s in (0, 3, 7) for b in (1, 2, 3)] + [(2, 408 // page)],
                       gap=1024 if how == 1 else 0, interleaved=how == 2)
        c.poison()
        after = 5 if how == 1 else 0
        pool, batch = c.device(table_gap=9 * how, rows_after=after, max_len=0)
        out = attend_shared(pool, batch, c.device_groups(batch, max_shared=0), c.q.to(DEV), rows_after=after)
        check_attention(c, out)
        assert (out[c.tokens:] == 7).all()
        if not after:  # (more rows are another call, whose splits may be others)
            assert want is None or torch.equal(want, out)
            want = out


def test_nothing_seen_is_zero():
    """All shared pages missing, own ones too in one sequence."""
    c = GroupCache("bf16", H7, 16, [(320, [(1, 3), (1, 20)])], seed=2, wide=WIDE // 16,
                   missing=[(b, s) for s in range(20) for b in (0, 1)] + [(0, 20)])
    c.poison()
    pool, batch = c.device(max_len=0)
    out = attend_shared(pool, batch, c.device_groups(batch), c.q.to(DEV))
    assert (out[0] == 0).all()
    check_attention(c, out)


@pytest.mark.parametrize("cache,heads", [("bf16", H7), ("e4m3", H05), ("f32", HF)])
def test_rising_logits(cache, heads):
    """Logits that rise along the keys by far more than the reference's slack, and fall again."""
    c = GroupCache(cache, heads, 32, [(700, [(1, 60), (1, 9), (3, 90)])], seed=3, wide=WIDE // 32)
    for n, by in ((200, 4.0), (350, 12.0), (690, 8.0), (720, 16.0)):
        for b in range(3):
            if n >= c.seqs[b][1]:
                continue
            for h in range(c.hkv):
                x = c.q[c.off[b], h * (c.hq // c.hkv)].float() * by
                if cache == "e4m3":
                    x = (x * 16).clamp(-448, 448)
                    c.scale["k"][c.table[b, n // 32], h] = 123
                c.raw["k"][c.table[b, n // 32], n % 32, h] = x.to(c.raw["k"].dtype)
    pool, batch = c.device(max_len=0)
    check_attention(c, attend_shared(pool, batch, c.device_groups(batch), c.q.to(DEV)))


def test_groups_that_are_none():
    """No groups, empty groups, offsets that reach past the batch: as page_attn."""
    c = GroupCache("bf16", H7, 16, [(3000, [(1, 9)] * 8)], seed=7)
    pool, batch = c.device()
    q = c.q.to(DEV)
    want = attend(pool, batch, q)
    import paper_2601_13631_amd as ckv
    none = ckv.PageGroups(torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(8, dtype=torch.int32, device=DEV))
    ckv.page_share(16, batch, none)
    assert torch.equal(attend_shared(pool, batch, none, q), want)
    for off in ([0, 0, 0], [8, 8], [0, 3, 3, 900], [-5, 4, 8], [2, 4, 6]):
        c.grp_off = np.array(off, np.int32)
        groups = ckv.PageGroups(torch.tensor(off, dtype=torch.int32, device=DEV),
                                torch.zeros(ckv.page_share_ints(len(off) - 1, 8), dtype=torch.int32, device=DEV))
        ckv.page_share(16, batch, groups)
        check_attention(c, attend_shared(pool, batch, groups, q))


@pytest.mark.parametrize("seed", range(6))
def test_share_of_many(seed):
    """Groups of hundreds of sequences, thousands of pages, tables that part anywhere or not at all."""
    import paper_2601_13631_amd as ckv
    rng = np.random.default_rng(seed)
    page, width = int(rng.choice((8, 16, 96))), int(rng.choice((3, 70, 1500, 5000)))
    sizes = rng.integers(0, 300, 5) if width < 1000 else rng.integers(0, 40, 5)
    n = int(sizes.sum()) + 3
    first = np.concatenate([[2], 2 + np.cumsum(sizes)])
    table = rng.integers(-1, 50, (n, width)).astype(np.int32)
    lens, new = rng.integers(1, width * page + 40, n), rng.integers(0, 4, n)
    for f, l in zip(first, first[1:]):
        table[f:l] = table[f] if l > f else 0
        if rng.random() < 0.7:
            lens[f:l] = width * page - rng.integers(0, 9, l - f)
        for b in rng.integers(f, l, 2) if l > f and rng.random() < 0.7 else ():
            table[b, int(rng.integers(0, width))] += 1
    off = np.concatenate([[0], np.cumsum(new)])
    want_g, want_s = [], np.zeros(n, int)
    for f, l in zip(first, first[1:]):
        active = [b for b in range(f, l) if new[b]]
        e = 0
        if active:
            agree = (table[active] == table[active[0]]).all(0)
            common = width if agree.all() else int(np.argmin(agree))
            e = max(min(common * page, min(lens[b] - new[b] + 1 for b in active)), 0) // 32 * 32
        want_g.append(e)
        want_s[f:l] = e
    t = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.int32)).to(DEV)  # noqa: E731
    batch = ckv.PageBatch(t(table), t(lens), t(off), int(off[-1]))
    shared = torch.full((ckv.page_share_ints(5, n),), -9, dtype=torch.int32, device=DEV)
    ckv.page_share(page, batch, ckv.PageGroups(t(first), shared))
    got = shared.cpu().numpy()
    assert (got[:5] == want_g).all() and (got[10:] == want_s).all()


@pytest.mark.parametrize("cache,heads", [("bf16", H7), ("e4m3", H14)])
def test_pages_far_apart(cache, heads):
    """Pages more than 4 GiB from the pool's begin."""
    c = GroupCache(cache, heads, 16, [(80, [(1, 3), (1, 20), (2, 40)])], seed=4, wide=WIDE // 16,
                   gap=(700 << 20) if cache == "e4m3" else 350 << 20)
    assert (c.n_pages - 1) * c.gap > 1 << 32
    c.poison()
    pool, batch = c.device(max_len=0)
    check_attention(c, attend_shared(pool, batch, c.device_groups(batch, max_shared=0), c.q.to(DEV)))


def draw(seed):
    rng = np.random.default_rng(3000 + seed)
    cache = ("bf16", "e4m3", "bf16", "e4m3", "f32")[seed % 5]
    d = 64 if cache == "f32" else int(rng.choice((64, 128)))
    hkv = int(rng.integers(1, 6))
    heads = (hkv * int(rng.integers(1, 9)), hkv, d)
    page = int(rng.choice((8, 16, 32, 64, 96)))
    groups = []
    for _ in range(int(rng.integers(1, 4))):
        most = int(rng.choice((1, 1, 3, 40)))
        members = [(int(rng.integers(0, most + 1)) if rng.random() < .2 else int(rng.integers(1, most + 1)),
                    int(np.exp(rng.uniform(0, np.log(200)))) - 1) for _ in range(int(rng.integers(1, 9)))]
        shared = int(np.exp(rng.uniform(0, np.log(2500))))
        groups.append((shared, [(min(n, shared + own), own) for n, own in members]))
    loose = [(1, int(rng.integers(1, 200))) for _ in range(int(rng.integers(0, 3)))]
    return rng, cache, heads, page, groups, loose


@pytest.mark.parametrize("seed", range(30))
def test_random(seed):
    rng, cache, heads, page, groups, loose = draw(seed)
    wide = rng.random() < 0.7
    c = GroupCache(cache, heads, page, groups, loose, seed=seed, wide=WIDE // page if wide else 0,
                   gap=int(rng.choice((0, 1024))))
    c.poison()
    sm = float(rng.choice((0.0, 0.2)))
    pool, batch = c.device(max_len=0 if wide else None)
    g = c.device_groups(batch, max_shared=0 if wide else None)
    check_attention(c, attend_shared(pool, batch, g, c.q.to(DEV), sm=sm), sm=sm)


@pytest.mark.parametrize("cache,heads", [("bf16", H7), ("e4m3", H14)])
def test_graph_and_streams(cache, heads):
    """One captured step on changing lengths, tables and queries, replayed with eager work between, and the same
    on a stream of its own."""
    import paper_2601_13631_amd as ckv
    every = [GroupCache(cache, heads, 16, [(s, [(1, 1 + 9 * i + k) for i in range(6)]), (s // 2, [(1, 30)] * 3)],
                        seed=k, wide=WIDE // 16, extra=2 + 400 - 3 * s // 32) for k, s in enumerate((1500, 800, 2000))]
    pages = max(c.n_pages for c in every)
    pool0, batch0 = every[0].device(max_len=0)
    raw = [torch.zeros((pages,) + t.shape[1:], dtype=torch.uint8, device=DEV).view(t.dtype) if t is not None and
           t.element_size() == 1 else None if t is None else torch.zeros((pages,) + t.shape[1:], dtype=t.dtype, device=DEV)
           for t in (pool0.k, pool0.v, pool0.k_scale, pool0.v_scale)]
    pool = ckv.PagePool(*raw)
    q, out = torch.zeros_like(every[0].q, device=DEV), torch.zeros_like(every[0].q, device=DEV)
    g = every[0].device_groups(batch0, max_shared=0)
    nbytes = ckv.page_attn_shared_workspace_bytes(pool, batch0, g, heads[0])
    assert nbytes > 0
    ws = torch.empty(nbytes, dtype=torch.uint8, device=DEV)

    def fill(c):
        for t, n in zip(raw, ("k", "v")):
            t[: c.n_pages].view(torch.uint8).copy_(c.raw[n].view(torch.uint8))
        for t, n in zip(raw[2:], ("k", "v")):
            if t is not None:
                t[: c.n_pages].copy_(c.scale[n])
        batch0.table.fill_(-1)
        batch0.table[:, : c.width].copy_(torch.from_numpy(c.table))
        batch0.lens.copy_(torch.from_numpy(c.lens))
        q.copy_(c.q)

    def step(stream=None):
        ckv.page_share(16, batch0, g, stream=stream)
        ckv.page_attn_shared(pool, batch0, g, q, out, ws, stream=stream)
    fill(every[0])
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for c in every + every[:1]:
        fill(c)
        out.fill_(7)
        graph.replay()
        replayed = out.clone()
        torch.cuda.synchronize()
        check_attention(c, replayed)
        out.fill_(7)
        step()
        assert torch.equal(out, replayed)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        out.fill_(7)
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, replayed)


def test_a_step_of_beams():
    """Eight steps of two requests of four beams: selection, fork, pages, copies, rows, attention; against
    dense attention over each beam's own history, and the host models of the tables."""
    import paper_2601_13631_amd as ckv
    page, heads, vocab, reqs, beams, layers = 16, (8, 2, 64), 97, 2, 4, 2
    hq, hkv, d = heads
    n, width, n_pages = reqs * beams, 12, 90
    gen = torch.Generator().manual_seed(11)
    table_kv = torch.randn(2, layers, vocab, hkv, d, generator=gen).bfloat16()   # a token's K and V rows
    table_q = torch.randn(layers, vocab, hq, d, generator=gen).bfloat16()
    head = (torch.randn(hq * d, vocab, generator=gen) * 0.5).to(DEV)
    kv, tq = table_kv.to(DEV), table_q.to(DEV)
    pools = [ckv.PagePool(*(torch.zeros(n_pages, page, hkv, d, dtype=torch.bfloat16, device=DEV) for _ in "kv"))
             for _ in range(layers)]
    every = ckv.PageLayers(pools)

    def ints(*shape, fill=0):
        return torch.full(shape, fill, dtype=torch.int32, device=DEV)
    a = dict(table=ints(n, width, fill=-1), lens=ints(n), history=ints(n, width * page))
    b = dict(table=ints(n, width, fill=-1), lens=ints(n), history=ints(n, width * page))
    refs, n_new, tok_off = ints(n_pages), ints(n), ints(n + 1)
    src, dst, counts = ints(n), ints(n), ints(4)
    scores = torch.full((reqs, beams), -float("inf"), device=DEV)
    scores[:, 0] = 0
    done = torch.zeros(reqs, beams, dtype=torch.uint8, device=DEV)
    logits = torch.zeros(reqs, beams, vocab, device=DEV)
    # prompts: one sequence of each request, 37 and 70 tokens
    host = [[], [], [], [], [], [], [], []]
    for r, m in enumerate((37, 70)):
        host[r * beams] = torch.randint(3, vocab, (m,), generator=gen).tolist()

    def run(tokens_of):
        """The rows of a step: `tokens_of` new ones per sequence; returns the last layer's output."""
        total = sum(len(t) for t in tokens_of)
        n_new.copy_(torch.tensor([len(t) for t in tokens_of], dtype=torch.int32))
        before = {k: x.cpu().numpy().copy() for k, x in (("table", a["table"]), ("lens", a["lens"]), ("refs", refs))}
        slots = torch.zeros(total, dtype=torch.int64, device=DEV)
        pos, seqs = ints(total), ints(total)
        step = ckv.PageStep(page, a["table"], a["table"], a["lens"], a["lens"], refs, refs, n_new, tok_off, src, dst,
                            counts, slots=slots, positions=pos, seqs=seqs)
        ckv.page_extend(step, torch.empty(ckv.page_extend_workspace_bytes(n_pages, n), dtype=torch.uint8, device=DEV))
        want = extend_model(page, before["table"], before["lens"], before["refs"], n_new.cpu().numpy(), total)
        for k, x in (("table", a["table"]), ("refs", refs), ("lens", a["lens"]), ("tok_off", tok_off), ("slots", slots),
                     ("positions", pos), ("seqs", seqs), ("copy_src", src), ("copy_dst", dst), ("counts", counts)):
            assert (x.cpu().numpy() == want[k]).all(), k
        assert int(counts[3]) == 0
        ckv.page_copy(every, src, dst)
        tok = torch.tensor([t for s in tokens_of for t in s], device=DEV)
        a["history"][seqs.long(), pos.long()] = tok.int()
        batch = ckv.PageBatch(a["table"], a["lens"], tok_off, total, max_tokens=max(len(t) for t in tokens_of))
        groups = ckv.PageGroups(torch.tensor([0, beams, n], dtype=torch.int32, device=DEV),
                                ints(ckv.page_share_ints(2, n)))
        ckv.page_share(page, batch, groups)
        for l, pool in enumerate(pools):
            ckv.page_append(pool, batch, kv[0, l][tok], kv[1, l][tok])
            q = tq[l][tok]
            out = torch.empty_like(q)
            ws = torch.empty(ckv.page_attn_shared_workspace_bytes(pool, batch, groups, hq), dtype=torch.uint8, device=DEV)
            ckv.page_attn_shared(pool, batch, groups, q, out, ws)
            got, row = out.cpu().double(), 0
            for s in range(n):
                h = torch.tensor(host[s])
                m = len(tokens_of[s])
                if m:
                    k, v = (x[l][h].double().repeat_interleave(hq // hkv, 1) for x in table_kv)
                    z = torch.einsum("thd,shd->hts", table_q[l][h[-m:]].double(), k) / d ** 0.5
                    z = z.masked_fill(torch.arange(len(h)) > torch.arange(len(h) - m, len(h))[:, None], -torch.inf)
                    w = torch.softmax(z, -1)
                    ref = torch.einsum("hts,shd->thd", w, v)
                    size = torch.einsum("hts,shd->thd", w, v.abs())
                    u = 2.0 ** -8
                    assert ((got[row:row + m] - ref).abs() <= 2 * u * ref.abs() + (u + 2.0 ** -11) * size).all()
                row += m
        return out

    out = run(host)
    last = tok_off.long()[1:] - 1
    for turn in range(8):
        logits.copy_((out[last.clamp(min=0)].float().reshape(n, -1) @ head).view(reqs, beams, vocab))
        parent, token, done2 = ints(reqs, beams), ints(reqs, beams), torch.zeros_like(done)
        scores2 = torch.zeros_like(scores)
        ws = torch.empty(ckv.beam_select_workspace_bytes(logits, beams), dtype=torch.uint8, device=DEV)
        ckv.beam_select(logits, scores, parent, token, scores2, ws, done=done, done_out=done2, eos=2)
        p, t, s, e = select_model(logits.cpu().numpy(), scores.cpu().numpy(), done.cpu().numpy(), beams, 2)
        assert (parent.cpu().numpy() == p).all() and (token.cpu().numpy() == t).all() and (done2.cpu().numpy() == e).all()
        assert np.abs(scores2.cpu().numpy() - s).max() < 1e-4
        fork = ckv.PageFork(page, a["table"], b["table"], a["lens"], b["lens"], refs, refs,
                            states=[(a["history"], b["history"])])
        want = fork_model(page, a["table"].cpu().numpy(), a["lens"].cpu().numpy(), refs.cpu().numpy(), p.reshape(-1))
        ckv.page_fork(fork, parent.view(-1))
        for x, y in zip((b["table"], b["lens"], refs), want):
            assert (x.cpu().numpy() == y).all()
        host = [list(host[i]) for i in p.reshape(-1)]
        new = [[int(x)] for x in t.reshape(-1)]
        for s_, x in zip(host, new):
            s_ += x
        scores, done, a, b = scores2, done2, b, a
        out = run(new)
        last = tok_off.long()[1:] - 1
        for i in range(n):
            assert a["history"][i, : len(host[i])].tolist() == host[i]
    held = a["table"].cpu().numpy()
    lens = a["lens"].cpu().numpy()
    used = np.zeros(n_pages, int)
    for i in range(n):
        np.add.at(used, held[i, : -(-lens[i] // page)], 1)
    assert (used == refs.cpu().numpy()).all()
