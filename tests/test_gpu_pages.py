"""The paged cache's operators against a host model in 64 bits: attention with and without a
window, append, copy and compact."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from pages_common import DEV, Cache, attend, check_attention, codes_to_f64  # noqa: E402

H05, H7, H14, HF, H1 = (14, 2, 64), (28, 4, 128), (40, 8, 128), (4, 1, 64), (3, 3, 64)

# (cache, heads, page, (new, length) per sequence, window, sinks)
ATTN = [
    ("bf16", H7, 16, [(1, 1)], 0, 0),                                   # one token, one key
    ("bf16", H7, 32, [(1, 33), (1, 32), (1, 31), (1, 1000)], 0, 0),     # page and step borders
    ("bf16", H05, 8, [(1, 7), (1, 8), (1, 9), (1, 257)], 0, 0),
    ("bf16", H14, 96, [(1, 95), (1, 97), (1, 777)], 0, 0),              # no power of two
    ("bf16", H1, 64, [(1, 500), (3, 3)], 0, 0),                         # no shared heads
    ("bf16", H7, 32, [(1, 20000)], 0, 0),                               # long: many splits
    ("bf16", H7, 64, [(37, 37), (1, 300), (0, 90), (130, 1000), (5, 64)], 0, 0),  # ragged, one idle
    ("bf16", H05, 16, [(200, 450), (64, 64)], 0, 0),
    ("bf16", H7, 32, [(1, 1000), (1, 64), (1, 65), (1, 3)], 64, 0),     # window as long as two steps
    ("bf16", H7, 16, [(1, 1000), (1, 5), (1, 70)], 1, 0),               # sees itself alone
    ("bf16", H05, 16, [(1, 900), (1, 40), (1, 64)], 50, 4),
    ("bf16", H14, 8, [(7, 500), (300, 700), (60, 61)], 100, 8),
    ("bf16", H7, 64, [(150, 900), (150, 150)], 97, 70),                 # sinks past one step
    ("bf16", H7, 32, [(40, 200), (1, 100)], 5000, 4),                   # window past everything
    ("bf16", H7, 32, [(40, 200), (1, 100)], 10, 5000),                  # sinks past everything
    ("bf16", H7, 16, [(4, 2), (3, 3), (2, 0)], 0, 0),                   # rows before position 0
    ("e4m3", H7, 16, [(1, 1), (1, 17), (1, 900)], 0, 0),
    ("e4m3", H14, 8, [(1, 333), (2, 77), (5, 5)], 0, 0),
    ("e4m3", H05, 32, [(1, 1000), (19, 400)], 200, 3),
    ("e4m3", H05, 8, [(4, 1000), (4, 9)], 64, 8),
    ("e4m3", H7, 96, [(1, 15000)], 0, 0),
    ("e4m3", H7, 64, [(140, 500), (0, 3), (70, 70)], 0, 0),
    ("e4m3", H14, 32, [(140, 500), (33, 1000)], 130, 40),
    ("f32", HF, 16, [(1, 1), (1, 100), (1, 1024)], 0, 0),
    ("f32", HF, 8, [(50, 333), (20, 20)], 0, 0),
    ("f32", (4, 2, 64), 32, [(96, 1000), (0, 5), (33, 64)], 128, 4),
    ("f32", HF, 96, [(1, 6000)], 0, 0),
    ("bf16", (48, 1, 128), 32, [(1, 700), (1, 1), (2, 90)], 0, 0),      # one KV head for 48, 16 and 20
    ("e4m3", (16, 1, 128), 16, [(1, 700), (2, 90)], 100, 4),
    ("bf16", (20, 1, 64), 8, [(1, 333), (1, 64)], 0, 0),
    ("f32", (20, 1, 64), 8, [(1, 333), (3, 64)], 0, 0),
    ("e4m3", (5, 5, 64), 16, [(130, 200), (1, 7)], 40, 0),              # KV heads that 8 does not divide
    ("bf16", (12, 6, 128), 32, [(150, 3000)], 0, 0),
    ("e4m3", (7, 7, 128), 8, [(140, 2000)], 700, 9),
]


@pytest.mark.parametrize("i", range(len(ATTN)))
def test_attention(i):
    cache, heads, page, seqs, window, sinks = ATTN[i]
    c = Cache(cache, heads, page, seqs, seed=i)
    c.poison(window, sinks)
    pool, batch = c.device()
    check_attention(c, attend(pool, batch, c.q.to(DEV), window, sinks), window, sinks)


@pytest.mark.parametrize("cache,heads", [("bf16", H7), ("bf16", H05), ("e4m3", H7), ("e4m3", H05), ("f32", HF)])
@pytest.mark.parametrize("new", [1, 60])
def test_attention_layouts(cache, heads, new):
    """Missing pages, pages and table rows that lie apart, K and V pages in turn, rows behind
    the last sequence, hints that do not hold."""
    seqs = [(new, 500), (1, 130), (new, new)]
    want = None
    for how in range(4):
        c = Cache(cache, heads, 16, seqs, seed=5, missing=[(0, 0), (0, 3), (0, 30), (1, 7)],
                  gap=1024 if how == 1 else 0, interleaved=how == 2)
        c.poison()
        hints = dict(max_tokens=0, max_len=0) if how == 0 else dict(max_tokens=1, max_len=3) if how == 3 else {}
        after = 5 if how == 1 else 0
        pool, batch = c.device(table_gap=9 * how, rows_after=after, **hints)
        out = attend(pool, batch, c.q.to(DEV), rows_after=after)
        check_attention(c, out)
        assert (out[c.tokens:] == 7).all()
        if how in (1, 2):
            assert want is None or torch.equal(want, out[:c.tokens])
            want = out[:c.tokens]


@pytest.mark.parametrize("cache,heads", [("bf16", H7), ("bf16", H05), ("e4m3", H7), ("e4m3", H05)])
@pytest.mark.parametrize("page", [8, 16, 96])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1800, 40)])
@pytest.mark.parametrize("max_len", [0, 40])
def test_missing_pages_far_in(cache, heads, page, window, sinks, max_len):
    """Pages missing here and there along thousands of keys, in one split (max_len 40) and in many."""
    rng = np.random.default_rng(page)
    seqs = [(90, 3333), (40, 1500)]
    missing = [(b, int(s)) for b, (_, n) in enumerate(seqs) for s in rng.choice(-(-n // page), 9, replace=False)]
    c = Cache(cache, heads, page, seqs, seed=page, missing=missing)
    c.poison(window, sinks)
    pool, batch = c.device(max_len=max_len)
    check_attention(c, attend(pool, batch, c.q.to(DEV), window, sinks), window, sinks)


@pytest.mark.parametrize("cache,heads", [("bf16", H7), ("e4m3", H7), ("f32", HF)])
@pytest.mark.parametrize("new", [1, 100])
def test_rows_without_keys_are_zero(cache, heads, new):
    c = Cache(cache, heads, 16, [(new, 300), (new, 300)], seed=9, missing=[(0, s) for s in range(19)])
    c.poison()
    pool, batch = c.device()
    out = attend(pool, batch, c.q.to(DEV))
    assert (out[:new] == 0).all()
    check_attention(c, out)


@pytest.mark.parametrize("cache,heads", [("bf16", H7), ("e4m3", H05), ("f32", HF)])
@pytest.mark.parametrize("new", [1, 90])
def test_rising_logits(cache, heads, new):
    """Logits that grow along the keys by far more than the reference's slack, and fall again."""
    c = Cache(cache, heads, 32, [(new, 700), (1, 600)], seed=3)
    for n in (200, 350, 690):
        slot, row = n // 32, n % 32
        for b in range(2):
            if n < c.seqs[b][1]:
                for h in range(c.hkv):
                    q = c.q[c.off[b], h * (c.hq // c.hkv)].float()
                    x = q * {200: 4.0, 350: 12.0, 690: 8.0}[n]
                    if cache == "e4m3":
                        x = (x * 16).clamp(-448, 448)
                        c.scale["k"][c.table[b, slot], h] = 123
                    c.raw["k"][c.table[b, slot], row, h] = x.to(c.raw["k"].dtype)
    pool, batch = c.device()
    check_attention(c, attend(pool, batch, c.q.to(DEV)))


def draw_attention(seed):
    """A random case: heads, page, ragged lengths, window, missing pages, layout, hints."""
    rng = np.random.default_rng(1000 + seed)
    cache = ("bf16", "e4m3", "bf16", "e4m3", "f32")[seed % 5]
    d = 64 if cache == "f32" else int(rng.choice((64, 128)))
    hkv = int(rng.integers(1, 8))
    heads = (hkv * int(rng.integers(1, 9)), hkv, d)
    page = int(rng.choice((8, 16, 32, 64, 96, 128)))
    top = int(np.exp(rng.uniform(0, np.log(3000))))
    many = int(np.exp(rng.uniform(0, np.log(300)))) if rng.random() < 0.6 else 1
    seqs = []
    for _ in range(int(rng.integers(1, 7))):
        n = int(rng.integers(0, many + 1))
        seqs.append((n, n + int(rng.integers(0, top + 1))))
    seqs[0] = (many, many + top)
    window = int(np.exp(rng.uniform(0, np.log(800)))) if rng.random() < 0.6 else 0
    sinks = int(rng.choice((0, 1, 4, 7, 64, 100)))
    missing = [(b, int(rng.integers(0, -(-m // page)))) for b, (n, m) in enumerate(seqs) if m and rng.random() < 0.4]
    return cache, heads, page, seqs, window, sinks, missing, rng


@pytest.mark.parametrize("seed", range(60))
def test_attention_random(seed):
    cache, heads, page, seqs, window, sinks, missing, rng = draw_attention(seed)
    c = Cache(cache, heads, page, seqs, seed=seed, missing=missing, interleaved=bool(rng.random() < 0.3))
    c.poison(window, sinks)
    hints = {} if rng.random() < 0.6 else dict(max_tokens=int(rng.integers(0, 50)), max_len=int(rng.integers(0, 2000)))
    after = int(rng.integers(0, 3))
    pool, batch = c.device(table_gap=int(rng.integers(0, 4)), rows_after=after, **hints)
    out = attend(pool, batch, c.q.to(DEV), window, sinks, rows_after=after)
    check_attention(c, out, window, sinks)
    assert (out[c.tokens:] == 7).all()
    assert torch.equal(out, attend(pool, batch, c.q.to(DEV), window, sinks, rows_after=after))  # bit for bit


@pytest.mark.parametrize("cache,heads,n,most", [("e4m3", (1, 1, 64), 5000, 3), ("bf16", (40, 1, 64), 130, 2),
                                                ("e4m3", (40, 2, 128), 65, 9), ("bf16", (1, 1, 128), 64, 1),
                                                ("e4m3", (36, 1, 64), 700, 1)])
def test_many_sequences(cache, heads, n, most):
    """More sequences than a wave has lanes, some with no token; what each is found by."""
    import paper_2601_13631_amd as ckv
    rng = np.random.default_rng(n)
    seqs = [(int(rng.integers(0, most + 1)), int(rng.integers(0, 20))) for _ in range(n)]
    seqs = [(a, a + b) for a, b in seqs]
    c = Cache(cache, heads, 8, seqs, seed=n)
    pool, batch = c.device()
    ckv.page_append(pool, batch, c.new_rows["k"].to(DEV), c.new_rows["v"].to(DEV))
    c.append()
    check_pages(c, pool.k, pool.v, pool.k_scale, pool.v_scale)
    check_attention(c, attend(pool, batch, c.q.to(DEV)))


def test_offsets_that_do_not_start_at_0():
    """Rows before the first sequence and behind the last belong to none."""
    import paper_2601_13631_amd as ckv
    for cache, heads in (("bf16", H7), ("e4m3", H7), ("f32", HF)):
        for new in (1, 45):
            c = Cache(cache, heads, 16, [(new, 200), (0, 20), (new, 90)], seed=3)
            pool, _ = c.device()
            lead, tail = 37, 5
            off = torch.from_numpy(c.off + lead).to(DEV)
            batch = ckv.PageBatch(torch.from_numpy(c.table).to(DEV), torch.from_numpy(c.lens).to(DEV), off,
                                  lead + c.tokens + tail, max_tokens=new)
            pad = lambda t: torch.cat([torch.full_like(t[:1], 9.0).repeat(lead, 1, 1), t,  # noqa: E731
                                       torch.full_like(t[:1], 9.0).repeat(tail, 1, 1)]).to(DEV)
            ckv.page_append(pool, batch, pad(c.new_rows["k"]), pad(c.new_rows["v"]))
            c.append()
            check_pages(c, pool.k, pool.v, pool.k_scale, pool.v_scale)
            out = attend(pool, batch, pad(c.q))
            assert (out[:lead] == 7).all() and (out[lead + c.tokens:] == 7).all()
            check_attention(c, out[lead:])


def test_lengths_past_the_table():
    """A sequence longer than its table: its queries see what the table holds."""
    import paper_2601_13631_amd as ckv
    for cache, heads in (("bf16", H7), ("e4m3", H05), ("f32", HF)):
        for new in (1, 70):
            c = Cache(cache, heads, 16, [(new, 200), (new, 90)], seed=3)
            c.table = np.ascontiguousarray(c.table[:, :4])
            c.width = 4
            pool = ckv.PagePool(*c.device_pages())
            batch = ckv.PageBatch(*(torch.from_numpy(x).to(DEV) for x in (c.table, c.lens, c.off)), c.tokens)
            check_attention(c, attend(pool, batch, c.q.to(DEV)))


def test_attention_scale():
    c = Cache("bf16", H7, 16, [(1, 200), (30, 90)], seed=2)
    pool, batch = c.device()
    check_attention(c, attend(pool, batch, c.q.to(DEV), sm=0.25), sm=0.25)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_pool_past_4_gib(cache):
    """Pages on both sides of 2^32 bytes, for one token and for many."""
    import paper_2601_13631_amd as ckv
    for new in (1, 150):
        c = Cache(cache, H7, 32, [(new, 400)], seed=6)
        k, v, ks, vs = c.device_pages()
        span = 32 * 4 * 128 * k.element_size()
        far = (5 << 30) // span
        total = far + c.n_pages
        place = np.array([p if p % 2 else far + p for p in range(c.n_pages)])
        big = []
        for t in (k, v):
            x = torch.empty((total,) + tuple(t.shape[1:]), dtype=t.dtype, device=DEV)
            x.view(torch.uint8)[torch.from_numpy(place).to(DEV)] = t.contiguous().view(torch.uint8)
            big.append(x)
        scales = [None, None]
        if cache == "e4m3":
            scales = [torch.zeros(total, 4, dtype=torch.uint8, device=DEV) for _ in range(2)]
            for s, t in zip(scales, (ks, vs)):
                s[torch.from_numpy(place).to(DEV)] = t
        pool = ckv.PagePool(*big, *scales)
        _, small = c.device()
        table = torch.from_numpy(place[c.table].astype(np.int32)).to(DEV)
        batch = ckv.PageBatch(table, small.lens, small.tok_off, c.tokens)
        check_attention(c, attend(pool, batch, c.q.to(DEV)))
        # append writes there too
        ckv.page_append(pool, batch, c.new_rows["k"].to(DEV), c.new_rows["v"].to(DEV))
        c.append()
        for x, n in zip(big, "kv"):
            got = x.view(torch.uint8)[torch.from_numpy(place).to(DEV)].view(x.dtype)
            assert np.array_equal(codes_to_f64(got), codes_to_f64(c.raw[n]))
        del big, pool


# ---- append -----------------------------------------------------------------------

APPEND = [
    (16, [(1, 1), (1, 16), (1, 17), (1, 300)]),      # a fresh page's first row, a page's last
    (8, [(3, 3), (20, 33), (0, 12), (8, 16)]),
    (32, [(100, 100), (31, 64), (70, 97)]),
    (96, [(200, 205), (1, 96), (1, 97)]),
    (64, [(500, 1000)]),
]


def check_pages(c: Cache, k, v, ks, vs):
    for t, n, s in ((k, "k", ks), (v, "v", vs)):
        got, want = codes_to_f64(t), codes_to_f64(c.raw[n])
        assert np.array_equal(got, want, equal_nan=True), n
        if s is not None:
            assert torch.equal(s.cpu(), c.scale[n]), n


@pytest.mark.parametrize("cache,heads", [("bf16", H7), ("e4m3", H7), ("e4m3", H05), ("f32", (4, 2, 64))])
@pytest.mark.parametrize("i", range(len(APPEND)))
@pytest.mark.parametrize("magnitude", [0.01, 3.0, 1e4])
def test_append(cache, heads, i, magnitude):
    """Every byte of the pool: new rows, older rows rounded to a scale that rose, all others."""
    import paper_2601_13631_amd as ckv
    page, seqs = APPEND[i]
    c = Cache(cache, heads, page, seqs, seed=i, missing=[(0, 0)] if i == 2 else ())
    c.new_rows = {n: (x.float() * magnitude).to(x.dtype) for n, x in c.new_rows.items()}
    pool, batch = c.device()
    ckv.page_append(pool, batch, c.new_rows["k"].to(DEV), c.new_rows["v"].to(DEV))
    c.append()
    check_pages(c, pool.k, pool.v, pool.k_scale, pool.v_scale)


def test_append_odd_values():
    """Zeros, the least and largest numbers, infinities and NaN; a page of zeros that grows."""
    import paper_2601_13631_amd as ckv
    c = Cache("e4m3", H05, 16, [(20, 20), (3, 5), (1, 1)], seed=1)
    big = float(torch.finfo(torch.bfloat16).max)
    for n in "kv":
        x = c.new_rows[n]
        x[:16] = 0
        x[16:20, 0] = torch.tensor([0.0, 1e-39, -1e-40, 2.0 ** -126])[:, None].to(x.dtype)
        x[17, 1, :6] = torch.tensor([float("nan"), float("inf"), -float("inf"), 2.0, 448.0, -449.0]).to(x.dtype)
        x[20] = big
        x[21, 0, 5] = float("inf")
        x[23] = float("nan")
    pool, batch = c.device()
    ckv.page_append(pool, batch, c.new_rows["k"].to(DEV), c.new_rows["v"].to(DEV))
    c.append()
    check_pages(c, pool.k, pool.v, pool.k_scale, pool.v_scale)


def test_append_outside_the_table():
    """Positions past the table and before position 0 are dropped; rows of no sequence too."""
    import paper_2601_13631_amd as ckv
    for cache, heads in (("bf16", H7), ("e4m3", H7)):
        c = Cache(cache, heads, 16, [(20, 40), (9, 5), (4, 30)], seed=4)
        pool, _ = c.device()
        narrow = torch.from_numpy(np.ascontiguousarray(c.table[:, :2])).to(DEV)
        batch = ckv.PageBatch(narrow, torch.from_numpy(c.lens).to(DEV), torch.from_numpy(c.off).to(DEV),
                              c.tokens + 3)
        rows = [torch.cat([c.new_rows[n], torch.full_like(c.new_rows[n][:3], 99.0)]).to(DEV) for n in "kv"]
        ckv.page_append(pool, batch, *rows)
        c.width, c.table = 2, c.table[:, :2]
        c.append()
        check_pages(c, pool.k, pool.v, pool.k_scale, pool.v_scale)


# ---- copy and compact -----------------------------------------------------------------

def layers_of(cache, n, page, pages, heads, interleaved=False):
    cs = [Cache(cache, heads, page, [(1, page * (pages - 2))], seed=i, interleaved=interleaved) for i in range(n)]
    import paper_2601_13631_amd as ckv
    return cs, ckv.PageLayers([ckv.PagePool(*c.device_pages()) for c in cs])


def bytes_of(t):
    return t.contiguous().view(torch.uint8).cpu()


@pytest.mark.parametrize("cache,heads", [("bf16", H7), ("e4m3", H05), ("f32", HF)])
@pytest.mark.parametrize("n,page,pages,interleaved", [(1, 16, 12, False), (3, 8, 40, True), (70, 32, 9, False),
                                                     (2, 96, 70, False)])
def test_copy(cache, heads, n, page, pages, interleaved):
    import paper_2601_13631_amd as ckv
    cs, layers = layers_of(cache, n, page, pages, heads, interleaved)
    before = [[t if t is None else t.clone() for t in (p.k, p.v, p.k_scale, p.v_scale)] for p in layers.pools]
    src = [2, 2, 5, -1, 3, pages, 6, 2 ** 31 - 1]
    dst = [0, 1, 7, 3, pages, 4, 6, 3]  # (6 to itself)
    ckv.page_copy(layers, *(torch.tensor(x, dtype=torch.int32, device=DEV) for x in (src, dst)))
    for p, old in zip(layers.pools, before):
        come = list(range(pages))
        for a, b in ((2, 0), (2, 1), (5, 7)):
            come[b] = a
        for t, o in zip((p.k, p.v, p.k_scale, p.v_scale), old):
            if t is not None:
                assert torch.equal(bytes_of(t), bytes_of(o)[come])
    ckv.page_copy(layers, *(torch.empty(0, dtype=torch.int32, device=DEV) for _ in range(2)))
    ckv.page_copy(ckv.PageLayers([]), *(torch.zeros(4, dtype=torch.int32, device=DEV) for _ in range(2)))


def host_compact(refs, table, n_pages):
    live = [p for p in range(n_pages) if refs[p] > 0]
    L = len(live)
    name, come = {p: p for p in live}, list(range(n_pages))
    out = [max(r, 0) for r in refs]
    for p, hole in zip([p for p in live if p >= L], [p for p in range(L) if refs[p] <= 0]):
        name[p], come[hole] = hole, p
        out[hole], out[p] = refs[p], 0
    follow = [name.get(e, -1) if 0 <= e < n_pages else e for e in table]
    return L, come, out, follow


@pytest.mark.parametrize("cache,heads", [("bf16", HF), ("e4m3", H05)])
@pytest.mark.parametrize("pages", [3, 64, 2047, 2048, 2049, 5000, 8192, 8193, 20000])
@pytest.mark.parametrize("share", [0.0, 0.02, 0.5, 0.97, 1.0])
def test_compact(cache, heads, pages, share):
    import paper_2601_13631_amd as ckv
    cs, layers = layers_of(cache, 2, 8, pages, heads)
    rng = np.random.default_rng(pages)
    refs = np.where(rng.random(pages) < share, rng.integers(1, 4, pages), -rng.integers(0, 2, pages)).astype(np.int32)
    table = rng.integers(-2, pages + 2, 777).astype(np.int32)
    L, come, want_refs, want_table = host_compact(refs.tolist(), table.tolist(), pages)
    before = [[t if t is None else bytes_of(t) for t in (p.k, p.v, p.k_scale, p.v_scale)] for p in layers.pools]
    ws = torch.full((ckv.page_compact_workspace_bytes(pages),), 0xFF, dtype=torch.uint8, device=DEV)
    for in_place in (False, True):  # (again from the same counts: the pages move as before)
        r, t = (torch.from_numpy(x).to(DEV) for x in (refs, table))
        ro, to = (r, t) if in_place else (torch.empty_like(r), torch.empty_like(t))
        n_live = torch.full((1,), -5, dtype=torch.int32, device=DEV)
        ckv.page_compact(layers, r, ro, t, to, n_live, ws)
        assert n_live.item() == L
        assert ro.tolist() == want_refs and to.tolist() == want_table
        for p, old in zip(layers.pools, before):
            for x, o in zip((p.k, p.v, p.k_scale, p.v_scale), old):
                if x is not None:
                    assert torch.equal(bytes_of(x), o[come])


def test_compact_without_pools_or_table():
    import paper_2601_13631_amd as ckv
    refs = torch.tensor([0, 1, 0, 2, 1], dtype=torch.int32, device=DEV)
    out, n = torch.empty_like(refs), torch.empty(1, dtype=torch.int32, device=DEV)
    ws = torch.empty(ckv.page_compact_workspace_bytes(5), dtype=torch.uint8, device=DEV)
    ckv.page_compact(ckv.PageLayers([]), refs, out, None, None, n, ws)
    assert out.tolist() == [2, 1, 1, 0, 0] and n.item() == 3


# ---- together ---------------------------------------------------------------------------

@pytest.mark.parametrize("cache,heads", [("bf16", H7), ("e4m3", H7), ("e4m3", H05), ("f32", HF)])
def test_serving_loop(cache, heads):
    """Two prompts appended and attended, one forked, decoding with a window, the first freed, the
    pool made compact: each step against the host model of the same cache."""
    import paper_2601_13631_amd as ckv
    page, n_pages, width = 16, 40, 12
    hq, hkv, d = heads
    c = Cache(cache, heads, page, [(0, page)] * 3, seed=8, extra=n_pages - 3)
    c.width, c.table = width, np.full((3, width), -1, np.int32)
    pool = ckv.PagePool(*c.device_pages())
    layers = ckv.PageLayers([pool])
    refs = np.zeros(n_pages, np.int32)
    g = torch.Generator().manual_seed(0)
    lens = [0, 0, 0]

    def step(new, window, sinks):
        for b, n in enumerate(new):
            lens[b] += n
            for s in range(-(-lens[b] // page)):
                if n and c.table[b, s] < 0:
                    c.table[b, s] = int(np.nonzero(refs == 0)[0][-1])  # from the back: compaction has work
                    refs[c.table[b, s]] = 1
        c.seqs = [(n, m) for n, m in zip(new, lens)]
        c.new, c.lens = np.array(new), np.array(lens, np.int32)
        c.off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        c.tokens = int(c.off[-1])
        wide = c.q.dtype
        c.q = torch.randn(c.tokens, hq, d, generator=g).to(wide)
        c.new_rows = {n: torch.randn(c.tokens, hkv, d, generator=g).to(wide) for n in "kv"}
        batch = ckv.PageBatch(torch.from_numpy(c.table).to(DEV), torch.from_numpy(c.lens).to(DEV),
                              torch.from_numpy(c.off).to(DEV), c.tokens, max_tokens=max(new))
        ckv.page_append(pool, batch, c.new_rows["k"].to(DEV), c.new_rows["v"].to(DEV))
        c.append()
        check_pages(c, pool.k, pool.v, pool.k_scale, pool.v_scale)
        check_attention(c, attend(pool, batch, c.q.to(DEV), window, sinks), window, sinks)

    step([70, 41, 0], 0, 0)
    # fork sequence 1: shared pages, its last one copied
    last = c.table[1, 2]
    own = int(np.nonzero(refs == 0)[0][-1])
    c.table[2] = c.table[1]
    c.table[2, 2] = own
    lens[2] = lens[1]
    refs[c.table[1, :2]] += 1
    refs[own] = 1
    ckv.page_copy(layers, *(torch.tensor([int(x)], dtype=torch.int32, device=DEV) for x in (last, own)))
    for n in "kv":
        c.raw[n].view(torch.uint8)[own] = c.raw[n].view(torch.uint8)[last].clone()
        if c.scale[n] is not None:
            c.scale[n][own] = c.scale[n][last]
    for _ in range(3):
        step([1, 1, 1], 0, 0)
    step([1, 9, 1], 24, 4)
    # the first sequence ends
    refs[c.table[0][c.table[0] >= 0]] -= 1
    c.table[0] = -1
    lens[0] = 0
    L, come, want_refs, want_table = host_compact(refs.tolist(), c.table.reshape(-1).tolist(), n_pages)
    table = torch.from_numpy(c.table).to(DEV)
    r = torch.from_numpy(refs).to(DEV)
    n_live = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.empty(ckv.page_compact_workspace_bytes(n_pages), dtype=torch.uint8, device=DEV)
    ckv.page_compact(layers, r, r, table, table, n_live, ws)
    assert n_live.item() == L and r.tolist() == want_refs
    refs[:] = r.cpu().numpy()
    c.table[:] = table.cpu().numpy()
    assert c.table.reshape(-1).tolist() == want_table
    for n in "kv":
        c.raw[n] = c.raw[n].view(torch.uint8)[come].view(c.raw[n].dtype).clone()
        if c.scale[n] is not None:
            c.scale[n] = c.scale[n][come].clone()
    step([30, 1, 1], 0, 0)
    step([0, 1, 40], 33, 1)


# ---- streams, graphs, refusals -------------------------------------------------------------

def serving_step(ckv, c, pool, layers, batch, q, out, ws, window):
    ckv.page_append(pool, batch, c["k"], c["v"])
    ckv.page_attn(pool, batch, q, out, ws, window=window, n_sinks=4)
    ckv.page_copy(layers, c["src"], c["dst"])
    ckv.page_compact(layers, c["refs"], c["refs_out"], c["table"], c["table_out"], c["live"], c["cws"])


@pytest.mark.parametrize("cache,heads", [("bf16", H7), ("e4m3", H7), ("f32", HF)])
@pytest.mark.parametrize("new", [1, 80])
@pytest.mark.parametrize("window", [0, 100])
def test_graphs(cache, heads, new, window):
    """Two captured graphs with workspaces of their own, replayed in turn with other inputs and
    lengths, against eager calls on a copy."""
    import paper_2601_13631_amd as ckv
    sides = []
    for g in range(2):
        c = Cache(cache, heads, 16, [(new, 2000 - 300 * g), (new, 100 + new)], seed=20 + g)
        two = []
        for _ in range(2):  # the graph's and the eager calls' own
            pool, batch = c.device(max_len=2000)
            x = {"k": c.new_rows["k"].to(DEV), "v": c.new_rows["v"].to(DEV)}
            x["src"], x["dst"] = (torch.tensor(i, dtype=torch.int32, device=DEV) for i in ([0, 1], [c.n_pages - 1, c.n_pages - 2]))
            refs = torch.ones(c.n_pages, dtype=torch.int32, device=DEV)
            refs[3::4] = 0
            x["refs"], x["refs_out"] = refs, torch.zeros_like(refs)
            x["table"] = batch.table.contiguous()
            x["table_out"] = torch.zeros_like(x["table"])
            x["live"] = torch.zeros(1, dtype=torch.int32, device=DEV)
            x["cws"] = torch.empty(ckv.page_compact_workspace_bytes(c.n_pages), dtype=torch.uint8, device=DEV)
            q = c.q.to(DEV)
            out = torch.zeros_like(q)
            ws = torch.empty(ckv.page_attn_workspace_bytes(pool, batch, q.shape[1], window, 4), dtype=torch.uint8, device=DEV)
            two.append((x, pool, ckv.PageLayers([pool]), batch, q, out, ws, window))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            serving_step(ckv, *two[0])
        sides.append((graph, *two))
    for i in range(4):
        for graph, a, b in sides:
            g = torch.Generator(DEV).manual_seed(i)
            fresh = torch.randn(a[4].shape, generator=g, device=DEV).to(a[4].dtype)
            for s in (a, b):
                s[4].copy_(fresh)
                s[3].lens.sub_(i)
            graph.replay()
            serving_step(ckv, *b)
            torch.cuda.synchronize()
            assert torch.equal(a[5], b[5])
            for n in ("k", "v", "k_scale", "v_scale"):
                u, v = getattr(a[1], n), getattr(b[1], n)
                assert u is None or torch.equal(bytes_of(u), bytes_of(v))
            for n in ("refs_out", "table_out", "live"):
                assert torch.equal(a[0][n], b[0][n])


def test_streams():
    """Calls on two streams at once, each with a workspace of its own, and a stream that is given."""
    import paper_2601_13631_amd as ckv
    cs = [Cache("bf16", H7, 32, [(1, 9000), (1, 500)], seed=i) for i in range(2)]
    made = [c.device() for c in cs]
    qs = [c.q.to(DEV) for c in cs]
    outs = [torch.zeros_like(q) for q in qs]
    wss = [torch.empty(ckv.page_attn_workspace_bytes(*m, 28), dtype=torch.uint8, device=DEV) for m in made]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for i in range(2):
            if i:
                ckv.page_attn(*made[i], qs[i], outs[i], wss[i], stream=streams[i])
            else:
                with torch.cuda.stream(streams[i]):
                    ckv.page_attn(*made[i], qs[i], outs[i], wss[i])
    torch.cuda.synchronize()
    for c, out in zip(cs, outs):
        check_attention(c, out)


def test_wrappers_refuse():
    import paper_2601_13631_amd as ckv
    c = Cache("bf16", H7, 16, [(3, 50)], seed=0)
    pool, batch = c.device()
    q = c.q.to(DEV)
    k = c.new_rows["k"].to(DEV)
    for bad in (q[:2], q.float(), q.cpu(), q.transpose(0, 1), q[..., :64]):
        with pytest.raises(ValueError):
            ckv.page_attn(pool, batch, bad, torch.empty_like(q))
    for bad in (q[:, :14], q.float(), torch.empty(q.shape[::-1], dtype=q.dtype, device=DEV).permute(2, 1, 0)):
        with pytest.raises(ValueError):
            ckv.page_attn(pool, batch, q, bad)
    with pytest.raises(ckv.CkvError):
        ckv.page_attn(pool, batch, q[:, :27].contiguous(), q[:, :27].contiguous())
    for bad in (dict(window=-1), dict(n_sinks=-1), dict(window=1 << 32)):
        with pytest.raises(ValueError):
            ckv.page_attn(pool, batch, q, torch.empty_like(q), **bad)
    for bad in (k[:2], k.float(), k[:, :2]):
        with pytest.raises(ValueError):
            ckv.page_append(pool, batch, bad, k)
    with pytest.raises(ValueError):
        ckv.PagePool(pool.k, pool.v, torch.zeros(c.n_pages, 4, dtype=torch.uint8, device=DEV))
    e = pool.k.to(torch.float8_e4m3fn)
    s = torch.zeros(c.n_pages, 4, dtype=torch.uint8, device=DEV)
    ckv.PagePool(e, e, s, s)
    for bad in ((None, None), (s, None), (s.int(), s), (s[:-1], s), (s.t().contiguous().t(), s)):
        with pytest.raises(ValueError):
            ckv.PagePool(e, e, *bad)
    with pytest.raises(ValueError):
        ckv.PagePool(pool.k.transpose(1, 2), pool.v.transpose(1, 2))
    with pytest.raises(ValueError):
        ckv.PagePool(pool.k[::2], pool.v[:pool.k[::2].shape[0]])
    for bad in (batch.table.long(), batch.table.t(), batch.table[0]):
        with pytest.raises(ValueError):
            ckv.PageBatch(bad, batch.lens, batch.tok_off, 3)
    with pytest.raises(ValueError):
        ckv.PageBatch(batch.table, batch.lens, batch.tok_off[:1], 3)
    i = torch.zeros(3, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        ckv.page_copy(ckv.PageLayers([pool]), i, i[:2])
    with pytest.raises(ValueError):
        ckv.page_copy(ckv.PageLayers([pool]), i.long(), i)


def test_wrappers_refuse_other_devices():
    """Handles made on another device than the call's (a device number that none has stands for it),
    and workspaces elsewhere or not contiguous."""
    import paper_2601_13631_amd as ckv
    c = Cache("bf16", H7, 16, [(3, 9000)], seed=0)
    q, i = c.q.to(DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    rows = [c.new_rows[n].to(DEV) for n in "kv"]
    for which in range(2):
        made = c.device()
        layers = ckv.PageLayers([made[0]])
        n = ckv.page_attn_workspace_bytes(*made, 28)
        assert n > 0
        ws = torch.empty(n, dtype=torch.uint8, device=DEV)
        made[which]._device = layers._device = 77
        with pytest.raises(ValueError, match="on device 77"):
            ckv.page_attn(*made, q, torch.empty_like(q), ws)
        with pytest.raises(ValueError, match="on device 77"):
            ckv.page_append(*made, *rows)
        with pytest.raises(ValueError, match="on device 77"):
            ckv.page_copy(layers, i, i)
        refs = torch.ones(c.n_pages, dtype=torch.int32, device=DEV)
        with pytest.raises(ValueError, match="on device 77"):
            ckv.page_compact(layers, refs, refs, None, None, i[:1], ws)
        with pytest.raises(ValueError, match="one device"):
            ckv.PageLayers([c.device()[0], _moved(c)])
    made = c.device()
    for bad in (ws.cpu(), ws[:1].expand(n), torch.empty(2 * n, dtype=torch.uint8, device=DEV)[::2]):
        with pytest.raises(ValueError, match="workspace"):
            ckv.page_attn(*made, q, torch.empty_like(q), bad)
        with pytest.raises(ValueError, match="workspace"):
            ckv.page_compact(ckv.PageLayers([]), i, i, None, None, i[:1], bad)


def _moved(c):
    pool = c.device()[0]
    pool._device = 77
    return pool
