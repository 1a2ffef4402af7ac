"""Sequences with thousands of keys of their own behind (or without) shared ones: their keys are taken in
several splits, whatever the hints say of the prefixes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from pages_common import DEV, check_attention  # noqa: E402
from shared_common import GroupCache, attend_shared  # noqa: E402

H7, H14, H05, HF = (28, 4, 128), (40, 8, 128), (14, 2, 64), (4, 1, 64)
WIDE = 1 << 18

# (cache, heads, page, groups, sequences of no group)
CASES = [
    ("bf16", H7, 16, [(320, [(1, 4000), (1, 5), (1, 1500)]), (64, [(1, 2600), (1, 0)])], [(1, 3001), (1, 7)]),
    ("bf16", H05, 32, [(640, [(1, 3000), (1, 900)]), (1, [(1, 2000)] * 2)], [(1, 5000)]),
    ("bf16", H7, 8, [(200, [(30, 2500), (30, 60), (7, 1300)])], [(40, 3000), (1, 1)]),           # prompts
    ("bf16", H05, 96, [(960, [(45, 2000), (60, 1100)])], [(50, 2222)]),
    ("e4m3", H14, 16, [(333, [(1, 3000)] * 3 + [(1, 2)] * 3)], [(1, 2000)]),
    ("e4m3", H05, 64, [(640, [(1, 2500), (1, 100), (2, 1900)])], [(1, 4001)]),
    ("e4m3", H7, 32, [(96, [(33, 2000), (64, 1500)])], [(20, 2600)]),                              # prompts
    ("f32", HF, 16, [(512, [(1, 3000), (1, 50), (3, 1700)])], [(2, 2500), (1, 1)]),
]


def attend(c, pool, batch, g):
    """page_attn_shared, and how many splits each token's own keys were taken in: the last numbers of a
    workspace of parts, 256 bytes at a time (bit 30: there are shared keys)."""
    import paper_2601_13631_amd as ckv
    q = c.q.to(DEV)
    out = torch.full_like(q, 7.0)
    nbytes = ckv.page_attn_shared_workspace_bytes(pool, batch, g, c.hq)
    assert nbytes > (4 * c.d + 8) * c.hq * c.tokens  # (in parts)
    ws = torch.full((nbytes,), 0xFF, dtype=torch.uint8, device=DEV)
    ckv.page_attn_shared(pool, batch, g, q, out, ws)
    splits = ws[-(-(-4 * c.tokens // 256) * 256):].view(torch.int32)[:c.tokens] & ((1 << 30) - 1)
    return out, splits.cpu().numpy()


@pytest.mark.parametrize("hints", ["unknown", "half", "all"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_attention(i, hints):
    cache, heads, page, groups, loose = CASES[i]
    # (what is said of the prefixes makes the batch one that goes in parts; the lengths are as they are)
    said = {"unknown": 0, "half": WIDE // 2, "all": WIDE - 64}[hints]
    c = GroupCache(cache, heads, page, groups, loose, seed=70 + i, wide=WIDE // page)
    c.poison()
    pool, batch = c.device(max_len=0)
    g = c.device_groups(batch, max_shared=said)
    out, splits = attend(c, pool, batch, g)
    check_attention(c, out)
    if hints != "half":  # (which promises sequences of 131,072 keys of their own)
        long = np.repeat(c.lens - c.shared()[2] >= 2048, c.new)
        assert long.any() and (splits[long] > 1).all()


@pytest.mark.parametrize("cache,heads,new", [("bf16", H7, 1), ("bf16", H7, 40), ("e4m3", H05, 1), ("f32", HF, 2)])
def test_nothing_shared(cache, heads, new):
    """Groups whose sequences share no page: every key is an own one, in splits."""
    c = GroupCache(cache, heads, 16, [(0, [(new, 3000), (new, 2000)]), (0, [(new, 1000), (new, 2 * new)])], seed=5,
                   wide=WIDE // 16)
    c.poison()
    pool, batch = c.device(max_len=0)
    g = c.device_groups(batch, max_shared=0)
    out, splits = attend(c, pool, batch, g)
    check_attention(c, out)
    assert (g.shared[:2] == 0).all() and splits[0] > 1 and splits[-1] == 1


@pytest.mark.parametrize("cache,heads,new", [("bf16", H7, 1), ("bf16", H7, 33), ("e4m3", H05, 1), ("e4m3", H7, 33), ("f32", HF, 1)])
def test_layouts(cache, heads, new):
    """Missing pages among thousands of own ones, rows that rise along them, pages and tables that lie apart,
    rows behind the last sequence; the same bits each time."""
    want = None
    for how in range(3):
        c = GroupCache(cache, heads, 16, [(400, [(new, 3000), (new, 1033), (new, new)])], [(new, 2200)], seed=6,
                       wide=WIDE // 16, missing=[(b, s) for b in (0, 1, 2, 3) for s in (2, 40, 41, 97)],
                       gap=1024 if how == 1 else 0, interleaved=how == 2)
        for b, n, by in ((1, 1000, 6.0), (1, 2500, 9.0), (2, 1400, 8.0), (0, 2000, 7.0)):
            for h in range(c.hkv):
                x = c.q[c.off[b], h * (c.hq // c.hkv)].float() * by
                if cache == "e4m3":
                    x = (x * 16).clamp(-448, 448)
                    c.scale["k"][c.table[b, n // 16], h] = 123
                c.raw["k"][c.table[b, n // 16], n % 16, h] = x.to(c.raw["k"].dtype)
        c.poison()
        after = 3 if how == 1 else 0
        pool, batch = c.device(table_gap=9 * how, rows_after=after, max_len=0)
        out = attend_shared(pool, batch, c.device_groups(batch, max_shared=0), c.q.to(DEV), rows_after=after)
        check_attention(c, out)
        assert (out[c.tokens:] == 7).all()
        if not after:
            assert want is None or torch.equal(want, out)
            want = out


@pytest.mark.parametrize("seed", range(12))
def test_random(seed):
    rng = np.random.default_rng(900 + seed)
    cache = ("bf16", "e4m3", "f32")[seed % 3]
    d = 64 if cache == "f32" else int(rng.choice((64, 128)))
    hkv = int(rng.integers(1, 5))
    heads, page = (hkv * int(rng.integers(1, 9)), hkv, d), int(rng.choice((8, 16, 32, 96)))
    most = int(rng.choice((1, 1, 45)))

    def own():
        n = int(rng.integers(1, most + 1))
        return n, n + int(np.exp(rng.uniform(0, np.log(3000))))
    groups = [(int(np.exp(rng.uniform(0, np.log(900)))), [own() for _ in range(int(rng.integers(1, 4)))])
              for _ in range(int(rng.integers(1, 3)))]
    c = GroupCache(cache, heads, page, groups + [(0, [own()])], [own()], seed=seed, wide=2 * WIDE // page)
    c.poison()
    pool, batch = c.device(max_len=0)
    g = c.device_groups(batch, max_shared=int(rng.choice((0, WIDE // 2, 2 * WIDE - 5))))
    check_attention(c, attend_shared(pool, batch, g, c.q.to(DEV)))
