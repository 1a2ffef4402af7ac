"""Logits far from zero, finite in fp32: a query whose softmax has one key gives that key's V row, in
page_attn and page_attn_shared, with few rows and many.

The keys are such that one logit is above all others by at least 4/5 of the largest size, or the only one, so
that every other weight is 0 in 64 bits as in 32 (from 1,000 on, that is 800 nats down).  The numerators' one term w
then stands in output and sum alike, as rounded: w v / w.  In fp32 that is the product w v (half a step of
2^-24 of the result), scaled by a power of two or by exp2(0) where parts meet (exact), 1 / w (rounded: one
step, two halves) and their product (half a step): 2^-22 of |v|.  bf16: the output's half step, 2^-8, and
the same in fp32."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from pages_common import DEV, Cache, attend  # noqa: E402
from shared_common import GroupCache, attend_shared  # noqa: E402

H7, H05, HF = (28, 4, 128), (14, 2, 64), (4, 2, 64)
SIZES = [1e4, 5e6, 1.5e9, 3.75e9, 1e25]
WIDE = 1 << 18


def split(c, size):
    """Parts of a logit's size that queries and keys have (8-bit keys none of it, and one scale)."""
    if c.cache == "e4m3":
        c.scale["k"].fill_(127)
        return size, 1.0
    return float(np.sqrt(size)), float(np.sqrt(size))


def single_out(c, size, sign):
    """K and q such that each row's logit is sign * size (times 1 to 2.5) at the key that its sequence
    picks, and -size or, where that is negative itself, -5 size elsewhere: q = t u_h and k_j = a_j u_h for one
    vector u_h a KV head.  Returns the V rows that come out, in 64 bits."""
    g = torch.Generator().manual_seed(17)
    G = c.hq // c.hkv
    u = (torch.randint(0, 2, (c.hkv, c.d), generator=g) * 2 - 1).float()  # (entries of one size: sums are exact)
    in_q, in_k = split(c, size)
    t = 1 + torch.rand(c.tokens, c.hq, 1, generator=g)
    c.q = (t * in_q * u.repeat_interleave(G, 0)[None]).to(c.q.dtype)
    want = torch.zeros(c.tokens, c.hq, c.d, dtype=torch.double)
    v = torch.from_numpy(c.values("v"))
    lens, off = c.lens, c.off
    k = torch.zeros(c.raw["k"].shape)
    for b in range(len(c.seqs)):
        # positions that every query of the sequence sees: one of them is picked
        see = int(lens[b] - c.new[b]) + 1
        pick = {"first": 0, "last": see - 1, "shared": getattr(c, "whole_pages", {}).get(b, see) - 1}[c.pick]
        for s in range(-(-int(lens[b]) // c.page)):
            k[c.table[b, s]] = u[None] * (in_k * (-1.0 if sign > 0 else -5.0))
        at, row = c.table[b, pick // c.page], pick % c.page
        c.picked.append((at, row))
        want[off[b]:off[b + 1]] = v[at, row].repeat_interleave(G, 0)[None]
    for at, row in c.picked:
        k[at, row] = u * in_k * (1.0 if sign > 0 else -1.0)
    c.raw["k"] = (k * (1.0 + 0.25 * torch.rand(c.hkv, 1, generator=g))).to(c.raw["k"].dtype)
    return want


def check(c, got, want):
    u = 2.0 ** -22 if c.cache == "f32" else 2.0 ** -8 + 2.0 ** -22
    err = (got.cpu().double()[:c.tokens] - want).abs()
    assert torch.isfinite(got).all()
    assert (err <= u * want.abs()).all(), float((err / want.abs().clamp(min=1e-30)).max())


def whole(cache, heads, seqs, pick):
    c = Cache(cache, heads, 16, seqs, seed=9)
    c.picked, c.pick = [], pick
    return c


def grouped(cache, heads, groups, pick, wide=0):
    c = GroupCache(cache, heads, 16, groups, [(1, 1)], seed=9, wide=wide)
    c.picked, c.pick = [], pick
    c.whole_pages = {b: groups[i][0] // 16 * 16 for i in range(len(groups))
                     for b in range(c.grp_off[i], c.grp_off[i + 1])}
    return c


# (new tokens, length): one token alone; a few keys; keys in several steps, stages and splits; prompts
FEW = [(1, 1), (1, 40), (1, 700), (2, 33)]
MANY = [(40, 40), (33, 300), (5, 700), (40, 1500)]
# (every sequence sees keys of its own)
GROUPS_FEW = [(64, [(1, 1), (1, 700)]), (333, [(1, 1), (1, 9), (1, 40)])]
GROUPS_MANY = [(64, [(40, 40), (33, 64)]), (333, [(45, 45), (3, 9)])]
LONG = [(1, 6000), (5, 3001)]
GROUPS_LONG = [(4000, [(1, 7), (1, 40)]), (333, [(1, 1500), (1, 9)])]
ROWS = [(40, 6000), (33, 3001)]
GROUPS_ROWS = [(4000, [(33, 40), (40, 70)]), (333, [(1, 1500), (5, 9)])]
WHOLE = [("f32", HF, FEW), ("f32", HF, MANY), ("bf16", H7, FEW), ("bf16", H7, MANY), ("bf16", H05, MANY),
         ("e4m3", H7, MANY), ("e4m3", H05, MANY)]
SHARED = [("f32", HF, GROUPS_FEW), ("f32", HF, GROUPS_MANY), ("bf16", H7, GROUPS_FEW), ("bf16", H7, GROUPS_MANY),
          ("bf16", H05, GROUPS_MANY), ("e4m3", H7, GROUPS_MANY), ("e4m3", H05, GROUPS_FEW)]
LEVEL = WHOLE + [("f32", HF, LONG), ("bf16", H7, LONG), ("bf16", H7, ROWS), ("e4m3", H05, ROWS)]
LEVEL_SHARED = SHARED + [("f32", HF, GROUPS_LONG), ("bf16", H7, GROUPS_LONG), ("bf16", H05, GROUPS_ROWS),
                         ("e4m3", H7, GROUPS_ROWS)]


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("cache,heads,seqs", WHOLE)
@pytest.mark.parametrize("pick", ["first", "last"])
def test_page_attn(cache, heads, seqs, size, sign, pick):
    c = whole(cache, heads, seqs, pick)
    want = single_out(c, size, sign)
    pool, batch = c.device()
    check(c, attend(pool, batch, c.q.to(DEV), sm=1.0 / c.d), want)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("cache,heads,groups", SHARED)
@pytest.mark.parametrize("pick", ["first", "shared", "last"])
@pytest.mark.parametrize("apart", [True, False])
def test_page_attn_shared(cache, heads, groups, size, sign, pick, apart):
    """The picked key the first or the last of the shared ones, or one of each sequence's own; in parts (by
    the hints) and each sequence by itself."""
    c = grouped(cache, heads, groups, pick, WIDE // 16 if apart else 0)
    want = single_out(c, size, sign)
    pool, batch = c.device(**(dict(max_len=0) if apart else {}))
    g = c.device_groups(batch, **(dict(max_shared=0) if apart else {}))
    check(c, attend_shared(pool, batch, g, c.q.to(DEV), sm=1.0 / c.d), want)


def level(c, size, sign):
    """Every key of a KV head alike, so that all that a row sees weigh the same: the mean of their V
    rows in 64 bits, and of their sizes."""
    g = torch.Generator().manual_seed(23)
    G = c.hq // c.hkv
    u = (torch.randint(0, 2, (c.hkv, c.d), generator=g) * 2 - 1).float()
    in_q, in_k = split(c, size)
    c.q = ((1 + torch.rand(c.tokens, c.hq, 1, generator=g)) * in_q * u.repeat_interleave(G, 0)[None]).to(c.q.dtype)
    c.raw["k"] = (sign * in_k * u).expand(c.raw["k"].shape).to(c.raw["k"].dtype).contiguous()
    mean, size = (torch.zeros(c.tokens, c.hq, c.d, dtype=torch.double) for _ in "ms")
    v = c.values("v")
    for b, (n, m) in enumerate(c.seqs):
        rows = torch.from_numpy(c.rows(v, b)).repeat_interleave(G, 1)[:m]
        count = torch.arange(1, m + 1, dtype=torch.double)[:, None, None]
        for x, into in ((rows, mean), (rows.abs(), size)):
            into[c.off[b]:c.off[b + 1]] = (x.cumsum(0) / count)[m - n:]
    return mean, size


def check_level(c, got, want):
    """Equal weights w: sums of n products and of n weights, a rounding of 2^-24 of the sum of sizes each and
    one for each of 2^8 steps, waves, splits and parts at most that they are joined from; for bf16 the
    output's half step."""
    mean, size = want
    n = 2 * (int(c.lens.max()) + 256) * 2.0 ** -24
    bound = n * size + (0 if c.cache == "f32" else 2.0 ** -8 * mean.abs())
    err = (got.cpu().double()[:c.tokens] - mean).abs()
    assert torch.isfinite(got).all()
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("cache,heads,seqs", LEVEL)
def test_page_attn_of_equal_keys(cache, heads, seqs, size, sign):
    c = Cache(cache, heads, 16, seqs, seed=10)
    want = level(c, size, sign)
    pool, batch = c.device()
    check_level(c, attend(pool, batch, c.q.to(DEV), sm=1.0 / c.d), want)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("cache,heads,groups", LEVEL_SHARED)
@pytest.mark.parametrize("apart", [True, False])
def test_page_attn_shared_of_equal_keys(cache, heads, groups, size, sign, apart):
    c = GroupCache(cache, heads, 16, groups, [(1, 1)], seed=10, wide=WIDE // 16 if apart else 0)
    want = level(c, size, sign)
    pool, batch = c.device(**(dict(max_len=0) if apart else {}))
    g = c.device_groups(batch, **(dict(max_shared=0) if apart else {}))
    check_level(c, attend_shared(pool, batch, g, c.q.to(DEV), sm=1.0 / c.d), want)
