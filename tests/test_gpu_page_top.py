"""8-bit pages whose scale byte is 247: 256 times the scale is 2^128, which bf16 does not hold, and what
was appended there was finite.  Codes of 256 and more are read as 240 times the scale."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from pages_common import DEV, Cache, attend, check_attention  # noqa: E402

H05, H7 = (14, 2, 64), (28, 4, 128)
TOP = 240 * 2.0 ** 120
BIG = float(torch.finfo(torch.bfloat16).max)


class Top(Cache):
    def values(self, n):
        return np.clip(super().values(n), -TOP, TOP)


def put(c, n, b, pos, h, code, byte=247):
    """Code values into row `pos` of sequence b, head h; the page's other codes become 0."""
    at, row = c.table[b, pos // c.page], pos % c.page
    c.raw[n][at, :, h] = torch.zeros(c.page, c.d).to(torch.float8_e4m3fn)
    c.raw[n][at, row, h] = torch.as_tensor(code, dtype=torch.float32).expand(c.d).to(torch.float8_e4m3fn)
    c.scale[n][at, h] = byte


# few rows (workgroups of 8 waves and, for many sequences, of 4) and many; pages of 8 and more tokens
SHAPES = [(heads, page, new, n) for heads in (H7, H05) for page in (8, 16, 96) for new, n in ((1, 2), (1, 140), (40, 2))]


@pytest.mark.parametrize("heads,page,new,n", SHAPES)
def test_appended_rows_come_back(heads, page, new, n):
    """Every query sees its own row alone: rows of the largest finite numbers are off by half a step
    of e4m3 at most, 2^-4 of them; an infinity beside them is read as the largest finite one."""
    import paper_2601_13631_amd as ckv
    c = Top("e4m3", heads, page, [(new, 3 * page + new + b % 5) for b in range(n)], seed=page)
    sign = torch.where(torch.rand(c.new_rows["v"].shape, generator=torch.Generator().manual_seed(1)) < 0.5, -1.0, 1.0)
    size = torch.tensor([BIG, 248.0 * 2.0 ** 120, 2.0 ** 127, 1.9375 * 2.0 ** 127])[torch.arange(c.tokens) % 4]
    given = sign * size[:, None, None]
    c.new_rows["v"] = given.to(torch.bfloat16)
    c.new_rows["v"][:, :, 0] = torch.where(torch.arange(c.tokens) % 3 == 0, float("inf"), c.new_rows["v"][:, :, 0].float().T).T.to(torch.bfloat16)
    pool, batch = c.device()
    ckv.page_append(pool, batch, c.new_rows["k"].to(DEV), c.new_rows["v"].to(DEV))
    c.append()
    out = attend(pool, batch, c.q.to(DEV), window=1)
    check_attention(c, out, window=1)
    got, want = out.cpu().double(), given.double().repeat_interleave(c.hq // c.hkv, 1)
    # the page's byte is 247 where one of its rows is above 448 * 2^119, as every page's is here but
    # for those with rows of 2^127 alone
    finite = torch.isfinite(c.new_rows["v"].double()).repeat_interleave(c.hq // c.hkv, 1)
    assert (got - want)[finite].abs().le(2.0 ** -4 * want[finite].abs()).all()
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("heads,page,new,n", SHAPES)
def test_largest_values_among_others(heads, page, new, n):
    """One row of V of the largest values among 700 that count alike, and splits to join."""
    length = 6000 if n == 2 else 700
    c = Top("e4m3", heads, page, [(new, length)] * n, seed=3)
    for b in range(n):
        for h in range(c.hkv):
            put(c, "v", b, 333, h, [256.0, -448.0, 288.0, -416.0][(b + h) % 4])
    pool, batch = c.device()
    out = attend(pool, batch, c.q.to(DEV), sm=1e-6)
    check_attention(c, out, sm=1e-6)


@pytest.mark.parametrize("heads,page,new,n", SHAPES)
def test_largest_keys(heads, page, new, n):
    """A row of K of the largest values, whose logits small queries keep small."""
    c = Top("e4m3", heads, page, [(new, 200 + new)] * n, seed=4)
    c.q = torch.where(c.q.abs() < 0.25, 0.25, c.q.float()).to(torch.bfloat16) * 2.0 ** -124  # (no less than 2^-126)
    for b in range(n):
        for h in range(c.hkv):
            code = torch.zeros(c.d)
            code[:3] = torch.tensor([448.0, 256.0, -288.0])
            put(c, "k", b, 77, h, code)
    pool, batch = c.device()
    out = attend(pool, batch, c.q.to(DEV), sm=1.0)
    check_attention(c, out, sm=1.0)


@pytest.mark.parametrize("heads,page,new,n", SHAPES)
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_a_largest_key_alone(heads, page, new, n, sign):
    """Queries that see one key of the largest values give its V row, whichever sign the logit has."""
    c = Top("e4m3", heads, page, [(new, page + new)] * n, seed=5)
    c.q = c.q.abs().clamp(0.25, 2.0) * 2.0 ** -124
    for x in c.table.reshape(-1):
        if x >= 0:
            c.raw["k"][x] = torch.full(c.raw["k"][x].shape, sign * 448.0).to(torch.float8_e4m3fn)
            c.scale["k"][x] = 247
    pool, batch = c.device()
    check_attention(c, attend(pool, batch, c.q.to(DEV), window=1, sm=0.125), window=1, sm=0.125)
