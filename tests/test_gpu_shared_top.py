"""8-bit pages of the largest scale among shared ones: workgroups of several row blocks and 128-row tiles
read codes of 256 and more as 240 times the scale, as page_attn does."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from pages_common import DEV, check_attention  # noqa: E402
from shared_common import GroupCache, attend_shared  # noqa: E402
from test_gpu_page_top import TOP, put  # noqa: E402

H05, H7, H14 = (14, 2, 64), (28, 4, 128), (40, 8, 128)
WIDE = 1 << 18


class Top(GroupCache):
    def values(self, n):
        return super().values(n).clip(-TOP, TOP)


# rows of a group, by the mean with the sequence of none: 28 (two blocks), 45 and 42 (three), 77 (tiles)
SHAPES = [(heads, page, n) for heads, n in ((H7, 3), (H14, 8), (H05, 5), (H7, 10)) for page in (8, 16, 96)]


def cache(heads, page, n, seed, shared=1000, own=130):
    return Top("e4m3", heads, page, [(shared, [(1, own)] * n)], [(1, 50)], seed=seed, wide=WIDE // page)


def attend(c, sm):
    pool, batch = c.device(max_len=0)
    return attend_shared(pool, batch, c.device_groups(batch, max_shared=0), c.q.to(DEV), sm=sm)


@pytest.mark.parametrize("heads,page,n", SHAPES)
@pytest.mark.parametrize("where", ["shared", "own"])
def test_largest_values_among_others(heads, page, n, where):
    """A row of V of the largest values among the shared keys, or one among the own, beside others that
    count alike.  (Two of one sign, 1.875 * 2^128 together, pass fp32's range before they are divided.)"""
    c = cache(heads, page, n, 3)
    for b, pos in [(1, 333)] if where == "shared" else [(b, 1100) for b in range(1, n + 1)]:
        for h in range(c.hkv):
            put(c, "v", b, pos, h, [256.0, -448.0, 288.0, -416.0][(b + h) % 4])
    check_attention(c, attend(c, 1e-6), sm=1e-6)


@pytest.mark.parametrize("heads,page,n", SHAPES)
def test_largest_keys(heads, page, n):
    """Rows of K of the largest values, whose logits small queries keep small."""
    c = cache(heads, page, n, 4)
    c.q = torch.where(c.q.abs() < 0.25, 0.25, c.q.float()).to(torch.bfloat16) * 2.0 ** -124  # (no less than 2^-126)
    code = torch.zeros(c.d)
    code[:3] = torch.tensor([448.0, 256.0, -288.0])
    for b, pos in [(1, 77), (1, 640)] + [(b, 1050) for b in range(1, n + 1)]:
        for h in range(c.hkv):
            put(c, "k", b, pos, h, code)
    check_attention(c, attend(c, 1.0), sm=1.0)
