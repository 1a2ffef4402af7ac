"""Beams whose logits are all far from zero, with maxima that rise along the vocabulary: the logarithm
of a beam's sum does not depend on where its logits lie."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from test_gpu_page_tables import T, check_select  # noqa: E402

OFFSETS = {"f32": (0.0, 100.0, -100.0, 500.0, -500.0, 1e4, -1e4, 1e5), "bf16": (0.0, 100.0, -100.0, 500.0, -500.0)}


def rising(kind, reqs, beams, vocab, offset, batches, seed):
    """Every wave of a scan has `batches` batches of 16,384 bytes over four waves in turn at most: of
    each the maximum is above the one before, by a step that the type holds at this offset."""
    per = 1024 if kind == "f32" else 2048
    step = max(1.0, 2 * abs(offset) * torch.finfo(T[kind]).eps)
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(reqs, beams, vocab, generator=g) * 0.25 * step
    return (x + (torch.arange(vocab) // per // 4 % batches) * step + offset).to(T[kind])


# With one request of two beams a workgroup has 16 batches, four a wave: three changes of the
# reference, as many as the bound of check_select has room for.
@pytest.mark.parametrize("kind,offset", [(k, o) for k, every in OFFSETS.items() for o in every])
def test_far_logits_rise_in_long_slices(kind, offset):
    vocab = 1000003 if kind == "f32" else 2000003
    x = rising(kind, 1, 2, vocab, offset, 4, 1)
    check_select(x, torch.tensor([[-1.0, -1.5]]), None, 4, -1)


# Enough rows for a workgroup each: three batches a wave at most.
@pytest.mark.parametrize("kind,offset", [("f32", 500.0), ("f32", -1e4), ("bf16", 500.0)])
def test_far_logits_rise_in_whole_rows(kind, offset):
    vocab = 9001 if kind == "f32" else 18001
    x = rising(kind, 1030, 1, vocab, offset, 3, 2)
    check_select(x, torch.full((1030, 1), -2.0), None, 2, -1)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_far_logits_of_beams_that_compete(kind):
    """The beams of a request differ in their offsets, which the logarithms take away again."""
    x = torch.cat([rising(kind, 1, 1, 200003, o, 4, i) for i, o in enumerate((-400.0, 0.0, 100.0, 450.0))], 1)
    check_select(x, torch.tensor([[-1.0, -1.25, -1.125, -1.0625]]), None, 12, -1)
