"""Equal beams whose two best tokens are equal: all four continuations tie, whatever the logarithm of the
beams' sums is."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from pages_common import DEV  # noqa: E402
from test_gpu_page_tables import T  # noqa: E402


# (a beam's sum is joined from 8, 64 and 1 slices; in the few cases in which lanes that hold the sums of
# different roundings would part, they do so for one request in thousands)
@pytest.mark.parametrize("kind,reqs,vocab,calls", [("f32", 64, 40001, 400), ("bf16", 64, 70001, 400),
                                                   ("f32", 8, 300007, 300), ("f32", 600, 2001, 50)])
def test_equal_tokens_of_equal_beams(kind, reqs, vocab, calls):
    import paper_2601_13631_amd as ckv
    g = torch.Generator(device=DEV).manual_seed(reqs)
    scores = torch.full((reqs, 2), -1.0, device=DEV)
    parent, token = (torch.empty(reqs, 4, dtype=torch.int32, device=DEV) for _ in "pt")
    best = torch.empty(reqs, 4, device=DEV)
    x = torch.empty(reqs, 2, vocab, dtype=T[kind], device=DEV)
    ws = torch.empty(ckv.beam_select_workspace_bytes(x, 4), dtype=torch.uint8, device=DEV)
    first = 2 * torch.arange(reqs, dtype=torch.int32, device=DEV)[:, None]
    lo, hi = vocab // 3, vocab - 5
    wrong = torch.zeros((), dtype=torch.long, device=DEV)
    for _ in range(calls):
        one = torch.randn(reqs, 1, vocab, generator=g, device=DEV)
        one[:, :, lo] = one[:, :, hi] = 9.0  # (6 is passed by one of 10^9 numbers)
        x.copy_(one)
        ckv.beam_select(x, scores, parent, token, best, ws)
        wrong += ((parent != first + torch.tensor([0, 0, 1, 1], dtype=torch.int32, device=DEV)) |
                  (token != torch.tensor([lo, hi, lo, hi], dtype=torch.int32, device=DEV))).any(1).sum()
    assert int(wrong) == 0
