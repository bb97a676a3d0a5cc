"""What stands in the padded rows of a batch reaches no bit of the others."""
import pytest
import torch

from tests.test_gpu_mixers import BF16, ctx, gen, rnd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks", [(1000, 0), (300, 4)])
@pytest.mark.parametrize("n", [513, 577, 70])
def test_window_rows_behind_a_sequence_do_not_move_its_maximum(ctx, n, window, sinks):      # noqa: F811
    """Padded queries of 60 times the size: their scores are hundreds, and their maxima move in tile after tile."""
    g = gen(43)
    T = 800
    q, k, v = (rnd(g, 1, T, h, 64, std=s, dtype=BF16) for h, s in ((4, 1.5), (2, 1.0), (2, 1.0)))
    lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
    outs = []
    for size in (1.0, 60.0):
        q2 = q.clone()
        q2[:, n:] *= size
        outs.append(ctx.lasad_window_attention(q2.cuda(), k.cuda(), v.cuda(), window, sinks=sinks, lengths=lengths, want_lse=True))
    (a, la), (b, lb) = outs
    assert torch.equal(a, b) and torch.equal(la, lb)
