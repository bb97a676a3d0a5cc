"""Whose memory the operators beside LASAD work in: calls on a stream other than the current one, and states
that are written where they were read."""
import pytest
import torch

from paper_2507_01652_b200 import binding

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    torch.cuda.set_device(0)
    c = binding.Lasad(0)
    yield c
    c.close()


def draw(seed, *shape, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def check_two_streams(ctx, call):
    """A call on the current stream, and the same at once on another one: both as it is alone.  The first has let go
    of its workspace and outputs when the second allocates, and is still at work."""
    alone = [t.clone() for t in call()]
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    kept = []
    for n in range(12):
        if n % 2:
            kept.append(call())
        else:
            call()                                     # (dropped: its outputs are free again too)
        kept.append(call(stream=other.cuda_stream))
    torch.cuda.synchronize()
    for got in kept:
        assert all(torch.equal(a, b) for a, b in zip(got, alone))
    assert ctx.device_status() == 0


def test_window_gradient_on_two_streams(ctx):
    q, do = draw(1, 1, 2305, 8, 64, dtype=BF16), draw(2, 1, 2305, 8, 64, dtype=BF16)
    k, v = draw(3, 1, 2305, 4, 64, dtype=BF16), draw(4, 1, 2305, 4, 64, dtype=BF16)
    o, lse = ctx.lasad_window_attention(q, k, v, 700, 3, want_lse=True)
    check_two_streams(ctx, lambda **s: ctx.lasad_window_attention_backward(q, k, v, o, lse, do, 700, 3, **s))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_cut_recurrence_on_two_streams(ctx, dtype):
    x, z, dy = (draw(n, 1, 5000, 256, dtype=dtype) for n in (1, 2, 3))

    def call(**s):
        y, h, saved = ctx.lasad_scan_forward(x, z, logits=True, save=True, **s)
        return (y, h, saved) + ctx.lasad_scan_backward(x, z, saved, dy, dh_out=h, logits=True, **s)
    check_two_streams(ctx, call)


def test_weight_gradients_on_two_streams(ctx):
    q, k, dq, dk = (draw(n, 4, 2000, 8, 64, dtype=BF16) for n in (1, 2, 3, 4))
    table, w = binding.rope_table(2000, 64, False, device="cuda"), draw(5, 64)
    check_two_streams(ctx, lambda **s: ctx.lasad_qk_norm_rope_backward(q, k, table, dq, dk, w, w, **s))
