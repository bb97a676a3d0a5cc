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


def test_streams_by_their_handles(ctx):
    """The default stream by its handle 0, a stream that is current, one that is being captured."""
    import ctypes
    x, z = draw(1, 1, 3000, 64), draw(2, 1, 3000, 64)
    want = ctx.lasad_scan_forward(x, z, logits=True)[:2]
    torch.cuda.synchronize()
    for handle in (0, ctypes.c_void_p(0), torch.cuda.current_stream().cuda_stream):
        got = ctx.lasad_scan_forward(x, z, logits=True, stream=handle)[:2]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = ctx.lasad_scan_forward(x, z, logits=True, stream=torch.cuda.current_stream().cuda_stream)[:2]
    for t in held:
        t.fill_(float("nan"))
    torch.empty(1 << 22, device="cuda").fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, want))


# ---------------------------------------------------------------------------------------------
# states written where they were read
# ---------------------------------------------------------------------------------------------
PIECES = [  # B, T, C, tokens of the first piece: pieces that are cut into segments (8 chunks of 128 and more) and whole
    (1, 3000, 64, 1500), (2, 2500, 34, 1100), (3, 2100, 96, 60), (1, 4700, 1536, 2350),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", PIECES)
def test_recurrence_carries_its_state_in_place(ctx, shape, dtype):
    """A sequence in two pieces with the state, and its gradient, in one piece of memory: the same bits as with
    memory of their own for each."""
    B, T, C, cut = shape
    x, z, dy = (draw(n, B, T, C, dtype=dtype) for n in (1, 2, 3))
    h_in, dh_out = draw(4, B, C), draw(5, B, C)
    kw = dict(grid_w=24, prefix_len=1, logits=True)
    halves = [(t[:, :cut], t[:, cut:]) for t in (x, z, dy)]

    def run(place):
        """place(t): where the state that replaces t goes."""
        h, u, ys, saves, grads = h_in.clone(), dh_out.clone(), [], [], []
        for n, t0 in ((0, 0), (1, cut)):
            y, h, saved = ctx.lasad_scan_forward(halves[0][n], halves[1][n], t0=t0, h_in=h, h_out=place(h), save=True, **kw)
            ys.append(y)
            saves.append(saved)
        for n, t0 in ((1, cut), (0, 0)):
            dx, dz, u = ctx.lasad_scan_backward(halves[0][n], halves[1][n], saves[n], halves[2][n], t0=t0, dh_out=u,
                                                dh_in=place(u), **kw)
            grads += [dx, dz]
        return ys + saves + grads + [h, u]
    apart = run(lambda t: None)
    for _ in range(5):
        for a, b in zip(run(lambda t: t), apart):
            assert torch.equal(a, b)
