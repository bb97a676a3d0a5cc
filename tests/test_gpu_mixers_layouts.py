"""Memory orders that models have: heads before tokens, tokens before the batch, queries, keys and values side by side.
Every call gives the bits that it gives for contiguous tensors."""
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


def heads_first(t):
    """The same values, in memory [B,H,T,d]."""
    return t.transpose(1, 2).contiguous().transpose(1, 2)


def tokens_first(t):
    """... [T,B,H,d] ([T,B,C])."""
    return t.transpose(0, 1).contiguous().transpose(0, 1)


def beside(*ts):
    """... of several tensors side by side, [B,T,all heads,d]."""
    return torch.cat(ts, 2).split([t.shape[2] for t in ts], 2)


LAYOUTS = {"heads first": lambda *ts: [heads_first(t) for t in ts], "tokens first": lambda *ts: [tokens_first(t) for t in ts],
           "beside": beside}


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("B,T,Hq,Hk,d", [(3, 200, 6, 2, 64), (1, 130, 2, 1, 64), (2, 150, 4, 4, 32), (4, 1, 2, 2, 64)])
def test_window_and_rotation_in_any_order_of_memory(ctx, B, T, Hq, Hk, d, layout, dtype):
    q, k, v = (draw(n, B, T, h, d, dtype=dtype) for n, h in ((1, Hq), (2, Hk), (3, Hk)))
    do, dk = draw(4, B, T, Hq, d, dtype=dtype), draw(5, B, T, Hk, d, dtype=dtype)
    lens = torch.tensor([max(T - 40 * b, 0) for b in range(B)], dtype=torch.int32, device="cuda")
    table = binding.rope_table(32, d, True, device="cuda")
    w = draw(6, d)

    def run(q, k, v, do, dk, outs):
        """outs(like, ..): tensors of these shapes to be written, or Nones."""
        o, lse = ctx.lasad_window_attention(q, k, v, 50, 2, lengths=lens, want_lse=True, o=outs(q)[0])
        dq_, dk_, dv_ = outs(q, k, v)
        grads = ctx.lasad_window_attention_backward(q, k, v, o, lse, do, 50, 2, lengths=lens, dq=dq_, dk=dk_, dv=dv_)
        a, b = outs(q, k)
        turned = ctx.lasad_qk_norm_rope(q, k, table, w, w, grid_w=24, prefix_len=1, q_out=a, k_out=b)
        a, b = outs(q, k)
        back = ctx.lasad_qk_norm_rope_backward(q, k, table, do, dk, w, w, grid_w=24, prefix_len=1, dq=a, dk=b)
        return (o, lse) + grads + turned + back
    want = run(q, k, v, do, dk, lambda *ts: [None] * len(ts))
    lay = LAYOUTS[layout]
    got = run(*lay(q, k, v), *lay(do, dk), lambda *ts: lay(*(torch.full_like(t, float("nan"), memory_format=torch.contiguous_format)
                                                            for t in ts)))
    for n, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a, b), n
    assert ctx.device_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hq,Hk,d,win", [(3, 8, 2, 64, 40), (5, 2, 2, 32, 7), (2, 4, 2, 64, 2000), (300, 8, 8, 64, 5)])
def test_step_and_store_in_any_order_of_memory(ctx, B, Hq, Hk, d, win, dtype):
    T, sinks = 30, 2
    k, v = draw(1, B, T, Hk, d, dtype=dtype), draw(2, B, T, Hk, d, dtype=dtype)
    q1, k1, v1 = (draw(n, B, h, d, dtype=dtype) for n, h in ((3, Hq), (4, Hk), (5, Hk)))
    lens = torch.tensor([b % (T + 1) for b in range(B)], dtype=torch.int32, device="cuda")

    def run(lay, lay1, k, v, q1, k1, v1):
        caches = lay(*(draw(6 + n, B, sinks + win, Hk, d, dtype=dtype) for n in range(2)))
        ctx.lasad_window_cache_store(*lay(k, v), *caches, win, sinks, lengths=lens)
        o = ctx.lasad_window_attention_step(*lay1(q1, k1, v1), *caches, lens, win, sinks)
        return [o] + list(caches)
    want = run(lambda *ts: ts, lambda *ts: ts, k, v, q1, k1, v1)
    for name, lay in LAYOUTS.items():
        one = lambda *ts: [t[:, 0] for t in lay(*(t[:, None] for t in ts))]      # noqa: E731
        for a, b in zip(run(lay, one, k, v, q1, k1, v1), want):
            assert torch.equal(a, b), name


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,C", [(3, 300, 64), (2, 1500, 64), (2, 1500, 30), (4, 5, 17), (3, 1, 64)])
def test_recurrence_in_any_order_of_memory(ctx, B, T, C, dtype):
    x, z, dy = (draw(n, B, T, C, dtype=dtype) for n in (1, 2, 3))
    h, dh = draw(4, B, C), draw(5, B, C)

    def run(x, z, dy, outs):
        y, hn, saved = ctx.lasad_scan_forward(x, z, grid_w=24, logits=True, h_in=h, save=True, y=outs[0])
        return (y, hn, saved) + ctx.lasad_scan_backward(x, z, saved, dy, dh_out=dh, grid_w=24, logits=True, dx=outs[1], dgate=outs[2])
    want = run(x, z, dy, [None] * 3)
    side = torch.cat((x, z, dy), 2).split(C, 2)
    empty = lambda: torch.full((B, T, C), float("nan"), dtype=dtype, device="cuda")      # noqa: E731
    for args in ([tokens_first(t) for t in (x, z, dy)], side):
        for outs in ([tokens_first(empty()) for _ in range(3)], torch.cat([empty()] * 3, 2).split(C, 2)):
            for a, b in zip(run(*args, outs), want):      # (single channels and pairs round alike)
                assert torch.equal(a, b)
