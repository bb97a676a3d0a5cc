"""The ways in which calls of real sizes are cut, against the float64 forms: the recurrence over whole tiles, segments
and both at once, the window's kernels with several units of work for every SM, and what the smaller cases leave out."""
import math

import pytest
import torch

from paper_2507_01652_b200 import binding
from tests import _mixers_ref as ref
from tests.test_gpu_mixers import check_window, d64, near, strided, window_case

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    torch.cuda.set_device(0)
    c = binding.Lasad(0)
    yield c
    c.close()


def draw(seed, *shape, dtype=F32, mean=0.0, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)


# ---------------------------------------------------------------------------------------------
# gated linear recurrence
# ---------------------------------------------------------------------------------------------
def tiles_past_a_round(dtype, backward):
    """Tiles of 32 channels: 20 more than CTAs that run at a time, so that the last round of tiles is cut."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    return sms * ((2 if backward else 3) if dtype == BF16 else (1 if backward else 2)) + 20


def check_scan(ctx, B, T, C, dtype, w=96, P=1, t0=0, tied=True, logits=True, gate=None):
    x, dy = draw(1, B, T, C, dtype=dtype), draw(2, B, T, C, dtype=dtype)
    if gate is None:
        z = draw(3, B, T, C, mean=1.5, std=2.0)
        gate = (z if logits else torch.sigmoid(z)).to(dtype)
    h_in, dh = draw(4, B, C), draw(5, B, C)
    kw = dict(grid_w=w, prefix_len=P, t0=t0, tied=tied, logits=logits)
    leaves = [t.double().requires_grad_() for t in (x, gate, h_in)]
    y, h = ref.scan(*leaves, w, P, t0, tied, logits)
    wants = torch.autograd.grad([y, h], leaves, [dy.double(), dh.double()], materialize_grads=True)
    got_y, got_h, saved = ctx.lasad_scan_forward(x, gate, h_in=h_in, save=True, **kw)
    near(got_y, y.detach().cpu(), dtype, "y")
    near(got_h, h.detach().cpu(), F32, "h_out")
    before = torch.stack([leaves[2].detach()] + [y[:, t - 1].detach() for t in range(128, T, 128)], 1)
    near(saved, before.cpu(), F32, "saved")
    back = ctx.lasad_scan_backward(x, gate, saved, dy, dh_out=dh, **kw)
    for n, a, b, t in zip(("dx", "dgate", "dh_in"), back, wants, (dtype, dtype, F32)):
        near(a, b.cpu(), t, n)
    only, none, nosave = ctx.lasad_scan_forward(x, gate, h_in=h_in, want_state=False, **kw)
    assert none is None and nosave is None and torch.equal(only, got_y)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tied,logits", [(True, True), (False, False)])
@pytest.mark.parametrize("shape", [
    (2, 500, 64),                                  # a few chunks, one after another: staging places used again
    (1, 1000, 64), (1, 1100, 96), (1, 2500, 96),   # cut into segments; the last one short, a last chunk of 104, 76, 68 tokens
    (2, 2500, 40),                                 # a tile that is not full
    (1, 1100, 6400),                               # so many tiles that none is cut
    (1, 5000, 17),                                 # single channels, cut
])
def test_recurrence_as_it_is_cut(ctx, shape, tied, logits, dtype):
    check_scan(ctx, *shape, dtype, tied=tied, logits=logits)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("backward", [False, True])
def test_recurrence_with_its_last_round_cut(ctx, dtype, backward):
    check_scan(ctx, 2, 1200, 16 * tiles_past_a_round(dtype, backward), dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("logits", [False, True])
@pytest.mark.parametrize("shape", [(2, 300, 64), (1, 1500, 64), (1, 1500, 33)])
def test_recurrence_gates_at_their_ends(ctx, shape, logits, dtype):
    """Gates of exactly 0 and 1, logits up to infinity, in the forward and the gradient; a NaN stays in its channel."""
    vals = [-math.inf, math.inf, -120.0, 120.0, 0.0] if logits else [0.0, 1.0, 0.5]
    g = torch.Generator(device="cuda").manual_seed(9)
    gate = torch.tensor(vals, device="cuda")[torch.randint(len(vals), shape, generator=g, device="cuda")].to(dtype)
    check_scan(ctx, *shape, dtype, w=16, tied=True, logits=logits, gate=gate)
    x, dy = draw(1, *shape, dtype=dtype), draw(2, *shape, dtype=dtype)
    others = torch.arange(shape[2], device="cuda") != 7

    def run():
        y, h, saved = ctx.lasad_scan_forward(x, gate, grid_w=16, logits=logits, save=True)
        return (y, h) + ctx.lasad_scan_backward(x, gate, saved, dy, grid_w=16, logits=logits)
    want = run()
    x[0, 200, 7] = float("nan")
    for a, b in zip(run(), want):
        assert torch.equal(a[..., others], b[..., others])
    assert bool(run()[0][0, 200, 7].isnan()) and bool(run()[0][0, :200, 7].isfinite().all())


# ---------------------------------------------------------------------------------------------
# norm and rotation
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("want_weights", [False, True])
def test_rotation_gradient_without_weights(ctx, want_weights, half, dtype):
    q, k = draw(1, 3, 50, 6, 64, dtype=dtype), draw(2, 3, 50, 2, 64, dtype=dtype, std=3.0)
    dq, dk = draw(3, 3, 50, 6, 64, dtype=dtype), draw(4, 3, 50, 2, 64, dtype=dtype)
    table = binding.rope_table(64, 64, True, device="cuda")
    kw = dict(grid_w=7, prefix_len=2, half=half, eps=1e-6)
    got = ctx.lasad_qk_norm_rope_backward(q, k, table, dq, dk, want_weights=want_weights, **kw)
    for n, (x, dy) in enumerate(((q, dq), (k, dk))):
        leaf, w = d64(x).requires_grad_(), torch.ones(64, dtype=torch.float64, requires_grad=True)
        y = ref.rope_one(leaf, w, 0, 7, 2, half, 1e-6)
        want, dw = torch.autograd.grad(y, (leaf, w), d64(dy))
        near(got[n], want, dtype, n)
        if want_weights:
            near(got[2 + n], dw, F32, ("dw", n), acc=2.0 ** -18)
        else:
            assert got[2 + n] is None


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rotation_over_many_tokens(ctx, dtype):
    """Runs of several tokens a warp in the gradient, runs that pass from a sequence to the next, and its sums over them."""
    B, T, Hq, Hk = 6, 1000, 5, 2
    q, k = draw(1, B, T, Hq, 64, dtype=dtype), draw(2, B, T, Hk, 64, dtype=dtype)
    dq, dk = draw(3, B, T, Hq, 64, dtype=dtype), draw(4, B, T, Hk, 64, dtype=dtype)
    wq, wk = draw(5, 64, mean=1.0, std=0.2), draw(6, 64, mean=1.0, std=0.2)
    pos = torch.tensor([0, 3, 500, 77, 1, 9], dtype=torch.int32, device="cuda")
    table = binding.rope_table(128, 64, True, device="cuda")
    kw = dict(q_weight=wq, k_weight=wk, grid_w=24, prefix_len=1, pos=pos, eps=1e-6)
    y = ctx.lasad_qk_norm_rope(q, k, table, **kw)
    back = ctx.lasad_qk_norm_rope_backward(q, k, table, dq, dk, **kw)
    for n, (x, w, dy) in enumerate(((q, wq, dq), (k, wk, dk))):
        leaf, lw = d64(x).requires_grad_(), d64(w).requires_grad_()
        want = ref.rope_one(leaf, lw, pos.cpu().long(), 24, 1, False, 1e-6)
        dx, dw = torch.autograd.grad(want, (leaf, lw), d64(dy))
        near(y[n], want.detach(), dtype, n)
        near(back[n], dx, dtype, n)
        near(back[2 + n], dw, F32, n, acc=2.0 ** -18)


# ---------------------------------------------------------------------------------------------
# window attention
# ---------------------------------------------------------------------------------------------
def spread(B, T):
    return tuple(T * b // (B - 1) for b in range(B))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [
    # more units (128 queries of a head) than three for every SM: a group of warps takes another one; lengths from 0 on
    # leave units without a tile between others
    (64, 300, 4, 2, 64, 37, 2, spread(64, 300)), (100, 300, 4, 4, 32, 300, 0, spread(100, 300)),
    (200, 130, 4, 1, 64, 20, 3, None), (1, 4000, 16, 2, 64, 64, 1, None),
])
def test_window_with_several_units_for_every_sm(ctx, shape, dtype):
    check_window(ctx, shape, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T", [(1, 1), (3, 200), (200, 130)])
def test_window_of_empty_sequences(ctx, B, T, dtype):
    q, k = (torch.full((B, T, h, 64), float("nan"), dtype=dtype, device="cuda") for h in (4, 2))
    kw = dict(window=16, sinks=1, lengths=torch.zeros(B, dtype=torch.int32, device="cuda"))
    o, lse = ctx.lasad_window_attention(q, k, k, want_lse=True, **kw)
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())
    assert all(bool((g == 0).all()) for g in ctx.lasad_window_attention_backward(q, k, k, q, lse, q, **kw))


@pytest.mark.parametrize("shape", [(3, 900, 6, 2, 64, 200, 5, (900, 513, 128)), (40, 257, 8, 4, 64, 37, 3, spread(40, 257))])
def test_window_on_tensor_cores_against_cuda_cores(ctx, shape):
    """Both implementations on the same bf16 tensors: apart by the bounds of both at most."""
    B, T, Hq, Hk, d, win, sinks, lengths = shape
    host, (q, k, v, do) = window_case(B, T, Hq, Hk, d, BF16, lengths, 3)
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    bounds = ref.window_bounds(*[d64(t) for t in host], win, sinks, None, lengths)
    got = []
    try:
        for impl in (1, 2):
            ctx.set_option(binding.LASAD_OPT_WINDOW_IMPL, impl)
            o, lse = ctx.lasad_window_attention(q, k, v, win, sinks, lengths=lens, want_lse=True)
            got.append((o, lse) + ctx.lasad_window_attention_backward(q, k, v, o, lse, do, win, sinks, lengths=lens))
    finally:
        ctx.set_option(binding.LASAD_OPT_WINDOW_IMPL, 0)
    near(got[0][1], d64(got[1][1]), F32, "lse", extra=2.0 ** -18)
    for name, a, b in zip(("o", "dq", "dk", "dv"), got[0][:1] + got[0][2:], got[1][:1] + got[1][2:]):
        assert bool(((d64(a) - d64(b)).abs() <= 2.04 * bounds[name] + 1e-30).all()), name


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("T,Hk,d,win,sinks", [(1, 1, 64, 1, 0), (50, 3, 32, 16, 2), (90, 2, 64, 24, 0), (20, 4, 64, 100, 5)])
def test_window_cache_store(ctx, T, Hk, d, win, sinks, pad, dtype):
    """Every slot has its last token or, where none has reached it, what it had."""
    lengths = [0, 1, min(sinks + 1, T), min(sinks + win, T), T, T // 2]
    B = len(lengths)
    k, v = draw(1, B, T, Hk, d, dtype=dtype), draw(2, B, T, Hk, d, dtype=dtype)
    for lens in (lengths, None):
        want = [draw(3 + n, B, sinks + win, Hk, d, dtype=dtype) for n in range(2)]
        caches = [strided(t.clone(), pad) for t in want]
        for b in range(B):
            for s in range(lengths[b] if lens else T):
                slot = s if s < sinks else sinks + (s - sinks) % win
                want[0][b, slot], want[1][b, slot] = k[b, s], v[b, s]
        ctx.lasad_window_cache_store(strided(k, pad), strided(v, pad), *caches, win, sinks,
                                     lengths=torch.tensor(lens, dtype=torch.int32, device="cuda") if lens else None)
        for a, b in zip(caches, want):
            assert torch.equal(a, b)
