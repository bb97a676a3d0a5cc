"""The operators beside LASAD on the GPU against their float64 forms.

Bounds come from the arithmetic: a bf16 output is within 2^-8 of its value (eight
significant bits, round to nearest), fp32
sums within a few 2^-24 per term of the sum of magnitudes (taken as 2^-20 of the largest result
where nothing tighter is formed)."""
import math

import pytest
import torch

from paper_2507_01652_b200 import binding
from tests import _mixers_ref as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    torch.cuda.set_device(0)
    c = binding.Lasad(0)
    yield c
    c.close()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rnd(g, *shape, dtype=F32, std=1.0, mean=0.0):
    return (torch.randn(*shape, generator=g) * std + mean).to(dtype)


def d64(t):
    return None if t is None else t.detach().cpu().double()


def near(got, want, dtype, what, extra=0.0, acc=2.0 ** -20):
    """Within the rounding of the output's type of the float64 value, and acc of the largest one."""
    got = d64(got)
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), what
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine], want[~fine]), what
    if not fine.any():
        return
    big = want[fine].abs().max()
    bound = (2.0 ** -8 if dtype == BF16 else 2.0 ** -22) * want.abs() * 1.01 + acc * big + extra
    over = ((got - want).abs() - bound)[fine]
    assert over.max() <= 0, (what, float((got - want).abs()[fine].max()), float(big))


def strided(t, pad):
    """The same values in memory with gaps after every row of every dimension but the last."""
    if not pad:
        return t
    big = torch.full([n + pad for n in t.shape[:-1]] + [t.shape[-1] + 2 * 8], float("nan"), dtype=t.dtype, device=t.device)
    view = big[tuple(slice(0, n) for n in t.shape[:-1]) + (slice(8, 8 + t.shape[-1]),)]
    view.copy_(t)
    return view


# ---------------------------------------------------------------------------------------------
# gated linear recurrence
# ---------------------------------------------------------------------------------------------
SCAN = [  # B, T, C, grid_w, prefix, t0
    (1, 1, 1, 0, 0, 0), (2, 2, 3, 2, 0, 0), (1, 7, 32, 3, 1, 0), (3, 8, 33, 1, 0, 5), (2, 127, 64, 16, 1, 0),
    (1, 128, 30, 0, 0, 7), (2, 129, 100, 16, 0, 0), (1, 1000, 2, 24, 3, 0), (1, 2500, 34, 64, 1, 12345678901),
    (5, 300, 130, 17, 400, 0), (300, 140, 32, 16, 1, 3),
]


def scan_case(B, T, C, dtype, tied, logits, seed=0):
    g = gen(seed + B * 1000 + T + C)
    x = rnd(g, B, T, C, dtype=dtype)
    z = rnd(g, B, T, C, mean=1.5, std=2.0)
    gate = (z if logits else torch.sigmoid(z)).to(dtype)
    return x, gate, rnd(g, B, C), rnd(g, B, T, C, dtype=dtype), rnd(g, B, C)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tied,logits", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("shape", SCAN)
def test_scan_matches_the_recurrence_and_its_gradient(ctx, shape, tied, logits, dtype):
    B, T, C, w, P, t0 = shape
    x, gate, h_in, dy, dh = scan_case(B, T, C, dtype, tied, logits)
    kw = dict(grid_w=w, prefix_len=P, t0=t0, tied=tied, logits=logits)
    leaves = [d64(t).requires_grad_() for t in (x, gate, h_in)]
    y, h = ref.scan(*leaves, w, P, t0, tied, logits)
    wants = torch.autograd.grad([y, h], leaves, [d64(dy), d64(dh)], materialize_grads=True)
    dx_, gate_ = x.cuda(), gate.cuda()
    got_y, got_h, saved = ctx.lasad_scan_forward(dx_, gate_, h_in=h_in.cuda(), save=True, **kw)
    near(got_y, y.detach(), dtype, "y")
    near(got_h, h.detach(), F32, "h_out")
    gx, gg, gh = ctx.lasad_scan_backward(dx_, gate_, saved, dy.cuda(), dh_out=dh.cuda(), **kw)
    for n, a, b, t in (("dx", gx, wants[0], dtype), ("dgate", gg, wants[1], dtype), ("dh_in", gh, wants[2], F32)):
        near(a, b, t, n)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_takes_strides_and_any_alignment(ctx, dtype):
    B, T, C = 3, 200, 65
    x, gate, h_in, dy, dh = scan_case(B, T, C, dtype, True, True)
    y, h = ref.scan(d64(x), d64(gate), d64(h_in), 16, 1, 0, True, True)
    big = torch.full((B + 1, T + 3, 2 * C + 3), float("nan"), dtype=dtype, device="cuda")
    xs, gs = big[:B, :T, 1:C + 1], big[:B, 3:, C + 2:2 * C + 2]
    xs.copy_(x)
    gs.copy_(gate)
    out = torch.full((B, T, C + 7), 7.0, dtype=dtype, device="cuda")
    got, _, _ = ctx.lasad_scan_forward(xs, gs, grid_w=16, prefix_len=1, logits=True, h_in=h_in.cuda(), y=out[:, :, 3:C + 3])
    near(got, y, dtype, "y")
    assert bool((out[:, :, :3] == 7).all()) and bool((out[:, :, C + 3:] == 7).all())


@pytest.mark.parametrize("logits", [False, True])
def test_scan_extreme_gates(ctx, logits):
    """Gates of exactly 0 and 1, logits up to infinity, and a NaN that stays in its channel."""
    vals = [0.0, 1.0, 0.5] if not logits else [-math.inf, math.inf, -120.0, 120.0, 0.0]
    T, C = 300, 40
    g = gen(4)
    gate = torch.tensor(vals)[torch.randint(len(vals), (1, T, C), generator=g)]
    x = rnd(g, 1, T, C)
    y, h = ref.scan(d64(x), d64(gate), None, 16, 1, 0, True, logits)
    got, got_h, _ = ctx.lasad_scan_forward(x.cuda(), gate.cuda(), grid_w=16, prefix_len=1, logits=logits)
    near(got, y, F32, "y")
    x[0, 5, 7] = float("nan")
    bad, _, _ = ctx.lasad_scan_forward(x.cuda(), gate.cuda(), grid_w=16, prefix_len=1, logits=logits)
    others = torch.arange(C) != 7
    assert torch.equal(bad[:, :, others.cuda()], got[:, :, others.cuda()])
    assert bool(torch.isnan(bad[0, 5, 7])) and bool(torch.isfinite(bad[0, :5, 7]).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [1, 6, 33, 640])
def test_scan_step_continues_a_prefill(ctx, C, dtype):
    B, T, w, P = 4, 40, 7, 1
    x, gate, h_in, _, _ = scan_case(B, T, C, dtype, True, True, seed=9)
    y, h = ref.scan(d64(x), d64(gate), d64(h_in), w, P, 0, True, True)
    dx, dg = x.cuda(), gate.cuda()
    cut = 22
    got, state, _ = ctx.lasad_scan_forward(dx[:, :cut], dg[:, :cut], grid_w=w, prefix_len=P, logits=True, h_in=h_in.cuda())
    for t in range(cut, T):
        if t % 2:
            yt, _ = ctx.lasad_scan_step(dx[:, t], dg[:, t], state, grid_w=w, prefix_len=P, t=t, logits=True)
        else:
            pos = torch.full((B,), t, dtype=torch.int32, device="cuda")
            yt, _ = ctx.lasad_scan_step(dx[:, t], dg[:, t], state, grid_w=w, prefix_len=P, pos=pos, logits=True)
        near(yt, y[:, t], dtype, t)
    near(state, h, F32, "state")


def test_scan_gradient_against_differences(ctx):
    """The fp32 forward along a random direction: (f(a + e) - f(a - e)) / 2.  The step of 2^-6 costs
    about step^2 of the derivative (2^-12), and rounding 2^-24 T / step of the sum, both below 1e-2."""
    B, T, C, w = 2, 150, 20, 16
    x, gate, h_in, dy, dh = [t.cuda() for t in scan_case(B, T, C, F32, True, True, seed=3)]
    f = lambda a, b, c: sum((s.double() * t.double()).sum() for s, t in zip(   # noqa: E731
        ctx.lasad_scan_forward(a, b, h_in=c, grid_w=w, logits=True)[:2], (dy, dh)))
    _, _, saved = ctx.lasad_scan_forward(x, gate, h_in=h_in, grid_w=w, logits=True, save=True)
    grads = ctx.lasad_scan_backward(x, gate, saved, dy, dh_out=dh, grid_w=w, logits=True)
    g = gen(8)
    for n in range(3):
        args, v = [x, gate, h_in], rnd(g, *(x, gate, h_in)[n].shape).cuda() * 2.0 ** -6
        up, down = list(args), list(args)
        up[n], down[n] = args[n] + v, args[n] - v
        want = (f(*up) - f(*down)) / 2
        got = (grads[n].double() * v.double()).sum()
        scale = (grads[n].double() * v.double()).square().sum().sqrt()
        assert abs(got - want) <= 1e-2 * max(scale, abs(want)), (n, float(got), float(want))


# ---------------------------------------------------------------------------------------------
# norm and rotation
# ---------------------------------------------------------------------------------------------
ROPE = [  # B, T, Hq, Hk, d, grid_w, prefix, t0, pos
    (1, 1, 1, 1, 32, 0, 0, 0, False), (2, 5, 3, 1, 64, 4, 1, 0, False), (3, 17, 7, 5, 32, 5, 0, 9, False),
    (4, 1, 20, 20, 64, 16, 1, 0, True), (2, 130, 12, 4, 64, 24, 3, 0, True), (1, 600, 9, 3, 64, 0, 0, 50, False),
    (2, 33, 2, 16, 32, 1, 0, 0, False), (70, 40, 6, 6, 64, 8, 2, 0, True),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("shape", ROPE)
def test_rope_matches_the_formula_and_its_gradient(ctx, shape, pad, half, dtype):
    B, T, Hq, Hk, d, w, P, t0, has_pos = shape
    g = gen(T * 7 + Hq)
    q, k = rnd(g, B, T, Hq, d, dtype=dtype), rnd(g, B, T, Hk, d, dtype=dtype, std=3.0)
    wq, wk = rnd(g, d, mean=1.0, std=0.2), rnd(g, d, mean=1.0, std=0.2)
    dq, dk = rnd(g, B, T, Hq, d, dtype=dtype), rnd(g, B, T, Hk, d, dtype=dtype)
    pos = torch.randint(0, 200, (B,), generator=g, dtype=torch.int32) if has_pos else None
    rows = 1000
    table = binding.rope_table(rows, d, w > 0, device="cuda")
    leaves = [d64(t).requires_grad_() for t in (q, k, wq, wk)]
    start = pos.long() if has_pos else t0
    yq = ref.rope_one(leaves[0], leaves[2], start, w, P, half, 1e-5)
    yk = ref.rope_one(leaves[1], leaves[3], start, w, P, half, 1e-5)
    wants = torch.autograd.grad([yq, yk], leaves, [d64(dq), d64(dk)])
    dev = lambda t: strided(t.cuda(), pad)    # noqa: E731
    kw = dict(q_weight=wq.cuda(), k_weight=wk.cuda(), grid_w=w, prefix_len=P, t0=t0, eps=1e-5, half=half,
              pos=pos.cuda() if has_pos else None)
    got = ctx.lasad_qk_norm_rope(dev(q), dev(k), table, **kw)
    near(got[0], yq.detach(), dtype, "q")
    near(got[1], yk.detach(), dtype, "k")
    back = ctx.lasad_qk_norm_rope_backward(dev(q), dev(k), table, dev(dq), dev(dk), **kw)
    for n, a, b, t in zip(("dq", "dk", "dwq", "dwk"), back, wants, (dtype, dtype, F32, F32)):
        # a weight's gradient is a sum over B T H terms of magnitude |dy x|: 2^-24 of their sum each
        near(a, b, t, n, acc=2.0 ** -18 if n[1] == "w" else 2.0 ** -20)


def test_rope_without_weights_in_place_and_without_weight_gradients(ctx):
    g = gen(1)
    q, k = rnd(g, 2, 9, 4, 64, dtype=BF16), rnd(g, 2, 9, 2, 64, dtype=BF16)
    table = binding.rope_table(64, 64, True, device="cuda")
    a, b = q.cuda(), k.cuda()
    ctx.lasad_qk_norm_rope(a, b, table, grid_w=3, prefix_len=1, q_out=a, k_out=b)
    near(a, ref.rope_one(d64(q), None, 0, 3, 1, False, 1e-6), BF16, "q")
    near(b, ref.rope_one(d64(k), None, 0, 3, 1, False, 1e-6), BF16, "k")
    out = ctx.lasad_qk_norm_rope_backward(q.cuda(), k.cuda(), table, a, b, grid_w=3, prefix_len=1, want_weights=False)
    assert out[2] is None and out[3] is None and bool(torch.isfinite(out[0]).all())


def test_rope_zero_rows_and_positions_past_the_table(ctx):
    """eps keeps a zero head at zero, gradient included; a position past the table takes its last row."""
    q = torch.zeros(1, 3, 2, 64, device="cuda")
    table = binding.rope_table(8, 64, False, device="cuda")
    a, _ = ctx.lasad_qk_norm_rope(q, q, table)
    assert bool((a == 0).all())
    x = rnd(gen(2), 2, 1, 2, 64).cuda()
    far = torch.tensor([7, 1000], dtype=torch.int32, device="cuda")
    y, _ = ctx.lasad_qk_norm_rope(x[:1].expand(2, 1, 2, 64).contiguous(), x, table, pos=far)
    assert torch.equal(y[0], y[1])
    d, _, _, _ = ctx.lasad_qk_norm_rope_backward(q, q, table, torch.ones_like(q), torch.ones_like(q))
    assert bool(torch.isfinite(d).all())


# ---------------------------------------------------------------------------------------------
# window attention
# ---------------------------------------------------------------------------------------------
WINDOW = [  # B, T, Hq, Hk, d, window, sinks, lengths
    (1, 1, 1, 1, 64, 1, 0, None), (1, 2, 1, 1, 32, 1, 1, None), (2, 63, 2, 1, 64, 5, 0, None),
    (1, 64, 3, 3, 64, 64, 2, None), (2, 65, 4, 2, 64, 1, 0, None), (1, 127, 2, 2, 64, 1000, 0, None),
    (1, 128, 2, 2, 64, 128, 0, None), (2, 129, 6, 2, 64, 33, 3, None), (1, 257, 2, 1, 64, 37, 17, None),
    (1, 300, 8, 1, 64, 128, 128, None), (1, 520, 2, 2, 64, 130, 1, None), (1, 700, 1, 1, 64, 64, 65, None),
    (5, 140, 2, 1, 64, 20, 3, (0, 1, 77, 128, 140)), (4, 300, 4, 4, 64, 300, 0, (300, 2, 129, 256)),
    (3, 400, 3, 1, 64, 100, 4, (399, 101, 260)), (2, 200, 2, 2, 32, 70, 2, (200, 33)),
    (1, 1100, 1, 1, 64, 513, 1, None),
]


def window_case(B, T, Hq, Hk, d, dtype, lengths, seed=0):
    g = gen(seed + T * 3 + Hq)
    q, do = rnd(g, B, T, Hq, d, dtype=dtype, std=1.5), rnd(g, B, T, Hq, d, dtype=dtype)
    k, v = rnd(g, B, T, Hk, d, dtype=dtype), rnd(g, B, T, Hk, d, dtype=dtype)
    dev = [t.cuda() for t in (q, k, v, do)]
    if lengths is not None:       # what stands past the end must not count
        for t, bad in zip(dev, (float("nan"), math.inf, float("nan"), -math.inf)):
            for b, n in enumerate(lengths):
                t[b, n:] = bad
    return (q, k, v, do), dev


def check_window(ctx, shape, dtype, pad=0, scale=None, seed=0):
    B, T, Hq, Hk, d, win, sinks, lengths = shape
    host, dev = window_case(B, T, Hq, Hk, d, dtype, lengths, seed)
    q, k, v, do = [strided(t, pad) for t in dev]
    lens = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    leaves = [d64(t).requires_grad_() for t in host[:3]]
    o, lse = ref.window(*leaves, win, sinks, scale, lengths)
    wants = torch.autograd.grad(o, leaves, d64(host[3]))
    half = dtype == BF16
    bounds = ref.window_bounds(*[d64(t) for t in host], win, sinks, scale, lengths,
                               u=2.0 ** -8 if half else 2.0 ** -23, acc=2.0 ** -20)
    kw = dict(window=win, sinks=sinks, scale=scale, lengths=lens)
    got_o, got_lse = ctx.lasad_window_attention(q, k, v, want_lse=True, **kw)

    def inside(name, got, want, bound):
        got = d64(got)
        assert torch.isfinite(got).all(), name
        over = (got - want).abs() - 1.02 * bound - 1e-30
        assert over.max() <= 0, (name, float((got - want).abs().max()), float(over.max()), float(want.abs().max()))

    inside("o", got_o, o.detach(), bounds["o"])
    near(got_lse, lse, F32, "lse", extra=2.0 ** -18)
    only_o, none = ctx.lasad_window_attention(q, k, v, **kw)
    assert none is None and torch.equal(only_o, got_o)
    back = ctx.lasad_window_attention_backward(q, k, v, got_o, got_lse, do, **kw)
    for name, g, want in zip(("dq", "dk", "dv"), back, wants):
        inside(name, g, want, bounds[name])
    assert ctx.device_status() == 0
    return (got_o, got_lse) + back


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", WINDOW)
def test_window_matches_the_formula_and_its_gradient(ctx, shape, dtype):
    check_window(ctx, shape, dtype)


@pytest.mark.parametrize("shape", [WINDOW[i] for i in (2, 7, 9, 12, 14)])
def test_window_on_cuda_cores_for_bf16(ctx, shape):
    ctx.set_option(binding.LASAD_OPT_WINDOW_IMPL, 1)
    try:
        check_window(ctx, shape, BF16)
    finally:
        ctx.set_option(binding.LASAD_OPT_WINDOW_IMPL, 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [WINDOW[7], WINDOW[14]])
def test_window_takes_strides(ctx, shape, dtype):
    check_window(ctx, shape, dtype, pad=1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0])
def test_window_other_scales(ctx, scale, dtype):
    check_window(ctx, (1, 150, 2, 1, 64, 40, 2, None), dtype, scale=scale)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_window_sharp_and_large_scores(ctx, dtype):
    """Scores of hundreds: one key takes all of the weight, and the running maximum has to move."""
    T, d = 400, 64
    g = gen(6)
    k = rnd(g, 1, T, 1, d, dtype=dtype)
    q = (k.float() * torch.linspace(0.5, 12, T)[None, :, None, None]).to(dtype).roll(-1, dims=1)
    v = rnd(g, 1, T, 1, d, dtype=dtype)
    o, lse = ref.window(d64(q), d64(k), d64(v), 300, 1)
    got, got_lse = ctx.lasad_window_attention(q.cuda(), k.cuda(), v.cuda(), 300, 1, want_lse=True)
    b = ref.window_bounds(d64(q), d64(k), d64(v), torch.zeros_like(o), 300, 1, u=2.0 ** -8 if dtype == BF16 else 2.0 ** -23)
    assert ((d64(got) - o).abs() <= 1.02 * b["o"]).all()
    near(got_lse, lse, F32, "lse", extra=2.0 ** -18)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_window_gradient_against_differences(ctx, dtype):
    """Along random directions of the float64 form: the form's difference quotient (step 1e-4, error
    1e-8) and the call's gradient; the call's own bound decides."""
    shape = (2, 130, 4, 2, 64, 50, 2, (130, 91))
    B, T, Hq, Hk, d, win, sinks, lengths = shape
    host, dev = window_case(B, T, Hq, Hk, d, dtype, lengths, 5)
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    o, lse = ctx.lasad_window_attention(*dev[:3], win, sinks, lengths=lens, want_lse=True)
    grads = ctx.lasad_window_attention_backward(*dev[:3], o, lse, dev[3], win, sinks, lengths=lens)
    h64 = [d64(t) for t in host]
    bounds = ref.window_bounds(*h64, win, sinks, None, lengths, u=2.0 ** -8 if dtype == BF16 else 2.0 ** -23)
    g = gen(77)
    for n, name in enumerate(("dq", "dk", "dv")):
        e = rnd(g, *h64[n].shape).double()
        up, down = list(h64[:3]), list(h64[:3])
        up[n], down[n] = h64[n] + 1e-4 * e, h64[n] - 1e-4 * e
        f = lambda a: (ref.window(*a, win, sinks, None, lengths)[0] * h64[3]).sum()    # noqa: E731
        want = (f(up) - f(down)) / 2e-4
        got = (d64(grads[n]) * e).sum()
        assert abs(got - want) <= (1.02 * bounds[name] * e.abs()).sum() + 1e-6 * abs(want), name


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_window_long_ragged_against_the_other_implementation_and_repeats(ctx, dtype):
    """A case large enough for every CTA shape: the same bits twice, and the batch's rows do not depend
    on what else is in the batch."""
    B, T, Hq, Hk, d, win, sinks = 3, 900, 6, 2, 64, 200, 5
    lengths = (900, 513, 128)
    _, dev = window_case(B, T, Hq, Hk, d, dtype, lengths, 2)
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")

    def run(b0, b1):
        q, k, v, do = [t[b0:b1].contiguous() for t in dev]
        o, lse = ctx.lasad_window_attention(q, k, v, win, sinks, lengths=lens[b0:b1].contiguous(), want_lse=True)
        return (o, lse) + ctx.lasad_window_attention_backward(q, k, v, o, lse, do, win, sinks,
                                                              lengths=lens[b0:b1].contiguous())
    first, again, one = run(0, 3), run(0, 3), run(1, 2)
    for a, b, c in zip(first, again, one):
        assert torch.equal(a, b) and torch.equal(a[1:2], c)


@pytest.mark.parametrize("T,win", [(2, 8), (40, 2), (300, 2)])
def test_window_gradient_where_rows_see_two_keys(ctx, T, win):
    """dP - Delta is small there against Delta itself, which the rounding of o must not reach: dq and dk within
    2^-8 in the 2-norm (2^-9 and less each from the output, P and dS; Delta from the bf16 o alone: 0.4 to 0.7 %)."""
    (q, k, v, do), dev = window_case(64, T, 4, 4, 64, BF16, None, 11)
    leaves = [d64(t).requires_grad_() for t in (q, k, v)]
    want = torch.autograd.grad(ref.window(*leaves, win)[0], leaves, d64(do))
    o, lse = ctx.lasad_window_attention(*dev[:3], win, want_lse=True)
    for a, b in zip(ctx.lasad_window_attention_backward(*dev[:3], o, lse, dev[3], win), want):
        assert (d64(a) - b).norm() <= 2.0 ** -8 * b.norm()


def test_window_back_to_back_in_a_warm_cache(ctx):
    """A long case over and over: tiles land at once, so that every wait meets the barrier's phase that
    is the hardest to tell from the next; no wait may give up, and every launch returns the same bits."""
    _, (q, k, v, do) = window_case(1, 2305, 8, 4, 64, BF16, None, 6)
    first = None
    for _ in range(30):
        o, lse = ctx.lasad_window_attention(q, k, v, 700, 3, want_lse=True)
        got = (o, lse) + ctx.lasad_window_attention_backward(q, k, v, o, lse, do, 700, 3)
        first = first or got
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_window_waits_are_bounded(ctx):
    """Waits that run out after one try: the kernels report it and leave, and the next calls are whole."""
    _, (q, k, v, do) = window_case(1, 700, 4, 4, 64, BF16, None, 7)
    o, lse = ctx.lasad_window_attention(q, k, v, 300, 1, want_lse=True)
    want = ctx.lasad_window_attention_backward(q, k, v, o, lse, do, 300, 1)
    try:
        ctx.set_option(binding.LASAD_OPT_WAIT_LIMIT, 1)
        ctx.lasad_window_attention(q, k, v, 300, 1)
        torch.cuda.synchronize()
        assert ctx.device_status() == binding.LASAD_ERR_TIMEOUT
        ctx.lasad_window_attention_backward(q, k, v, o, lse, do, 300, 1)
        torch.cuda.synchronize()
        assert ctx.device_status() == binding.LASAD_ERR_TIMEOUT
    finally:
        ctx.set_option(binding.LASAD_OPT_WAIT_LIMIT, 0)
    assert torch.equal(ctx.lasad_window_attention(q, k, v, 300, 1)[0], o)
    assert all(torch.equal(a, b) for a, b in zip(ctx.lasad_window_attention_backward(q, k, v, o, lse, do, 300, 1), want))
    assert ctx.device_status() == 0


STEP = [  # B, Hq, Hk, d, window, sinks
    (1, 1, 1, 64, 1, 0), (3, 2, 1, 64, 5, 0), (4, 3, 3, 32, 16, 2), (2, 8, 1, 64, 200, 1), (5, 12, 4, 64, 64, 1),
    (2, 10, 1, 64, 33, 3), (1, 24, 8, 64, 1500, 1), (40, 4, 4, 64, 70, 4),
    # so many heads that each has one warp; few, with clusters of CTAs along the slots
    (130, 20, 20, 64, 6, 1), (400, 18, 6, 32, 9, 0), (700, 40, 4, 64, 3, 1), (2, 4, 2, 32, 3000, 2), (3, 16, 2, 64, 700, 0),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", STEP)
def test_window_step_matches_the_formula(ctx, shape, dtype):
    B, Hq, Hk, d, win, sinks = shape
    g = gen(B + win)
    q, k, v = rnd(g, B, Hq, d, dtype=dtype, std=2.0), rnd(g, B, Hk, d, dtype=dtype), rnd(g, B, Hk, d, dtype=dtype)
    kc, vc = (rnd(g, B, sinks + win, Hk, d, dtype=dtype) for _ in range(2))
    for pos in ([max(-1, sinks - 1)] * B, [b * 3 - 1 for b in range(B)], [win + sinks + 5 * b for b in range(B)],
                [2 ** 31 - 1 - b for b in range(B)]):
        # slots that no token has reached hold anything
        dk, dv = kc.cuda(), vc.cuda()
        for b, p in enumerate(pos):
            dk[b, max(p + 1, 0):] = float("nan")
            dv[b, max(p + 1, 0):] = math.inf
        before = dk.clone()
        if max(pos) < 10 ** 6:
            o, wk, wv = ref.window_step(d64(q), d64(k), d64(v), d64(kc), d64(vc), pos, win, sinks)
        else:                # all slots in use: the same as at a position of the same slot
            low = [win + sinks + (p - sinks) % win for p in pos]
            o, wk, wv = ref.window_step(d64(q), d64(k), d64(v), d64(kc), d64(vc), low, win, sinks)
            low = [sinks + win * (1 + b) + (p - sinks) % win for b, p in enumerate(pos)]
            o, wk, wv = ref.window_step(d64(q), d64(k), d64(v), d64(kc), d64(vc), low, win, sinks)
        p32 = torch.tensor(pos, dtype=torch.int32, device="cuda")
        got = ctx.lasad_window_attention_step(q.cuda(), k.cuda(), v.cuda(), dk, dv, p32, win, sinks)
        # fp32 throughout: the output's rounding, and the exponent's 2^-20 |q||k| scale on weights of a mean of v
        near(got, o, dtype, pos, acc=2.0 ** -16)
        for b, p in enumerate(pos):
            used = min(max(p + 1, 0), sinks + win)
            assert torch.equal(d64(dk[b, :used]), wk[b, :used]) and torch.equal(d64(dv[b, :used]), wv[b, :used])
            assert torch.equal(dk[b, used:].isnan(), before[b, used:].isnan())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_window_generation_continues_a_prefill(ctx, dtype):
    """Prefill, store, then tokens one at a time: the same as the whole sequence at once."""
    B, T, Hq, Hk, d, win, sinks = 3, 90, 4, 2, 64, 24, 2
    host, (q, k, v, _) = window_case(B, T, Hq, Hk, d, dtype, None, 8)
    o, _ = ref.window(*[d64(t) for t in host[:3]], win, sinks)
    b_o = ref.window_bounds(*[d64(t) for t in host], win, sinks, u=2.0 ** -8 if dtype == BF16 else 2.0 ** -23)["o"]
    lengths = [1, 25, 70]
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    kc = torch.full((B, sinks + win, Hk, d), float("nan"), dtype=dtype, device="cuda")
    vc = kc.clone()
    ctx.lasad_window_cache_store(k[:, :70], v[:, :70], kc, vc, win, sinks, lengths=lens)
    for n in range(20):
        pos = [L + n for L in lengths]
        at = torch.tensor(pos, device="cuda")
        rows = torch.arange(B, device="cuda")
        got = ctx.lasad_window_attention_step(q[rows, at], k[rows, at], v[rows, at], kc, vc, at.int(), win, sinks)
        want, bound = o[range(B), pos], b_o[range(B), pos]
        assert ((d64(got) - want).abs() <= 1.02 * bound).all(), n


# ---------------------------------------------------------------------------------------------
# streams, graphs, counters, refusals
# ---------------------------------------------------------------------------------------------
def test_calls_on_another_stream_and_in_a_graph(ctx):
    g = gen(1)
    x, gate = rnd(g, 1, 2000, 64, dtype=BF16).cuda(), rnd(g, 1, 2000, 64, dtype=BF16).cuda()
    q, k, v = [rnd(g, 1, 200, 4, 64, dtype=BF16).cuda() for _ in range(3)]
    table = binding.rope_table(64, 64, True, device="cuda")

    def step():
        y, h, saved = ctx.lasad_scan_forward(x, gate, grid_w=16, logits=True, save=True)
        gx = ctx.lasad_scan_backward(x, gate, saved, y, dh_out=h, grid_w=16, logits=True)
        a, b = ctx.lasad_qk_norm_rope(q, k, table, grid_w=16)
        o, lse = ctx.lasad_window_attention(a, b, v, 50, 1, want_lse=True)
        ga = ctx.lasad_window_attention_backward(a, b, v, o, lse, o, 50, 1)
        gq = ctx.lasad_qk_norm_rope_backward(q, k, table, ga[0], ga[1], grid_w=16)
        return (y, h, a, b, o, lse) + gx + ga + gq

    want = step()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        there = step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(want, there, held):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_raw_stream_handle_keeps_its_workspace(ctx):
    """A call on a raw stream while the current one allocates and fills memory of the same size."""
    x, gate = rnd(gen(1), 1, 4000, 64).cuda(), rnd(gen(2), 1, 4000, 64).cuda()
    want = ctx.lasad_scan_forward(x, gate, logits=True)[0]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    outs = []
    for _ in range(20):
        outs.append(ctx.lasad_scan_forward(x, gate, logits=True, stream=s.cuda_stream)[0])
        torch.empty(1 << 16, device="cuda").fill_(float("nan"))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_hybrid_block_example():
    """The operators together: a training step lowers the loss, and a prefix continued token by token
    gives the rows of one pass (bf16 projections of bf16 sums on both sides: a few roundings)."""
    from examples import hybrid_block
    losses = hybrid_block.train(steps=10)
    assert losses[-1] < 0.9 * losses[0]
    assert hybrid_block.generate(T=120) < 2e-2


def test_launches_are_counted(ctx):
    n = ctx.launch_count
    x = torch.zeros(1, 1, 32, device="cuda")
    ctx.lasad_scan_forward(x, x)
    assert ctx.launch_count == n + 1


def code(fn, *a, **kw):
    with pytest.raises(binding.LasadError) as e:
        fn(*a, **kw)
    return e.value.code


def test_refusals(ctx):
    INV, UNS = binding.LASAD_ERR_INVALID_ARG, binding.LASAD_ERR_UNSUPPORTED
    x = torch.zeros(2, 4, 32, device="cuda")
    assert code(ctx.lasad_scan_forward, x, x, grid_w=-1) == INV
    assert code(ctx.lasad_scan_forward, x, x, prefix_len=-1) == INV
    assert code(ctx.lasad_scan_forward, x, x, t0=-1) == INV
    assert code(ctx.lasad_scan_forward, x[:, :1].expand(2, 4, 32), x) == INV
    assert code(ctx.lasad_scan_forward, x[:, :0], x[:, :0]) == INV
    q = torch.zeros(1, 3, 4, 64, device="cuda")
    table = binding.rope_table(8, 64, False, device="cuda")
    assert code(ctx.lasad_qk_norm_rope, q, q, table, t0=6) == INV        # past the table
    assert code(ctx.lasad_qk_norm_rope, q, q, table, eps=-1.0) == INV
    assert code(ctx.lasad_qk_norm_rope, q, q, table, eps=float("nan")) == INV
    t48 = torch.zeros(8, 24, 2, device="cuda")
    q48 = torch.zeros(1, 3, 4, 48, device="cuda")
    assert code(ctx.lasad_qk_norm_rope, q48, q48, t48) == UNS
    assert code(ctx.lasad_window_attention, q48, q48, q48, 4) == UNS
    assert code(ctx.lasad_window_attention, q, q, q, 0) == INV
    assert code(ctx.lasad_window_attention, q, q, q, 4, -1) == INV
    assert code(ctx.lasad_window_attention, q, q, q, 4, 129) == UNS
    assert code(ctx.lasad_window_attention, q, q, q, 4, scale=float("inf")) == INV
    k3 = torch.zeros(1, 3, 3, 64, device="cuda")
    assert code(ctx.lasad_window_attention, q, k3, k3, 4) == INV         # 3 does not divide 4
    flat = torch.zeros(3 * 4 * 64 + 8, device="cuda")
    off = flat[1:1 + 3 * 4 * 64].view(1, 3, 4, 64)
    assert code(ctx.lasad_window_attention, off, q, q, 4) == INV         # not on 16 bytes
    pos = torch.zeros(1, dtype=torch.int32, device="cuda")
    q1 = torch.zeros(1, 4, 64, device="cuda")
    with pytest.raises(ValueError):
        ctx.lasad_window_attention_step(q1, q1, q1, torch.zeros(1, 9, 4, 64, device="cuda"),
                                        torch.zeros(1, 9, 4, 64, device="cuda"), pos, 10)
    with pytest.raises(ValueError):
        ctx.lasad_window_attention(q, q, q.bfloat16(), 4)
    with pytest.raises(ValueError):
        ctx.lasad_window_attention(q, q, q, 4, lengths=torch.zeros(1, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        ctx.lasad_scan_forward(x, x.bfloat16())
    with pytest.raises(ValueError):
        ctx.lasad_scan_forward(x.cpu(), x)
    with pytest.raises(ValueError):
        ctx.lasad_scan_backward(x, x, torch.zeros(2, 2, 32, device="cuda"), x)
    with pytest.raises(TypeError):
        ctx.lasad_scan_forward(x.half(), x.half())


def test_null_arguments_are_refused(ctx):
    import ctypes

    from paper_2507_01652_b200 import mixers
    lib = binding.load_library()
    for cls, calls in ((mixers.ScanParams, ("lasad_scan_forward", "lasad_scan_backward", "lasad_scan_step")),
                       (mixers.RopeParams, ("lasad_qk_norm_rope", "lasad_qk_norm_rope_backward")),
                       (mixers.WindowParams, ("lasad_window_attention", "lasad_window_attention_backward",
                                              "lasad_window_attention_step", "lasad_window_cache_store"))):
        p = cls()
        for name in calls:
            n = len(mixers.PROTOTYPES[name][1]) - 2
            assert getattr(lib, name)(None, ctypes.byref(p), *[None] * n) == binding.LASAD_ERR_INVALID_ARG
            assert getattr(lib, name)(ctx._h, None, *[None] * n) == binding.LASAD_ERR_INVALID_ARG
            assert getattr(lib, name)(ctx._h, ctypes.byref(p), *[None] * n) == binding.LASAD_ERR_INVALID_ARG
