"""Edges of the operators beside LASAD: gates that are nearly shut, grids and positions near the ends of their types,
calls that have to be refused."""
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


def draw(seed, *shape, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("C", [64, 33])
@pytest.mark.parametrize("tied", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gate_gradient_at_row_ends_of_nearly_shut_gates(ctx, dtype, tied, C):
    """Logits from -15 to -60 (lambda from 3e-7 to 1e-26).  On a row's last token the tied gate's gradient is
    -g x lambda (1 - lambda), as small as lambda, and 0 untied.  Each value on its own: lambda carries (|z| + 4) 2^-23
    (2^-17), the products and g, which is dy and a share of lambda from the right, a few 2^-24; a bf16 gradient
    its rounding of 2^-8."""
    B, T, w = 2, 200, 5
    x, dy = draw(1, B, T, C, dtype=dtype), draw(2, B, T, C, dtype=dtype)
    z = -15 - 45 * torch.rand(B, T, C, generator=torch.Generator().manual_seed(3))
    z = z.to(dtype)
    leaves = [t.double().requires_grad_() for t in (x, z)]
    y, _ = ref.scan(*leaves, None, w, 0, 0, tied, True)
    # (autograd forms the derivative of sigmoid(-z) as s (1 - s), which is 0 in 64 bits too from z = -37 on: the
    # formula instead, with g = dx / (1 - lambda) where tied)
    dx, dz = torch.autograd.grad(y, leaves, dy.double())
    z64 = z.double()
    want = -dx * x.double() * torch.sigmoid(z64) if tied else dz
    _, _, saved = ctx.lasad_scan_forward(x.cuda(), z.cuda(), grid_w=w, tied=tied, logits=True, save=True)
    _, got, _ = ctx.lasad_scan_backward(x.cuda(), z.cuda(), saved, dy.cuda(), grid_w=w, tied=tied, logits=True)
    ends = [t for t in range(T) if ref.ends_row(t, w, 0)]
    got, want = got.cpu().double()[:, ends], want[:, ends]
    if not tied:
        assert bool((got == 0).all()) and bool((want == 0).all())
        return
    assert bool(((got - want).abs() <= (2.0 ** -16 + (2.0 ** -8 if dtype == BF16 else 0)) * want.abs()).all())


@pytest.mark.parametrize("C", [64, 33])
@pytest.mark.parametrize("w", [2 ** 30 + 50, 2 ** 31 - 60, 2 ** 31 - 1])
def test_recurrence_on_rows_near_2_to_31_tokens(ctx, w, C):
    """A walk over the end of a grid row whose width, and the tokens' columns on it, fill an int32: the row's last
    token lets h through whole, the ones 128 and 256 further on do not."""
    T, P = 400, 3
    t0 = P + w - 1 - 130                       # the row ends at token 130 of the call
    x, gate, dy = draw(1, 1, T, C), torch.sigmoid(draw(2, 1, T, C)), draw(3, 1, T, C)
    leaves = [t.double().requires_grad_() for t in (x, gate)]
    y, _ = ref.scan(*leaves, None, w, P, t0, True, False)
    assert [t for t in range(T) if ref.ends_row(t0 + t, w, P)] == [130]
    want = torch.autograd.grad(y, leaves, dy.double())
    kw = dict(grid_w=w, prefix_len=P, t0=t0)
    got, _, saved = ctx.lasad_scan_forward(x.cuda(), gate.cuda(), save=True, **kw)
    back = ctx.lasad_scan_backward(x.cuda(), gate.cuda(), saved, dy.cuda(), **kw)
    for a, b in zip((got,) + back[:2], (y.detach(),) + want):
        # fp32: 2^-22 of each value and 2^-20 of the largest (sums of some tens of terms)
        assert bool(((a.cpu().double() - b).abs() <= 2.0 ** -22 * b.abs() + 2.0 ** -20 * b.abs().max()).all())
    state = torch.zeros(1, C, device="cuda")
    for t in range(128, 133):
        pos = None if t0 + t > 2 ** 31 - 1 else torch.tensor([t0 + t], dtype=torch.int32, device="cuda")
        before = state.clone()
        step, _ = ctx.lasad_scan_step(x[:, t].cuda(), gate[:, t].cuda(), state, t=t0 + t, grid_w=w, prefix_len=P, pos=pos)
        lam = torch.ones_like(gate[:, t]) if t == 130 else gate[:, t]
        want_h = lam.double() * before.cpu().double() + (1 - gate[:, t].double()) * x[:, t].double()
        assert bool(((step.cpu().double() - want_h).abs() <= 2.0 ** -21).all())


def refused(fn, *a, **kw):
    with pytest.raises(binding.LasadError) as e:
        fn(*a, **kw)
    return e.value.code == binding.LASAD_ERR_INVALID_ARG


def test_positions_that_are_no_numbers_are_refused(ctx):
    """t0 past 2^62: a sum that wraps round at 2^63 would look like a position before the table's end."""
    x, q = torch.zeros(1, 4, 32, device="cuda"), torch.zeros(1, 4, 2, 64, device="cuda")
    table, grid = (binding.rope_table(16, 64, g, device="cuda") for g in (False, True))
    for t0 in (2 ** 63 - 1, 2 ** 63 - 4, 2 ** 62 + 1):
        assert refused(ctx.lasad_scan_forward, x, x, t0=t0)
        assert refused(ctx.lasad_scan_backward, x, x, torch.zeros(1, 1, 32, device="cuda"), x, t0=t0)
        assert refused(ctx.lasad_qk_norm_rope, q, q, table, t0=t0)
        assert refused(ctx.lasad_qk_norm_rope, q, q, grid, grid_w=8, t0=t0)
        assert refused(ctx.lasad_qk_norm_rope_backward, q, q, table, q, q, t0=t0)
    assert refused(ctx.lasad_scan_step, x[:, 0], x[:, 0], torch.zeros(1, 32, device="cuda"), t=2 ** 63 - 1)
    y, _, _ = ctx.lasad_scan_forward(x, x, t0=2 ** 62, grid_w=7)        # the largest ones are positions
    assert bool((y == 0).all())


@pytest.mark.parametrize("t0,T,fits", [
    (1 + 96 * 5 + 2, 3, True),          # row 5, columns 2 to 4
    (1 + 96 * 5 + 2, 6, True),          # ... to column 7, the table's last row
    (1 + 96 * 5 + 2, 7, False),         # ... to column 8
    (1 + 96 * 7, 1, True), (1 + 96 * 8, 1, False),
    (1 + 96 * 4 + 94, 4, False),        # over the end of a row: column 95
    (0, 9, True), (0, 10, False), (0, 1, True),
])
def test_rotation_takes_every_position_that_its_table_has(ctx, t0, T, fits):
    """A table of 8 rows for a grid of 96 columns and one token before it: a call is refused where a token's row or
    column is not in the table, and only there."""
    q = draw(1, 1, T, 2, 64).cuda()
    table = binding.rope_table(8, 64, True, device="cuda")
    kw = dict(grid_w=96, prefix_len=1, t0=t0)
    if not fits:
        assert refused(ctx.lasad_qk_norm_rope, q, q, table, **kw)
        assert refused(ctx.lasad_qk_norm_rope_backward, q, q, table, q, q, **kw)
        return
    y, _ = ctx.lasad_qk_norm_rope(q, q, table, **kw)
    ctx.lasad_qk_norm_rope_backward(q, q, table, q, q, **kw)
    want = ref.rope_one(q.cpu().double(), None, t0, 96, 1, False, 1e-6)
    # fp32: 2^-22 of each value and 2^-20 of the largest
    assert bool(((y.cpu().double() - want).abs() <= 2.0 ** -22 * want.abs() + 2.0 ** -20 * want.abs().max()).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_windows_longer_than_any_sequence(ctx, dtype):
    """They hide nothing, whatever their size: the same bits as a window of the sequence's length."""
    q, k, v, do = (draw(n, 2, 150, h, 64, dtype=dtype).cuda() for n, h in ((1, 4), (2, 2), (3, 2), (4, 4)))

    def run(window):
        o, lse = ctx.lasad_window_attention(q, k, v, window, 1, want_lse=True)
        return (o, lse) + ctx.lasad_window_attention_backward(q, k, v, o, lse, do, window, 1)
    want = run(150)
    for window in (151, 2 ** 30 + 1, 2 ** 31 - 1, 2 ** 32 + 3, 2 ** 63 - 1):
        assert all(torch.equal(a, b) for a, b in zip(run(window), want)), window
