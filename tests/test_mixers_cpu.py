"""What can be said of the operators beside LASAD without a GPU: the structs' layout, the rotation
table, and that the float64 forms the GPU tests compare with are the formulas' own gradients."""
import ctypes
import math

import pytest
import torch

from paper_2507_01652_b200 import binding, mixers
from tests import _mixers_ref as ref


def test_struct_layouts():
    assert ctypes.sizeof(mixers.ScanParams) == 32 + 8 + 5 * 16
    assert mixers.ScanParams.t0.offset == 32
    assert ctypes.sizeof(mixers.RopeParams) == 48 + 8 + 8 * 24
    assert mixers.RopeParams.t0.offset == 48
    assert ctypes.sizeof(mixers.WindowParams) == 40 + 10 * 24
    assert mixers.WindowParams.q_stride.offset == 40


def test_rope_table_is_exact_at_long_positions():
    t = binding.rope_table(100001, 64, False)
    assert t.shape == (100001, 32, 2)
    for m in (0, 5, 31):
        a = 100000 * 10000.0 ** (-m / 32)
        assert abs(float(t[100000, m, 0]) - math.cos(a)) < 1e-7 and abs(float(t[100000, m, 1]) - math.sin(a)) < 1e-7
    assert binding.rope_table(5, 64, True).shape == (5, 16, 2)


def test_no_cpu_path():
    if torch.cuda.is_available():
        pytest.skip("checks the behaviour without a device")
    with pytest.raises(RuntimeError):
        binding.Lasad()


@pytest.mark.parametrize("tied,logits", [(True, True), (True, False), (False, False)])
def test_scan_gradient_formula(tied, logits):
    """dx, dlambda, dh_in as the kernel forms them, against autograd of the recurrence."""
    torch.manual_seed(0)
    B, T, C, w, P = 2, 23, 3, 5, 1
    x, z = torch.randn(B, T, C).double().requires_grad_(), torch.randn(B, T, C).double()
    gate = (z if logits else torch.sigmoid(z)).requires_grad_()
    h0 = torch.randn(B, C).double().requires_grad_()
    dy, dh = torch.randn(B, T, C).double(), torch.randn(B, C).double()
    y, h = ref.scan(x, gate, h0, w, P, 0, tied, logits)
    want = torch.autograd.grad([y, h], [x, gate, h0], [dy, dh])
    lam = torch.sigmoid(gate) if logits else gate
    gain = 1 - lam if tied else torch.ones_like(lam)
    u, dx, dg = dh, [None] * T, [None] * T
    for t in range(T - 1, -1, -1):
        g = dy[:, t] + u
        row_end = ref.ends_row(t, w, P)
        prev = h0 if t == 0 else y[:, t - 1]
        d = (0 if row_end else prev) - (x[:, t] if tied else 0)
        dx[t], dg[t] = gain[:, t] * g, d * g * (lam * (1 - lam))[:, t] if logits else d * g
        u = g if row_end else lam[:, t] * g
    for a, b in zip((torch.stack(dx, 1), torch.stack(dg, 1), u), want):
        assert torch.allclose(a, b, rtol=1e-12, atol=1e-12)


def test_window_reference_rows_and_gradient_against_differences():
    torch.manual_seed(1)
    q, k, v = [torch.randn(1, 30, h, 8).double() for h in (2, 1, 1)]
    o, lse = ref.window(q, k, v, 7, 2, lengths=[21])
    t = 15          # sees 0, 1 and 9..15
    s = [0, 1] + list(range(9, 16))
    p = torch.softmax(k[0, s, 0] @ q[0, t, 1] / math.sqrt(8), 0)
    assert torch.allclose(o[0, t, 1], p @ v[0, s, 0])
    assert bool((o[0, 21:] == 0).all()) and bool((lse[0, :, 21:] == -math.inf).all())
    g = torch.randn_like(o)
    leaves = [a.clone().requires_grad_() for a in (q, k, v)]
    grads = torch.autograd.grad(ref.window(*leaves, 7, 2, lengths=[21])[0], leaves, g)
    for n in range(3):
        e = torch.randn_like(leaves[n])
        f = lambda x: (ref.window(*[x if m == n else a for m, a in enumerate((q, k, v))], 7, 2, lengths=[21])[0] * g).sum()  # noqa: E731
        base = (q, k, v)[n]
        diff = (f(base + 1e-5 * e) - f(base - 1e-5 * e)) / 2e-5
        assert abs(diff - (grads[n] * e).sum()) < 1e-6 * (1 + abs(diff))


def test_ring_slots_hold_what_a_token_sees():
    for win, sinks in ((1, 0), (4, 2), (7, 0), (3, 5)):
        for p in range(40):
            tokens = [s for s in range(p + 1) if p - s < win or s < sinks]
            slots = sorted(s if s < sinks else sinks + (s - sinks) % win for s in tokens)
            # the slots in use are the first ones, whatever the order
            assert slots == list(range(min(p + 1, sinks + win)))
