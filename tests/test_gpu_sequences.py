"""The operators of a layer that attends to whole sequences on the GPU against their float64 forms.

Bounds come from the arithmetic, as in test_gpu_mixers: what a rounding to the type of the weights or of the output
costs (bf16 2^-8, both sides of it), and 2^-20 of the sum of magnitudes for fp32 sums and exponentials.  What
is rounded to 8 bits is compared for equality."""
import ctypes
import math

import pytest
import torch

from paper_2507_01652_b200 import binding, sequences
from tests import _sequences_ref as ref
from tests.test_gpu_mixers import BF16, F32, ctx, d64, gen, near, rnd, strided  # noqa: F401

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def inside(name, got, want, bound):
    got = d64(got)
    assert torch.isfinite(got).all(), name
    over = (got - want).abs() - 1.02 * bound - 1e-30
    assert over.max() <= 0, (name, float((got - want).abs().max()), float(over.max()), float(want.abs().max()))


# ---------------------------------------------------------------------------------------------
# packed sequences
# ---------------------------------------------------------------------------------------------
PACKED = [  # lengths, rows behind the last, Hq, Hk, d
    ((1,), 0, 1, 1, 64), ((2, 1), 0, 2, 1, 32), ((63,), 1, 3, 3, 64), ((64, 65), 0, 4, 2, 64), ((0, 5, 0, 0, 7, 0), 3, 2, 1, 64),
    ((127, 128, 129), 0, 2, 2, 64), ((0,), 70, 2, 1, 64), ((255, 1, 257), 130, 4, 1, 64), ((33,) * 9, 0, 6, 2, 32),
    ((500, 13, 260), 5, 8, 8, 64), ((1, 2, 3, 4, 5, 6, 7, 8, 9), 200, 1, 1, 64), ((700,), 0, 6, 2, 64), ((384, 385, 383), 0, 3, 1, 32),
    ((128, 256), 0, 2, 2, 64), ((1100,), 300, 2, 1, 64),
]


def packed_case(lengths, tail, Hq, Hk, d, dtype, seed=0):
    g = gen(seed + sum(lengths) * 3 + Hq)
    offsets = [0]
    for n in lengths:
        offsets.append(offsets[-1] + n)
    N = offsets[-1] + tail
    q, do = rnd(g, N, Hq, d, dtype=dtype, std=1.5), rnd(g, N, Hq, d, dtype=dtype)
    k, v = rnd(g, N, Hk, d, dtype=dtype), rnd(g, N, Hk, d, dtype=dtype)
    dev = [t.cuda() for t in (q, k, v, do)]
    for t, bad in zip(dev, (float("nan"), math.inf, float("nan"), -math.inf)):       # what nobody owns must not count
        t[offsets[-1]:] = bad
    return (q, k, v, do), dev, offsets, torch.tensor(offsets, dtype=torch.int32, device="cuda")


def check_packed(ctx, shape, dtype, pad=0, scale=None, seed=0):
    host, dev, offsets, at = packed_case(*shape, dtype, seed)
    q, k, v, do = [strided(t, pad) for t in dev]
    leaves = [d64(t).requires_grad_() for t in host[:3]]
    o, lse = ref.packed(*leaves, offsets, scale)
    wants = torch.autograd.grad(o, leaves, d64(host[3]), materialize_grads=True)
    bounds = ref.packed_bounds(*[d64(t) for t in host], offsets, scale, u=2.0 ** -8 if dtype == BF16 else 2.0 ** -23)
    got_o, got_lse = ctx.lasad_packed_attention(q, k, v, at, scale=scale, want_lse=True)
    inside("o", got_o, o.detach(), bounds["o"])
    near(got_lse, lse, F32, "lse", extra=2.0 ** -18)
    only_o, none = ctx.lasad_packed_attention(q, k, v, at, scale=scale)
    assert none is None and torch.equal(only_o, got_o)
    back = ctx.lasad_packed_attention_backward(q, k, v, got_o, got_lse, do, at, scale=scale)
    for name, g, want in zip(("dq", "dk", "dv"), back, wants):
        inside(name, g, want, bounds[name])
    assert ctx.device_status() == 0
    return (got_o, got_lse) + back


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", PACKED)
def test_packed_matches_the_formula_and_its_gradient(ctx, shape, dtype):      # noqa: F811
    check_packed(ctx, shape, dtype)


@pytest.mark.parametrize("shape", [PACKED[n] for n in (4, 7, 8)])
def test_packed_on_cuda_cores_for_bf16(ctx, shape):      # noqa: F811
    try:
        ctx.set_option(binding.LASAD_OPT_WINDOW_IMPL, 1)
        check_packed(ctx, shape, BF16)
    finally:
        ctx.set_option(binding.LASAD_OPT_WINDOW_IMPL, 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [PACKED[n] for n in (4, 7, 8)])
def test_packed_takes_strides(ctx, shape, dtype):      # noqa: F811
    check_packed(ctx, shape, dtype, pad=2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0])
def test_packed_other_scales(ctx, scale, dtype):      # noqa: F811
    check_packed(ctx, ((150, 40), 0, 2, 1, 64), dtype, scale=scale)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_packed_heads_first_and_one_tensor_for_all(ctx, dtype):      # noqa: F811
    """q, k and v as views of one projection's output, and memory with the heads first."""
    (q, k, v, _), _, offsets, at = packed_case((70, 200), 0, 4, 2, 64, dtype)
    want = ctx.lasad_packed_attention(q.cuda(), k.cuda(), v.cuda(), at)[0]
    one = torch.cat((q, k, v), 1).cuda()
    assert torch.equal(ctx.lasad_packed_attention(one[:, :4], one[:, 4:6], one[:, 6:], at)[0], want)
    first = [t.transpose(0, 1).contiguous().cuda().transpose(0, 1) for t in (q, k, v)]
    out = torch.empty(4, 270, 64, dtype=dtype, device="cuda").transpose(0, 1)
    assert torch.equal(ctx.lasad_packed_attention(*first, at, o=out)[0], want)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_packed_sharp_and_large_scores(ctx, dtype):      # noqa: F811
    """Scores of hundreds: one key takes all of the weight, and the running maximum has to move."""
    T = 400
    g = gen(6)
    k = rnd(g, T, 1, 64, dtype=dtype)
    q = (k.float() * torch.linspace(0.5, 12, T)[:, None, None]).to(dtype).roll(-1, dims=0)
    v = rnd(g, T, 1, 64, dtype=dtype)
    o, lse = ref.packed(d64(q), d64(k), d64(v), [0, 300, T])
    at = torch.tensor([0, 300, T], dtype=torch.int32, device="cuda")
    got, got_lse = ctx.lasad_packed_attention(q.cuda(), k.cuda(), v.cuda(), at, want_lse=True)
    b = ref.packed_bounds(d64(q), d64(k), d64(v), torch.zeros_like(o), [0, 300, T], u=2.0 ** -8 if dtype == BF16 else 2.0 ** -23)
    inside("o", got, o, b["o"])
    near(got_lse, lse, F32, "lse", extra=2.0 ** -18)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_packed_a_nan_stays_in_its_sequence(ctx, dtype):      # noqa: F811
    _, (q, k, v, do), offsets, at = packed_case((90, 140, 60), 0, 2, 1, 64, dtype)
    o, lse = ctx.lasad_packed_attention(q, k, v, at, want_lse=True)
    grads = ctx.lasad_packed_attention_backward(q, k, v, o, lse, do, at)
    for t in (q, k, v, do):
        t[100] = float("nan")
        t[101] = math.inf
    o2, lse2 = ctx.lasad_packed_attention(q, k, v, at, want_lse=True)
    grads2 = ctx.lasad_packed_attention_backward(q, k, v, o2, lse2, do, at)
    for r in (slice(0, 90), slice(230, 290)):
        assert torch.equal(o[r], o2[r]) and torch.equal(lse[:, r], lse2[:, r])
        assert all(torch.equal(a[r], b[r]) for a, b in zip(grads, grads2))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_packed_gradient_against_differences(ctx, dtype):      # noqa: F811
    """Along random directions of the float64 form: the form's difference quotient (step 1e-4, error 1e-8) and the
    call's gradient; the call's own bound decides."""
    host, dev, offsets, at = packed_case((130, 91), 0, 4, 2, 64, dtype, 5)
    o, lse = ctx.lasad_packed_attention(*dev[:3], at, want_lse=True)
    grads = ctx.lasad_packed_attention_backward(*dev[:3], o, lse, dev[3], at)
    h64 = [d64(t) for t in host]
    bounds = ref.packed_bounds(*h64, offsets, u=2.0 ** -8 if dtype == BF16 else 2.0 ** -23)
    g = gen(77)
    for n, name in enumerate(("dq", "dk", "dv")):
        e = rnd(g, *h64[n].shape).double()
        up, down = list(h64[:3]), list(h64[:3])
        up[n], down[n] = h64[n] + 1e-4 * e, h64[n] - 1e-4 * e
        f = lambda a: (ref.packed(*a, offsets)[0] * h64[3]).sum()    # noqa: E731
        want = (f(up) - f(down)) / 2e-4
        got = (d64(grads[n]) * e).sum()
        assert abs(got - want) <= (1.02 * bounds[name] * e.abs()).sum() + 1e-6 * abs(want), name


@pytest.mark.parametrize("lengths", [(2,) * 64, (3, 2, 1) * 30, (40,) * 8])
def test_packed_gradient_where_rows_see_few_keys(ctx, lengths):      # noqa: F811
    """dP - Delta is small there against Delta itself, which the rounding of o must not reach: 2^-8 in the 2-norm."""
    (q, k, v, do), dev, offsets, at = packed_case(lengths, 0, 4, 4, 64, BF16, 11)
    leaves = [d64(t).requires_grad_() for t in (q, k, v)]
    want = torch.autograd.grad(ref.packed(*leaves, offsets)[0], leaves, d64(do))
    o, lse = ctx.lasad_packed_attention(*dev[:3], at, want_lse=True)
    for a, b in zip(ctx.lasad_packed_attention_backward(*dev[:3], o, lse, dev[3], at), want):
        assert (d64(a) - b).norm() <= 2.0 ** -8 * b.norm()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_packed_repeats_and_does_not_depend_on_neighbours(ctx, dtype):      # noqa: F811
    _, dev, offsets, at = packed_case((900, 513, 128, 1), 7, 6, 2, 64, dtype, 2)

    def run(lo, hi, at):
        q, k, v, do = [t[lo:hi].contiguous() for t in dev]
        o, lse = ctx.lasad_packed_attention(q, k, v, at, want_lse=True)
        return (o, lse) + ctx.lasad_packed_attention_backward(q, k, v, o, lse, do, at)
    first, again = run(0, 1549, at), run(0, 1549, at)
    one = run(900, 1413, torch.tensor([0, 513], dtype=torch.int32, device="cuda"))
    for a, b, c in zip(first, again, one):
        assert torch.equal(a, b)
        assert torch.equal(a[:, 900:1413] if a.dim() == 2 else a[900:1413], c)


def test_packed_offsets_that_do_not_ascend_stay_inside(ctx):      # noqa: F811
    """Undefined results, but memory around the tensors stays as it was."""
    for bad in ([0, 500, 100, 300], [-5, 2 ** 31 - 1, 0, 10], [300, 200, 100, 0], [7, 7, 7, 7]):
        at = torch.tensor(bad, dtype=torch.int32, device="cuda")
        for dtype in (F32, BF16):
            big = [torch.full((700, 2, 64), 0.25, dtype=dtype, device="cuda") for _ in range(8)]
            q, k, v, o, do, dq, dk, dv = [t[200:500] for t in big]
            lse = torch.zeros(2, 300, device="cuda")
            ctx.lasad_packed_attention(q, k, v, at, o=o, lse=lse)
            ctx.lasad_packed_attention_backward(q, k, v, o, lse, do, at, dq=dq, dk=dk, dv=dv)
            assert all(bool((t[:200] == 0.25).all()) and bool((t[500:] == 0.25).all()) for t in big)
    assert ctx.device_status() == 0


def both_ways(ctx, dev, at, **kw):      # noqa: F811
    """What the tensor cores and the CUDA cores make of it."""
    q, k, v, do = dev
    out = []
    try:
        for impl in (2, 1):
            ctx.set_option(binding.LASAD_OPT_WINDOW_IMPL, impl)
            o, lse = ctx.lasad_packed_attention(q, k, v, at, want_lse=True, **kw)
            out.append((o, lse) + ctx.lasad_packed_attention_backward(q, k, v, o, lse, do, at, **kw))
    finally:
        ctx.set_option(binding.LASAD_OPT_WINDOW_IMPL, 0)
    return out


@pytest.mark.parametrize("lengths,tail,Hq,Hk,d", [
    ((257,) * 32, 0, 12, 12, 64), ((129,) * 40, 5, 16, 4, 64), ((1,) * 300, 0, 8, 8, 64), ((3000, 1, 300, 2049), 700, 6, 2, 64),
    ((1025,) * 4, 0, 24, 8, 64), ((0, 640, 0, 0, 641, 1) * 6, 3, 10, 5, 32), ((65, 64, 63) * 50, 0, 5, 1, 64)])
def test_packed_many_units_on_both_implementations(ctx, lengths, tail, Hq, Hk, d):      # noqa: F811
    """So many units that every CTA takes several, some of which one of its row tiles has none of: both
    implementations round p and ds and their outputs by at most 2^-8 each, so they are within 2^-7 of one another in the
    2-norm (the statistics, in fp32, within 2^-18).  Where rows see one key dP - Delta is 0, and what is left of it is the fp32
    rounding of sums of 64 products of size 1, |do||v| 2^-23 or less, on keys of size 1: 2^-18 for an element is far above."""
    _, dev, offsets, at = packed_case(lengths, tail, Hq, Hk, d, BF16, 3)
    for name, a, b in zip(("o", "lse", "dq", "dk", "dv"), *both_ways(ctx, dev, at)):
        a, b = a.double(), b.double()
        if name == "lse":
            live = b > -math.inf
            assert torch.equal(live, a > -math.inf) and float((a - b)[live].abs().max()) <= 2.0 ** -18 * float(b[live].abs().max())
        else:
            assert float((a - b).norm()) <= 2.0 ** -7 * float(b.norm()) + 2.0 ** -18 * math.sqrt(b.numel()), name
            assert bool((a[offsets[-1]:] == 0).all())
    assert ctx.device_status() == 0


def test_packed_back_to_back_in_a_warm_cache(ctx):      # noqa: F811
    """Over and over with nothing in between: no wait may give up, and every launch returns the same bits."""
    _, (q, k, v, do), _, at = packed_case((2305, 700, 129, 1), 0, 8, 4, 64, BF16, 6)
    first = None
    for _ in range(30):
        o, lse = ctx.lasad_packed_attention(q, k, v, at, want_lse=True)
        got = (o, lse) + ctx.lasad_packed_attention_backward(q, k, v, o, lse, do, at)
        first = first or got
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_packed_waits_are_bounded(ctx):      # noqa: F811
    """Waits that run out after one try: the kernels report it and leave, and the next calls are whole."""
    _, (q, k, v, do), _, at = packed_case((700, 300), 0, 4, 4, 64, BF16, 7)
    o, lse = ctx.lasad_packed_attention(q, k, v, at, want_lse=True)
    want = ctx.lasad_packed_attention_backward(q, k, v, o, lse, do, at)
    try:
        ctx.set_option(binding.LASAD_OPT_WAIT_LIMIT, 1)
        ctx.lasad_packed_attention(q, k, v, at)
        torch.cuda.synchronize()
        assert ctx.device_status() == binding.LASAD_ERR_TIMEOUT
        ctx.lasad_packed_attention_backward(q, k, v, o, lse, do, at)
        torch.cuda.synchronize()
        assert ctx.device_status() == binding.LASAD_ERR_TIMEOUT
    finally:
        ctx.set_option(binding.LASAD_OPT_WAIT_LIMIT, 0)
    assert torch.equal(ctx.lasad_packed_attention(q, k, v, at)[0], o)
    assert all(torch.equal(a, b) for a, b in zip(ctx.lasad_packed_attention_backward(q, k, v, o, lse, do, at), want))
    assert ctx.device_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_packed_rows_far_apart(ctx, dtype):      # noqa: F811
    """Places past 2^31 elements: rows 8 M elements apart."""
    host, dev, offsets, at = packed_case((150, 130), 0, 2, 1, 64, dtype, 9)
    o, lse = ctx.lasad_packed_attention(*dev[:3], at, want_lse=True)
    want = (o,) + ctx.lasad_packed_attention_backward(*dev[:3], o, lse, dev[3], at)
    apart = 8 << 20
    big = torch.zeros(280 * apart, dtype=dtype, device="cuda")
    view = lambda n, t: torch.as_strided(big, t.shape, (apart, 64, 1), n * 256)       # noqa: E731
    far = [view(n, t).copy_(t) for n, t in enumerate((*dev, o))]
    outs = [view(8 + n, t) for n, t in enumerate(want)]
    ctx.lasad_packed_attention(*far[:3], at, o=outs[0], lse=lse)
    ctx.lasad_packed_attention_backward(*far[:3], far[4], lse, far[3], at, dq=outs[1], dk=outs[2], dv=outs[3])
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


# ---------------------------------------------------------------------------------------------
# paged cache
# ---------------------------------------------------------------------------------------------
def cache_of(g, P, Hk, page, d, low=-6, high=6):
    """A pool in use: any e4m3 numbers but NaN, and any powers of two as scales."""
    codes = lambda: torch.randint(0, 127, (P, Hk, page, d), generator=g) + 128 * torch.randint(0, 2, (P, Hk, page, d), generator=g)   # noqa: E731
    scales = lambda: 2.0 ** torch.randint(low, high + 1, (P, Hk), generator=g).float()   # noqa: E731
    return dict(k_pages=codes().to(torch.uint8).view(E4M3), v_pages=codes().to(torch.uint8).view(E4M3),
                k_scales=scales(), v_scales=scales())


def to_dev(cache, pad=0):
    out = {}
    for n, t in cache.items():
        if pad and n.endswith("pages"):
            big = torch.full([s + 1 for s in t.shape[:-1]] + [t.shape[-1] + 32], 0x7f, dtype=torch.uint8, device="cuda").view(E4M3)
            view = big[tuple(slice(0, s) for s in t.shape[:-1]) + (slice(16, 16 + t.shape[-1]),)]
            view.view(torch.uint8).copy_(t.view(torch.uint8))
            out[n] = view
        else:
            out[n] = t.cuda()
    return out


def to_64(cache):
    return {n: t.cpu().double() for n, t in cache.items()}


def same_cache(got, want):
    for n, t in got.items():
        assert torch.equal(t.cpu().double().nan_to_num(nan=1e9), want[n].nan_to_num(nan=1e9)), n


APPEND = [  # new tokens of each sequence (None: one each, no offsets), first positions, Hq, Hk, d, page, table entries
    (None, (0,), 1, 1, 64, 16, 1), (None, (0, 15, 16, -1, 33, 47), 4, 2, 64, 16, 3), (None, (127, 128, 5), 3, 1, 32, 128, 2),
    ((1,), (0,), 2, 2, 64, 32, 1), ((40, 0, 17, 3), (0, 5, 9, -1), 4, 2, 64, 16, 4), ((100, 33), (31, 64), 6, 2, 64, 32, 5),
    ((64, 65, 1), (0, 0, 63), 2, 1, 32, 64, 2), ((300,), (100,), 8, 4, 64, 128, 4), ((5, 200), (1000, 30), 2, 2, 64, 16, 10),
]


def append_case(shape, dtype, seed=0):
    lengths, pos, Hq, Hk, d, page, entries = shape
    g = gen(seed + Hq + page)
    B = len(pos)
    offsets = None
    N = B
    if lengths is not None:
        offsets = [0]
        for n in lengths:
            offsets.append(offsets[-1] + n)
        N = offsets[-1] + 3                                    # three rows that nobody has
    k, v, q = (rnd(g, N, h, d, dtype=dtype, std=s) for h, s in ((Hk, 3.0), (Hk, 0.2), (Hq, 1.0)))
    k[0, 0, 0] = 0.0
    block_table = torch.randperm(B * entries + 2, generator=g)[: B * entries].view(B, entries).int()
    return k, v, q, offsets, list(pos), block_table, cache_of(g, B * entries + 2, Hk, page, d)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("grid_w,prefix,half", [(0, 0, False), (0, 0, True), (7, 1, False), (5, 3, True), (None, 0, False)])
@pytest.mark.parametrize("shape", APPEND)
def test_append_matches_the_definition(ctx, shape, grid_w, prefix, half, dtype):      # noqa: F811
    k, v, q, offsets, pos, bt, cache = append_case(shape, dtype)
    d, page, entries = shape[4:]
    table = None if grid_w is None else binding.rope_table(60 if grid_w else 900, d, bool(grid_w))
    grid_w = grid_w or 0
    dev, want = to_dev(cache, pad=1 if half else 0), to_64(cache)
    ref.append(k, v, want, bt, pos, offsets, table, grid_w, prefix, half)
    dq = ctx.lasad_paged_append(strided(k.cuda(), 1 if half else 0), v.cuda(), **dev, block_table=bt.cuda(),
                                pos=torch.tensor(pos, dtype=torch.int32, device="cuda"),
                                offsets=None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda"),
                                q=strided(q.cuda(), 1 if half else 0), table=None if table is None else table.cuda(), grid_w=grid_w,
                                prefix_len=prefix, half=half)
    same_cache(dev, want)
    turned = torch.zeros_like(d64(q))
    for b, r in enumerate(ref.rows(offsets or range(len(pos) + 1))):
        for i in range(r.start, r.stop):
            if pos[b] >= 0:
                x = d64(q[i])
                turned[i] = x if table is None else ref.turned(x, table, pos[b] + i - r.start, grid_w, prefix, half)
    near(dq, turned, dtype, "q")
    assert ctx.device_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_append_extreme_values(ctx, dtype):      # noqa: F811
    """Zeros, the largest and smallest numbers, infinities and NaN, and scales that have to grow or may not shrink."""
    page, d = 16, 64
    k, v, q, offsets, pos, bt, cache = append_case(((16, 3, 5, 2, 8), (0, 4, 15, 8, 3), 1, 2, d, page, 2), dtype, 4)
    v[0:16] = 0.0
    v[16] = 1e30
    k[17, 0, 3], k[17, 1, 5] = math.inf, float("nan")
    k[19:24] *= 1e-25
    v[24:26] = -448 * 2.0 ** 40
    k[26:30, :, 0] = 448.0 * 2.0 ** torch.arange(4)[:, None].float()
    k[30:34] = 3e38
    dev, want = to_dev(cache), to_64(cache)
    ref.append(k, v, want, bt, pos, offsets)
    ctx.lasad_paged_append(k.cuda(), v.cuda(), **dev, block_table=bt.cuda(), pos=torch.tensor(pos, dtype=torch.int32, device="cuda"),
                           offsets=torch.tensor(offsets, dtype=torch.int32, device="cuda"))
    same_cache(dev, want)


def test_append_drops_what_has_no_page(ctx):      # noqa: F811
    """Entries outside the pool, positions past the table, far positions: nothing but the pool's own pages changes."""
    k, v, q, offsets, pos, bt, cache = append_case(((40, 40, 40, 2), (0, 20, 2 ** 31 - 41, 70), 2, 2, 64, 16, 4), BF16, 1)
    bt[0, 1], bt[1, 2], bt[0, 2] = -1, 2 ** 31 - 1, bt.numel() + 2
    dev, want = to_dev(cache, pad=1), to_64(cache)
    ref.append(k, v, want, bt, pos, offsets)
    ctx.lasad_paged_append(k.cuda(), v.cuda(), **dev, block_table=bt.cuda(), pos=torch.tensor(pos, dtype=torch.int32, device="cuda"),
                           offsets=torch.tensor(offsets, dtype=torch.int32, device="cuda"))
    same_cache(dev, want)
    big = dev["k_pages"]._base
    assert bool((big.view(torch.uint8)[:, :, :, :16] == 0x7f).all()) and bool((big.view(torch.uint8)[-1] == 0x7f).all())


PAGED = [  # positions, Hq, Hk, d, page, table entries
    ((0,), 1, 1, 64, 16, 1), ((-1, 0, 15, 16, 31), 2, 1, 64, 16, 2), ((63, 64, 100), 8, 8, 64, 32, 4), ((5, 400), 12, 4, 32, 64, 7),
    ((1000,), 24, 8, 64, 64, 16), ((300, 17), 20, 1, 64, 128, 3), ((700, 3), 40, 1, 32, 16, 44), ((257, 256, 255, 254), 3, 3, 64, 16, 17),
    ((5000, 1), 6, 2, 64, 128, 40), ((2047,), 9, 1, 64, 32, 64), ((99999,), 2, 2, 64, 16, 30),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", PAGED)
def test_paged_attention_matches_the_formula(ctx, shape, dtype):      # noqa: F811
    pos, Hq, Hk, d, page, entries = shape
    B = len(pos)
    g = gen(page + Hq)
    q = rnd(g, B, Hq, d, dtype=dtype)
    bt = torch.randperm(B * entries + 2, generator=g)[: B * entries].view(B, entries).int()
    cache = cache_of(g, B * entries + 2, Hk, page, d, low=-9, high=-6)
    cache["v_scales"] *= 2.0 ** torch.randint(-3, 4, cache["v_scales"].shape, generator=g).float()
    # weights carry 2^-11 (fp16); the output is rounded once: at most half a step, eps / 2 of its value
    o, lse, err = ref.paged(d64(q), to_64(cache), bt, pos, u=2.0 ** -11 if dtype == BF16 else 2.0 ** -22)
    for b, p in enumerate(pos):                   # slots that no token has reached hold anything
        for i in range(p + 1, entries * page):
            for n in ("k", "v"):
                cache[n + "_pages"].view(torch.uint8)[bt[b, i // page], :, i % page] = 0x7f
    for pad in (0, 1):
        dev = to_dev(cache, pad)
        got, got_lse = ctx.lasad_paged_attention(strided(q.cuda(), pad), **dev, block_table=bt.cuda(),
                                                 pos=torch.tensor(pos, dtype=torch.int32, device="cuda"), want_lse=True)
        inside("o", got, o, err + torch.finfo(dtype).eps / 2 * o.abs())
        near(got_lse, lse, F32, "lse", extra=2.0 ** -18)
    assert ctx.device_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_paged_attention_over_scales_far_apart(ctx, dtype):      # noqa: F811
    """Value scales from 2^-40 to 2^40 and scores of hundreds in one sequence, queries from 1e-30 to 1e30 with a scale
    that brings them back."""
    g = gen(3)
    page, entries, pos = 16, 20, (319, 200)
    cache = cache_of(g, 2 * entries, 2, page, 64, low=-7, high=-3)
    cache["v_scales"] = 2.0 ** torch.linspace(-40, 40, 2 * entries * 2).round().view(2 * entries, 2)[torch.randperm(2 * entries, generator=g)]
    bt = torch.arange(2 * entries).view(2, entries).int()
    dev = to_dev(cache)
    p32 = torch.tensor(pos, dtype=torch.int32, device="cuda")
    for size in (1.0, 2.0 ** -100, 2.0 ** 100):
        q = rnd(g, 2, 4, 64, std=2.0, dtype=dtype) * size
        scale = 0.125 / size
        o, lse, err = ref.paged(d64(q), to_64(cache), bt, pos, scale, u=2.0 ** -11 if dtype == BF16 else 2.0 ** -22)
        got, got_lse = ctx.lasad_paged_attention(q.cuda(), **dev, block_table=bt.cuda(), pos=p32, scale=scale, want_lse=True)
        inside("o", got, o, err + torch.finfo(dtype).eps / 2 * o.abs())
        near(got_lse, lse, F32, "lse", extra=2.0 ** -18)


def test_paged_attention_passes_over_pages_that_are_none(ctx):      # noqa: F811
    g = gen(8)
    page, entries, pos = 16, 40, (639, 639, 100, 50)
    cache = cache_of(g, 100, 1, page, 64, low=-9, high=-6)
    bt = torch.randint(0, 100, (4, entries), generator=g).int()                  # (pages may be shared)
    bt[0, ::3], bt[1, 5:], bt[2], bt[3, 0] = -1, 100, -7, 2 ** 31 - 1
    q = rnd(g, 4, 2, 64)
    o, lse, err = ref.paged(d64(q), to_64(cache), bt, pos, u=2.0 ** -22)
    got, got_lse = ctx.lasad_paged_attention(q.cuda(), **to_dev(cache), block_table=bt.cuda(),
                                             pos=torch.tensor(pos, dtype=torch.int32, device="cuda"), want_lse=True)
    inside("o", got, o, err + 2.0 ** -24 * o.abs())
    near(got_lse, lse, F32, "lse", extra=2.0 ** -18)
    assert bool((got[2] == 0).all()) and bool((got_lse[2] == -math.inf).all())


def test_paged_attention_a_nan_stays_in_its_sequence(ctx):      # noqa: F811
    g = gen(9)
    cache = cache_of(g, 8, 2, 16, 64, low=-9, high=-6)
    bt, pos = torch.arange(8).view(2, 4).int().cuda(), torch.tensor([60, 50], dtype=torch.int32, device="cuda")
    q = rnd(g, 2, 4, 64, dtype=BF16).cuda()
    a, _ = ctx.lasad_paged_attention(q, **to_dev(cache), block_table=bt, pos=pos)
    cache["v_pages"].view(torch.uint8)[1, 0, 3, 7] = 0x7f
    b, _ = ctx.lasad_paged_attention(q, **to_dev(cache), block_table=bt, pos=pos)
    assert torch.equal(a[1], b[1]) and torch.equal(a[0, 2:], b[0, 2:])
    assert bool(b[0, :2, 7].isnan().all()) and bool(b[0, :2, :7].isfinite().all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("entries", [4, 130])       # one part, and parts that are joined
def test_paged_attention_keeps_a_nan_of_the_query(ctx, entries, dtype):      # noqa: F811
    """Where every score of a sequence is NaN so is its output, however its tokens are cut.  Other sequences and key
    heads keep their bits.  The head that shares the key head shares the warps, which move their running maximum as soon as
    one column has none, and so at other steps than before: a move multiplies by an exponential (2^-22), a warp has at most
    4 steps of a part here (256 tokens, 4 warps, 16 tokens a step), and 4 x 2^-22 is below the 2 x 2^-20 that the
    formula's bound has for exponentials.  So it is held to that bound."""
    g = gen(10)
    cache = cache_of(g, entries, 2, 16, 64, low=-9, high=-6)
    bt = torch.arange(entries).int().repeat(3, 1).cuda()
    pos = torch.tensor([16 * entries - 1, 16 * entries - 1, -1], dtype=torch.int32, device="cuda")
    q = rnd(g, 3, 4, 64, dtype=dtype).cuda()
    a, la = ctx.lasad_paged_attention(q, **to_dev(cache), block_table=bt, pos=pos, want_lse=True)
    q[1, 2, 5] = float("nan")
    b, lb = ctx.lasad_paged_attention(q, **to_dev(cache), block_table=bt, pos=pos, want_lse=True)
    assert bool(b[1, 2].isnan().all()) and bool(lb[1, 2].isnan())
    o, lse, err = ref.paged(d64(q[:2, 3:]).repeat(1, 2, 1), {n: x[:, 1:] for n, x in to_64(cache).items()}, bt.cpu(),
                            pos[:2].tolist(), u=2.0 ** -11 if dtype == BF16 else 2.0 ** -22)
    inside("the other head", b[1, 3], o[1, 0], err[1, 0] + torch.finfo(dtype).eps / 2 * o[1, 0].abs())
    near(lb[1, 3], lse[1, 0], F32, "lse", extra=2.0 ** -18)
    b[1, 2:], lb[1, 2:] = a[1, 2:], la[1, 2:]
    assert torch.equal(a, b) and torch.equal(la, lb)


@pytest.mark.parametrize("strides", [(64, 64, 1 << 30), (1 << 31, 64, 64), (64, 64, 1 << 62), (1 << 62, 64, 64)])
@pytest.mark.parametrize("which", ["k_pages_stride", "v_pages_stride"])
def test_pools_too_large_to_count_are_refused(ctx, which, strides):      # noqa: F811
    """The last place of a pool decides, whichever stride takes it there.  (Asking for the workspace launches nothing.)"""
    p = sequences.PagedParams(2, 0, 4, 2, 64, 1, 128, 64, 4, 0, 0, 0, 0, 0.125)
    for n in ("k_pages_stride", "v_pages_stride"):
        setattr(p, n, (ctypes.c_int64 * 3)(2 * 128 * 64, 128 * 64, 64))
    for n in ("q_stride", "o_stride"):
        setattr(p, n, (ctypes.c_int64 * 2)(256, 64))
    assert ctx._lib.lasad_paged_attention_workspace(ctx._h, ctypes.byref(p)) >= 0
    setattr(p, which, (ctypes.c_int64 * 3)(*strides))
    assert ctx._lib.lasad_paged_attention_workspace(ctx._h, ctypes.byref(p)) == binding.LASAD_ERR_UNSUPPORTED


def test_pages_far_apart_and_tokens_first(ctx):      # noqa: F811
    """A pool whose pages are 3 GiB apart (places past 2^32 bytes), and one with the slots ahead of the heads."""
    g = gen(12)
    cache = cache_of(g, 4, 2, 16, 64, low=-9, high=-6)
    bt, pos = torch.tensor([[3, 0, 2, 1]], dtype=torch.int32).cuda(), torch.tensor([49], dtype=torch.int32, device="cuda")
    k, v, q = (rnd(g, 1, h, 64, dtype=BF16).cuda() for h in (2, 2, 4))
    apart = 3 << 30
    big = torch.zeros(3 * apart + (1 << 20), dtype=torch.uint8, device="cuda").view(E4M3)
    results = []
    for how in ("together", "apart", "tokens first"):
        dev = to_dev(cache)
        for n, name in enumerate(("k_pages", "v_pages")):
            t = dev[name]
            if how == "apart":
                dev[name] = torch.as_strided(big, t.shape, (apart, 16 * 64, 64, 1), n * 4096)
            elif how == "tokens first":
                dev[name] = torch.empty(4, 16, 2, 64, dtype=torch.uint8, device="cuda").view(E4M3).transpose(1, 2)
            if how != "together":
                dev[name].view(torch.uint8).copy_(t.view(torch.uint8))
        ctx.lasad_paged_append(k, v, **dev, block_table=bt, pos=pos)
        o, lse = ctx.lasad_paged_attention(q, **dev, block_table=bt, pos=pos, want_lse=True)
        results.append([o, lse] + [dev[n].view(torch.uint8).clone() for n in ("k_pages", "v_pages")] + [dev["k_scales"], dev["v_scales"]])
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))


@pytest.mark.parametrize("shape", [(300, 4, 4, 40), (40, 24, 8, 700), (2, 6, 2, 3000), (1, 24, 1, 5000)])
def test_paged_attention_by_every_plan(ctx, shape):      # noqa: F811
    """A warp, a CTA and many CTAs for a (sequence, key head): against the attention of a prompt's last token over the cache's
    own values, in float64 on the device."""
    B, Hq, Hk, n = shape
    g, page = gen(B), 32
    entries = -(-n // page)
    cache = to_dev(cache_of(g, B * entries, Hk, page, 64, low=-9, high=-6))
    bt = torch.randperm(B * entries, generator=g).view(B, entries).int().cuda()
    pos = torch.randint(-1, n, (B,), generator=g).int()
    pos[-1] = n - 1
    for dtype in (F32, BF16):
        q = rnd(g, B, Hq, 64, dtype=dtype).cuda()
        got, lse = ctx.lasad_paged_attention(q, **cache, block_table=bt, pos=pos.cuda(), want_lse=True)
        for b in list(range(min(B, 12))) + [B - 1]:
            if int(pos[b]) < 0:
                assert bool((got[b] == 0).all()) and bool((lse[b] == -math.inf).all())
                continue
            kk, vv = ((cache[m + "_pages"][bt[b].long()].double() * cache[m + "_scales"][bt[b].long()].double()[..., None, None])
                      .transpose(0, 1).flatten(1, 2)[:, : int(pos[b]) + 1].repeat_interleave(Hq // Hk, 0) for m in ("k", "v"))
            x = torch.einsum("hd,hnd->hn", q[b].double(), kk) / 8
            p = torch.softmax(x, -1)
            o = torch.einsum("hn,hnd->hd", p, vv)
            # weights: 2^-11 (bf16) or 2^-22; exponents 2^-20 of their size; the output's own rounding
            size = torch.einsum("hd,hnd->hn", q[b].double().abs(), kk.abs()) / 8
            e = (2.0 ** -11 if dtype == BF16 else 2.0 ** -22) + 2.0 ** -20 * (2 + size + x.abs().amax(-1, keepdim=True))
            bound = torch.einsum("hn,hnd->hd", p * e, vv.abs()) + torch.finfo(dtype).eps / 2 * o.abs() + 2.0 ** -30
            assert bool(((got[b].double() - o).abs() <= 1.02 * bound).all()), (b, dtype)
            near(lse[b], torch.logsumexp(x, -1).cpu(), F32, "lse", extra=2.0 ** -18)


# ---------------------------------------------------------------------------------------------
# the layer as it is used
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_prompts_then_tokens(ctx, dtype):      # noqa: F811
    """A batch's prompts go into the cache and through packed attention, then every sequence grows token by token:
    each token's output is what the definition gives for the cache as it then stands, and near what attention over
    the whole, unrounded sequence gives (2^-4 of a key or value, as e4m3 has, gathered like noise)."""
    B, Hq, Hk, d, page, entries, w, prefix = 3, 4, 2, 64, 16, 5, 8, 1
    prompts, new = (0, 17, 40), 20
    g = gen(5)
    total = [n + new for n in prompts]
    xs = [[rnd(g, n, h, d, dtype=dtype) for h in (Hq, Hk, Hk)] for n in total]
    table = binding.rope_table(16, d, True)
    bt = torch.randperm(B * entries, generator=g).view(B, entries).int()
    cache = cache_of(g, B * entries, Hk, page, d)
    dev, want = to_dev(cache), to_64(cache)
    kw = dict(table=table.cuda(), grid_w=w, prefix_len=prefix, block_table=bt.cuda())
    offsets = [0, 0, 17, 57]
    q, k, v = (torch.cat([x[i][:n] for x, n in zip(xs, prompts)]) for i in range(3))
    at = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    pos = torch.zeros(B, dtype=torch.int32, device="cuda")
    qt = ctx.lasad_paged_append(k.cuda(), v.cuda(), **dev, pos=pos, offsets=at, q=q.cuda(), **kw)
    ref.append(k, v, want, bt, [0] * B, offsets, table, w, prefix)
    same_cache(dev, want)
    # packed attention on the same rotation
    kt = torch.cat([torch.stack([ref.turned(d64(k[offsets[b] + i]), table, i, w, prefix) for i in range(n)])
                    for b, n in enumerate(prompts) if n]).to(dtype)
    o, _ = ctx.lasad_packed_attention(qt, kt.cuda(), v.cuda(), at)
    bound = ref.packed_bounds(d64(qt), d64(kt), d64(v), torch.zeros_like(d64(q)), offsets, u=2.0 ** -8 if dtype == BF16 else 2.0 ** -23)
    inside("prompts", o, ref.packed(d64(qt), d64(kt), d64(v), offsets)[0], bound["o"])
    pos = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    graph, side = None, torch.cuda.Stream()
    inq, ink, inv = (torch.zeros(B, h, d, dtype=dtype, device="cuda") for h in (Hq, Hk, Hk))
    out = torch.empty_like(inq)
    for step in range(new):
        q1, k1, v1 = (torch.stack([x[i][n + step] for x, n in zip(xs, prompts)]) for i in range(3))
        for to, x in ((inq, q1), (ink, k1), (inv, v1)):
            to.copy_(x)
        if step == 3:                             # from here on a captured step
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=side):
                qt = ctx.lasad_paged_append(ink, inv, **dev, pos=pos, q=inq, **kw)
                ctx.lasad_paged_attention(qt, **dev, block_table=kw["block_table"], pos=pos, o=out)
        if graph is not None:
            graph.replay()
        else:
            qt = ctx.lasad_paged_append(ink, inv, **dev, pos=pos, q=inq, **kw)
            ctx.lasad_paged_attention(qt, **dev, block_table=kw["block_table"], pos=pos, o=out)
        now = [n + step for n in prompts]
        ref.append(k1, v1, want, bt, now, None, table, w, prefix)
        same_cache(dev, want)
        q64 = d64(qt)
        o, _, err = ref.paged(q64, want, bt, now, u=2.0 ** -11 if dtype == BF16 else 2.0 ** -22)
        inside(("step", step), out, o, err + torch.finfo(dtype).eps / 2 * o.abs())
        for b, n in enumerate(now):
            kk = torch.stack([ref.turned(d64(xs[b][1][i]), table, i, w, prefix) for i in range(n + 1)])
            whole = torch.stack([torch.softmax(kk[:, h // 2] @ q64[b, h] / 8, 0) @ d64(xs[b][2][: n + 1, h // 2]) for h in range(Hq)])
            assert (d64(out[b]) - whole).norm() <= 2.0 ** -3 * d64(xs[b][2][: n + 1]).norm() / math.sqrt(n + 1)
        pos += 1
    assert ctx.device_status() == 0


def test_calls_on_two_streams_and_in_graphs_that_share_nothing(ctx):      # noqa: F811
    from tests.test_gpu_mixers_memory import check_two_streams
    _, (q, k, v, do), offsets, at = packed_case((800, 1200, 3), 0, 8, 4, 64, BF16, 1)
    o, lse = ctx.lasad_packed_attention(q, k, v, at, want_lse=True)
    check_two_streams(ctx, lambda **s: ctx.lasad_packed_attention_backward(q, k, v, o, lse, do, at, **s))
    check_two_streams(ctx, lambda **s: ctx.lasad_packed_attention(q, k, v, at, want_lse=True, **s))
    g = gen(1)
    cache, bt = to_dev(cache_of(g, 80, 2, 64, 64, low=-9, high=-6)), torch.arange(80).view(2, 40).int().cuda()
    qs, pos = rnd(g, 2, 4, 64, dtype=BF16).cuda(), torch.tensor([2500, 100], dtype=torch.int32, device="cuda")
    check_two_streams(ctx, lambda **s: ctx.lasad_paged_attention(qs, **cache, block_table=bt, pos=pos, want_lse=True, **s))


def test_refusals_of_the_library(ctx):      # noqa: F811
    at = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    x = lambda *s, **kw: torch.zeros(*s, device="cuda", **kw)       # noqa: E731
    calls = []
    calls.append(lambda: ctx.lasad_packed_attention(x(5, 2, 48), x(5, 2, 48), x(5, 2, 48), at))                       # head size
    calls.append(lambda: ctx.lasad_packed_attention(x(5, 3, 64), x(5, 2, 64), x(5, 2, 64), at))                       # heads
    calls.append(lambda: ctx.lasad_packed_attention(x(5, 2, 65)[:, :, 1:], x(5, 2, 64), x(5, 2, 64), at))             # alignment
    calls.append(lambda: ctx.lasad_packed_attention(x(5, 1, 64).expand(5, 2, 64), x(5, 2, 64), x(5, 2, 64), at, o=x(5, 1, 64).expand(5, 2, 64)))
    calls.append(lambda: ctx.lasad_packed_attention(x(5, 2, 64), x(5, 2, 64), x(5, 2, 64), at, scale=math.inf))
    calls.append(lambda: ctx.lasad_packed_attention(x(0, 2, 64), x(0, 2, 64), x(0, 2, 64), at))
    def cache(page=16, d=64, P=4, Hk=2):                              # noqa: E306
        return dict(k_pages=x(P, Hk, page, d).to(E4M3), v_pages=x(P, Hk, page, d).to(E4M3), k_scales=x(P, Hk), v_scales=x(P, Hk),
                    block_table=x(2, 2, dtype=torch.int32), pos=x(2, dtype=torch.int32))
    for c in (cache(page=24), cache(page=8), cache(page=256), cache(d=48)):
        d = c["k_pages"].shape[3]
        calls.append(lambda c=c, d=d: ctx.lasad_paged_append(x(2, 2, d), x(2, 2, d), **c))
        calls.append(lambda c=c, d=d: ctx.lasad_paged_attention(x(2, 2, d), **c))
    calls.append(lambda: ctx.lasad_paged_append(x(2, 2, 64), x(2, 2, 64), **cache(), q=x(2, 3, 64)))
    calls.append(lambda: ctx.lasad_paged_append(x(2, 2, 64), x(2, 2, 64), **cache(), table=x(5, 16, 2), grid_w=3, prefix_len=-1))
    calls.append(lambda: ctx.lasad_paged_append(x(2, 2, 72)[:, :, 4:68], x(2, 2, 65)[:, :, 1:], **cache()))
    calls.append(lambda: ctx.lasad_paged_attention(x(2, 2, 64), **cache(), scale=math.nan))
    for n, call in enumerate(calls):
        before = ctx.launch_count
        with pytest.raises((binding.LasadError, ValueError)):
            call()
        assert ctx.launch_count == before, n
    torch.cuda.synchronize()
