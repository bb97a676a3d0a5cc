"""What can be said of the operators of a layer that attends to whole sequences without a GPU: the structs' layout,
the rounding to 8 bits that the GPU tests compare with, refusals, and that outputs belong to the call's stream."""
import ctypes
import math

import pytest
import torch

from paper_2507_01652_b200 import binding, sequences
from tests import _sequences_ref as ref
from tests.test_mixers_devices_cpu import there
from tests.test_stream_memory_cpu import CURRENT, OTHER, Memory, m, world  # noqa: F401


@pytest.fixture(autouse=True)
def streams(monkeypatch):
    monkeypatch.setattr(sequences, "_stream", lambda device, s: CURRENT if s is None else s)


def test_struct_layouts():
    assert ctypes.sizeof(sequences.PackedParams) == 32 + 8 * 16
    assert sequences.PackedParams.q_stride.offset == 32
    assert ctypes.sizeof(sequences.PagedParams) == 56 + 2 * 24 + 4 * 16
    assert sequences.PagedParams.k_pages_stride.offset == 56


def test_null_arguments_need_no_device():
    lib = binding.load_library()
    p, g = sequences.PackedParams(), sequences.PagedParams()
    assert lib.lasad_packed_attention(None, ctypes.byref(p), *[None] * 7) == binding.LASAD_ERR_INVALID_ARG
    assert lib.lasad_packed_attention_workspace(None, ctypes.byref(p)) == binding.LASAD_ERR_INVALID_ARG
    assert lib.lasad_packed_attention_backward(None, ctypes.byref(p), *[None] * 12) == binding.LASAD_ERR_INVALID_ARG
    assert lib.lasad_paged_append(None, ctypes.byref(g), *[None] * 13) == binding.LASAD_ERR_INVALID_ARG
    assert lib.lasad_paged_attention(None, ctypes.byref(g), *[None] * 11) == binding.LASAD_ERR_INVALID_ARG
    assert lib.lasad_paged_attention_workspace(None, ctypes.byref(g)) == binding.LASAD_ERR_INVALID_ARG


def test_rounding_to_8_bits_is_the_types_own():
    x = torch.cat((torch.randn(4000, generator=torch.Generator().manual_seed(1)) * 20, torch.linspace(-500, 500, 999),
                   torch.tensor([0.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -11, 17.0, 19.0, 448.0, 464.0, 1e9])))
    want = x.clamp(-448, 448).to(torch.float8_e4m3fn).double()
    assert torch.equal(ref.nearest(x.double()), want)
    assert bool(ref.nearest(torch.tensor([math.nan], dtype=torch.float64)).isnan().all())
    for big, e in ((448.0, 0), (448.1, 1), (1.75, -8), (1.7500001, -7), (0.0, -40), (1e-30, -40), (1e30, 40)):
        assert ref.scale_of(torch.tensor([0.0, -big, math.inf, math.nan], dtype=torch.float64)) == 2.0 ** e


def test_appending_in_pieces_is_appending_at_once():
    """Powers of two move no digits: what grew token by token is what is written at once, but for the numbers that
    leave the normal range of the page's last scale (below 2^-6 of it)."""
    g = torch.Generator().manual_seed(3)
    n, Hk, page, d = 37, 2, 16, 8
    k, v = torch.randn(n, Hk, d, generator=g), torch.randn(n, Hk, d, generator=g) * torch.linspace(0.1, 9, n)[:, None, None]
    table = torch.tensor([[2, 0, 1]])
    new = lambda: dict(k_pages=torch.zeros(3, Hk, page, d, dtype=torch.float64), v_pages=torch.zeros(3, Hk, page, d, dtype=torch.float64),   # noqa: E731
                       k_scales=torch.ones(3, Hk, dtype=torch.float64), v_scales=torch.ones(3, Hk, dtype=torch.float64))
    once, grown = new(), new()
    ref.append(k, v, once, table, [0], [0, n])
    for i in range(n):
        ref.append(k[i:i + 1], v[i:i + 1], grown, table, [i])
    for name in ("k", "v"):
        assert torch.equal(once[name + "_scales"], grown[name + "_scales"])
        a, b = once[name + "_pages"], grown[name + "_pages"]
        normal = a.abs() >= 2.0 ** -6
        assert torch.equal(a[normal], b[normal]) and float((a - b).abs().max()) <= 2.0 ** -9
        x = torch.stack([ref.seen_tokens(once, name, table, 0, n - 1, h) for h in range(Hk)], 1)
        full = (k, v)["kv".index(name)].double()
        step = once[name + "_scales"][table[0, torch.arange(n) // page]][..., None] * 2.0 ** -10
        assert bool(((x - full).abs() <= torch.maximum(full.abs() * 2.0 ** -4, step)).all())


def arguments(packed_rows=True):
    q, k = m(7, 4, 64), m(7, 2, 64)
    offsets, lse = m(3, dtype=torch.int32), m(4, 7)
    e4 = torch.float8_e4m3fn
    cache = dict(k_pages=m(5, 2, 16, 64, dtype=e4), v_pages=m(5, 2, 16, 64, dtype=e4), k_scales=m(5, 2), v_scales=m(5, 2),
                 block_table=m(2, 3, dtype=torch.int32), pos=m(2, dtype=torch.int32))
    return dict(
        lasad_packed_attention=dict(q=q, k=k, v=k, offsets=offsets, o=q, lse=lse),
        lasad_packed_attention_backward=dict(q=q, k=k, v=k, o=q, lse=lse, do=q, offsets=offsets, dq=q, dk=k, dv=k, workspace=m(64)),
        lasad_paged_append=dict(k=k, v=k, q=q, q_out=q, offsets=offsets, table=m(9, 32, 2), **cache),
        lasad_paged_attention=dict(q=m(2, 4, 64), o=m(2, 4, 64), lse=m(2, 4), workspace=m(64), **cache),
    )


CASES = [(c, n) for c, kw in arguments().items() for n, t in kw.items() if isinstance(t, Memory)]


@pytest.mark.parametrize("call,name", CASES)
@pytest.mark.parametrize("made_before", [False, True])
def test_a_tensor_of_another_device_is_refused(world, call, name, made_before):      # noqa: F811
    ctx, _ = world
    kw = arguments()[call]
    if made_before:
        getattr(ctx, call)(**kw)
    with pytest.raises(ValueError):
        getattr(ctx, call)(**{**kw, name: there(kw[name])})


@pytest.mark.parametrize("call,name", CASES)
def test_other_shapes_and_types_are_refused(world, call, name):      # noqa: F811
    ctx, _ = world
    kw = arguments()[call]
    t = kw[name]
    if name == "workspace":
        bad = [m(3)]
    else:
        more = lambda i: [n + (1 if i == j else 0) for j, n in enumerate(t.shape)]   # noqa: E731
        bad = [m(*more(i), dtype=t.dtype) for i in range(t.dim())] + [m(*t.shape, dtype=torch.float64), m(*t.shape, 1, dtype=t.dtype)]
    free = {"table": 0, "block_table": 1}      # another number of rows of the table, or of pages of a sequence, is a call
    if call != "lasad_paged_append":
        free["offsets"] = 0                    # and so is another number of sequences where nothing else counts them
    if name in free:
        del bad[free[name]]
    for other in bad:
        with pytest.raises((ValueError, TypeError)):
            getattr(ctx, call)(**{**kw, name: other})


@pytest.mark.parametrize("call", ["lasad_paged_append", "lasad_paged_attention"])
@pytest.mark.parametrize("name", ["k_pages", "v_pages", "v_scales"])
def test_a_cache_is_asked_for_whole(world, call, name):      # noqa: F811
    ctx, _ = world
    with pytest.raises(ValueError, match=name):
        getattr(ctx, call)(**{**arguments()[call], name: None})


@pytest.mark.parametrize("call,name", [(c, n) for c, n in CASES if n in ("offsets", "block_table", "pos", "k_scales")
                                       and (c, n) != ("lasad_paged_append", "offsets")] + [("lasad_packed_attention_backward", "lse")])
def test_what_is_needed_is_asked_for(world, call, name):      # noqa: F811
    ctx, _ = world
    with pytest.raises(ValueError):
        getattr(ctx, call)(**{**arguments()[call], name: None})


def test_one_row_for_each_sequence_without_offsets(world):      # noqa: F811
    ctx, _ = world
    kw = arguments()["lasad_paged_append"]
    with pytest.raises(ValueError):
        ctx.lasad_paged_append(**{**kw, "offsets": None})
    with pytest.raises(ValueError):
        ctx.lasad_paged_append(**{**kw, "q": None})


@pytest.mark.parametrize("call,outs", [("lasad_packed_attention", ("o", "lse")), ("lasad_packed_attention_backward", ("dq", "dk", "dv", "workspace")),
                                       ("lasad_paged_append", ("q_out",)), ("lasad_paged_attention", ("o", "lse", "workspace"))])
def test_what_a_call_allocates_is_its_streams(world, call, outs):      # noqa: F811
    ctx, made = world
    kw = {n: t for n, t in arguments()[call].items() if n not in outs}
    if "lse" in outs:
        kw["want_lse"] = True
    for stream, owner in ((None, CURRENT), (OTHER, OTHER)):
        made.clear()
        getattr(ctx, call)(stream=stream, **kw)
        assert len(made) == len(outs) and all(t.owner == owner for t in made)
