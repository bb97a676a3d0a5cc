"""Which stream owns what a call allocates, without a GPU: every call of ``Lasad`` that takes ``stream`` runs
against a library that does nothing and an allocator that writes down the stream it was asked on."""
import contextlib
import types

import pytest
import torch

from paper_2507_01652_b200 import binding

CURRENT, OTHER = 11, 22


class Memory:
    """A CPU tensor that passes for one of cuda:0."""
    device = torch.device("cuda", 0)
    is_cuda = True

    def __init__(self, t, owner=None):
        self.t, self.owner, self.readers = t, owner, []

    def __getattr__(self, name):
        return getattr(self.t, name)

    def __getitem__(self, at):
        return Memory(self.t[at], self.owner)

    def get_device(self):
        return 0

    def record_stream(self, s):
        self.readers.append(s.cuda_stream)


class Library:
    """Every entry point succeeds; workspace queries ask for 64 bytes."""

    def __getattr__(self, name):
        fn = lambda *a: 64 if name.endswith("_workspace") else 0      # noqa: E731
        fn.__name__ = name
        return fn


@pytest.fixture
def world(monkeypatch):
    now, made = [CURRENT], []

    def empty(*shape, dtype=None, device=None):
        shape = shape[0] if len(shape) == 1 else shape
        made.append(Memory(torch.zeros(shape, dtype=dtype), now[0]))
        return made[-1]

    @contextlib.contextmanager
    def stream(s):
        before, now[0] = now[0], s.cuda_stream
        yield
        now[0] = before

    handle = lambda h, device=None: types.SimpleNamespace(cuda_stream=h)      # noqa: E731
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch, "empty_like", lambda t: empty(t.shape, dtype=t.dtype))
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", handle)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: handle(now[0]))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(binding._mixers, "_stream", lambda device, s: CURRENT if s is None else s)
    monkeypatch.setattr(binding, "_stream", lambda device, s: CURRENT if s is None else s)
    ctx = binding.Lasad.__new__(binding.Lasad)
    ctx._lib, ctx._h, ctx.device, ctx._calls = Library(), None, 0, {}
    return ctx, made


def m(*shape, dtype=torch.float32):
    return Memory(torch.zeros(shape, dtype=dtype), CURRENT)


def calls(ctx):
    x, st = m(2, 5, 8), m(2, 8)
    q, k = m(2, 5, 4, 64), m(2, 5, 2, 64)
    q1, k1, cache = m(2, 4, 64), m(2, 2, 64), [m(2, 5, 2, 64) for _ in range(2)]
    pos, lse, table, w = m(2, dtype=torch.int32), m(2, 4, 5), m(9, 16, 2), m(64)
    decay, state = m(4), m(2, 4, 64, 64)
    return dict(
        scan_forward=lambda **s: ctx.lasad_scan_forward(x, x, save=True, **s),
        scan_backward=lambda **s: ctx.lasad_scan_backward(x, x, m(2, 1, 8), x, **s),
        scan_step=lambda **s: ctx.lasad_scan_step(x[:, 0], x[:, 0], st, **s),
        rope=lambda **s: ctx.lasad_qk_norm_rope(q, k, table, grid_w=3, **s),
        rope_backward=lambda **s: ctx.lasad_qk_norm_rope_backward(q, k, table, q, k, w, w, grid_w=3, **s),
        window=lambda **s: ctx.lasad_window_attention(q, k, k, 4, want_lse=True, **s),
        window_backward=lambda **s: ctx.lasad_window_attention_backward(q, k, k, q, lse, q, 4, **s),
        window_step=lambda **s: ctx.lasad_window_attention_step(q1, k1, k1, *cache, pos, 4, 1, **s),
        forward=lambda **s: ctx.lasad_forward(q, q, q, decay, 3, **s),
        forward_gated=lambda **s: ctx.lasad_forward_gated(q, q, q, q, 3, **s),
        forward_fused=lambda **s: ctx.lasad_forward_fused(q, q, q, q, 3, **s),
        decode=lambda **s: ctx.lasad_decode_step(q1, q1, q1, decay, state, 3, 0, 1, **s),
        decode_gated=lambda **s: ctx.lasad_decode_step_gated(q1, q1, q1, q1, state, 3, 0, 1, **s),
        decode_pos=lambda **s: ctx.lasad_decode_step_pos(q1, q1, q1, decay, state, pos, **s),
        decode_fused=lambda **s: ctx.lasad_decode_step_fused(q1, q1, q1, q1, state, 3, 0, 1, **s),
    )


@pytest.mark.parametrize("name", sorted(calls(None)))
def test_memory_belongs_to_the_stream_that_writes_it(world, name):
    """A block of the current stream's pool may still be written by what that stream has to do when a call on
    another stream starts; an output is read on the current stream and must outlive that."""
    ctx, made = world
    out = calls(ctx)[name](stream=OTHER)
    assert made and all(t.owner == OTHER for t in made)
    returned = [t for t in (out if isinstance(out, tuple) else (out,)) if any(t is one for one in made)]
    assert returned and all(t.readers == [CURRENT] for t in returned)
    # (a workspace is nobody's but the call's)
    assert all(t.readers == [] for t in made if not any(t is one for one in returned))


@pytest.mark.parametrize("name", sorted(calls(None)))
def test_memory_of_the_current_stream_without_one(world, name):
    ctx, made = world
    calls(ctx)[name]()
    assert made and all(t.owner == CURRENT and t.readers == [] for t in made)
