"""Marshalling of the operators that stand beside LASAD in a hybrid stack (``include/lasad.h``).

``Mixers`` is the part of ``binding.Lasad`` that holds them: the gated linear recurrence with the
spatial rule (``lasad_scan_*``), the norm and rotation of queries and keys (``lasad_qk_norm_rope*``)
and attention over a sliding window with visible first tokens (``lasad_window_*``).  Gradients are
explicit calls; outputs that are not passed in are allocated.  Every call is asynchronous on
``stream`` (a raw handle; the current one by default), and what a call allocates belongs to that
stream: a workspace is free again once the stream has passed the call, an output once the current stream
too has passed the point where it was dropped.
"""
from __future__ import annotations

import ctypes
import math

import torch

from .marshal import _check_cuda, _dtype_code, _empty, _ptr, _stream, _strides3, _strides_decode

LASAD_SCAN_TIED = 1
LASAD_SCAN_LOGITS = 2
LASAD_SCAN_CHUNK = 128
LASAD_ROPE_HALF = 1

_I32, _I64, _F32, _VP = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p


class ScanParams(ctypes.Structure):
    """Mirror of ``lasad_scan_params``."""
    _fields_ = ([(n, _I32) for n in ("B", "T", "C", "grid_w", "prefix_len", "dtype", "flags", "reserved")]
                + [("t0", _I64)]
                + [(n, _I64 * 2) for n in ("x_stride", "gate_stride", "y_stride", "dx_stride", "dgate_stride")])


class RopeParams(ctypes.Structure):
    """Mirror of ``lasad_rope_params``."""
    _fields_ = ([(n, _I32) for n in ("B", "T", "Hq", "Hk", "d", "dtype", "grid_w", "prefix_len", "table_rows", "flags")]
                + [("eps", _F32), ("reserved", _I32), ("t0", _I64)]
                + [(n, _I64 * 3) for n in ("q_stride", "k_stride", "q_out_stride", "k_out_stride",
                                           "dq_out_stride", "dk_out_stride", "dq_stride", "dk_stride")])


class WindowParams(ctypes.Structure):
    """Mirror of ``lasad_window_params``."""
    _fields_ = ([(n, _I32) for n in ("B", "T", "Hq", "Hk", "d", "dtype", "window", "sinks")]
                + [("scale", _F32), ("reserved", _I32)]
                + [(n, _I64 * 3) for n in ("q_stride", "k_stride", "v_stride", "o_stride", "do_stride", "dq_stride",
                                           "dk_stride", "dv_stride", "k_cache_stride", "v_cache_stride")])


_SP, _RP, _WP = (ctypes.POINTER(c) for c in (ScanParams, RopeParams, WindowParams))
PROTOTYPES = {
    "lasad_scan_workspace": (_I64, [_VP, _SP]),
    "lasad_scan_forward": (ctypes.c_int, [_VP, _SP] + [_VP] * 8),
    "lasad_scan_backward": (ctypes.c_int, [_VP, _SP] + [_VP] * 10),
    "lasad_scan_step": (ctypes.c_int, [_VP, _SP] + [_VP] * 7),
    "lasad_qk_norm_rope": (ctypes.c_int, [_VP, _RP] + [_VP] * 9),
    "lasad_qk_norm_rope_workspace": (_I64, [_VP, _RP]),
    "lasad_qk_norm_rope_backward": (ctypes.c_int, [_VP, _RP] + [_VP] * 14),
    "lasad_window_attention": (ctypes.c_int, [_VP, _WP] + [_VP] * 7),
    "lasad_window_attention_workspace": (_I64, [_VP, _WP]),
    "lasad_window_attention_backward": (ctypes.c_int, [_VP, _WP] + [_VP] * 12),
    "lasad_window_attention_step": (ctypes.c_int, [_VP, _WP] + [_VP] * 8),
    "lasad_window_cache_store": (ctypes.c_int, [_VP, _WP] + [_VP] * 6),
}


def rope_table(rows: int, d: int, grid: bool, base: float = 10000.0, device=None) -> torch.Tensor:
    """The (cos, sin) table of ``lasad_qk_norm_rope``, fp32 [rows, pairs, 2], from angles in 64 bits:
    row x base^(-m / pairs), with d/4 pairs for positions on a grid and d/2 for plain ones."""
    pairs = d // (4 if grid else 2)
    a = torch.arange(rows, dtype=torch.float64)[:, None] * base ** (-torch.arange(pairs, dtype=torch.float64) / pairs)
    return torch.stack((a.cos(), a.sin()), dim=-1).to(torch.float32).to(device)


# What a call looks like: the shape, strides, type and device of every tensor, or None.  A call that
# looks like one before it has been checked and has its params struct and workspace size already
# (checking and building them costs more than the rest of the call); scalars are set again each time.
# A context keeps its own (``_calls``): like the context, they serve one host thread at a time.
def _look(t):
    return None if t is None else (t.shape, t.stride(), t.dtype, t.get_device())


def _like(t, stream):
    """An output of t's shape, with contiguous channels."""
    return torch.empty_like(t) if stream is None and t.is_contiguous() else _empty(t.shape, t.dtype, t.device, stream)


class _Entry:
    __slots__ = ("p", "ref", "ws")

    def __init__(self, p):
        self.p, self.ref, self.ws = p, ctypes.byref(p), None


def _same(what, *ts):
    """The tensors that are there have one dtype."""
    for t in ts[1:]:
        if t is not None and t.dtype != ts[0].dtype:
            raise ValueError(f"{what} must share one dtype")


def _f32(name, t, shape):
    if t is not None and (t.dtype != torch.float32 or not t.is_contiguous() or tuple(t.shape) != shape):
        raise ValueError(f"{name} must be contiguous float32 {list(shape)}")


def _i32(name, t, n):
    if t is not None and (t.dtype != torch.int32 or not t.is_contiguous() or t.numel() != n):
        raise ValueError(f"{name} must be contiguous int32 [B]")


def _shape(name, t, shape):
    if t is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")


def _strides2(t):
    if t is None:
        return (_I64 * 2)()
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError("channels must be contiguous")
    return (_I64 * 2)(t.stride(0), t.stride(1) if t.dim() == 3 else 0)


class Mixers:
    """The calls beside LASAD; a base of ``binding.Lasad``, which has the library and the context."""

    def _here(self, *ts):
        """The tensors that are there are on the context's device."""
        _check_cuda(*ts)
        for t in ts:
            if t is not None and t.get_device() != self.device:
                raise ValueError(f"all tensors must be on cuda:{self.device}, the context's device, not on {t.device}")

    def _new(self, key, p):
        if len(self._calls) > 256:
            self._calls.clear()
        e = self._calls[key] = _Entry(p)
        return e

    def _workspace(self, e, query, like, given, stream):
        if e.ws is None:
            n = query(self._h, e.ref)
            if n < 0:
                self._raise(int(n), query.__name__)
            e.ws = int(n)
        if given is not None:
            if given.get_device() != self.device or not given.is_contiguous() or given.numel() * given.element_size() < e.ws:
                raise ValueError(f"workspace must be contiguous memory of cuda:{self.device} of at least {e.ws} bytes")
            return given
        if not e.ws:
            return None
        return _empty(e.ws, torch.uint8, like.device, stream, returned=False)

    # ---- gated linear recurrence ------------------------------------------------------------
    def _scan(self, key, kind, x, gate, y, dx, dgate, states, saved, pos):
        """Checks a call that looks like none before it.  states: (name, tensor) of [B,C]."""
        self._here(x, gate, y, dx, dgate, saved, pos, *(t for _, t in states))
        _same("x, gate and their outputs and gradients", x, gate, y, dx, dgate)
        if x.dim() != (2 if kind == "step" else 3):
            raise ValueError("expected [B,C]" if kind == "step" else "expected [B,T,C]")
        for name, t in (("gate", gate), ("y", y), ("dx", dx), ("dgate", dgate)):
            _shape(name, t, x.shape)
        B, T, C = (x.shape[0], 1, x.shape[1]) if kind == "step" else x.shape
        for name, t in states:
            _f32(name, t, (B, C))
        _f32("saved", saved, (B, -(-T // LASAD_SCAN_CHUNK), C))
        _i32("pos", pos, B)
        return self._new(key, ScanParams(B, T, C, 0, 0, _dtype_code(x), 0, 0, 0, *[_strides2(t) for t in (x, gate, y, dx, dgate)]))

    @staticmethod
    def _scan_set(p, grid_w, prefix_len, t0, tied, logits):
        p.grid_w, p.prefix_len, p.t0 = grid_w, prefix_len, t0
        p.flags = (LASAD_SCAN_TIED if tied else 0) | (LASAD_SCAN_LOGITS if logits else 0)

    def lasad_scan_forward(self, x, gate, grid_w=0, prefix_len=0, t0=0, tied=True, logits=False, h_in=None, y=None,
                           h_out=None, want_state=True, save=False, workspace=None, stream=None):
        """Gated linear recurrence with the spatial rule over [B,T,C]; returns (y, h_out, saved).
        ``gate`` holds lambda, or with ``logits`` its pre-activation; ``tied`` scales x by 1 - lambda.
        ``save`` keeps the states that ``lasad_scan_backward`` needs.  ``h_out`` may be ``h_in``: a sequence
        taken in pieces carries its state in place."""
        if y is None:
            y = _like(x, stream)
        key = ("scan", _look(x), _look(gate), _look(h_in), _look(y), _look(h_out))
        e = self._calls.get(key) or self._scan(key, "forward", x, gate, y, None, None, (("h_in", h_in), ("h_out", h_out)), None, None)
        p = e.p
        self._scan_set(p, grid_w, prefix_len, t0, tied, logits)
        if h_out is None and want_state:
            h_out = _empty((p.B, p.C), torch.float32, x.device, stream)
        saved = _empty((p.B, -(-p.T // LASAD_SCAN_CHUNK), p.C), torch.float32, x.device, stream) if save else None
        ws = self._workspace(e, self._lib.lasad_scan_workspace, x, workspace, stream)
        rc = self._lib.lasad_scan_forward(self._h, e.ref, x.data_ptr(), gate.data_ptr(), _ptr(h_in), y.data_ptr(), _ptr(h_out),
                                          _ptr(saved), _ptr(ws), _stream(x.device, stream))
        if rc:
            self._raise(rc, "lasad_scan_forward")
        return y, h_out, saved

    def lasad_scan_backward(self, x, gate, saved, dy, dh_out=None, grid_w=0, prefix_len=0, t0=0, tied=True, logits=False,
                            dx=None, dgate=None, dh_in=None, want_state=True, workspace=None, stream=None):
        """The gradient of ``lasad_scan_forward``; returns (dx, dgate, dh_in).  ``dh_in`` may be ``dh_out``."""
        if dx is None:
            dx = _like(x, stream)
        if dgate is None:
            dgate = _like(x, stream)
        key = ("scan'", _look(x), _look(gate), _look(saved), _look(dy), _look(dh_out), _look(dx), _look(dgate),
               _look(dh_in))
        e = self._calls.get(key)
        if e is None:
            if saved is None:
                raise ValueError("saved is what lasad_scan_forward returns with save=True")
            e = self._scan(key, "backward", x, gate, dy, dx, dgate, (("dh_out", dh_out), ("dh_in", dh_in)), saved, None)
        p = e.p
        self._scan_set(p, grid_w, prefix_len, t0, tied, logits)
        if dh_in is None and want_state:
            dh_in = _empty((p.B, p.C), torch.float32, x.device, stream)
        ws = self._workspace(e, self._lib.lasad_scan_workspace, x, workspace, stream)
        rc = self._lib.lasad_scan_backward(self._h, e.ref, x.data_ptr(), gate.data_ptr(), saved.data_ptr(), dy.data_ptr(),
                                           _ptr(dh_out), dx.data_ptr(), dgate.data_ptr(), _ptr(dh_in), _ptr(ws),
                                           _stream(x.device, stream))
        if rc:
            self._raise(rc, "lasad_scan_backward")
        return dx, dgate, dh_in

    def lasad_scan_step(self, x, gate, h_in, grid_w=0, prefix_len=0, t=0, pos=None, tied=True, logits=False, y=None,
                        h_out=None, stream=None):
        """One token of the recurrence, x and gate [B,C]; ``t`` or ``pos`` (int32 [B]) gives its
        position.  The state is updated in place unless ``h_out`` is given.  Returns (y, h_out)."""
        if y is None:
            y = _like(x, stream)
        if h_out is None:
            h_out = h_in
        key = ("scan1", _look(x), _look(gate), _look(h_in), _look(y), _look(h_out), _look(pos))
        e = self._calls.get(key) or self._scan(key, "step", x, gate, y, None, None, (("h_in", h_in), ("h_out", h_out)), None, pos)
        self._scan_set(e.p, grid_w, prefix_len, t, tied, logits)
        rc = self._lib.lasad_scan_step(self._h, e.ref, x.data_ptr(), gate.data_ptr(), h_in.data_ptr(), y.data_ptr(),
                                       h_out.data_ptr(), _ptr(pos), _stream(x.device, stream))
        if rc:
            self._raise(rc, "lasad_scan_step")
        return y, h_out

    # ---- norm and rotation of queries and keys ----------------------------------------------
    def _rope(self, key, q, k, table, q_weight, k_weight, pos, grid, outs):
        """Checks a call that looks like none before it.  outs: the (up to six) tensors after q and k
        in the order of the params' strides, or None."""
        self._here(q, k, table, q_weight, k_weight, pos, *outs)
        _same("q, k and their outputs and gradients", q, k, *outs)
        if q.dim() != 4 or k.dim() != 4:
            raise ValueError("expected [B,T,H,d]")
        B, T, Hq, d = q.shape
        _shape("k", k, (B, T, k.shape[2], d))
        for n, t in enumerate(outs):
            _shape("an output or gradient of " + ("k" if n % 2 else "q"), t, k.shape if n % 2 else q.shape)
        _f32("table", table, (table.shape[0], d // (4 if grid else 2), 2))
        _f32("q_weight", q_weight, (d,))
        _f32("k_weight", k_weight, (d,))
        _i32("pos", pos, B)
        return self._new(key, RopeParams(B, T, Hq, k.shape[2], d, _dtype_code(q), 0, 0, table.shape[0], 0, 0.0, 0, 0, _strides3(q),
                                    _strides3(k), *[(_I64 * 3)() if t is None else _strides3(t) for t in outs]))

    @staticmethod
    def _rope_set(p, grid_w, prefix_len, t0, half, eps):
        p.grid_w, p.prefix_len, p.t0, p.eps, p.flags = grid_w, prefix_len, t0, eps, LASAD_ROPE_HALF if half else 0

    def lasad_qk_norm_rope(self, q, k, table, q_weight=None, k_weight=None, grid_w=0, prefix_len=0, t0=0, pos=None,
                           eps=1e-6, half=False, q_out=None, k_out=None, stream=None):
        """RMS norm of every head of q [B,T,Hq,d] and k [B,T,Hk,d] and their rotation by position
        (``table`` from ``rope_table``), in one pass; returns (q_out, k_out)."""
        if q_out is None:
            q_out = _like(q, stream)
        if k_out is None:
            k_out = _like(k, stream)
        key = ("rope", grid_w > 0, _look(q), _look(k), _look(table), _look(q_weight), _look(k_weight), _look(pos),
               _look(q_out), _look(k_out))
        e = self._calls.get(key) or self._rope(key, q, k, table, q_weight, k_weight, pos, grid_w > 0,
                                          (q_out, k_out, None, None, None, None))
        self._rope_set(e.p, grid_w, prefix_len, t0, half, eps)
        rc = self._lib.lasad_qk_norm_rope(self._h, e.ref, q.data_ptr(), k.data_ptr(), table.data_ptr(), _ptr(q_weight),
                                          _ptr(k_weight), _ptr(pos), q_out.data_ptr(), k_out.data_ptr(), _stream(q.device, stream))
        if rc:
            self._raise(rc, "lasad_qk_norm_rope")
        return q_out, k_out

    def lasad_qk_norm_rope_backward(self, q, k, table, dq_out, dk_out, q_weight=None, k_weight=None, grid_w=0,
                                    prefix_len=0, t0=0, pos=None, eps=1e-6, half=False, dq=None, dk=None,
                                    want_weights=True, workspace=None, stream=None):
        """The gradient of ``lasad_qk_norm_rope`` from its inputs; returns (dq, dk, dq_weight,
        dk_weight), the last two fp32 [d] (None without ``want_weights``)."""
        if dq is None:
            dq = _like(q, stream)
        if dk is None:
            dk = _like(k, stream)
        key = ("rope'", grid_w > 0, _look(q), _look(k), _look(table), _look(q_weight), _look(k_weight), _look(pos),
               _look(dq_out), _look(dk_out), _look(dq), _look(dk))
        e = self._calls.get(key) or self._rope(key, q, k, table, q_weight, k_weight, pos, grid_w > 0,
                                          (None, None, dq_out, dk_out, dq, dk))
        self._rope_set(e.p, grid_w, prefix_len, t0, half, eps)
        dwq = dwk = ws = None
        if want_weights:
            dwq, dwk = _empty(e.p.d, torch.float32, q.device, stream), _empty(e.p.d, torch.float32, q.device, stream)
            ws = self._workspace(e, self._lib.lasad_qk_norm_rope_workspace, q, workspace, stream)
        rc = self._lib.lasad_qk_norm_rope_backward(self._h, e.ref, q.data_ptr(), k.data_ptr(), table.data_ptr(), _ptr(q_weight),
                                                   _ptr(k_weight), _ptr(pos), dq_out.data_ptr(), dk_out.data_ptr(),
                                                   dq.data_ptr(), dk.data_ptr(), _ptr(dwq), _ptr(dwk), _ptr(ws),
                                                   _stream(q.device, stream))
        if rc:
            self._raise(rc, "lasad_qk_norm_rope_backward")
        return dq, dk, dwq, dwk

    # ---- attention over a sliding window ----------------------------------------------------
    _ORDER = ("q", "k", "v", "o", "do", "dq", "dk", "dv", "k_cache", "v_cache")

    def _window(self, key, kind, window, sinks, lse, ints, **ts):
        """Checks a call that looks like none before it.  ints: (name, tensor) of int32 [B]; the other
        tensors by name: those of a step have no token dimension, caches always have slots."""
        self._here(lse, ints[1], *ts.values())
        first = ts["q"] if "q" in ts else ts["k"]
        _same("all tensors", first, *ts.values())
        k = ts["k"]
        dims = 3 if kind == "step" else 4
        for n, t in ts.items():
            if t.dim() != (4 if n.endswith("cache") else dims):
                raise ValueError(f"{n} must have {4 if n.endswith('cache') else dims} dimensions")
        B, d, Hk = k.shape[0], k.shape[-1], k.shape[-2]
        Hq = ts["q"].shape[-2] if "q" in ts else Hk
        T = 1 if kind == "step" else k.shape[1]
        rows = (B,) if kind == "step" else (B, T)
        for n, t in ts.items():
            _shape(n, t, (B, sinks + window, Hk, d) if n.endswith("cache")
                   else (*rows, Hq if n in ("q", "o", "do", "dq") else Hk, d))
        _i32(ints[0], ints[1], B)
        _f32("lse", lse, (B, Hq, T))
        st = [(_I64 * 3)() if n not in ts else (_strides3 if ts[n].dim() == 4 else _strides_decode)(ts[n]) for n in self._ORDER]
        # (a struct's int32 would take a longer window's lowest bits; no sequence is longer than the longest of them)
        return self._new(key, WindowParams(B, T, Hq, Hk, d, _dtype_code(first), min(window, 2 ** 31 - 1), sinks, 0.0, 0, *st))

    def lasad_window_attention(self, q, k, v, window, sinks=0, scale=None, lengths=None, o=None, lse=None,
                               want_lse=False, stream=None):
        """Causal softmax attention of q [B,T,Hq,d] over the last ``window`` tokens and the first
        ``sinks`` ones of k, v [B,T,Hk,d]; ``lengths`` int32 [B] ends the sequences early, ``scale`` is
        1/sqrt(d) by default.  Returns (o, lse); lse, fp32 [B,Hq,T], only with ``want_lse`` (the
        gradient needs it)."""
        if o is None:
            o = _like(q, stream)
        key = ("window", window, sinks, _look(q), _look(k), _look(v), _look(lengths), _look(o), _look(lse))
        e = self._calls.get(key) or self._window(key, "forward", window, sinks, lse, ("lengths", lengths), q=q, k=k, v=v, o=o)
        p = e.p
        p.scale = 1.0 / math.sqrt(p.d) if scale is None else scale
        if lse is None and want_lse:
            lse = _empty((p.B, p.Hq, p.T), torch.float32, q.device, stream)
        rc = self._lib.lasad_window_attention(self._h, e.ref, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(lengths),
                                              o.data_ptr(), _ptr(lse), _stream(q.device, stream))
        if rc:
            self._raise(rc, "lasad_window_attention")
        return o, lse

    def lasad_window_attention_backward(self, q, k, v, o, lse, do, window, sinks=0, scale=None, lengths=None, dq=None,
                                        dk=None, dv=None, workspace=None, stream=None):
        """The gradient of ``lasad_window_attention`` from its inputs and outputs; returns (dq, dk, dv)."""
        dq = _like(q, stream) if dq is None else dq
        dk = _like(k, stream) if dk is None else dk
        dv = _like(v, stream) if dv is None else dv
        key = ("window'", window, sinks, _look(q), _look(k), _look(v), _look(o), _look(lse), _look(do),
               _look(lengths), _look(dq), _look(dk), _look(dv))
        e = self._calls.get(key)
        if e is None:
            if lse is None:
                raise ValueError("lse is what lasad_window_attention returns with want_lse=True")
            e = self._window(key, "backward", window, sinks, lse, ("lengths", lengths), q=q, k=k, v=v, o=o, do=do, dq=dq, dk=dk,
                             dv=dv)
        p = e.p
        p.scale = 1.0 / math.sqrt(p.d) if scale is None else scale
        ws = self._workspace(e, self._lib.lasad_window_attention_workspace, q, workspace, stream)
        rc = self._lib.lasad_window_attention_backward(self._h, e.ref, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                                       lse.data_ptr(), do.data_ptr(), _ptr(lengths), dq.data_ptr(),
                                                       dk.data_ptr(), dv.data_ptr(), _ptr(ws), _stream(q.device, stream))
        if rc:
            self._raise(rc, "lasad_window_attention_backward")
        return dq, dk, dv

    def lasad_window_attention_step(self, q, k, v, k_cache, v_cache, pos, window, sinks=0, scale=None, o=None,
                                    stream=None):
        """One new token per sequence, q [B,Hq,d], k, v [B,Hk,d], against ring caches [B, sinks +
        window, Hk, d], which get the token's k and v.  ``pos`` int32 [B]: the tokens' positions
        (negative: the sequence takes no part).  Returns o [B,Hq,d]."""
        if o is None:
            o = _like(q, stream)
        key = ("window1", window, sinks, _look(q), _look(k), _look(v), _look(k_cache), _look(v_cache), _look(pos),
               _look(o))
        e = self._calls.get(key)
        if e is None:
            if pos is None:
                raise ValueError("pos must be contiguous int32 [B]")
            e = self._window(key, "step", window, sinks, None, ("pos", pos), q=q, k=k, v=v, o=o, k_cache=k_cache,
                             v_cache=v_cache)
        p = e.p
        p.scale = 1.0 / math.sqrt(p.d) if scale is None else scale
        rc = self._lib.lasad_window_attention_step(self._h, e.ref, q.data_ptr(), k.data_ptr(), v.data_ptr(), k_cache.data_ptr(),
                                                   v_cache.data_ptr(), pos.data_ptr(), o.data_ptr(), _stream(q.device, stream))
        if rc:
            self._raise(rc, "lasad_window_attention_step")
        return o

    def lasad_window_cache_store(self, k, v, k_cache, v_cache, window, sinks=0, lengths=None, stream=None):
        """Puts the keys and values of a prefill, [B,T,Hk,d], into the ring caches of the step."""
        key = ("store", window, sinks, _look(k), _look(v), _look(k_cache), _look(v_cache), _look(lengths))
        e = self._calls.get(key) or self._window(key, "store", window, sinks, None, ("lengths", lengths), k=k, v=v, k_cache=k_cache,
                                            v_cache=v_cache)
        rc = self._lib.lasad_window_cache_store(self._h, e.ref, k.data_ptr(), v.data_ptr(), _ptr(lengths), k_cache.data_ptr(),
                                                v_cache.data_ptr(), _stream(k.device, stream))
        if rc:
            self._raise(rc, "lasad_window_cache_store")
