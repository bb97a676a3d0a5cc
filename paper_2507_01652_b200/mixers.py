"""Marshalling of the operators that stand beside LASAD in a hybrid stack (``include/lasad.h``).

``Mixers`` is the part of ``binding.Lasad`` that holds them: the gated linear recurrence with the
spatial rule (``lasad_scan_*``), the norm and rotation of queries and keys (``lasad_qk_norm_rope*``)
and attention over a sliding window with visible first tokens (``lasad_window_*``).  Gradients are
explicit calls; outputs that are not passed in are allocated.  Every call is asynchronous on
``stream`` (a raw handle; the current one by default).  Workspaces come from torch's allocator and
are its again once the stream has passed the call.
"""
from __future__ import annotations

import ctypes
import math

import torch

from .marshal import _check_cuda, _dtype_code, _ptr, _stream, _strides3, _strides_decode

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
    "lasad_window_attention_step_workspace": (_I64, [_VP, _WP]),
    "lasad_window_attention_step": (ctypes.c_int, [_VP, _WP] + [_VP] * 9),
    "lasad_window_cache_store": (ctypes.c_int, [_VP, _WP] + [_VP] * 6),
}


def rope_table(rows: int, d: int, grid: bool, base: float = 10000.0, device=None) -> torch.Tensor:
    """The (cos, sin) table of ``lasad_qk_norm_rope``, fp32 [rows, pairs, 2], from angles in 64 bits:
    row x base^(-m / pairs), with d/4 pairs for positions on a grid and d/2 for plain ones."""
    pairs = d // (4 if grid else 2)
    a = torch.arange(rows, dtype=torch.float64)[:, None] * base ** (-torch.arange(pairs, dtype=torch.float64) / pairs)
    return torch.stack((a.cos(), a.sin()), dim=-1).to(torch.float32).to(device)


# Params structs (and workspace sizes) by what they depend on; building their arrays costs more than
# the rest of a call.  Scalars that may change from call to call are set again each time.
_cache = {}


def _cached(key, make):
    e = _cache.get(key)
    if e is None:
        if len(_cache) > 256:
            _cache.clear()
        e = _cache[key] = make()
    return e


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
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError("channels must be contiguous")
    return (_I64 * 2)(t.stride(0), t.stride(1) if t.dim() == 3 else 0)


class Mixers:
    """The calls beside LASAD; a base of ``binding.Lasad``, which has the library and the context."""

    def _workspace(self, e, query, device, given, stream):
        if e.ws is None:
            n = query(self._h, e.ref)
            if n < 0:
                self._raise(int(n), query.__name__)
            e.ws = int(n)
        if given is not None:
            if given.numel() * given.element_size() < e.ws:
                raise ValueError(f"workspace must have at least {e.ws} bytes")
            return given
        if not e.ws:
            return None
        ws = torch.empty(e.ws, dtype=torch.uint8, device=device)
        if stream is not None:       # not handed out again before that stream has passed the call
            ws.record_stream(torch.cuda.ExternalStream(stream, device=device))
        return ws

    # ---- gated linear recurrence ------------------------------------------------------------
    def _scan(self, kind, x, gate, y, dx, dgate, grid_w, prefix_len, t0, tied, logits):
        key = (kind, self.device, x.dtype, x.shape, x.stride(), gate.stride(), y.stride(),
               None if dx is None else dx.stride(), None if dgate is None else dgate.stride())

        def make():
            if x.dim() != (2 if kind == "step" else 3):
                raise ValueError("expected [B,C]" if kind == "step" else "expected [B,T,C]")
            B, T, C = (x.shape[0], 1, x.shape[1]) if kind == "step" else x.shape
            none = (_I64 * 2)()
            return _Entry(ScanParams(B, T, C, 0, 0, _dtype_code(x), 0, 0, 0, _strides2(x), _strides2(gate), _strides2(y),
                                     none if dx is None else _strides2(dx), none if dgate is None else _strides2(dgate)))

        e = _cached(key, make)
        e.p.grid_w, e.p.prefix_len, e.p.t0 = grid_w, prefix_len, t0
        e.p.flags = (LASAD_SCAN_TIED if tied else 0) | (LASAD_SCAN_LOGITS if logits else 0)
        return e

    def lasad_scan_forward(self, x, gate, grid_w=0, prefix_len=0, t0=0, tied=True, logits=False, h_in=None, y=None,
                           h_out=None, want_state=True, save=False, workspace=None, stream=None):
        """Gated linear recurrence with the spatial rule over [B,T,C]; returns (y, h_out, saved).
        ``gate`` holds lambda, or with ``logits`` its pre-activation; ``tied`` scales x by 1 - lambda.
        ``save`` keeps the states that ``lasad_scan_backward`` needs."""
        _check_cuda(x, gate, h_in, y, h_out)
        _same("x, gate, y", x, gate, y)
        _shape("gate", gate, x.shape)
        _shape("y", y, x.shape)
        if x.dim() != 3:
            raise ValueError("expected [B,T,C]")
        B, T, C = x.shape
        _f32("h_in", h_in, (B, C))
        _f32("h_out", h_out, (B, C))
        if y is None:
            y = torch.empty((B, T, C), dtype=x.dtype, device=x.device)
        if h_out is None and want_state:
            h_out = torch.empty((B, C), dtype=torch.float32, device=x.device)
        saved = None
        if save:
            saved = torch.empty((B, -(-T // LASAD_SCAN_CHUNK), C), dtype=torch.float32, device=x.device)
        e = self._scan("prefill", x, gate, y, None, None, grid_w, prefix_len, t0, tied, logits)
        ws = self._workspace(e, self._lib.lasad_scan_workspace, x.device, workspace, stream)
        rc = self._lib.lasad_scan_forward(self._h, e.ref, _ptr(x), _ptr(gate), _ptr(h_in), _ptr(y), _ptr(h_out), _ptr(saved),
                                          _ptr(ws), _stream(x.device, stream))
        if rc:
            self._raise(rc, "lasad_scan_forward")
        return y, h_out, saved

    def lasad_scan_backward(self, x, gate, saved, dy, dh_out=None, grid_w=0, prefix_len=0, t0=0, tied=True, logits=False,
                            dx=None, dgate=None, dh_in=None, want_state=True, workspace=None, stream=None):
        """The gradient of ``lasad_scan_forward``; returns (dx, dgate, dh_in)."""
        _check_cuda(x, gate, saved, dy, dh_out, dx, dgate, dh_in)
        _same("x, gate, dy, dx, dgate", x, gate, dy, dx, dgate)
        for name, t in (("gate", gate), ("dy", dy), ("dx", dx), ("dgate", dgate)):
            _shape(name, t, x.shape)
        if x.dim() != 3:
            raise ValueError("expected [B,T,C]")
        B, T, C = x.shape
        _f32("saved", saved, (B, -(-T // LASAD_SCAN_CHUNK), C))
        _f32("dh_out", dh_out, (B, C))
        _f32("dh_in", dh_in, (B, C))
        if dx is None:
            dx = torch.empty((B, T, C), dtype=x.dtype, device=x.device)
        if dgate is None:
            dgate = torch.empty((B, T, C), dtype=x.dtype, device=x.device)
        if dh_in is None and want_state:
            dh_in = torch.empty((B, C), dtype=torch.float32, device=x.device)
        e = self._scan("backward", x, gate, dy, dx, dgate, grid_w, prefix_len, t0, tied, logits)
        ws = self._workspace(e, self._lib.lasad_scan_workspace, x.device, workspace, stream)
        rc = self._lib.lasad_scan_backward(self._h, e.ref, _ptr(x), _ptr(gate), _ptr(saved), _ptr(dy), _ptr(dh_out), _ptr(dx),
                                           _ptr(dgate), _ptr(dh_in), _ptr(ws), _stream(x.device, stream))
        if rc:
            self._raise(rc, "lasad_scan_backward")
        return dx, dgate, dh_in

    def lasad_scan_step(self, x, gate, h_in, grid_w=0, prefix_len=0, t=0, pos=None, tied=True, logits=False, y=None,
                        h_out=None, stream=None):
        """One token of the recurrence, x and gate [B,C]; ``t`` or ``pos`` (int32 [B]) gives its
        position.  The state is updated in place unless ``h_out`` is given.  Returns (y, h_out)."""
        _check_cuda(x, gate, h_in, y, h_out, pos)
        _same("x, gate, y", x, gate, y)
        _shape("gate", gate, x.shape)
        _shape("y", y, x.shape)
        if x.dim() != 2:
            raise ValueError("expected [B,C]")
        B, C = x.shape
        _f32("h_in", h_in, (B, C))
        _f32("h_out", h_out, (B, C))
        _i32("pos", pos, B)
        if y is None:
            y = torch.empty((B, C), dtype=x.dtype, device=x.device)
        if h_out is None:
            h_out = h_in
        e = self._scan("step", x, gate, y, None, None, grid_w, prefix_len, t, tied, logits)
        rc = self._lib.lasad_scan_step(self._h, e.ref, _ptr(x), _ptr(gate), _ptr(h_in), _ptr(y), _ptr(h_out), _ptr(pos),
                                       _stream(x.device, stream))
        if rc:
            self._raise(rc, "lasad_scan_step")
        return y, h_out

    # ---- norm and rotation of queries and keys ----------------------------------------------
    def _rope(self, q, k, table, outs, grid_w, prefix_len, t0, half, eps):
        """outs: the (up to six) tensors after q and k in the order of the params' strides, or None."""
        key = ("rope", self.device, q.dtype, q.shape, k.shape, q.stride(), k.stride(), table.shape,
               tuple(None if t is None else t.stride() for t in outs))

        def make():
            if q.dim() != 4 or k.dim() != 4:
                raise ValueError("expected [B,T,H,d]")
            B, T, Hq, d = q.shape
            return _Entry(RopeParams(B, T, Hq, k.shape[2], d, _dtype_code(q), 0, 0, table.shape[0], 0, 0.0, 0, 0,
                                     _strides3(q), _strides3(k),
                                     *[(_I64 * 3)() if t is None else _strides3(t) for t in outs]))

        e = _cached(key, make)
        p = e.p
        p.grid_w, p.prefix_len, p.t0, p.eps, p.flags = grid_w, prefix_len, t0, eps, LASAD_ROPE_HALF if half else 0
        return e

    @staticmethod
    def _rope_check(q, k, table, q_weight, k_weight, pos, grid_w, like_q, like_k):
        _check_cuda(q, k, table, q_weight, k_weight, pos, *like_q, *like_k)
        _same("q, k and their outputs", q, k, *like_q, *like_k)
        if q.dim() != 4:
            raise ValueError("expected [B,T,H,d]")
        B, T, _, d = q.shape
        _shape("k", k, (B, T, k.shape[2] if k.dim() == 4 else 0, d))
        for t in like_q:
            _shape("an output or gradient of q", t, q.shape)
        for t in like_k:
            _shape("an output or gradient of k", t, k.shape)
        _f32("table", table, (table.shape[0], d // (4 if grid_w else 2), 2))
        _f32("q_weight", q_weight, (d,))
        _f32("k_weight", k_weight, (d,))
        _i32("pos", pos, B)

    def lasad_qk_norm_rope(self, q, k, table, q_weight=None, k_weight=None, grid_w=0, prefix_len=0, t0=0, pos=None,
                           eps=1e-6, half=False, q_out=None, k_out=None, stream=None):
        """RMS norm of every head of q [B,T,Hq,d] and k [B,T,Hk,d] and their rotation by position
        (``table`` from ``rope_table``), in one pass; returns (q_out, k_out)."""
        self._rope_check(q, k, table, q_weight, k_weight, pos, grid_w, (q_out,), (k_out,))
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if k_out is None:
            k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
        e = self._rope(q, k, table, (q_out, k_out, None, None, None, None), grid_w, prefix_len, t0, half, eps)
        rc = self._lib.lasad_qk_norm_rope(self._h, e.ref, _ptr(q), _ptr(k), _ptr(table), _ptr(q_weight), _ptr(k_weight),
                                          _ptr(pos), _ptr(q_out), _ptr(k_out), _stream(q.device, stream))
        if rc:
            self._raise(rc, "lasad_qk_norm_rope")
        return q_out, k_out

    def lasad_qk_norm_rope_backward(self, q, k, table, dq_out, dk_out, q_weight=None, k_weight=None, grid_w=0,
                                    prefix_len=0, t0=0, pos=None, eps=1e-6, half=False, dq=None, dk=None,
                                    want_weights=True, workspace=None, stream=None):
        """The gradient of ``lasad_qk_norm_rope`` from its inputs; returns (dq, dk, dq_weight,
        dk_weight), the last two fp32 [d] (None without ``want_weights``)."""
        self._rope_check(q, k, table, q_weight, k_weight, pos, grid_w, (dq_out, dq), (dk_out, dk))
        if dq is None:
            dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if dk is None:
            dk = torch.empty(k.shape, dtype=k.dtype, device=k.device)
        dw = torch.empty((2, q.shape[3]), dtype=torch.float32, device=q.device) if want_weights else (None, None)
        dwq, dwk = dw[0], dw[1]
        e = self._rope(q, k, table, (None, None, dq_out, dk_out, dq, dk), grid_w, prefix_len, t0, half, eps)
        ws = self._workspace(e, self._lib.lasad_qk_norm_rope_workspace, q.device, workspace, stream) if want_weights else None
        rc = self._lib.lasad_qk_norm_rope_backward(self._h, e.ref, _ptr(q), _ptr(k), _ptr(table), _ptr(q_weight),
                                                   _ptr(k_weight), _ptr(pos), _ptr(dq_out), _ptr(dk_out), _ptr(dq), _ptr(dk),
                                                   _ptr(dwq), _ptr(dwk), _ptr(ws), _stream(q.device, stream))
        if rc:
            self._raise(rc, "lasad_qk_norm_rope_backward")
        return dq, dk, dwq, dwk

    # ---- attention over a sliding window ----------------------------------------------------
    _ORDER = ("q", "k", "v", "o", "do", "dq", "dk", "dv", "k_cache", "v_cache")

    def _window(self, kind, window, sinks, scale, **ts):
        """The params for the named tensors; those of a step have no token dimension, caches always have slots."""
        key = (kind, self.device, window, sinks) + tuple((n, t.dtype, t.shape, t.stride()) for n, t in ts.items())

        def make():
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
                want = ((B, sinks + window, Hk, d) if n.endswith("cache")
                        else (*rows, Hq if n in ("q", "o", "do", "dq") else Hk, d))
                _shape(n, t, want)
            st = [(_I64 * 3)() if n not in ts else (_strides3 if ts[n].dim() == 4 else _strides_decode)(ts[n])
                  for n in self._ORDER]
            return _Entry(WindowParams(B, T, Hq, Hk, d, _dtype_code(first), window, sinks, 0.0, 0, *st))

        e = _cached(key, make)
        e.p.scale = 1.0 / math.sqrt(e.p.d) if scale is None else scale
        return e

    def lasad_window_attention(self, q, k, v, window, sinks=0, scale=None, lengths=None, o=None, lse=None,
                               want_lse=False, stream=None):
        """Causal softmax attention of q [B,T,Hq,d] over the last ``window`` tokens and the first
        ``sinks`` ones of k, v [B,T,Hk,d]; ``lengths`` int32 [B] ends the sequences early, ``scale`` is
        1/sqrt(d) by default.  Returns (o, lse); lse, fp32 [B,Hq,T], only with ``want_lse`` (the
        gradient needs it)."""
        _check_cuda(q, k, v, lengths, o, lse)
        if o is None:
            o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        e = self._window("forward", window, sinks, scale, q=q, k=k, v=v, o=o)
        p = e.p
        _i32("lengths", lengths, p.B)
        _f32("lse", lse, (p.B, p.Hq, p.T))
        if lse is None and want_lse:
            lse = torch.empty((p.B, p.Hq, p.T), dtype=torch.float32, device=q.device)
        rc = self._lib.lasad_window_attention(self._h, e.ref, _ptr(q), _ptr(k), _ptr(v), _ptr(lengths), _ptr(o), _ptr(lse),
                                              _stream(q.device, stream))
        if rc:
            self._raise(rc, "lasad_window_attention")
        return o, lse

    def lasad_window_attention_backward(self, q, k, v, o, lse, do, window, sinks=0, scale=None, lengths=None, dq=None,
                                        dk=None, dv=None, workspace=None, stream=None):
        """The gradient of ``lasad_window_attention`` from its inputs and outputs; returns (dq, dk, dv)."""
        _check_cuda(q, k, v, o, lse, do, lengths, dq, dk, dv)
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
        dk = torch.empty(k.shape, dtype=k.dtype, device=k.device) if dk is None else dk
        dv = torch.empty(v.shape, dtype=v.dtype, device=v.device) if dv is None else dv
        e = self._window("backward", window, sinks, scale, q=q, k=k, v=v, o=o, do=do, dq=dq, dk=dk, dv=dv)
        p = e.p
        _i32("lengths", lengths, p.B)
        _f32("lse", lse, (p.B, p.Hq, p.T))
        ws = self._workspace(e, self._lib.lasad_window_attention_workspace, q.device, workspace, stream)
        rc = self._lib.lasad_window_attention_backward(self._h, e.ref, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(do),
                                                       _ptr(lengths), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(ws),
                                                       _stream(q.device, stream))
        if rc:
            self._raise(rc, "lasad_window_attention_backward")
        return dq, dk, dv

    def lasad_window_attention_step(self, q, k, v, k_cache, v_cache, pos, window, sinks=0, scale=None, o=None,
                                    workspace=None, stream=None):
        """One new token per sequence, q [B,Hq,d], k, v [B,Hk,d], against ring caches [B, sinks +
        window, Hk, d], which get the token's k and v.  ``pos`` int32 [B]: the tokens' positions
        (negative: the sequence takes no part).  Returns o [B,Hq,d]."""
        _check_cuda(q, k, v, k_cache, v_cache, pos, o)
        if o is None:
            o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        e = self._window("step", window, sinks, scale, q=q, k=k, v=v, o=o, k_cache=k_cache, v_cache=v_cache)
        if pos is None:
            raise ValueError("pos must be contiguous int32 [B]")
        _i32("pos", pos, e.p.B)
        ws = self._workspace(e, self._lib.lasad_window_attention_step_workspace, q.device, workspace, stream)
        rc = self._lib.lasad_window_attention_step(self._h, e.ref, _ptr(q), _ptr(k), _ptr(v), _ptr(k_cache), _ptr(v_cache),
                                                   _ptr(pos), _ptr(o), _ptr(ws), _stream(q.device, stream))
        if rc:
            self._raise(rc, "lasad_window_attention_step")
        return o

    def lasad_window_cache_store(self, k, v, k_cache, v_cache, window, sinks=0, lengths=None, stream=None):
        """Puts the keys and values of a prefill, [B,T,Hk,d], into the ring caches of the step."""
        _check_cuda(k, v, k_cache, v_cache, lengths)
        e = self._window("store", window, sinks, 1.0, k=k, v=v, k_cache=k_cache, v_cache=v_cache)
        _i32("lengths", lengths, e.p.B)
        rc = self._lib.lasad_window_cache_store(self._h, e.ref, _ptr(k), _ptr(v), _ptr(lengths), _ptr(k_cache), _ptr(v_cache),
                                                _stream(k.device, stream))
        if rc:
            self._raise(rc, "lasad_window_cache_store")
