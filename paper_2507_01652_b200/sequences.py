"""Marshalling of the operators of a layer that attends to whole sequences (``include/lasad.h``).

``Sequences`` is the part of ``binding.Lasad`` that holds them: causal attention over packed sequences
(``lasad_packed_attention*``), appending rotated keys and values to a paged cache in 8 bits
(``lasad_paged_append``) and attention of one token per sequence over that cache
(``lasad_paged_attention``).  Gradients, streams, workspaces and outputs are handled as in ``mixers``.
"""
from __future__ import annotations

import ctypes
import math

import torch

from .marshal import _dtype_code, _empty, _ptr, _stream
from .mixers import LASAD_ROPE_HALF, _F32, _I32, _I64, _VP, _f32, _like, _look, _same, _shape

E4M3 = torch.float8_e4m3fn


class PackedParams(ctypes.Structure):
    """Mirror of ``lasad_packed_params``."""
    _fields_ = ([(n, _I32) for n in ("N", "S", "Hq", "Hk", "d", "dtype")] + [("scale", _F32), ("reserved", _I32)]
                + [(n, _I64 * 2) for n in ("q_stride", "k_stride", "v_stride", "o_stride", "do_stride", "dq_stride",
                                           "dk_stride", "dv_stride")])


class PagedParams(ctypes.Structure):
    """Mirror of ``lasad_paged_params``."""
    _fields_ = ([(n, _I32) for n in ("B", "N", "Hq", "Hk", "d", "dtype", "page", "pages", "table_pages", "grid_w",
                                     "prefix_len", "table_rows", "flags")] + [("scale", _F32)]
                + [(n, _I64 * 3) for n in ("k_pages_stride", "v_pages_stride")]
                + [(n, _I64 * 2) for n in ("q_stride", "k_stride", "v_stride", "o_stride")])


_KP, _GP = ctypes.POINTER(PackedParams), ctypes.POINTER(PagedParams)
PROTOTYPES = {
    "lasad_packed_attention": (ctypes.c_int, [_VP, _KP] + [_VP] * 7),
    "lasad_packed_attention_workspace": (_I64, [_VP, _KP]),
    "lasad_packed_attention_backward": (ctypes.c_int, [_VP, _KP] + [_VP] * 12),
    "lasad_paged_append": (ctypes.c_int, [_VP, _GP] + [_VP] * 13),
    "lasad_paged_attention": (ctypes.c_int, [_VP, _GP] + [_VP] * 11),
    "lasad_paged_attention_workspace": (_I64, [_VP, _GP]),
}


def _rows(name, t):
    """Element strides of (row, head) of a [N,H,d] view with contiguous channels."""
    if t is None:
        return (_I64 * 2)()
    if t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{name} must be [rows,H,d] with contiguous channels")
    return (_I64 * 2)(t.stride(0), t.stride(1))


def _ints(name, t, shape):
    if t is not None and (t.dtype != torch.int32 or not t.is_contiguous() or tuple(t.shape) != shape):
        raise ValueError(f"{name} must be contiguous int32 {list(shape)}")


class Sequences:
    """The calls of a layer that attends to whole sequences; a base of ``binding.Lasad`` beside ``Mixers``."""

    # ---- packed sequences -------------------------------------------------------------------
    _PACKED = ("q", "k", "v", "o", "do", "dq", "dk", "dv")

    def _packed(self, key, offsets, lse, **ts):
        """Checks a call that looks like none before it."""
        if offsets is None:
            raise ValueError("offsets is missing")
        self._here(offsets, lse, *ts.values())
        q, k = ts["q"], ts["k"]
        _same("all tensors", q, *ts.values())
        strides = [_rows(n, ts.get(n)) for n in self._PACKED]
        N, Hq, d = q.shape
        for n, t in ts.items():
            _shape(n, t, (N, Hq if n in ("q", "o", "do", "dq") else k.shape[1], d))
        if offsets.dim() != 1 or offsets.dtype != torch.int32 or not offsets.is_contiguous() or offsets.numel() < 2:
            raise ValueError("offsets must be contiguous int32 [sequences + 1]")
        _f32("lse", lse, (Hq, N))
        return self._new(key, PackedParams(N, offsets.numel() - 1, Hq, k.shape[1], d, _dtype_code(q), 0.0, 0, *strides))

    def lasad_packed_attention(self, q, k, v, offsets, scale=None, o=None, lse=None, want_lse=False, stream=None):
        """Causal softmax attention of q [N,Hq,d] over k, v [N,Hk,d], sequence i being rows ``offsets``[i] to
        ``offsets``[i+1] - 1 (int32 [S+1]); rows of no sequence get zeros.  ``scale`` is 1/sqrt(d) by
        default.  Returns (o, lse); lse, fp32 [Hq,N], only with ``want_lse`` (the gradient needs it)."""
        if o is None:
            o = _like(q, stream)
        key = ("packed", _look(q), _look(k), _look(v), _look(offsets), _look(o), _look(lse))
        e = self._calls.get(key) or self._packed(key, offsets, lse, q=q, k=k, v=v, o=o)
        p = e.p
        p.scale = 1.0 / math.sqrt(p.d) if scale is None else scale
        if lse is None and want_lse:
            lse = _empty((p.Hq, p.N), torch.float32, q.device, stream)
        rc = self._lib.lasad_packed_attention(self._h, e.ref, q.data_ptr(), k.data_ptr(), v.data_ptr(), offsets.data_ptr(),
                                              o.data_ptr(), _ptr(lse), _stream(q.device, stream))
        if rc:
            self._raise(rc, "lasad_packed_attention")
        return o, lse

    def lasad_packed_attention_backward(self, q, k, v, o, lse, do, offsets, scale=None, dq=None, dk=None, dv=None,
                                        workspace=None, stream=None):
        """The gradient of ``lasad_packed_attention`` from its inputs and outputs; returns (dq, dk, dv)."""
        dq = _like(q, stream) if dq is None else dq
        dk = _like(k, stream) if dk is None else dk
        dv = _like(v, stream) if dv is None else dv
        key = ("packed'", _look(q), _look(k), _look(v), _look(o), _look(lse), _look(do), _look(offsets), _look(dq),
               _look(dk), _look(dv))
        e = self._calls.get(key)
        if e is None:
            if lse is None:
                raise ValueError("lse is what lasad_packed_attention returns with want_lse=True")
            e = self._packed(key, offsets, lse, q=q, k=k, v=v, o=o, do=do, dq=dq, dk=dk, dv=dv)
        p = e.p
        p.scale = 1.0 / math.sqrt(p.d) if scale is None else scale
        ws = self._workspace(e, self._lib.lasad_packed_attention_workspace, q, workspace, stream)
        rc = self._lib.lasad_packed_attention_backward(self._h, e.ref, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                                       lse.data_ptr(), do.data_ptr(), offsets.data_ptr(), dq.data_ptr(),
                                                       dk.data_ptr(), dv.data_ptr(), _ptr(ws), _stream(q.device, stream))
        if rc:
            self._raise(rc, "lasad_packed_attention_backward")
        return dq, dk, dv

    # ---- paged cache ------------------------------------------------------------------------
    def _paged(self, key, q, k, v, o, k_pages, v_pages, k_scales, v_scales, block_table, pos, offsets, table, grid, lse):
        """Checks a call that looks like none before it."""
        self._here(q, k, v, o, k_pages, v_pages, k_scales, v_scales, block_table, pos, offsets, table, lse)
        for n, t in (("k_pages", k_pages), ("v_pages", v_pages), ("block_table", block_table), ("pos", pos),
                     ("k_scales", k_scales), ("v_scales", v_scales)):
            if t is None:
                raise ValueError(f"{n} is missing")
        first = k if q is None else q
        _same("q, k, v and their outputs", first, q, k, v, o)
        strides = [_rows(n, t) for n, t in (("q", q), ("k", k), ("v", v), ("o", o))]
        for n, t in (("k_pages", k_pages), ("v_pages", v_pages)):
            if t.dtype != E4M3 or t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
                raise ValueError(f"{n} must be float8_e4m3fn [pages,Hk,page,d] with contiguous channels")
        P, Hk, page, d = k_pages.shape
        _shape("v_pages", v_pages, (P, Hk, page, d))
        N = first.shape[0]
        Hq = Hk if q is None else q.shape[1]
        for n, t, h in (("q", q, Hq), ("o", o, Hq), ("k", k, Hk), ("v", v, Hk)):
            _shape(n, t, (N, h, d))
        _f32("k_scales", k_scales, (P, Hk))
        _f32("v_scales", v_scales, (P, Hk))
        if block_table.dim() != 2:
            raise ValueError("block_table must be int32 [B,pages of a sequence]")
        B = block_table.shape[0]
        _ints("block_table", block_table, (B, block_table.shape[1]))
        _ints("pos", pos, (B,))
        _ints("offsets", offsets, (B + 1,))
        if offsets is None and N != B:
            raise ValueError(f"expected one row for each of the {B} sequences, got {N}")
        _f32("lse", lse, (B, Hq))
        if table is not None:
            _f32("table", table, (table.shape[0], d // (4 if grid else 2), 2))
        return self._new(key, PagedParams(B, N, Hq, Hk, d, _dtype_code(first), page, P, block_table.shape[1], 0, 0,
                                          0 if table is None else table.shape[0], 0, 0.0,
                                          *[(_I64 * 3)(*t.stride()[:3]) for t in (k_pages, v_pages)], *strides))

    def lasad_paged_append(self, k, v, k_pages, v_pages, k_scales, v_scales, block_table, pos, offsets=None, q=None,
                           table=None, grid_w=0, prefix_len=0, half=False, q_out=None, stream=None):
        """Puts k, v [N,Hk,d] into the paged cache (``k_pages``, ``v_pages`` float8_e4m3fn [P,Hk,page,d],
        ``k_scales``, ``v_scales`` fp32 [P,Hk], ``block_table`` int32 [B,pages]), one token for each of the B
        sequences or, with ``offsets`` int32 [B+1], each one's rows of a pack, from position ``pos`` int32 [B]
        on (negative: the sequence takes no part).  With ``table`` (from ``rope_table``) keys are rotated by
        position on the way, and so is ``q`` [N,Hq,d] if it is given.  Returns q_out (None without q)."""
        if q is not None and q_out is None:
            q_out = _like(q, stream)
        if q is None and q_out is not None:
            raise ValueError("q_out is for q")
        key = ("append", grid_w > 0, _look(k), _look(v), _look(k_pages), _look(v_pages), _look(k_scales), _look(v_scales),
               _look(block_table), _look(pos), _look(offsets), _look(q), _look(table), _look(q_out))
        e = self._calls.get(key) or self._paged(key, q, k, v, q_out, k_pages, v_pages, k_scales, v_scales, block_table, pos,
                                                offsets, table, grid_w > 0, None)
        p = e.p
        p.grid_w, p.prefix_len, p.flags = grid_w, prefix_len, LASAD_ROPE_HALF if half else 0
        rc = self._lib.lasad_paged_append(self._h, e.ref, k.data_ptr(), v.data_ptr(), _ptr(q), _ptr(table), _ptr(offsets),
                                          pos.data_ptr(), block_table.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                                          k_scales.data_ptr(), v_scales.data_ptr(), _ptr(q_out), _stream(k.device, stream))
        if rc:
            self._raise(rc, "lasad_paged_append")
        return q_out

    def lasad_paged_attention(self, q, k_pages, v_pages, k_scales, v_scales, block_table, pos, scale=None, o=None, lse=None,
                              want_lse=False, workspace=None, stream=None):
        """Softmax attention of one token per sequence, q [B,Hq,d], over the tokens 0 to ``pos`` (int32 [B]) of the
        paged cache, its own among them (``lasad_paged_append`` comes first); a negative position gives zeros.
        Returns (o, lse); lse, fp32 [B,Hq], only with ``want_lse``."""
        if o is None:
            o = _like(q, stream)
        key = ("paged", _look(q), _look(k_pages), _look(v_pages), _look(k_scales), _look(v_scales), _look(block_table),
               _look(pos), _look(o), _look(lse))
        e = self._calls.get(key) or self._paged(key, q, None, None, o, k_pages, v_pages, k_scales, v_scales, block_table, pos,
                                                None, None, False, lse)
        p = e.p
        p.scale = 1.0 / math.sqrt(p.d) if scale is None else scale
        if lse is None and want_lse:
            lse = _empty((p.B, p.Hq), torch.float32, q.device, stream)
        ws = self._workspace(e, self._lib.lasad_paged_attention_workspace, q, workspace, stream)
        rc = self._lib.lasad_paged_attention(self._h, e.ref, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                                             k_scales.data_ptr(), v_scales.data_ptr(), block_table.data_ptr(), pos.data_ptr(),
                                             o.data_ptr(), _ptr(lse), _ptr(ws), _stream(q.device, stream))
        if rc:
            self._raise(rc, "lasad_paged_attention")
        return o, lse
