"""What the marshalling modules share: dtype codes, raw pointers and streams of torch tensors."""
from __future__ import annotations

import ctypes

import torch

LASAD_F32 = 0
LASAD_BF16 = 1


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return LASAD_F32
    if t.dtype == torch.bfloat16:
        return LASAD_BF16
    raise TypeError(f"q, k, v, o must be float32 or bfloat16, got {t.dtype}")


def _ptr(t):
    # (an int is accepted where the prototype says c_void_p; None is a null pointer)
    return None if t is None else t.data_ptr()


try:
    _raw_stream = torch._C._cuda_getCurrentRawStream     # the current stream's handle without a Stream object
except AttributeError:       # pragma: no cover - older torch
    _raw_stream = None


def _stream(device, stream):
    if stream is not None:
        return stream
    if _raw_stream is not None:
        return _raw_stream(device.index if device.index is not None else torch.cuda.current_device())
    return torch.cuda.current_stream(device).cuda_stream


def _check_cuda(*ts):
    for t in ts:
        if t is not None and not t.is_cuda:
            raise ValueError("all tensors must be CUDA tensors (there is no CPU path)")


def _strides3(t: torch.Tensor):
    """Element strides of (batch, token, head) for a [B,T,H,d] view with contiguous channels."""
    if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
        raise ValueError("expected [B,T,H,d] with contiguous channels")
    return (ctypes.c_int64 * 3)(t.stride(0), t.stride(1), t.stride(2))


def _strides_decode(t: torch.Tensor):
    if t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError("expected [B,H,d] with contiguous channels")
    return (ctypes.c_int64 * 3)(t.stride(0), 0, t.stride(1))
