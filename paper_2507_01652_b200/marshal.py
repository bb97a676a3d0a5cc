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


def _empty(shape, dtype, device, stream, returned=True):
    """Memory that a call on ``stream`` (a raw handle; None: the current stream) writes.

    The allocator hands a block on as soon as its owner lets go of it, in the order of the stream it belongs
    to: memory of the current stream may still be in use by what that stream has to do, and memory that
    another stream has to write must not go back to the current one.  So it is that stream's own.  What is
    ``returned`` will be read on the current stream, which the allocator then waits for as well."""
    if stream is None or device.type != "cuda":         # (the call refuses what is not on a GPU)
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(torch.cuda.ExternalStream(getattr(stream, "value", stream) or 0, device=device)):
        t = torch.empty(shape, dtype=dtype, device=device)
    if returned:
        t.record_stream(torch.cuda.current_stream(device))
    return t


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
