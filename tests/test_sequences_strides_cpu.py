"""Outputs whose rows share memory are refused by the library (several CTAs would write the same bytes).  Without a GPU: strides
are looked at ahead of the head size, so of two calls with a head size that no kernel has, the one with good
strides is UNSUPPORTED and the other INVALID_ARG.  The context is memory that neither of them looks at."""
import ctypes

import pytest

from paper_2507_01652_b200 import binding, sequences

D, N, HQ, HK = 48, 10, 4, 2
PACKED = ("q", "k", "v", "o", "do", "dq", "dk", "dv")
PAGED = ("q", "k", "v", "o")
PAGE, PAGES = 16, 5


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def packed(lib, backward, **strides):
    p = sequences.PackedParams(N, 1, HQ, HK, D, binding.LASAD_BF16, 0.125, 0)
    for n in PACKED:
        h = HK if n in ("k", "v", "dk", "dv") else HQ
        setattr(p, n + "_stride", (ctypes.c_int64 * 2)(*strides.get(n, (h * D, D))))
    ctx = ctypes.create_string_buffer(1 << 16)
    if backward:
        return lib.lasad_packed_attention_backward(ctx, ctypes.byref(p), *[None] * 12)
    return lib.lasad_packed_attention(ctx, ctypes.byref(p), *[None] * 7)


def paged(lib, append, pages=None, **strides):
    p = sequences.PagedParams(N, N, HQ, HK, D, binding.LASAD_BF16, PAGE, PAGES, 3, 0, 0, 0, 0, 0.125)
    for n in PAGED:
        h = HK if n in ("k", "v") else HQ
        setattr(p, n + "_stride", (ctypes.c_int64 * 2)(*strides.get(n, (h * D, D))))
    for n in ("k", "v"):
        setattr(p, n + "_pages_stride", (ctypes.c_int64 * 3)(*(pages if pages and n == strides.get("which", n) else (HK * PAGE * D, PAGE * D, D))))
    ctx = ctypes.create_string_buffer(1 << 16)
    if append:
        some = ctypes.c_void_p(16)                # (q, so that its strides count; not followed: the call is refused)
        return lib.lasad_paged_append(ctx, ctypes.byref(p), None, None, some, *[None] * 10)
    return lib.lasad_paged_attention(ctx, ctypes.byref(p), *[None] * 11)


# (token, head): rows inside one another, beside one another by 16 bytes, half over each other, heads over the next tokens
SHARED = [(8, D), (16, D), (D, D), (D * 3, D), (D, D * 9), (D, 8), (0, D), (HQ * D, 0), (1 << 40, 8), (8, 1 << 62)]
APART = [(HQ * D, D), (HQ * D + 16, D), (D, N * D), (D, N * D + 8), (1 << 40, D), (D * 20, D * 3), (D, 1 << 62), (1 << 62, D)]


@pytest.mark.parametrize("shared", SHARED)
def test_an_output_with_rows_in_the_same_memory_is_refused(lib, shared):
    for n in ("dq", "o"):
        back = n != "o"
        assert packed(lib, back, **{n: shared}) == binding.LASAD_ERR_INVALID_ARG, n
    for append in (True, False):
        assert paged(lib, append, o=shared) == binding.LASAD_ERR_INVALID_ARG


@pytest.mark.parametrize("strides", [(8, D), (D, D), (D, D * 9)])
def test_gradients_of_shared_heads_too(lib, strides):
    for n in ("dk", "dv"):
        assert packed(lib, True, **{n: strides}) == binding.LASAD_ERR_INVALID_ARG
        assert packed(lib, True, **{n: (D, D * 10)}) == binding.LASAD_ERR_UNSUPPORTED
        assert packed(lib, False, **{n: strides}) == binding.LASAD_ERR_UNSUPPORTED       # (a forward does not have it)


@pytest.mark.parametrize("apart", APART)
def test_other_orders_of_memory_are_taken(lib, apart):
    for back, n in ((False, "o"), (True, "dq"), (True, "o"), (False, "q"), (True, "do")):
        assert packed(lib, back, **{n: apart}) == binding.LASAD_ERR_UNSUPPORTED, n
    for append in (True, False):
        assert paged(lib, append, o=apart) == binding.LASAD_ERR_UNSUPPORTED


@pytest.mark.parametrize("overlapping", [(8, D), (D, D)])
def test_rows_that_are_only_read_may_overlap(lib, overlapping):
    """(Sliding views of one tensor; nothing is written there.)"""
    for n in ("q", "k", "v"):
        assert packed(lib, True, **{n: overlapping}) == binding.LASAD_ERR_UNSUPPORTED
        assert packed(lib, True, **{n: (0, D)}) == binding.LASAD_ERR_INVALID_ARG         # (nor repeated)


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("pages", [(16, PAGE * D, D), (HK * PAGE * D, PAGE * D, 16), (HK * PAGE * D, 16, D), (PAGE * D, PAGE * D, D),
                                   (HK * PAGE * D, D, D), (D, PAGE * D, D), (PAGE * HK * D, D, D * HK - 16), (0, PAGE * D, D)])
def test_pools_that_are_written_to_have_no_slot_twice(lib, which, pages):
    assert paged(lib, True, pages, which=which) == binding.LASAD_ERR_INVALID_ARG


@pytest.mark.parametrize("pages", [(HK * PAGE * D, PAGE * D, D), (HK * PAGE * D, D, HK * D), (1 << 33, 64, 128), (PAGE * D, PAGES * PAGE * D, D),
                                   (D, PAGES * D, PAGES * HK * D), (2 * HK * PAGE * D, PAGE * D, D), (1 << 62, PAGE * D, D)])
def test_pools_in_other_orders_are_taken(lib, pages):
    assert paged(lib, True, pages) == binding.LASAD_ERR_UNSUPPORTED
