// TMA descriptors and TMEM helpers of the window attention's tensor-core kernels.
#pragma once
#include "lasad_mixers.cuh"
#include "lasad_tc_ptx.cuh"
#include "lasad_tc_tma.cuh"

namespace lasad {
namespace tcx {

// [B,T,H,d] bf16 with element strides -> 4-D map (d, h, t, b); box = `rows` tokens of one head and 64
// channels, rows of 128 bytes with the 128-byte swizzle.  What lies outside reads as zeros and is not
// stored: tokens past T, and with d = 32 the upper half of the channels, so the kernels have one
// width (the zeros add nothing to a product).  That makes twice the products that d = 32 needs, which the
// kernels are not bound by: 1 x 9217 tokens, 24 query and 8 key heads, window 1536, forward 157 us and with its
// gradient 549, at d = 64 162 and 595.
inline bool encode_rows_map(CUtensorMap* map, const void* base, int d, int B, int T, int H, const long long* strides, int rows)
{
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    auto bytes = [](long long elems) { return (cuuint64_t)(elems > 0 ? elems * 2 : 128); };
    const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)H, (cuuint64_t)T, (cuuint64_t)B};
    const cuuint64_t gstr[3] = {bytes(strides[2]), bytes(strides[1]), bytes(strides[0])};
    const cuuint32_t box[4] = {64u, 1u, (cuuint32_t)rows, 1u};
    const cuuint32_t estr[4] = {1u, 1u, 1u, 1u};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, gstr, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// [N,H,d] bf16 with element strides of (token, head): the same map with one batch element.
inline bool encode_packed_map(CUtensorMap* map, const void* base, int d, int N, int H, const long long (&s)[2], int rows)
{
    const long long strides[3] = {0, s[0], s[1]};
    return encode_rows_map(map, base, d, 1, N, H, strides, rows);
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr unsigned kDrainLimit = 1u << 26;

// bits lo .. hi of a word (none where hi < lo)
__device__ __forceinline__ uint32_t bit_range(int lo, int hi)
{
    lo = max(lo, 0);
    hi = min(hi, 31);
    return hi < lo ? 0u : (0xffffffffu >> (31 - hi)) & (0xffffffffu << lo);
}

// Which of the keys s0 .. s0 + 31 token t sees (a sequence of n tokens; t itself is not checked).
__device__ __forceinline__ uint32_t seen_bits(int t, int s0, int window, int sinks, int n)
{
    const int last = min(t, n - 1) - s0;
    return bit_range(t - window + 1 - s0, last) | bit_range(0, min(last, sinks - 1 - s0));
}

// A value that all lanes of the warp have, in a form that the compiler knows to be one: addresses and
// descriptors of tcgen05 instructions built from such values stay in uniform registers.
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }

// mbar_wait of a whole warp: every lane goes on, or none does, so that what follows may need all of them.
// (The first try, which most often succeeds, costs 90 clocks, the general loop 130.)
__device__ __forceinline__ bool warp_wait(void* bar, unsigned parity, unsigned limit, volatile int* abort_flag, int* status)
{
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, limit, abort_flag, status));
}

// Copies `bytes` (a multiple of 16, both ends on 16 bytes) of this GPU's memory; they count on `bar`.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, unsigned bytes, void* bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                 "l"(src), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

// Zeroes one 128-byte row of a tile.
__device__ __forceinline__ void zero_row(unsigned char* row)
{
    uint4* p = reinterpret_cast<uint4*>(row);
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = make_uint4(0, 0, 0, 0);
}

// the largest of three
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// {a0 + b0, a1 + b1}, in place
__device__ __forceinline__ void add2(float& a0, float& a1, float b0, float b1)
{
    unsigned long long pa, pb;
    asm("mov.b64 %0, {%1, %2};" : "=l"(pa) : "f"(a0), "f"(a1));
    asm("mov.b64 %0, {%1, %2};" : "=l"(pb) : "f"(b0), "f"(b1));
    asm("add.rn.f32x2 %0, %0, %1;" : "+l"(pa) : "l"(pb));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a0), "=f"(a1) : "l"(pa));
}
// {a0 * b + c, a1 * b + c}
__device__ __forceinline__ void fma2s(float a0, float a1, float b, float c, float& r0, float& r1)
{
    fma2(a0, a1, b, c, c, r0, r1);
}

}  // namespace tcx
}  // namespace lasad
