// Appending to a paged cache in 8 bits, with the rotation by position on the way.
//
// A page has `page` tokens of every key head; of each head's keys (and values) in a page the cache holds e4m3
// numbers c and one scale s, a power of two, x ~ c s.  The new tokens of a page and head bring
//
//     s' = the smallest 2^e, -40 <= e <= 40, with max |x| <= 448 2^e        (448: the largest e4m3 number)
//
// and the page takes s = s' where its first token is new, else s = max(s, s'); where that has grown, the
// tokens that were there are rounded again, c <- e4m3(c s_old / s).  A power of two moves no digits: numbers
// that stay normal (2^-6 .. 448) are exact through it, so a cache that grew token by token holds what one
// written at once does, but for what falls below 2^-6 of the scale.  The maximum takes no account of infinities
// and NaN; an infinity is stored as 448 s, a NaN as NaN.
//
// Keys turn in 64 bits and are rounded to 32 once, ahead of the rounding to 8: of a product and a difference
// in 32 bits the last digit depends on the order of operations, and next to a border between two e4m3 numbers
// that would be a step of 1/16.  (fp64 multiply-adds run at half of the fp32 rate here.)  Queries turn in 32
// bits and go back to their own type.
//
// Bound by memory: k, v and q in, a byte a value and q out.
#include "lasad_full.cuh"
#include "lasad_tc_ptx.cuh"

namespace lasad {
namespace {

constexpr int kWarps = 8, kStep = 16;        // kStep: tokens of a warp

// 448 = 1.75 x 2^8: with |x| = m 2^e the exponent is e - 8 where m <= 1.75, else e - 7.
__device__ __forceinline__ int scale_exponent(float amax)
{
    const uint32_t bits = __float_as_uint(amax);
    const int e = (int)(bits >> 23) - 127;                 // (a denormal: far below kScaleLow)
    return max(kScaleLow, min(kScaleHigh, (bits & 0x7fffffu) <= 0x600000u ? e - 8 : e - 7));
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
__device__ __forceinline__ float finite_size(float x)
{
    const float a = fabsf(x);
    return a <= 3.4028235e38f ? a : 0.0f;                  // (a NaN compares false)
}
// lo and hi as two e4m3 numbers, saturating; lo in the low byte
__device__ __forceinline__ uint32_t to_e4m3(float lo, float hi)
{
    unsigned short r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// the two numbers of the low 16 bits
__device__ __forceinline__ float2 from_e4m3(uint32_t x)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)x));
    float2 r;
    asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(r.x), "=f"(r.y) : "r"(h));
    return r;
}

// Channels of lane `sub` of a row's D / 8 lanes: with HALF sub * 4 .. + 3 and their partners D / 2 further, else
// sub * 8 .. + 7; x[0..3] are the pairs' first channels, x[4..7] their partners.
template <typename T, int D, bool HALF> __device__ __forceinline__ void load_pairs(const T* row, int sub, float (&x)[8])
{
    using namespace tcx;
    if constexpr (sizeof(T) == 2) {
        uint32_t w[4];
        if (HALF) {
            const uint2 a = *reinterpret_cast<const uint2*>(row + sub * 4), b = *reinterpret_cast<const uint2*>(row + D / 2 + sub * 4);
            w[0] = a.x, w[1] = a.y, w[2] = b.x, w[3] = b.y;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(w[i]), x[2 * i + 1] = bf16_hi(w[i]);
        } else {
            const uint4 a = *reinterpret_cast<const uint4*>(row + sub * 8);
            w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = bf16_lo(w[i]), x[4 + i] = bf16_hi(w[i]);
        }
    } else {
        const float4 a = *reinterpret_cast<const float4*>(row + (HALF ? sub * 4 : sub * 8));
        const float4 b = *reinterpret_cast<const float4*>(row + (HALF ? D / 2 + sub * 4 : sub * 8 + 4));
        if (HALF) {
            x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
        } else {
            x[0] = a.x, x[4] = a.y, x[1] = a.z, x[5] = a.w, x[2] = b.x, x[6] = b.y, x[3] = b.z, x[7] = b.w;
        }
    }
}
template <typename T, int D, bool HALF> __device__ __forceinline__ void store_pairs(T* row, int sub, const float (&x)[8])
{
    using namespace tcx;
    if constexpr (sizeof(T) == 2) {
        if (HALF) {
            *reinterpret_cast<uint2*>(row + sub * 4) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
            *reinterpret_cast<uint2*>(row + D / 2 + sub * 4) = make_uint2(pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
        } else {
            *reinterpret_cast<uint4*>(row + sub * 8) =
                make_uint4(pack_bf16(x[0], x[4]), pack_bf16(x[1], x[5]), pack_bf16(x[2], x[6]), pack_bf16(x[3], x[7]));
        }
    } else if (HALF) {
        *reinterpret_cast<float4*>(row + sub * 4) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4*>(row + D / 2 + sub * 4) = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        *reinterpret_cast<float4*>(row + sub * 8) = make_float4(x[0], x[4], x[1], x[5]);
        *reinterpret_cast<float4*>(row + sub * 8 + 4) = make_float4(x[2], x[6], x[3], x[7]);
    }
}
// The same places of a row of bytes, from x times f.
template <int D, bool HALF> __device__ __forceinline__ void store_bytes(unsigned char* row, int sub, const float (&x)[8], float f)
{
    if (HALF) {
        *reinterpret_cast<uint32_t*>(row + sub * 4) = to_e4m3(x[0] * f, x[1] * f) | to_e4m3(x[2] * f, x[3] * f) << 16;
        *reinterpret_cast<uint32_t*>(row + D / 2 + sub * 4) = to_e4m3(x[4] * f, x[5] * f) | to_e4m3(x[6] * f, x[7] * f) << 16;
    } else {
        *reinterpret_cast<uint2*>(row + sub * 8) = make_uint2(to_e4m3(x[0] * f, x[4] * f) | to_e4m3(x[1] * f, x[5] * f) << 16,
                                                              to_e4m3(x[2] * f, x[6] * f) | to_e4m3(x[3] * f, x[7] * f) << 16);
    }
}

// cos and sin of a lane's four pairs for the token at position i.
template <int D> __device__ __forceinline__ void angles(const PagedArgs& a, long long i, int sub, float (&c)[4], float (&s)[4])
{
    int m = sub * 4, width = D / 2;
    long long row = i;
    if (a.grid_w > 0) {
        const long long j = i - a.prefix_len;
        if (j < 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) c[e] = 1.0f, s[e] = 0.0f;
            return;
        }
        // (positions are 32 bits wide, and so is what a call adds)
        const unsigned q = (unsigned)j / (unsigned)a.grid_w;
        width = D / 4;
        row = m < width ? q : (unsigned)j - q * (unsigned)a.grid_w;
        if (m >= width) m -= width;
    }
    row = min(row, (long long)a.table_rows - 1);
    const float4* t = reinterpret_cast<const float4*>(a.table + (row * width + m) * 2);
    const float4 u = t[0], v = t[1];
    c[0] = u.x, s[0] = u.y, c[1] = u.z, s[1] = u.w, c[2] = v.x, s[2] = v.y, c[3] = v.z, s[3] = v.w;
}

// The new tokens of sequence b: their place in memory, their number and the first one's position.  A sequence
// that begins before 0 takes no part.
struct Fresh {
    int at, n;
    long long pos;
};
__device__ __forceinline__ Fresh fresh_of(const PagedArgs& a, int b)
{
    Fresh f;
    f.at = a.offsets ? max(0, min(a.offsets[b], a.N)) : b;
    f.n = a.offsets ? max(0, min(a.offsets[b + 1], a.N) - f.at) : 1;
    f.pos = a.pos[b];
    return f;
}

// One page and head: `page` / kStep warps, kStep tokens each; first keys, then values.
template <typename T, int D, bool HALF, bool TURN>
__device__ __forceinline__ void write_page(const PagedArgs& a, int unit, float (&top)[2][kWarps])
{
    constexpr int LANES = D / 8, ROWS = 32 / LANES, ACC = kStep / ROWS;     // lanes of a row, rows of an access, accesses
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % LANES, mine = lane / LANES;
    const int W = a.page / kStep, team = warp / W, w = warp - team * W;     // a page's warps
    unit = unit * (kWarps / W) + team;
    const int at = unit / a.Hk, h = unit - at * a.Hk;
    // the page: of sequence b its page number j (see region_tiles for numbers without a table)
    int b = at, j = 0;
    bool live;
    if (a.offsets) {
        int lo = 0, hi = a.B;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (max(0, min(a.offsets[mid], a.N)) / a.page + 2 * mid <= at) lo = mid;
            else hi = mid;
        }
        b = lo;
        j = at - (max(0, min(a.offsets[b], a.N)) / a.page + 2 * b);
        live = j >= 0;
    } else {
        live = b < a.B;
    }
    Fresh f{0, 0, 0};
    if (live) f = fresh_of(a, b);
    live = live && f.pos >= 0 && f.n > 0;
    const long long page0 = live ? (f.pos / a.page + j) * a.page : 0;       // the position of the page's first slot
    live = live && page0 < f.pos + f.n && page0 / a.page < a.table_pages;
    int id = -1;
    if (live) id = a.block_table[(long long)b * a.table_pages + page0 / a.page];
    live = live && id >= 0 && id < a.pages;
    // slots first .. last - 1 are new
    const int first = live ? (int)max(0LL, f.pos - page0) : 0, last = live ? (int)min((long long)a.page, f.pos + f.n - page0) : 0;
    const long long row0 = f.at + (page0 - f.pos);                          // the row of the page's slot 0
    for (int kv = 0; kv < 2; ++kv) {
        const T* src = static_cast<const T*>(kv ? a.v : a.k) + h * (kv ? a.vs[1] : a.ks[1]);
        const long long stride = kv ? a.vs[0] : a.ks[0];
        float x[ACC][8], size = 0.0f;
#pragma unroll
        for (int i = 0; i < ACC; ++i) {
            const int slot = w * kStep + i * ROWS + mine;
            if (slot < first || slot >= last) continue;
            load_pairs<T, D, HALF>(src + (row0 + slot) * stride, sub, x[i]);
            if (TURN && kv == 0) {
                float c[4], s[4];
                angles<D>(a, page0 + slot, sub, c, s);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const double x0 = x[i][e], x1 = x[i][4 + e], cd = c[e], sd = s[e];
                    x[i][e] = (float)(x0 * cd - x1 * sd);
                    x[i][4 + e] = (float)(x0 * sd + x1 * cd);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) size = fmaxf(size, finite_size(x[i][e]));
        }
#pragma unroll
        for (int k = 16; k >= 1; k >>= 1) size = fmaxf(size, __shfl_xor_sync(0xffffffffu, size, k));
        if (lane == 0) top[kv][warp] = size;
        __syncthreads();
        for (int k = 0; k < W; ++k) size = fmaxf(size, top[kv][team * W + k]);
        float* scale = (kv ? a.vscale : a.kscale) + (long long)id * a.Hk + h;
        unsigned char* dst = kv ? a.vp + id * a.vps[0] + h * a.vps[1] : a.kp + id * a.kps[0] + h * a.kps[1];
        const long long slots = kv ? a.vps[2] : a.kps[2];
        float now = power_of_two(scale_exponent(size)), was = now;
        if (live && first > 0) {
            was = *scale;
            now = fmaxf(now, was);
        }
        __syncthreads();                                                    // (everyone has read the scale)
        if (!live) continue;
        if (w == 0 && lane == 0) *scale = now;
        if (now > was) {
            const float f8 = was / now;
            for (int slot = w * ROWS + mine; slot < first; slot += W * ROWS) {
                unsigned char* row = dst + slot * slots + sub * 8;
                uint2 old = *reinterpret_cast<const uint2*>(row);
                uint32_t r[2] = {old.x, old.y};
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float2 u = from_e4m3(r[e] & 0xffffu), v = from_e4m3(r[e] >> 16);
                    r[e] = to_e4m3(u.x * f8, u.y * f8) | to_e4m3(v.x * f8, v.y * f8) << 16;
                }
                *reinterpret_cast<uint2*>(row) = make_uint2(r[0], r[1]);
            }
        }
        const float inv = 1.0f / now;
#pragma unroll
        for (int i = 0; i < ACC; ++i) {
            const int slot = w * kStep + i * ROWS + mine;
            if (slot >= first && slot < last) store_bytes<D, HALF>(dst + slot * slots, sub, x[i], inv);
        }
    }
}

// A row of lanes has a token; it goes over the query heads.
template <typename T, int D, bool HALF, bool TURN>
__device__ __forceinline__ void turn_queries(const PagedArgs& a, int cta)
{
    constexpr int LANES = D / 8, ROWS = 32 / LANES;
    const int sub = threadIdx.x % LANES;
    const long long row = (long long)cta * kWarps * ROWS + threadIdx.x / LANES;
    if (row >= a.N) return;
    // its sequence and position
    int b = (int)row;
    bool live = b < a.B;
    long long pos = 0;
    if (a.offsets) {
        int lo = -1, hi = a.B + 1;                  // the last offset that is not behind the row
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.offsets[mid] <= row) lo = mid;
            else hi = mid;
        }
        b = lo;
        live = b >= 0 && b < a.B;
        if (live) pos = row - a.offsets[b];
    }
    if (live) {
        const int first = a.pos[b];
        live = first >= 0;
        pos += first;
    }
    float c[4] = {1.0f, 1.0f, 1.0f, 1.0f}, s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (TURN && live) angles<D>(a, pos, sub, c, s);
    const T* src = static_cast<const T*>(a.q) + row * a.qs[0];
    T* dst = static_cast<T*>(a.q_out) + row * a.qos[0];
    for (int h = 0; h < a.Hq; ++h) {
        float x[8], y[8];
        load_pairs<T, D, HALF>(src + h * a.qs[1], sub, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[e] = live ? TURN ? x[e] * c[e] - x[4 + e] * s[e] : x[e] : 0.0f;
            y[4 + e] = live ? TURN ? x[e] * s[e] + x[4 + e] * c[e] : x[4 + e] : 0.0f;
        }
        store_pairs<T, D, HALF>(dst + h * a.qos[1], sub, y);
    }
}

template <typename T, int D, bool HALF, bool TURN>
__global__ void __launch_bounds__(32 * kWarps) paged_append_kernel(const PagedArgs a, int page_ctas)
{
    __shared__ float top[2][kWarps];
    pdl_wait();
    if ((int)blockIdx.x < page_ctas) write_page<T, D, HALF, TURN>(a, blockIdx.x, top);
    else turn_queries<T, D, HALF, TURN>(a, blockIdx.x - page_ctas);
}

template <typename T, int D> cudaError_t launch_t(const PagedArgs& a, cudaStream_t st)
{
    const int per_cta = kWarps / (a.page / kStep);
    // pages that a sequence of n new tokens touches: at most n / page + 2, and none is numbered twice
    const long long pages = a.offsets ? (long long)a.N / a.page + 2LL * a.B : a.B;
    const long long page_ctas = (pages * a.Hk + per_cta - 1) / per_cta;
    constexpr int rows = kWarps * 32 / (D / 8);
    const long long ctas = page_ctas + (a.q ? ((long long)a.N + rows - 1) / rows : 0);
    auto kernel = a.table ? (a.half ? paged_append_kernel<T, D, true, true> : paged_append_kernel<T, D, false, true>)
                          : paged_append_kernel<T, D, false, false>;
    return launch_dependent(kernel, dim3((unsigned)ctas), dim3(32 * kWarps), 0, st, a, (int)page_ctas);
}

}  // namespace

cudaError_t launch_paged_append(const PagedArgs& a, cudaStream_t st)
{
    if (a.bf16) return a.d == 64 ? launch_t<__nv_bfloat16, 64>(a, st) : launch_t<__nv_bfloat16, 32>(a, st);
    return a.d == 64 ? launch_t<float, 64>(a, st) : launch_t<float, 32>(a, st);
}

}  // namespace lasad
