// One token per sequence against a paged cache in 8 bits (e4m3 numbers c with one scale s per page and head, x = c s):
//
//     o = sum_j p_j v_j ,   p_j = e^(scale q.k_j) / sum   over the tokens 0 .. pos of the sequence.
//
// Bound by reading the cache once, 2 d bytes a token and key head.  A warp takes steps of 16 tokens, straight from
// memory into the fragments of two products on mma.sync.m16n8k16 (the rows are the query heads that share
// the key head: 16 of them, of which few are used, so the tensor cores have time to spare and tcgen05's 128 rows
// would only add a way through shared memory).  e4m3 numbers are exact in fp16, so keys and values enter
// without a rounding; the page's key scale multiplies the fp32 score.  The order of a product's inner index is
// free, so a lane reads 16 neighbouring channels of a key and 8 of a value.
//
// The page's value scale goes into the exponent: with x_j = scale q.k_j log2(e) + log2 s_j a warp sums
//
//     O = sum_j w_j c_j ,  l = sum_j w_j / s_j ,   w_j = 2^(x_j - M) ,      o = O / l ,  lse = (M + log2 l) ln 2
//
// so that w stays in the range of fp16 however far the scales of two pages are apart.  M lies 11 below a lagging
// maximum, which moves only when some row has grown by more than 4: w is at most 2^15, and it keeps its eleven
// digits down to 2^-25 of the largest and some down to 2^-35.  w is rounded to fp16 (2^-11 of each term) where q is bf16; where q is
// fp32, q and w enter as sums of two fp16 numbers (22 bits).  q is brought near 1 by a power of two first, so that
// fp16 holds it.
//
// The tokens of a sequence are cut into parts where there are few (sequence, key head) pairs; then the parts'
// (M, l, O) go to memory and a second kernel joins them.
#include "lasad_full.cuh"
#include "lasad_tc_ptx.cuh"

#include <cuda_fp16.h>

#include <algorithm>

namespace lasad {
namespace {

constexpr int kWarps = 4, kStep = 16, kMinPart = 256;    // kMinPart: tokens of a part, at least
constexpr int kAhead = 2;                                // steps of a warp in flight beside the one it works on
constexpr float kLift = 11.0f, kLag = 4.0f;              // of the largest x over M; how far it may be over that
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// two e4m3 numbers to two fp16 ones
__device__ __forceinline__ uint32_t f16_of(uint32_t x)
{
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)x));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// what fp16 leaves of lo and hi
__device__ __forceinline__ uint32_t rest_f16(float lo, float hi, uint32_t packed)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&packed));
    return pack_f16(lo - f.x, hi - f.y);
}

// The tokens of a sequence and how they are cut: part p has tokens p * size .. of n.
struct Cut {
    int n, size, parts;
};
__device__ __forceinline__ Cut cut_of(const PagedArgs& a, int b)
{
    Cut c;
    c.n = min((long long)a.pos[b] + 1, (long long)a.table_pages * a.page);
    c.n = max(c.n, 0);
    c.size = max(((c.n + a.splits - 1) / a.splits + kStep - 1) / kStep * kStep, a.splits > 1 ? kMinPart : kStep);
    c.parts = (c.n + c.size - 1) / c.size;
    return c;
}

// A lane's share of 16 tokens: of tokens g and 8 + g the keys' channels t D / 4 .. (g = lane / 4, t = lane % 4), of tokens
// 2 t, 2 t + 1, 8 + 2 t, 9 + 2 t the values' channels g D / 8 .. .
template <int D> struct Step {
    uint32_t k[2][D / 16], v[4][D / 32];
    float ks, lv, iv;            // the key scale, log2 of the value scale and its reciprocal; ks < 0: no such page
    int at;                      // its first token
};

// PAIR: fp32 queries.  LOW: at most 8 query heads, rows 8 to 15 are empty.
template <int D, bool PAIR, bool LOW>
__global__ void __launch_bounds__(32 * kWarps) paged_attention_kernel(const PagedArgs a, int row_tiles)
{
    constexpr int KK = D / 16;                               // inner steps of q.k; words of a lane's key piece
    constexpr int DN = D / 8;                                // column tiles of O
    __shared__ float part[kWarps][16][D + 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int G = a.Hq / a.Hk;
    // blockIdx.x = ((part * B + sequence) * Hk + key head) * row_tiles + row tile
    int rest = blockIdx.x;
    const int rt = rest % row_tiles;
    rest /= row_tiles;
    const int hk = rest % a.Hk;
    rest /= a.Hk;
    const int b = rest % a.B, p = rest / a.B;
    const int rows = min(16, G - rt * 16), h0 = hk * G + rt * 16;
    pdl_wait();
    const Cut cut = cut_of(a, b);
    if (p >= max(cut.parts, 1)) return;
    const int lo = p * cut.size, hi = min(cut.n, lo + cut.size);

    // q as fp16 fragments: inner step kk, register r: row g + 8 (r & 1), channels t D / 4 + 4 kk + 2 (r >> 1) and the next
    uint32_t qa[KK][4], ql[PAIR ? KK : 1][4];
    float factor[2];                                         // scale log2(e) and what q was divided by
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float x[D / 4], top = 0.0f;
#pragma unroll
        for (int e = 0; e < D / 4; ++e) x[e] = 0.0f;
        const int row = g + 8 * i;
        if ((!LOW || i == 0) && row < rows) {
            const long long at = b * a.qs[0] + (h0 + row) * a.qs[1] + t * (D / 4);
            if (PAIR) {
#pragma unroll
                for (int e = 0; e < D / 16; ++e) {
                    const float4 v = reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + at)[e];
                    x[4 * e] = v.x, x[4 * e + 1] = v.y, x[4 * e + 2] = v.z, x[4 * e + 3] = v.w;
                }
            } else {
#pragma unroll
                for (int e = 0; e < D / 32; ++e) {
                    const uint4 v = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + at)[e];
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[8 * e + 2 * k] = tcx::bf16_lo(w[k]), x[8 * e + 2 * k + 1] = tcx::bf16_hi(w[k]);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < D / 4; ++e) top = fmaxf(top, fabsf(x[e]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // |q| < 2 after division by 2^e (a power that fp32 has, and its reciprocal too)
        const int e2 = max(-120, min(120, (int)(__float_as_uint(top) >> 23) - 127));
        const float down = __uint_as_float((uint32_t)(127 - e2) << 23);
        factor[i] = a.scale * kLog2e * __uint_as_float((uint32_t)(127 + e2) << 23);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float u = x[4 * kk + 2 * r] * down, v = x[4 * kk + 2 * r + 1] * down;
                qa[kk][2 * r + i] = pack_f16(u, v);
                if (PAIR) ql[kk][2 * r + i] = rest_f16(u, v, qa[kk][2 * r + i]);
            }
    }

    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f}, o[DN][4];
#pragma unroll
    for (int n = 0; n < DN; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.0f;

    // The warp's steps: number i is at lo + (i kWarps + warp) kStep.  Pages and scales of 32 of them are fetched at a
    // time, one by each lane.
    const int steps = (max(hi - lo, 0) + kStep - 1) / kStep, mine = (steps - warp + kWarps - 1) / kWarps;
    const int* ids = a.block_table + (long long)b * a.table_pages;
    int id = -1;
    float ks = 0.0f, vs = 1.0f;
    auto fetch_pages = [&](int i) {                          // steps i .. i + 31
        id = -1;
        if (i + lane < mine) id = ids[(lo + ((i + lane) * kWarps + warp) * kStep) / a.page];
        if (id >= a.pages) id = -1;
        if (id >= 0) {
            ks = a.kscale[(long long)id * a.Hk + hk];
            vs = a.vscale[(long long)id * a.Hk + hk];
        }
    };
    auto load = [&](Step<D>& s, int i) {
        if ((i & 31) == 0) fetch_pages(i);
        const int page = __shfl_sync(0xffffffffu, id, i & 31);
        s.ks = __shfl_sync(0xffffffffu, ks, i & 31);
        const float v = __shfl_sync(0xffffffffu, vs, i & 31);
        s.lv = log2f(v);
        s.iv = 1.0f / v;
        s.at = lo + (i * kWarps + warp) * kStep;
        const int slot = s.at % a.page, live = page >= 0 && i < mine ? hi - s.at : 0;    // tokens of the step that count
        if (live <= 0) s.at = hi;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const unsigned char* at = a.kp + page * a.kps[0] + hk * a.kps[1] + (slot + 8 * n + g) * a.kps[2] + t * (D / 4);
            if (8 * n + g < live) {
                if constexpr (D == 64) {
                    const uint4 v = *reinterpret_cast<const uint4*>(at);
                    s.k[n][0] = v.x, s.k[n][1] = v.y, s.k[n][2] = v.z, s.k[n][3] = v.w;
                } else {
                    const uint2 v = *reinterpret_cast<const uint2*>(at);
                    s.k[n][0] = v.x, s.k[n][1] = v.y;
                }
            } else {
#pragma unroll
                for (int e = 0; e < D / 16; ++e) s.k[n][e] = 0u;
            }
        }
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const int token = 2 * t + (n & 1) + 8 * (n >> 1);
            const unsigned char* at = a.vp + page * a.vps[0] + hk * a.vps[1] + (slot + token) * a.vps[2] + g * (D / 8);
            if (token < live) {
                if constexpr (D == 64) {
                    const uint2 v = *reinterpret_cast<const uint2*>(at);
                    s.v[n][0] = v.x, s.v[n][1] = v.y;
                } else {
                    s.v[n][0] = *reinterpret_cast<const uint32_t*>(at);
                }
            } else {
#pragma unroll
                for (int e = 0; e < D / 32; ++e) s.v[n][e] = 0u;
            }
        }
    };
    auto work = [&](const Step<D>& s) {
        // scores: c[n][0..1] of row g and tokens 8 n + 2 t, + 1, c[n][2..3] of row g + 8
        float c[2][4];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            c[n][0] = c[n][1] = c[n][2] = c[n][3] = 0.0f;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                const uint32_t b0 = f16_of(s.k[n][kk]), b1 = f16_of(s.k[n][kk] >> 16);
                mma16816(c[n], qa[kk], b0, b1);
                if (PAIR) mma16816(c[n], ql[kk], b0, b1);
            }
        }
        const int live = hi - s.at;
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < (LOW ? 1 : 2); ++i) {
            const float f = s.ks * factor[i];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float& x = c[n][2 * i + e];
                    x = 8 * n + 2 * t + e < live ? fmaf(x, f, s.lv) : -INFINITY;
                    top[i] = fmaxf(top[i], x);
                }
        }
        bool grow = top[0] > m[0] + (kLift + kLag);
        if (!LOW) grow = grow || top[1] > m[1] + (kLift + kLag);
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
            for (int i = 0; i < (LOW ? 1 : 2); ++i) {
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
                const float now = fmaxf(m[i], top[i] - kLift), f = now == m[i] ? 1.0f : tcx::ex2_approx(m[i] - now);
                m[i] = now;
                l[i] *= f;
#pragma unroll
                for (int n = 0; n < DN; ++n) o[n][2 * i] *= f, o[n][2 * i + 1] *= f;
            }
        }
        uint32_t w[4] = {0u, 0u, 0u, 0u}, wl[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < (LOW ? 1 : 2); ++i) {
            const float base = m[i] == -INFINITY ? 0.0f : m[i];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const float x0 = tcx::ex2_approx(c[n][2 * i] - base), x1 = tcx::ex2_approx(c[n][2 * i + 1] - base);
                l[i] = fmaf(x0 + x1, s.iv, l[i]);
                w[2 * n + i] = pack_f16(x0, x1);
                if (PAIR) wl[2 * n + i] = rest_f16(x0, x1, w[2 * n + i]);
            }
        }
        // O += w V: register pairs (token 2 t, 2 t + 1) and (8 + 2 t, 9 + 2 t) of channel g D / 8 + n
#pragma unroll
        for (int q = 0; q < D / 32; ++q)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint32_t sel = half ? 0x7362u : 0x5140u;
                const uint32_t x = __byte_perm(s.v[0][q], s.v[1][q], sel), y = __byte_perm(s.v[2][q], s.v[3][q], sel);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t b0 = f16_of(k ? x >> 16 : x), b1 = f16_of(k ? y >> 16 : y);
                    float (&acc)[4] = o[4 * q + 2 * half + k];
                    mma16816(acc, w, b0, b1);
                    if (PAIR) mma16816(acc, wl, b0, b1);
                }
            }
    };
    Step<D> ring[kAhead + 1];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load(ring[i], i);
    for (int i = 0; i < mine; i += kAhead + 1) {
#pragma unroll
        for (int k = 0; k <= kAhead; ++k) {
            if (i + k >= mine) break;
            load(ring[(k + kAhead) % (kAhead + 1)], i + k + kAhead);
            work(ring[k]);
        }
    }

    // the warps' parts meet in shared memory
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
        float* to = part[warp][g + 8 * i];
        if (t == 0) to[D] = m[i], to[D + 1] = l[i];
#pragma unroll
        for (int n = 0; n < DN; ++n) {
            to[2 * t * (D / 8) + n] = o[n][2 * i];
            to[(2 * t + 1) * (D / 8) + n] = o[n][2 * i + 1];
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < rows * D; e += 32 * kWarps) {
        const int row = e / D, d = e - row * D;
        float M = -INFINITY, L = 0.0f, O = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, part[w][row][D]);
        const float base = M == -INFINITY ? 0.0f : M;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float f = tcx::ex2_approx(part[w][row][D] - base);
            L = fmaf(part[w][row][D + 1], f, L);
            O = fmaf(part[w][row][d], f, O);
        }
        if (a.splits > 1) {
            float* to = a.ws + (((long long)b * a.Hq + h0 + row) * a.splits + p) * (D + 2);
            to[d] = O;
            if (d == 0) to[D] = M, to[D + 1] = L;
        } else {
            const float v = L == 0.0f ? 0.0f : O / L;
            const long long at = b * a.os[0] + (h0 + row) * a.os[1] + d;
            if (PAIR) static_cast<float*>(a.o)[at] = v;
            else static_cast<__nv_bfloat16*>(a.o)[at] = __float2bfloat16_rn(v);
            if (d == 0 && a.lse) a.lse[(long long)b * a.Hq + h0 + row] = L == 0.0f ? -INFINITY : M * kLn2 + logf(L);
        }
    }
}

// Joins the parts of a row: a warp has one.
template <int D, bool F32>
__global__ void __launch_bounds__(128) paged_join_kernel(const PagedArgs a)
{
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    pdl_wait();
    if (row >= (long long)a.B * a.Hq) return;
    const int b = (int)(row / a.Hq), h = (int)(row - (long long)b * a.Hq);
    const Cut cut = cut_of(a, b);
    const float* from = a.ws + row * a.splits * (D + 2);
    float M = -INFINITY, L = 0.0f, O[D / 32];
#pragma unroll
    for (int e = 0; e < D / 32; ++e) O[e] = 0.0f;
    for (int p = lane; p < cut.parts; p += 32) M = fmaxf(M, from[p * (D + 2) + D]);
#pragma unroll
    for (int k = 16; k >= 1; k >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, k));
    const float base = M == -INFINITY ? 0.0f : M;
    for (int p = 0; p < cut.parts; ++p) {
        const float f = tcx::ex2_approx(from[p * (D + 2) + D] - base);
        L = fmaf(from[p * (D + 2) + D + 1], f, L);
#pragma unroll
        for (int e = 0; e < D / 32; ++e) O[e] = fmaf(from[p * (D + 2) + lane + 32 * e], f, O[e]);
    }
#pragma unroll
    for (int e = 0; e < D / 32; ++e) {
        const float v = L == 0.0f ? 0.0f : O[e] / L;
        const long long at = b * a.os[0] + h * a.os[1] + lane + 32 * e;
        if (F32) static_cast<float*>(a.o)[at] = v;
        else static_cast<__nv_bfloat16*>(a.o)[at] = __float2bfloat16_rn(v);
    }
    if (lane == 0 && a.lse) a.lse[row] = L == 0.0f ? -INFINITY : M * kLn2 + logf(L);
}

template <int D, bool PAIR> cudaError_t launch_t(const PagedArgs& a, cudaStream_t st)
{
    const int G = a.Hq / a.Hk, row_tiles = (G + 15) / 16;
    const unsigned ctas = (unsigned)((long long)a.splits * a.B * a.Hk * row_tiles);
    auto kernel = G <= 8 ? paged_attention_kernel<D, PAIR, true> : paged_attention_kernel<D, PAIR, false>;
    const cudaError_t e = launch_dependent(kernel, dim3(ctas), dim3(32 * kWarps), 0, st, a, row_tiles);
    if (e != cudaSuccess || a.splits == 1) return e;
    return launch_dependent(paged_join_kernel<D, PAIR>, dim3((unsigned)(((long long)a.B * a.Hq + 3) / 4)), dim3(128), 0, st, a);
}

}  // namespace

// Enough parts for sixteen CTAs per SM, none below kMinPart tokens.
int paged_splits(const PagedArgs& a)
{
    const long long units = (long long)a.B * a.Hk * ((a.Hq / a.Hk + 15) / 16), want = (16LL * a.sms + units - 1) / units;
    const long long most = ((long long)a.table_pages * a.page + kMinPart - 1) / kMinPart;
    return (int)std::max(1LL, std::min({want, most, 256LL}));
}

size_t paged_workspace_bytes(const PagedArgs& a)
{
    return a.splits > 1 ? (size_t)a.B * a.Hq * a.splits * (a.d + 2) * sizeof(float) : 0;
}

cudaError_t launch_paged_attention(const PagedArgs& a, cudaStream_t st)
{
    if (a.bf16) return a.d == 64 ? launch_t<64, false>(a, st) : launch_t<32, false>(a, st);
    return a.d == 64 ? launch_t<64, true>(a, st) : launch_t<32, true>(a, st);
}

}  // namespace lasad
