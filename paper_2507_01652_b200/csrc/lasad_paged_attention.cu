// One token per sequence against a paged cache in 8 bits (e4m3 numbers c with one scale s per page and head, x = c s):
//
//     o = sum_j p_j v_j ,   p_j = e^(scale q.k_j) / sum   over the tokens 0 .. pos of the sequence.
//
// Bound by reading the cache once, 2 d bytes a token and key head.  A warp takes steps of 16 tokens, copied to shared
// memory three (d = 64) or seven steps ahead, and from there into the fragments of two products on mma.sync.m16n8k16:
// tokens are the rows of the first, channels those of the second; the columns are the query heads that share the key
// head, 8 at a time, of which few are used, so the tensor cores have time to spare and tcgen05's 128 rows
// would only be emptier.  e4m3 numbers are exact in fp16, so keys and values enter without a rounding; the page's key
// scale multiplies the fp32 score.  The order of a product's inner index is free, and so is that of its rows, so a lane
// reads 16 neighbouring channels of a key and 8 of a value.
// Measured: 64 sequences of 9217 tokens, 24 query and 8 key heads: 5.9 TB/s (loads into registers three steps ahead, which
// were waited for all the same, 4.65; twice as many steps on their way 5.3); of 1 to 9217
// tokens 64.8 us, 4.7 TB/s.
//
// The page's value scale goes into the exponent: with x_j = scale q.k_j log2(e) + log2 s_j a warp sums
//
//     O = sum_j w_j c_j ,  l = sum_j w_j / s_j ,   w_j = 2^(x_j - M) ,      o = O / l ,  lse = (M + log2 l) ln 2
//
// so that w stays in the range of fp16 however far the scales of two pages are apart.  M lies 11 below a lagging
// maximum, which moves only when some row has grown by more than 4: w is at most 2^15, and it keeps its eleven
// digits down to 2^-25 of the largest and some down to 2^-35.  w is rounded to fp16 (2^-11 of each term) where q is bf16;
// where q is fp32, q and w enter as sums of two fp16 numbers (22 bits).  q is brought near 1 by a power of two first,
// so that fp16 holds it.
//
// The tokens of a sequence are cut into parts where there are few (sequence, key head) pairs; then the parts'
// (M, l, O) go to memory and a second kernel joins them (2 x 24 heads of 8 key heads, 9217 tokens: 9.5 us; joined by the
// CTAs of a cluster in shared memory 12.7, where two kernels then took 11.6).  Twice or half as many parts: 69.4 or 66.7 us
// for 64 sequences of 1 to 9217 tokens, as it is 64.8.  Where there are many pairs a warp has one (256 x 20 heads, up to
// 577 tokens: 40.6 us; four warps 49.6), and then the order of the lengths counts: 40.6 and 39.4 us where they ascend and
// descend, 46.4 shuffled, 36.0 for as many tokens in equal sequences (cut into parts, 64 sequences of 1 to 9217: 64.7, 63.9,
// 64.6, 59.2).  fp32 queries: 43.7 and 71.5 us for the two.
#include "lasad_full.cuh"
#include "lasad_tc_ptx.cuh"
#include "lasad_tc_tma.cuh"

#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

namespace lasad {
namespace {

constexpr int kCtaWarps = 4, kStep = 16, kMinPart = 256;  // kMinPart: tokens of a part, at least
constexpr int kColTiles = 3;                              // columns of a warp: at most 24 query heads
constexpr float kLift = 11.0f, kLag = 4.0f;               // of the largest x over M; how far it may be over that
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816_new(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
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
// An 8 x 8 tile of fp16 numbers, lane 4 i + j with (i, 2 j) and (i, 2 j + 1), turned over.
__device__ __forceinline__ uint32_t transposed(uint32_t x)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
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

// A step in shared memory: rows of D bytes, the 16-byte pieces of 64-byte rows turned by half the row's number, so that what
// the lanes of a quarter warp read lies in different banks.
template <int D> struct Step {
    unsigned char k[kStep * D], v[kStep * D];
};
template <int D> __device__ __forceinline__ int piece_at(int row, int piece)
{
    return row * D + (D == 64 ? ((piece + (row >> 1)) & 3) * 16 : piece * 16);
}
// The token that row i of a product's tile of 8 stands for (the order is free): what a lane reads of the values, tokens
// 2 t, 2 t + 1 of 8, then meets no bank twice, and neither do two neighbouring rows of the keys.
__device__ __forceinline__ int token_of(int i) { return i ^ ((i >> 1) & 1); }

// 16 bytes to shared memory, or zeros
__device__ __forceinline__ void copy16(void* to, const unsigned char* from, bool live)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tcx::smem_u32(to)), "l"(from), "r"(live ? 16 : 0) : "memory");
}

// A unit is a sequence, a key head, up to 8 NR of its query heads and a part of the tokens; WARPS warps have it.  PAIR:
// fp32 queries.
template <int D, bool PAIR, int NR, int WARPS>
__global__ void __launch_bounds__(32 * kCtaWarps) paged_attention_kernel(const PagedArgs a, int col_blocks)
{
    constexpr int KK = D / 16;                               // inner steps of q.k; words of a lane's key piece
    constexpr int MT = D / 16;                               // row tiles of O
    constexpr int DEPTH = 256 / D;                           // steps of a warp in shared memory (8 KB)
    extern __shared__ __align__(16) unsigned char steps_raw[];
    static_assert(8 * NR * (D + 2) * 4 <= DEPTH * sizeof(Step<D>), "a warp's part of the result takes the place of its steps");
    auto part = reinterpret_cast<float (*)[8 * NR][D + 2]>(steps_raw);
    const int lane = threadIdx.x & 31, warp = WARPS > 1 ? threadIdx.x >> 5 : 0, g = lane >> 2, t = lane & 3;
    const int G = a.Hq / a.Hk;
    // unit = ((part * B + sequence) * Hk + key head) * col_blocks + block of query heads
    long long unit = WARPS > 1 ? blockIdx.x : (long long)blockIdx.x * kCtaWarps + (threadIdx.x >> 5);
    const int cb = (int)(unit % col_blocks);
    unit /= col_blocks;
    const int hk = (int)(unit % a.Hk);
    unit /= a.Hk;
    const int b = (int)(unit % a.B), p = (int)(unit / a.B);
    const int heads = min(8 * NR, G - cb * 8 * NR), h0 = hk * G + cb * 8 * NR;
    pdl_wait();
    if (p >= a.splits) return;                               // (behind the last unit)
    const Cut cut = cut_of(a, b);
    if (p >= max(cut.parts, 1)) return;
    const int lo = p * cut.size, hi = min(cut.n, lo + cut.size);

    // The warp's steps: number i is at lo + (i WARPS + warp) kStep.  Pages and scales of 32 of them are fetched at a
    // time, one by each lane, a batch ahead of the one that is worked on.
    const int steps = (max(hi - lo, 0) + kStep - 1) / kStep, mine = (steps - warp + WARPS - 1) / WARPS;
    const int* ids = a.block_table + (long long)b * a.table_pages;
    struct Pages {
        uint32_t k, v;                                       // where the step's keys and values begin, in 16 bytes; k of no page: kNone
        float ks, vs;                                        // the scales
    };
    constexpr uint32_t kNone = 0xffffffffu;
    auto fetch_pages = [&](int i) {                          // of steps i .. i + 31
        Pages f{kNone, 0u, 0.0f, 1.0f};
        const int at = lo + ((i + lane) * WARPS + warp) * kStep;
        int id = -1;
        if (i + lane < mine) id = ids[at / a.page];
        if (id >= 0 && id < a.pages) {
            const int slot = at & (a.page - 1);
            f.k = (uint32_t)((id * a.kps[0] + slot * a.kps[2]) >> 4);
            f.v = (uint32_t)((id * a.vps[0] + slot * a.vps[2]) >> 4);
            f.ks = a.kscale[(long long)id * a.Hk + hk];
            f.vs = a.vscale[(long long)id * a.Hk + hk];
        }
        return f;
    };
    Pages now = fetch_pages(0), next = fetch_pages(32);
    int batch = 0;                                           // the first step of `now`
    // A lane copies pieces of 16 bytes: of keys and values 32 at a time, rows row0, row0 + ROWS ..
    constexpr int PIECES = D / 16, ROWS = 32 / PIECES;
    Step<D>* const ring = reinterpret_cast<Step<D>*>(steps_raw) + (threadIdx.x >> 5) * DEPTH;
    const int row0 = lane / PIECES, piece = lane % PIECES;
    const unsigned char* const at_k = a.kp + hk * a.kps[1] + row0 * a.kps[2] + piece * 16;
    const unsigned char* const at_v = a.vp + hk * a.vps[1] + row0 * a.vps[2] + piece * 16;
    const long long next_k = ROWS * a.kps[2], next_v = ROWS * a.vps[2];
    auto load = [&](int i) {
        const uint32_t from_k = __shfl_sync(0xffffffffu, i - batch < 32 ? now.k : next.k, i & 31);
        const uint32_t from_v = __shfl_sync(0xffffffffu, i - batch < 32 ? now.v : next.v, i & 31);
        if (i < mine) {
            // (what does not count is 0, whatever stands there: a weight of 0 times a NaN is not 0)
            const int live = from_k != kNone ? hi - (lo + (i * WARPS + warp) * kStep) : 0;
            const unsigned char* k = at_k + (live > 0 ? from_k : 0) * 16ull;
            const unsigned char* v = at_v + (live > 0 ? from_v : 0) * 16ull;
            Step<D>& s = ring[i & (DEPTH - 1)];
#pragma unroll
            for (int n = 0; n < kStep / ROWS; ++n) {
                const int row = row0 + n * ROWS;
                copy16(s.k + piece_at<D>(row, piece), k + n * next_k, row < live);
                copy16(s.v + piece_at<D>(row, piece), v + n * next_v, row < live);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < DEPTH - 1; ++i) load(i);

    // q as fp16 fragments: inner step kk, register r: column g (query head), channels t D / 4 + 4 kk + 2 r and the next
    uint32_t qb[NR][KK][2], ql[PAIR ? NR : 1][PAIR ? KK : 1][2];
    float mine_factor[NR];                                   // scale log2(e) and what q was divided by, of column g
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        float x[D / 4], top = 0.0f;
#pragma unroll
        for (int e = 0; e < D / 4; ++e) x[e] = 0.0f;
        if (8 * n + g < heads) {
            const long long at = b * a.qs[0] + (h0 + 8 * n + g) * a.qs[1] + t * (D / 4);
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
        mine_factor[n] = a.scale * kLog2e * __uint_as_float((uint32_t)(127 + e2) << 23);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float u = x[4 * kk + 2 * r] * down, v = x[4 * kk + 2 * r + 1] * down;
                qb[n][kk][r] = pack_f16(u, v);
                if (PAIR) ql[n][kk][r] = rest_f16(u, v, qb[n][kk][r]);
            }
    }
    // scores have columns 2 t and 2 t + 1 (i) in a lane
    float factor[NR][2], M[NR][2], l[NR][2], o[NR][MT][4];   // (M is -infinity until a row has seen something)
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            factor[n][i] = __shfl_sync(0xffffffffu, mine_factor[n], 4 * (2 * t + i));
            M[n][i] = -INFINITY;
            l[n][i] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < MT; ++k) o[n][k][0] = o[n][k][1] = o[n][k][2] = o[n][k][3] = 0.0f;
    }

    float lv = log2f(now.vs), iv = 1.0f / now.vs;            // of the value scales: log2 and reciprocal
    auto live_of = [&](int i) { return now.k == kNone ? 0 : hi - (lo + ((i + lane) * WARPS + warp) * kStep); };
    int lives = live_of(0);                                  // tokens that count
    // a lane's places in a step: keys of tokens g and 8 + g, values of tokens 2 t, 2 t + 1 and 8 further
    const int at_key = D == 64 ? piece_at<D>(token_of(g), t) : token_of(g) * D + t * 8;
    const int at_value0 = D == 64 ? piece_at<D>(token_of(2 * t), g >> 1) + (g & 1) * 8 : token_of(2 * t) * D + g * 4;
    const int at_value1 = D == 64 ? piece_at<D>(token_of(2 * t + 1), g >> 1) + (g & 1) * 8 : token_of(2 * t + 1) * D + g * 4;
    auto work = [&](int i) {
        struct {
            uint32_t k[2][D / 16], v[4][D / 32];
        } s;
        const Step<D>& from = ring[i & (DEPTH - 1)];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            if constexpr (D == 64) {
                const uint4 x = *reinterpret_cast<const uint4*>(from.k + at_key + 8 * n * D);
                s.k[n][0] = x.x, s.k[n][1] = x.y, s.k[n][2] = x.z, s.k[n][3] = x.w;
                const uint2 y = *reinterpret_cast<const uint2*>(from.v + at_value0 + 8 * n * D);
                const uint2 z = *reinterpret_cast<const uint2*>(from.v + at_value1 + 8 * n * D);
                s.v[2 * n][0] = y.x, s.v[2 * n][1] = y.y, s.v[2 * n + 1][0] = z.x, s.v[2 * n + 1][1] = z.y;
            } else {
                const uint2 x = *reinterpret_cast<const uint2*>(from.k + at_key + 8 * n * D);
                s.k[n][0] = x.x, s.k[n][1] = x.y;
                s.v[2 * n][0] = *reinterpret_cast<const uint32_t*>(from.v + at_value0 + 8 * n * D);
                s.v[2 * n + 1][0] = *reinterpret_cast<const uint32_t*>(from.v + at_value1 + 8 * n * D);
            }
        }
        const float step_ks = __shfl_sync(0xffffffffu, now.ks, i & 31), step_lv = __shfl_sync(0xffffffffu, lv, i & 31);
        const float step_iv = __shfl_sync(0xffffffffu, iv, i & 31);
        const int step_live = __shfl_sync(0xffffffffu, lives, i & 31);
        // scores: c[0..1] of token g, c[2..3] of token 8 + g
        float c[NR][4];
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            const uint32_t f[4] = {f16_of(s.k[0][kk]), f16_of(s.k[1][kk]), f16_of(s.k[0][kk] >> 16), f16_of(s.k[1][kk] >> 16)};
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                if (kk == 0) mma16816_new(c[n], f, qb[n][kk][0], qb[n][kk][1]);
                else mma16816(c[n], f, qb[n][kk][0], qb[n][kk][1]);
                if (PAIR) mma16816(c[n], f, ql[n][kk][0], ql[n][kk][1]);
            }
        }
        // c becomes x - M; over kLift + kLag somewhere, M moves
        bool grow = false;
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float f = step_ks * factor[n][e], base = step_lv - (M[n][e] == -INFINITY ? 0.0f : M[n][e]);
                c[n][e] = fmaf(c[n][e], f, base);
                c[n][2 + e] = fmaf(c[n][2 + e], f, base);
                grow = grow || M[n][e] == -INFINITY || fmaxf(c[n][e], c[n][2 + e]) > kLift + kLag;
            }
        if (step_live < kStep) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (token_of(g) + 8 * (e >> 1) >= step_live) c[n][e] = -INFINITY;
        }
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = fmaxf(c[n][e], c[n][2 + e]);
#pragma unroll
                    for (int k = 4; k <= 16; k <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
                    // (top is over M, or over 0 where there is none yet)
                    const float old = M[n][e], was = old == -INFINITY ? 0.0f : old;
                    if (top == -INFINITY || (old != -INFINITY && top <= kLift)) continue;
                    M[n][e] = was + (top - kLift);
                    const float f = old == -INFINITY ? 0.0f : tcx::ex2_approx(old - M[n][e]);
                    c[n][e] -= M[n][e] - was, c[n][2 + e] -= M[n][e] - was;
                    l[n][e] *= f;
#pragma unroll
                    for (int k = 0; k < MT; ++k) o[n][k][e] *= f, o[n][k][2 + e] *= f;
                }
        }
        uint32_t w[NR][2], wl[PAIR ? NR : 1][2];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float x0 = tcx::ex2_approx(c[n][2 * k]), x1 = tcx::ex2_approx(c[n][2 * k + 1]);
                l[n][0] = fmaf(x0, step_iv, l[n][0]);
                l[n][1] = fmaf(x1, step_iv, l[n][1]);
                const uint32_t packed = pack_f16(x0, x1);
                w[n][k] = transposed(packed);                // tokens 8 k + 2 t, + 1 of column g
                if (PAIR) wl[n][k] = transposed(rest_f16(x0, x1, packed));
            }
        }
        // O += V^T w: row tile 2 q + half has channels g D / 8 + 4 q + 2 half (rows g) and the next (rows 8 + g)
#pragma unroll
        for (int q = 0; q < D / 32; ++q)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint32_t sel = half ? 0x7362u : 0x5140u;
                const uint32_t x = __byte_perm(s.v[0][q], s.v[1][q], sel), y = __byte_perm(s.v[2][q], s.v[3][q], sel);
                const uint32_t f[4] = {f16_of(x), f16_of(x >> 16), f16_of(y), f16_of(y >> 16)};
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    mma16816(o[n][2 * q + half], f, w[n][0], w[n][1]);
                    if (PAIR) mma16816(o[n][2 * q + half], f, wl[n][0], wl[n][1]);
                }
            }
    };
    for (int i = 0; i < mine; ++i) {
        if (i - batch == 32) {
            now = next;
            batch = i;
            lv = log2f(now.vs), iv = 1.0f / now.vs, lives = live_of(i);
            next = fetch_pages(i + 32);
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 2) : "memory");
        __syncwarp();                                        // (step i is there, and step i - 1 has been read by all lanes)
        load(i + DEPTH - 1);
        work(i);
    }
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int k = 4; k <= 16; k <<= 1) l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], k);

    // M, l and O of query head `col` of the unit's: a lane has E neighbouring channels from d on
    auto finish = [&](int col, int d, float M, float L, const float* O, auto count) {
        constexpr int E = decltype(count)::value;
        const int h = h0 + col;
        if (a.splits > 1) {
            float* to = a.ws + (((long long)b * a.Hq + h) * a.splits + p) * (D + 2);
#pragma unroll
            for (int e = 0; e < E; e += 2) *reinterpret_cast<float2*>(to + d + e) = make_float2(O[e], O[e + 1]);
            if (d == 0) *reinterpret_cast<float2*>(to + D) = make_float2(M, L);
            return;
        }
        const float inv = L == 0.0f ? 0.0f : 1.0f / L;
        const long long at = b * a.os[0] + h * a.os[1] + d;
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const float x = L == 0.0f ? 0.0f : O[e] * inv, y = L == 0.0f ? 0.0f : O[e + 1] * inv;
            if (PAIR) *reinterpret_cast<float2*>(static_cast<float*>(a.o) + at + e) = make_float2(x, y);
            else *reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(a.o) + at + e) = tcx::pack_bf16(x, y);
        }
        if (d == 0 && a.lse) a.lse[(long long)b * a.Hq + h] = L == 0.0f ? -INFINITY : M * kLn2 + logf(L);
    };
    if (WARPS > 1) __syncthreads();                          // (their steps have been read)
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float x[D / 8];                                  // channels g D / 8 .. of column 8 n + 2 t + i
#pragma unroll
            for (int k = 0; k < MT; ++k) x[2 * k] = o[n][k][i], x[2 * k + 1] = o[n][k][2 + i];
            const int col = 8 * n + 2 * t + i;
            if (WARPS == 1) {
                if (col < heads) finish(col, g * (D / 8), M[n][i], l[n][i], x, std::integral_constant<int, D / 8>{});
            } else {
                float* to = part[warp][col];
#pragma unroll
                for (int e = 0; e < D / 8; e += 2) *reinterpret_cast<float2*>(to + g * (D / 8) + e) = make_float2(x[e], x[e + 1]);
                if (g == 0) *reinterpret_cast<float2*>(to + D) = make_float2(M[n][i], l[n][i]);
            }
        }
    if (WARPS == 1) return;
    // the warps' parts meet in shared memory
    __syncthreads();
    for (int e = threadIdx.x; e < heads * (D / 2); e += 32 * WARPS) {
        const int col = e / (D / 2), d = 2 * (e - col * (D / 2));
        float M = -INFINITY, L = 0.0f, O[2] = {0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < WARPS; ++w) M = fmaxf(M, part[w][col][D]);
        const float base = M == -INFINITY ? 0.0f : M;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float f = tcx::ex2_approx(part[w][col][D] - base);
            L = fmaf(part[w][col][D + 1], f, L);
            O[0] = fmaf(part[w][col][d], f, O[0]);
            O[1] = fmaf(part[w][col][d + 1], f, O[1]);
        }
        finish(col, d, M, L, O, std::integral_constant<int, 2>{});
    }
}

// Joins the parts of a row: a CTA has one, its warps every eighth part each.  The first kBatch of a warp's are asked for
// before it is known how many there are (what stands in the others is not used).
constexpr int kJoinWarps = 8, kBatch = 4;
template <int D, bool F32>
__global__ void __launch_bounds__(32 * kJoinWarps) paged_join_kernel(const PagedArgs a)
{
    constexpr int E = D / 32;
    __shared__ float tops[kJoinWarps], sums[kJoinWarps][D + 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int b = blockIdx.x / a.Hq, h = blockIdx.x - b * a.Hq;
    const float* from = a.ws + (long long)blockIdx.x * a.splits * (D + 2);
    float M = -INFINITY, L = 0.0f, O[E];
#pragma unroll
    for (int e = 0; e < E; ++e) O[e] = 0.0f;
    pdl_wait();
    int parts = a.splits;
    for (int p0 = warp; p0 < parts; p0 += kJoinWarps * kBatch) {
        float m[kBatch], l[kBatch], o[kBatch][E];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const float* at = from + min(p0 + k * kJoinWarps, a.splits - 1) * (D + 2);
            const float2 ml = *reinterpret_cast<const float2*>(at + D);
            m[k] = ml.x, l[k] = ml.y;
#pragma unroll
            for (int e = 0; e < E; ++e) o[k][e] = at[lane * E + e];
        }
        if (p0 == warp) parts = cut_of(a, b).parts;
        float top = M;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (p0 + k * kJoinWarps >= parts) {              // (memory that nobody has written)
                m[k] = -INFINITY, l[k] = 0.0f;
#pragma unroll
                for (int e = 0; e < E; ++e) o[k][e] = 0.0f;
            }
            top = fmaxf(top, m[k]);
        }
        // (a part without a maximum is added, too: its sums are 0, or NaN where its scores are, and that has to stay)
        const float base = top == -INFINITY ? 0.0f : top, f0 = tcx::ex2_approx(M - base);
        M = top;
        L *= f0;
#pragma unroll
        for (int e = 0; e < E; ++e) O[e] *= f0;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const float f = tcx::ex2_approx(m[k] - base);
            L = fmaf(l[k], f, L);
#pragma unroll
            for (int e = 0; e < E; ++e) O[e] = fmaf(o[k][e], f, O[e]);
        }
    }
    if (lane == 0) tops[warp] = M, sums[warp][D] = L;
#pragma unroll
    for (int e = 0; e < E; ++e) sums[warp][lane * E + e] = O[e];
    __syncthreads();
    if (threadIdx.x >= D) return;
    const int d = threadIdx.x;
    M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) M = fmaxf(M, tops[w]);
    const float base = M == -INFINITY ? 0.0f : M;
    float x = 0.0f;
    L = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) {
        const float f = tcx::ex2_approx(tops[w] - base);
        x = fmaf(sums[w][d], f, x), L = fmaf(sums[w][D], f, L);
    }
    const float v = L == 0.0f ? 0.0f : x / L;
    const long long at = b * a.os[0] + h * a.os[1] + d;
    if (F32) static_cast<float*>(a.o)[at] = v;
    else static_cast<__nv_bfloat16*>(a.o)[at] = __float2bfloat16_rn(v);
    if (d == 0 && a.lse) a.lse[blockIdx.x] = L == 0.0f ? -INFINITY : M * kLn2 + logf(L);
}

long long units_of(const PagedArgs& a) { return (long long)a.B * a.Hk * ((a.Hq / a.Hk + 8 * kColTiles - 1) / (8 * kColTiles)); }
// A warp for a unit where there are enough of them to fill the SMs, else a CTA of four.
bool solo(const PagedArgs& a) { return a.splits == 1 && units_of(a) >= 16LL * a.sms; }

template <int D, bool PAIR, int NR> cudaError_t launch_n(const PagedArgs& a, cudaStream_t st)
{
    constexpr size_t smem = (size_t)kCtaWarps * (256 / D) * sizeof(Step<D>);
    const long long units = units_of(a) * a.splits;
    const int blocks = (a.Hq / a.Hk + 8 * kColTiles - 1) / (8 * kColTiles);
    static bool done1[64], done2[64];
    cudaError_t e = tcx::allow_dynamic_smem(paged_attention_kernel<D, PAIR, NR, 1>, smem, done1);
    if (e == cudaSuccess) e = tcx::allow_dynamic_smem(paged_attention_kernel<D, PAIR, NR, kCtaWarps>, smem, done2);
    if (e != cudaSuccess) return e;
    if (solo(a))
        return launch_dependent(paged_attention_kernel<D, PAIR, NR, 1>, dim3((unsigned)((units + kCtaWarps - 1) / kCtaWarps)),
                                dim3(32 * kCtaWarps), smem, st, a, blocks);
    return launch_dependent(paged_attention_kernel<D, PAIR, NR, kCtaWarps>, dim3((unsigned)units), dim3(32 * kCtaWarps), smem, st, a, blocks);
}
template <int D, bool PAIR> cudaError_t launch_t(const PagedArgs& a, cudaStream_t st)
{
    const int G = a.Hq / a.Hk;
    const cudaError_t e = G <= 8 ? launch_n<D, PAIR, 1>(a, st) : G <= 16 ? launch_n<D, PAIR, 2>(a, st) : launch_n<D, PAIR, kColTiles>(a, st);
    if (e != cudaSuccess || a.splits == 1) return e;
    return launch_dependent(paged_join_kernel<D, PAIR>, dim3((unsigned)((long long)a.B * a.Hq)), dim3(32 * kJoinWarps), 0, st, a);
}

}  // namespace

// Enough parts for sixteen CTAs per SM, none below kMinPart tokens; a short table is not cut (a second launch costs what a
// CTA does in four parts' time).
int paged_splits(const PagedArgs& a)
{
    const long long units = units_of(a), tokens = (long long)a.table_pages * a.page, want = (16LL * a.sms + units - 1) / units;
    if (tokens <= 4 * kMinPart) return 1;
    return (int)std::max(1LL, std::min({want, (tokens + kMinPart - 1) / kMinPart, 256LL}));
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
