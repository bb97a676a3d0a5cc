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
// Bound by memory where prompts are long: k, v and q in, a byte a value and q out.  Prompts: a page's keys, or values, of some heads for a team of
// page / 16 warps, so that its maximum needs no second reading, the next head's rows on their way meanwhile; queries by CTAs of
// their own, eight heads at a time (8 x 9217 tokens, 24 query and 8 key heads, 680 MB: 139 us, 4.9 TB/s; four heads at a time 154;
// keys, then values, by the same warps and one query head at a time 326; fp32, 1284 MB: 236).  64 prompts of 1 to 577 tokens, 16 and 4
// heads, 104 MB: 31.5 us, 3.3 TB/s; the search for a row's sequence is little of that, as the same tokens of 8 sequences
// take 29.3 and of one 28.6.  One token per sequence: 3.9 us for 256 x 20 heads (by the prompts' kernel 11.6).
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
// sub * 8 .. + 7; as they come from memory, and in get() as the pairs' first channels x[0..3] and their partners x[4..7].
template <typename T, int D, bool HALF> struct Piece;
template <int D, bool HALF> struct Piece<__nv_bfloat16, D, HALF> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const __nv_bfloat16* row, int sub)
    {
        if (HALF) {
            const uint2 a = *reinterpret_cast<const uint2*>(row + sub * 4), b = *reinterpret_cast<const uint2*>(row + D / 2 + sub * 4);
            w[0] = a.x, w[1] = a.y, w[2] = b.x, w[3] = b.y;
        } else {
            const uint4 a = *reinterpret_cast<const uint4*>(row + sub * 8);
            w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
        }
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        using namespace tcx;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (HALF) x[2 * i] = bf16_lo(w[i]), x[2 * i + 1] = bf16_hi(w[i]);
            else x[i] = bf16_lo(w[i]), x[4 + i] = bf16_hi(w[i]);
        }
    }
};
template <int D, bool HALF> struct Piece<float, D, HALF> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* row, int sub)
    {
        a = *reinterpret_cast<const float4*>(row + (HALF ? sub * 4 : sub * 8));
        b = *reinterpret_cast<const float4*>(row + (HALF ? D / 2 + sub * 4 : sub * 8 + 4));
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        if (HALF) {
            x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
        } else {
            x[0] = a.x, x[4] = a.y, x[1] = a.z, x[5] = a.w, x[2] = b.x, x[6] = b.y, x[3] = b.z, x[7] = b.w;
        }
    }
};
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

// Rows of e4m3 numbers in 8 channels of a lane, times f (a power of two at most 1) and rounded again: slots slot, slot + by .. of
// those below n, a few of them in flight.
template <int kFlight>
__device__ __forceinline__ void round_again(unsigned char* dst, long long slots, int slot, int by, int n, float f)
{
    for (; slot < n; slot += by * kFlight) {
        uint2 old[kFlight];
#pragma unroll
        for (int k = 0; k < kFlight; ++k)
            if (slot + k * by < n) old[k] = *reinterpret_cast<const uint2*>(dst + (slot + k * by) * slots);
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
            if (slot + k * by >= n) break;
            uint32_t r[2] = {old[k].x, old[k].y};
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float2 u = from_e4m3(r[e] & 0xffffu), v = from_e4m3(r[e] >> 16);
                r[e] = to_e4m3(u.x * f, u.y * f) | to_e4m3(v.x * f, v.y * f) << 16;
            }
            *reinterpret_cast<uint2*>(dst + (slot + k * by) * slots) = make_uint2(r[0], r[1]);
        }
    }
}
__device__ __forceinline__ void turn_key(float (&x)[8], const float (&c)[4], const float (&s)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const double x0 = x[e], x1 = x[4 + e], cd = c[e], sd = s[e];
        x[e] = (float)(x0 * cd - x1 * sd);
        x[4 + e] = (float)(x0 * sd + x1 * cd);
    }
}

// One new token per sequence: a row of lanes has the key or value of one head, so a warp has D / 8 of them side by side,
// and what it reads of them is asked for before it is known where they go.
template <typename T, int D, bool HALF, bool TURN>
__device__ __forceinline__ void write_token(const PagedArgs& a, int cta)
{
    constexpr int LANES = D / 8, ROWS = 32 / LANES;
    const int lane = threadIdx.x & 31, sub = lane % LANES;
    const long long all = (long long)a.B * a.Hk, at = (long long)cta * kWarps * ROWS + threadIdx.x / LANES;
    const bool there = at < 2 * all;                                        // (all lanes stay for the shuffles)
    const int kv = at >= all, unit = there ? (int)(at - kv * all) : 0, b = unit / a.Hk, h = unit - b * a.Hk;
    Piece<T, D, HALF> piece;
    piece.load(static_cast<const T*>(kv && there ? a.v : a.k) + b * (kv && there ? a.vs[0] : a.ks[0]) + h * (kv && there ? a.vs[1] : a.ks[1]), sub);
    const int pos = a.pos[b], page = pos / a.page, slot = pos - page * a.page;
    bool live = there && pos >= 0 && page < a.table_pages;
    const int id = live ? a.block_table[(long long)b * a.table_pages + page] : -1;
    live = live && id >= 0 && id < a.pages;
    float* const scale = (kv ? a.vscale : a.kscale) + (long long)id * a.Hk + h;
    const float was = live && slot > 0 ? *scale : 0.0f;
    float x[8], size = 0.0f;
    piece.get(x);
    if (TURN && !kv && live) {
        float c[4], s[4];
        angles<D>(a, pos, sub, c, s);
        turn_key(x, c, s);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) size = fmaxf(size, finite_size(x[e]));
#pragma unroll
    for (int k = LANES / 2; k >= 1; k >>= 1) size = fmaxf(size, __shfl_xor_sync(0xffffffffu, size, k));
    const float now = fmaxf(power_of_two(scale_exponent(size)), was);       // (the shuffles say that all lanes have read it)
    unsigned char* const dst = kv ? a.vp + id * a.vps[0] + h * a.vps[1] : a.kp + id * a.kps[0] + h * a.kps[1];
    const long long slots = kv ? a.vps[2] : a.kps[2];
    if (live) {
        if (sub == 0) *scale = now;
        store_bytes<D, HALF>(dst + slot * slots, sub, x, 1.0f / now);
    }
    // where a scale has grown the whole warp rounds the earlier tokens again
    unsigned grown = __ballot_sync(0xffffffffu, live && slot > 0 && now > was && sub == 0);
    while (grown) {
        const int from = __ffs(grown) - 1;
        grown &= grown - 1;
        const unsigned long long page_at = __shfl_sync(0xffffffffu, (unsigned long long)dst, from);
        const long long by = __shfl_sync(0xffffffffu, slots, from);
        const int n = __shfl_sync(0xffffffffu, slot, from);
        const float f = __shfl_sync(0xffffffffu, was / now, from);
        round_again<4>(reinterpret_cast<unsigned char*>(page_at) + sub * 8, by, lane / LANES, ROWS, n, f);
    }
}

// A page's keys or values of some heads: `page` / kStep warps (a team), kStep tokens each; head after head, the next one's
// rows on their way while one is worked on.
template <typename T, int D, bool HALF, bool TURN>
__device__ __forceinline__ void write_page(const PagedArgs& a, int cta, int numbers, int per, int groups, float (&tops)[2][kWarps])
{
    constexpr int LANES = D / 8, ROWS = 32 / LANES, ACC = kStep / ROWS;     // lanes of a row, rows of an access, accesses
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % LANES, mine = lane / LANES;
    const int W = a.page / kStep, team = warp / W, w = warp - team * W;     // a page's warps
    // unit = (page number * groups + group of heads) * 2 + values
    int unit = cta * (kWarps / W) + team;
    const int kv = unit & 1;
    unit >>= 1;
    const int at = unit / groups, h0 = (unit - at * groups) * per, h1 = min(h0 + per, a.Hk);
    if (at >= numbers) return;
    // the page: of sequence b its page number j (see region_tiles for numbers without a table)
    int lo = 0, hi = a.B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (max(0, min(a.offsets[mid], a.N)) / a.page + 2 * mid <= at) lo = mid;
        else hi = mid;
    }
    const int b = lo, j = at - (max(0, min(a.offsets[b], a.N)) / a.page + 2 * b);
    if (j < 0) return;
    // its new tokens: their place in memory, their number and the first one's position
    const int from = max(0, min(a.offsets[b], a.N)), n = max(0, min(a.offsets[b + 1], a.N) - from);
    const long long pos = a.pos[b];
    if (pos < 0 || n == 0) return;
    const long long page0 = (pos / a.page + j) * a.page;                    // the position of the page's first slot
    if (page0 >= pos + n || page0 / a.page >= a.table_pages) return;
    const int id = a.block_table[(long long)b * a.table_pages + page0 / a.page];
    if (id < 0 || id >= a.pages) return;
    // slots first .. last - 1 are new; the row of slot 0
    const int first = (int)max(0LL, pos - page0), last = (int)min((long long)a.page, pos + n - page0);
    const long long row0 = from + (page0 - pos), stride = kv ? a.vs[0] : a.ks[0], next_head = kv ? a.vs[1] : a.ks[1];
    const T* src = static_cast<const T*>(kv ? a.v : a.k) + (row0 + w * kStep + mine) * stride;
    const long long slots = kv ? a.vps[2] : a.kps[2];
    auto fresh = [&](int i) {
        const int slot = w * kStep + i * ROWS + mine;
        return slot >= first && slot < last;
    };
    auto fetch = [&](Piece<T, D, HALF> (&to)[ACC], int h) {
#pragma unroll
        for (int i = 0; i < ACC; ++i)
            if (fresh(i)) to[i].load(src + i * ROWS * stride + h * next_head, sub);
    };
    Piece<T, D, HALF> now[ACC];
    fetch(now, h0);
    float c[ACC][4], s[ACC][4];
    if (TURN && kv == 0) {
#pragma unroll
        for (int i = 0; i < ACC; ++i) angles<D>(a, page0 + w * kStep + i * ROWS + mine, sub, c[i], s[i]);
    }
    for (int h = h0; h < h1; ++h) {
        float* scale = (kv ? a.vscale : a.kscale) + (long long)id * a.Hk + h;
        unsigned char* dst = kv ? a.vp + id * a.vps[0] + h * a.vps[1] : a.kp + id * a.kps[0] + h * a.kps[1];
        const float was = first > 0 ? *scale : 0.0f;
        Piece<T, D, HALF> next[ACC];
        if (h + 1 < h1) fetch(next, h + 1);
        float x[ACC][8], size = 0.0f;
#pragma unroll
        for (int i = 0; i < ACC; ++i) {
            if (!fresh(i)) continue;
            now[i].get(x[i]);
            if (TURN && kv == 0) turn_key(x[i], c[i], s[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) size = fmaxf(size, finite_size(x[i][e]));
        }
#pragma unroll
        for (int k = 16; k >= 1; k >>= 1) size = fmaxf(size, __shfl_xor_sync(0xffffffffu, size, k));
        if (W > 1) {
            // (two places in turn: who is a head ahead has met the others since they read this one's)
            float (&top)[kWarps] = tops[h & 1];
            if (lane == 0) top[warp] = size;
            asm volatile("barrier.cta.sync %0, %1;" ::"r"(1 + team), "r"(32 * W) : "memory");
            for (int k = 0; k < W; ++k) size = fmaxf(size, top[team * W + k]);
        } else {
            __syncwarp();                                                   // (everyone has read the scale)
        }
        const float now_s = fmaxf(power_of_two(scale_exponent(size)), was);
        if (w == 0 && lane == 0) *scale = now_s;
        if (first > 0 && now_s > was) round_again<1>(dst + sub * 8, slots, w * ROWS + mine, W * ROWS, first, was / now_s);
        const float inv = 1.0f / now_s;
#pragma unroll
        for (int i = 0; i < ACC; ++i) {
            if (fresh(i)) store_bytes<D, HALF>(dst + (w * kStep + i * ROWS + mine) * slots, sub, x[i], inv);
            now[i] = next[i];
        }
    }
}

// A row of lanes has a token and some of its query heads, kTogether at a time.
constexpr int kTogether = 8;
template <typename T, int D, bool HALF, bool TURN>
__device__ __forceinline__ void turn_queries(const PagedArgs& a, int cta, int per, int groups)
{
    constexpr int LANES = D / 8, ROWS = 32 / LANES;
    const int sub = threadIdx.x % LANES;
    const int group = cta % groups, h0 = group * per, h1 = min(h0 + per, a.Hq);
    const long long row = (long long)(cta / groups) * kWarps * ROWS + threadIdx.x / LANES;
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
    for (int h = h0; h < h1; h += kTogether) {
        Piece<T, D, HALF> piece[kTogether];
#pragma unroll
        for (int k = 0; k < kTogether; ++k)
            if (h + k < h1) piece[k].load(src + (h + k) * a.qs[1], sub);
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
            if (h + k >= h1) break;
            float x[8], y[8];
            piece[k].get(x);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[e] = live ? TURN ? x[e] * c[e] - x[4 + e] * s[e] : x[e] : 0.0f;
                y[4 + e] = live ? TURN ? x[e] * s[e] + x[4 + e] * c[e] : x[4 + e] : 0.0f;
            }
            store_pairs<T, D, HALF>(dst + (h + k) * a.qos[1], sub, y);
        }
    }
}

// How a launch is cut: CTAs for pages, then CTAs for queries.
struct Plan {
    int page_ctas, numbers, kv_per, kv_groups, q_per, q_groups;
};

// STEP: one token per sequence.  (Two CTAs have an SM: with one, prompts of 8 x 9217 tokens take 250 us instead of 140.)
template <typename T, int D, bool HALF, bool TURN, bool STEP>
__global__ void __launch_bounds__(32 * kWarps, 2) paged_append_kernel(const PagedArgs a, const Plan plan)
{
    __shared__ float tops[2][kWarps];
    pdl_wait();
    if ((int)blockIdx.x < plan.page_ctas) {
        if constexpr (STEP) write_token<T, D, HALF, TURN>(a, blockIdx.x);
        else write_page<T, D, HALF, TURN>(a, blockIdx.x, plan.numbers, plan.kv_per, plan.kv_groups, tops);
    } else turn_queries<T, D, HALF, TURN>(a, blockIdx.x - plan.page_ctas, plan.q_per, plan.q_groups);
}

// Of n heads as many for a warp as leave 32 warps per SM when all tokens' take `warps` a head group.
int heads_per(int n, long long warps, int sms)
{
    const long long groups = (32LL * sms + warps - 1) / warps;
    return groups >= n ? 1 : (int)((n + groups - 1) / groups);
}

template <typename T, int D> cudaError_t launch_t(const PagedArgs& a, cudaStream_t st)
{
    const int team = a.page / kStep, per_cta = kWarps / team;
    constexpr int rows = kWarps * 32 / (D / 8);
    Plan plan{};
    // pages that a sequence of n new tokens touches: at most n / page + 2, and none is numbered twice
    plan.numbers = a.N / a.page + 2 * a.B;
    plan.kv_per = heads_per(a.Hk, 2LL * plan.numbers * team, a.sms);
    plan.kv_groups = (a.Hk + plan.kv_per - 1) / plan.kv_per;
    plan.q_per = heads_per(a.Hq, (a.N + rows / kWarps - 1) / (rows / kWarps), a.sms);
    plan.q_per = (plan.q_per + kTogether - 1) / kTogether * kTogether;
    plan.q_groups = (a.Hq + plan.q_per - 1) / plan.q_per;
    plan.page_ctas = a.offsets ? (int)((2LL * plan.numbers * plan.kv_groups + per_cta - 1) / per_cta) : (int)((2LL * a.B * a.Hk + rows - 1) / rows);
    const long long ctas = plan.page_ctas + (a.q ? ((long long)a.N + rows - 1) / rows * plan.q_groups : 0);
    auto kernel = a.offsets ? (a.table ? (a.half ? paged_append_kernel<T, D, true, true, false> : paged_append_kernel<T, D, false, true, false>)
                                       : paged_append_kernel<T, D, false, false, false>)
                            : (a.table ? (a.half ? paged_append_kernel<T, D, true, true, true> : paged_append_kernel<T, D, false, true, true>)
                                       : paged_append_kernel<T, D, false, false, true>);
    return launch_dependent(kernel, dim3((unsigned)ctas), dim3(32 * kWarps), 0, st, a, plan);
}

}  // namespace

cudaError_t launch_paged_append(const PagedArgs& a, cudaStream_t st)
{
    if (a.bf16) return a.d == 64 ? launch_t<__nv_bfloat16, 64>(a, st) : launch_t<__nv_bfloat16, 32>(a, st);
    return a.d == 64 ? launch_t<float, 64>(a, st) : launch_t<float, 32>(a, st);
}

}  // namespace lasad
