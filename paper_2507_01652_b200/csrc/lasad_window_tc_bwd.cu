// Gradient of the window attention on the tensor cores (bf16), in two kernels of one form:
//
//     keys:     a CTA has 128 keys of one key head and goes over the queries that see them
//     queries:  a CTA has 128 queries of one head and goes over the keys that they see
//
// so that every sum stays in one CTA (no atomics: results repeat bit for bit, and the heads that
// share a key head are added in order).  With X1, X2 the CTA's own rows (K, V or Q, dO) and Y1, Y2 a
// tile of 64 rows that it passes (Q, dO or K, V), a tile costs the products
//
//     S = X1 Y1^T ,  dP = X2 Y2^T ,        P = 2^(S c - lse log2(e)) ,  dS = P * (dP - Delta)
//     A1 += dS Y1  (dK or dQ) ,            keys only: A2 += P Y2  (dV)
//
// all of them tcgen05 128 x 64 x 64 with the left operand in TMEM: X1 and X2 are put there once, and P
// and dS are written over S and dP.  (A left operand from shared memory would cost 4 KB beside the 2 KB
// of the right one per 32-clock instruction, more than the 128 bytes per clock that an SM reads.)
// scale is applied to dK and dQ once, at the end.  Delta and, for the keys of the sinks, the sums
// over the queries whose window has left them come from launch_window_prep.
//
// What bounds it: per tile 512 clocks of exponentials (16 per SM and clock) against four (three)
// products of 128 clocks.  Two groups of eight warps take the tiles in turn, each with its own S
// and dP columns, so that one group's exponentials run under the other's products: 448 (384) of
// the SM's 512 TMEM columns, one CTA per SM.  Against one kernel that makes all five products once
// and adds dQ by atomics this makes S, dP and P twice; it buys results that repeat, and no 32-bit dQ in
// memory.
//
// Warps 0-7 and 8-15: the two groups, two threads per own row, 32 of a tile's 64 columns each (a
// group of four warps with 64 columns each left a scheduler two warps, too few to hide the
// latency of TMEM and of the exponentials).  Warp 16: MMA issue.  Warp 17: TMA.
#include "lasad_window_tma.cuh"

namespace lasad {
namespace {

using namespace tcx;

constexpr int kRows = 128, kCols = 64, kStages = 4, kGroup = 256, kThreads = 2 * kGroup + 64;
constexpr int kTile = kCols * 128;                         // bytes of a passing tile
constexpr uint32_t kColX1 = 0, kColX2 = 32, kColS = 64, kColDP = 128, kGroupCols = 128, kColA1 = 320, kColA2 = 384;
constexpr int kTmemCols = 512;

struct Smem {
    unsigned char y1[kStages][kTile];
    unsigned char y2[kStages][kTile];
    float lse[2][2][kCols], delta[2][2][kCols];            // keys: of each group's tiles, by column, two in turn
    unsigned long long full[kStages], free[kStages];       // Y1 and Y2 have landed; their products have been made
    unsigned long long x_ready;                            // X1 and X2 are in TMEM (2 kGroup arrivals)
    unsigned long long s_full[2];                          // S and dP of a group's tile are there (and all products before are done)
    unsigned long long p_ready[2];                         // P and dS are (kGroup arrivals)
    unsigned long long st_ready[2];                        // keys: lse and delta are (kGroup arrivals)
    unsigned long long done, drain;
    uint32_t tmem_base;
    int abort_flag;
};

struct Params {
    int B, T, Hq, Hk, d, window, sinks;
    float scale, scale2;                                   // scale2 = scale log2(e)
    const int* lengths;
    const float* lse;
    const float* delta;
    const float* sums;                                     // keys: of the sinks, [B,Hk,chunks,sinks,2,d]
    const __nv_bfloat16* x1;
    const __nv_bfloat16* x2;
    long long x1s[3], x2s[3];
    __nv_bfloat16* a1;
    __nv_bfloat16* a2;
    long long a1s[3], a2s[3];
    int* status;
    unsigned wait_limit;
};

// 32 channels of a row of an own operand into 16 TMEM columns.
__device__ __forceinline__ void half_row_to_tmem(uint32_t col, const __nv_bfloat16* row, bool live)
{
    uint32_t r[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (live) v = *reinterpret_cast<const uint4*>(row + 8 * i);
        r[4 * i] = v.x, r[4 * i + 1] = v.y, r[4 * i + 2] = v.z, r[4 * i + 3] = v.w;
    }
    tmem_st16(col, r);
}

template <bool KEYS>
__global__ void __launch_bounds__(kThreads, 1)
window_backward_tc_kernel(const __grid_constant__ CUtensorMap tm_y1, const __grid_constant__ CUtensorMap tm_y2, const Params p)
{
    extern __shared__ unsigned char smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    volatile int* abort_flag = &sm.abort_flag;
    const unsigned limit = p.wait_limit;
    // the CTAs with most tiles first: the first key tiles, the last query tiles
    const int tiles = (p.T + kRows - 1) / kRows, heads = p.B * (KEYS ? p.Hk : p.Hq), G = p.Hq / p.Hk;
    const int at = (int)(blockIdx.x / (unsigned)heads), bh = blockIdx.x % (unsigned)heads;
    const int r0 = (KEYS ? at : tiles - 1 - at) * kRows;
    const int b = bh / (KEYS ? p.Hk : p.Hq), h = bh - b * (KEYS ? p.Hk : p.Hq);

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm.full[s], 1);
            mbar_init(&sm.free[s], 1);
        }
        mbar_init(&sm.x_ready, 2 * kGroup);
        for (int w = 0; w < 2; ++w) {
            mbar_init(&sm.s_full[w], 1);
            mbar_init(&sm.p_ready[w], kGroup);
            mbar_init(&sm.st_ready[w], kGroup);
        }
        mbar_init(&sm.done, 1);
        mbar_init(&sm.drain, 1);
        sm.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // (TMEM only after the kernel before has ended, the next kernel only after the TMEM: see the forward)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == 16) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem_base)),
                     "r"(kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tmem = (uint32_t)uniform((int)sm.tmem_base);

    const int len = uniform(p.lengths ? max(0, min(p.lengths[b], p.T)) : p.T);
    // the tiles that pass.  keys: the query tiles r0/64 .. of every head of the group; queries: the
    // sinks' tiles that lie before the window, then the window's
    int per = 0, lo = 0, extra = 0, n = 0;
    if (r0 < len) {
        if (KEYS) {
            const int last = (int)min((long long)r0 + kRows + p.window - 1, (long long)len);
            lo = r0 / kCols;
            per = (last + kCols - 1) / kCols - lo;
            n = per * G;
        } else {
            lo = r0 >= p.window ? (r0 - p.window + 1) / kCols : 0;
            extra = min(lo, (p.sinks + kCols - 1) / kCols);
            n = extra + (min(r0 + kRows, len) + kCols - 1) / kCols - lo;
        }
    }
    auto first_of = [&](int i) { return (KEYS ? lo + i % per : i < extra ? i : lo + i - extra) * kCols; };
    auto head_of = [&](int i) { return KEYS ? h * G + i / per : h / G; };

    if (warp == 17) {
        if (elect_one()) {
            int issued = 0;
            for (; issued < n; ++issued) {
                const int s = issued % kStages;
                if (issued >= kStages && !mbar_wait(&sm.free[s], (issued / kStages - 1) & 1, limit, abort_flag, p.status)) break;
                mbar_arrive_expect_tx(&sm.full[s], 2 * kTile);
                tma_load_4d(sm.y1[s], &tm_y1, &sm.full[s], 0, head_of(issued), first_of(issued), b);
                tma_load_4d(sm.y2[s], &tm_y2, &sm.full[s], 0, head_of(issued), first_of(issued), b);
            }
            // leave only when every issued load has landed
            for (int j = max(0, issued - kStages); j < issued; ++j)
                for (unsigned it = 0; it < kDrainLimit; ++it)
                    if (mbar_try_wait(&sm.full[j % kStages], (j / kStages) & 1)) break;
        }
        __syncwarp();
    } else if (warp == 16) {
        const uint64_t dy1 = make_desc(smem_u32(sm.y1[0])), dy2 = make_desc(smem_u32(sm.y2[0]));
        constexpr uint64_t stage = kTile >> 4;
        constexpr uint32_t idesc_s = make_idesc(128, 64, 0, 0);    // X (tmem) x Y (K-major)
        constexpr uint32_t idesc_a = make_idesc(128, 64, 0, 1);    // P, dS (tmem) x Y (MN-major)
        // (the elected lane) S and dP of tile i
        auto scores = [&](int i) {
            const int s = i % kStages, w = i & 1;
            const uint32_t at_s = tmem + kColS + w * kGroupCols, at_dp = tmem + kColDP + w * kGroupCols;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) mma_ts(at_s, tmem + kColX1 + 8 * kk, dy1 + s * stage + 2 * kk, idesc_s, kk > 0);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) mma_ts(at_dp, tmem + kColX2 + 8 * kk, dy2 + s * stage + 2 * kk, idesc_s, kk > 0);
        };
        auto landed = [&](int i) { return warp_wait(&sm.full[i % kStages], (i / kStages) & 1, limit, abort_flag, p.status); };
        bool ok = n > 0 && warp_wait(&sm.x_ready, 0, limit, abort_flag, p.status);
        for (int i = 0; ok && i < min(n, 2); ++i) {
            if (!(ok = landed(i))) break;
            tc_fence_after();
            if (elect_one()) {
                scores(i);
                mma_commit(&sm.s_full[i]);
            }
            __syncwarp();
        }
        for (int i = 0; ok && i < n; ++i) {
            const int s = i % kStages, w = i & 1;
            // (the wait for a tile that has most often landed long ago stands ahead of the one for P)
            if (i + 2 < n && !(ok = landed(i + 2))) break;
            if (!(ok = warp_wait(&sm.p_ready[w], (i >> 1) & 1, limit, abort_flag, p.status))) break;
            tc_fence_after();
            if (elect_one()) {
                const uint32_t at_p = tmem + kColS + w * kGroupCols, at_ds = tmem + kColDP + w * kGroupCols;
                // 16 passing rows: 8 columns of P or dS (rows 32-63 stand 32 columns on), 2048 bytes of Y
                if (KEYS)
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        mma_ts(tmem + kColA2, at_p + 32 * (kk >> 1) + 8 * (kk & 1), dy2 + s * stage + 128 * kk, idesc_a, i > 0 || kk > 0);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    mma_ts(tmem + kColA1, at_ds + 32 * (kk >> 1) + 8 * (kk & 1), dy1 + s * stage + 128 * kk, idesc_a, i > 0 || kk > 0);
                mma_commit(&sm.free[s]);
                // the group's next S and dP, over this P and dS (the products run in the order they were issued)
                if (i + 2 < n) {
                    scores(i + 2);
                    mma_commit(&sm.s_full[w]);
                }
                if (i == n - 1) mma_commit(&sm.done);
            }
            __syncwarp();
        }
        if (elect_one()) {
            mma_commit(&sm.drain);
            for (unsigned it = 0; it < kDrainLimit; ++it)
                if (mbar_try_wait(&sm.drain, 0)) break;
        }
        __syncwarp();
    } else {
        const int group = warp >> 3, c = (warp >> 2) & 1;         // c: which 32 of the columns
        const int row = (warp & 3) * 32 + lane, r = r0 + row, gt = tid & (kGroup - 1);
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const int rw0 = r0 + (warp & 3) * 32, rw1 = rw0 + 31;     // the warp's rows
        // X1 by group 0, X2 by group 1, half a row each
        {
            const __nv_bfloat16* x = group == 0 ? p.x1 + b * p.x1s[0] + r * p.x1s[1] + h * p.x1s[2]
                                                : p.x2 + b * p.x2s[0] + r * p.x2s[1] + h * p.x2s[2];
            half_row_to_tmem(lanes + (group == 0 ? kColX1 : kColX2) + 16 * c, x + 32 * c, r < len && 32 * c < p.d);
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&sm.x_ready);

        float row_lse = 0.0f, row_delta = 0.0f;
        if (!KEYS && r < len) {
            row_lse = -p.lse[(long long)bh * p.T + r] * kLog2e;
            row_delta = -p.delta[(long long)bh * p.T + r];
        }
        // keys: this thread's part of the tile's 64 lse (threads 0-63) and Delta (64-127; the rest has none), one tile ahead
        auto stat = [&](int i) {
            const int q = first_of(i) + (gt & 63);
            if (gt >= 128 || q >= len) return 0.0f;
            const long long x = ((long long)b * p.Hq + head_of(i)) * p.T + q;
            return gt < 64 ? -p.lse[x] * kLog2e : -p.delta[x];
        };
        float ahead = KEYS && group < n ? stat(group) : 0.0f;
        bool ok = true;
        for (int i = group; i < n; i += 2) {
            const int s = i % kStages, c0 = first_of(i);
            if (KEYS) {
                // (a buffer is written again two tiles on, when every thread has arrived for the one between)
                if (gt < 128) (gt < 64 ? sm.lse : sm.delta)[group][(i >> 1) & 1][gt & 63] = ahead;
                mbar_arrive(&sm.st_ready[group]);
                if (i + 2 < n) ahead = stat(i + 2);
                if (!(ok = warp_wait(&sm.st_ready[group], (i >> 1) & 1, limit, abort_flag, p.status))) break;
            }
            if (!(ok = warp_wait(&sm.s_full[group], (i >> 1) & 1, limit, abort_flag, p.status))) break;
            tc_fence_after();
            const uint32_t at_s = lanes + kColS + group * kGroupCols, at_dp = lanes + kColDP + group * kGroupCols;
            {
                // what the warp's rows and these 32 columns have to do with each other: 0 nothing, 1 part, 2 all
                const int s0 = c0 + 32 * c, s1 = s0 + 31;
                bool any, all;
                if (KEYS) {
                    any = s1 >= rw0 && s0 < len && rw0 < len && s0 - rw1 < p.window;
                    all = s0 >= rw1 && s1 < len && rw1 < len && s1 - rw0 < p.window;
                } else {
                    any = s0 <= rw1 && s0 < len && rw0 < len && (rw0 - s1 < p.window || s0 < p.sinks);
                    all = s1 <= rw0 && rw1 < len && (rw1 - s0 < p.window || s1 < p.sinks);
                }
                uint32_t pp[16], pd[16];
                if (any) {
                    uint32_t sv[32], dv[32];
                    tmem_ld32(at_s + 32 * c, sv);
                    tmem_ld32(at_dp + 32 * c, dv);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float x0, x1, g0 = __uint_as_float(dv[2 * e]), g1 = __uint_as_float(dv[2 * e + 1]);
                        float2 ls = make_float2(row_lse, row_lse), de = make_float2(row_delta, row_delta);
                        if (KEYS) {
                            ls = *reinterpret_cast<const float2*>(&sm.lse[group][(i >> 1) & 1][32 * c + 2 * e]);
                            de = *reinterpret_cast<const float2*>(&sm.delta[group][(i >> 1) & 1][32 * c + 2 * e]);
                        }
                        fma2(__uint_as_float(sv[2 * e]), __uint_as_float(sv[2 * e + 1]), p.scale2, ls.x, ls.y, x0, x1);
                        x0 = ex2_approx(x0);
                        x1 = ex2_approx(x1);
                        add2(g0, g1, de.x, de.y);
                        mul2_pair(g0, g1, x0, x1);
                        pp[e] = pack_bf16(x0, x1);
                        pd[e] = pack_bf16(g0, g1);
                    }
                    if (!all) {          // (what is masked may be NaN: its bits go)
                        const uint32_t bits = r >= len ? 0u : KEYS ? bit_range(r - s0, min(r + p.window - 1, len - 1) - s0)
                                                                   : seen_bits(r, s0, p.window, p.sinks, len);
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const uint32_t keep = ((bits >> (2 * e)) & 1u ? 0x0000ffffu : 0u) | ((bits >> (2 * e + 1)) & 1u ? 0xffff0000u : 0u);
                            pp[e] &= keep;
                            pd[e] &= keep;
                        }
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) pp[e] = pd[e] = 0u;
                }
                // over the columns that this thread has read
                if (KEYS) tmem_st16(at_s + 32 * c, pp);
                tmem_st16(at_dp + 32 * c, pd);
            }
            // rows past the sequence's end do not count, whatever they hold
            if (len < p.T && c0 + kCols > len) {
                const int y = gt & 63;
                if (c0 + y >= len) {
                    if (gt < 64) zero_row(sm.y1[s] + y * 128);
                    else if (KEYS && gt < 128) zero_row(sm.y2[s] + y * 128);
                }
                fence_proxy_async();
            }
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(&sm.p_ready[group]);
        }
        if (ok && n > 0) ok = warp_wait(&sm.done, 0, limit, abort_flag, p.status);
        tc_fence_after();
        // group 0: A1 (dK, dQ), times scale; group 1: A2 (dV)
        if (ok && (KEYS || group == 0)) {
            const float f = group == 0 ? p.scale : 1.0f;
            __nv_bfloat16* out = group == 0 ? p.a1 + b * p.a1s[0] + r * p.a1s[1] + h * p.a1s[2]
                                            : p.a2 + b * p.a2s[0] + r * p.a2s[1] + h * p.a2s[2];
            const int chunks = (p.T + kPrepRows - 1) / kPrepRows, sinks = min(p.sinks, p.T);
            const float* sums = p.sums + ((long long)bh * chunks * sinks + r) * 2 * p.d + group * p.d;
            {
                uint32_t a[32];
                if (n > 0) {
                    tmem_ld32(lanes + (group == 0 ? kColA1 : kColA2) + 32 * c, a);
                    tmem_wait_ld();
                }
                const bool live = r < p.T && 32 * c < p.d;
#pragma unroll
                for (int e = 0; e < 32; ++e) a[e] = n == 0 || r >= len ? 0u : __float_as_uint(__uint_as_float(a[e]) * f);
                if (KEYS && live && r < sinks && p.window < len)
                    for (int k = p.window / kPrepRows; k < (len + kPrepRows - 1) / kPrepRows; ++k)
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const float4 v = *reinterpret_cast<const float4*>(sums + (long long)k * sinks * 2 * p.d + 32 * c + e);
                            a[e] = __float_as_uint(__uint_as_float(a[e]) + v.x);
                            a[e + 1] = __float_as_uint(__uint_as_float(a[e + 1]) + v.y);
                            a[e + 2] = __float_as_uint(__uint_as_float(a[e + 2]) + v.z);
                            a[e + 3] = __float_as_uint(__uint_as_float(a[e + 3]) + v.w);
                        }
                if (live)
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    uint4 v;
                    v.x = pack_bf16(__uint_as_float(a[e]), __uint_as_float(a[e + 1]));
                    v.y = pack_bf16(__uint_as_float(a[e + 2]), __uint_as_float(a[e + 3]));
                    v.z = pack_bf16(__uint_as_float(a[e + 4]), __uint_as_float(a[e + 5]));
                    v.w = pack_bf16(__uint_as_float(a[e + 6]), __uint_as_float(a[e + 7]));
                    *reinterpret_cast<uint4*>(out + 32 * c + e) = v;
                }
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 16) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

void copy3(long long (&to)[3], const long long (&from)[3])
{
    for (int i = 0; i < 3; ++i) to[i] = from[i];
}

}  // namespace

cudaError_t launch_window_backward_tc(const WindowArgs& a, cudaStream_t st)
{
    CUtensorMap mq, mg, mk, mv;
    if (!encode_rows_map(&mq, a.q, a.d, a.B, a.T, a.Hq, a.qs, kCols) || !encode_rows_map(&mg, a.dout, a.d, a.B, a.T, a.Hq, a.dos, kCols) ||
        !encode_rows_map(&mk, a.k, a.d, a.B, a.T, a.Hk, a.ks, kCols) || !encode_rows_map(&mv, a.v, a.d, a.B, a.T, a.Hk, a.vs, kCols))
        return cudaErrorInvalidValue;
    static bool done1[64], done2[64];
    const size_t smem = sizeof(Smem) + 1024;
    cudaError_t e = allow_dynamic_smem(window_backward_tc_kernel<true>, smem, done1);
    if (e == cudaSuccess) e = allow_dynamic_smem(window_backward_tc_kernel<false>, smem, done2);
    if (e != cudaSuccess) return e;
    const unsigned tiles = (unsigned)((a.T + kRows - 1) / kRows);
    Params p{};
    p.B = a.B, p.T = a.T, p.Hq = a.Hq, p.Hk = a.Hk, p.d = a.d, p.window = a.window, p.sinks = a.sinks;
    p.scale = a.scale, p.scale2 = a.scale * kLog2e;
    p.lengths = a.lengths, p.lse = a.lse, p.delta = a.ws, p.sums = a.ws + window_delta_floats(a);
    p.status = a.status, p.wait_limit = a.wait_limit;
    typedef const __nv_bfloat16* in;
    typedef __nv_bfloat16* out;
    p.x1 = static_cast<in>(a.k), p.x2 = static_cast<in>(a.v), p.a1 = static_cast<out>(a.dk), p.a2 = static_cast<out>(a.dv);
    copy3(p.x1s, a.ks), copy3(p.x2s, a.vs), copy3(p.a1s, a.dks), copy3(p.a2s, a.dvs);
    e = launch_dependent(window_backward_tc_kernel<true>, dim3(tiles * a.B * a.Hk), dim3(kThreads), smem, st, mq, mg, p);
    if (e != cudaSuccess) return e;
    p.x1 = static_cast<in>(a.q), p.x2 = static_cast<in>(a.dout), p.a1 = static_cast<out>(a.dq), p.a2 = nullptr;
    copy3(p.x1s, a.qs), copy3(p.x2s, a.dos), copy3(p.a1s, a.dqs);
    return launch_dependent(window_backward_tc_kernel<false>, dim3(tiles * a.B * a.Hq), dim3(kThreads), smem, st, mk, mv, p);
}

}  // namespace lasad
