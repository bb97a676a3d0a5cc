// Gradient of the packed causal attention on the tensor cores (bf16), in two kernels of one form:
//
//     queries:  a CTA has 128 queries of one head and goes over the keys of its sequence up to the diagonal
//     keys:     a CTA has 128 keys of one key head and goes over the queries behind them, of every head of the group
//
// so that every sum stays in one CTA (no atomics: results repeat bit for bit, and the heads that share a key head
// are added in order).  With X1, X2 the CTA's own rows (Q, dO or K, V) and Y1, Y2 a tile of 64 rows that it
// passes (K, V or Q, dO), a tile costs the products
//
//     S = X1 Y1^T ,  dP = X2 Y2^T ,        P = 2^(S c - lse log2(e)) ,  dS = P * (dP - Delta)
//     A1 += dS Y1  (dQ or dK) ,            A2 += P Y1  or  P Y2 (dV)
//
// all of them tcgen05 128 x 64 x 64 with the left operand in TMEM: X1 and X2 are put there once, P and dS per tile.
// (A left operand from shared memory would cost 4 KB beside the 2 KB of the right one per 32-clock instruction, more
// than the 128 bytes per clock that an SM reads.)  scale is applied to dQ and dK once, at the end.
//
// Delta.  The queries kernel runs first and starts from Delta' = sum_c do_c o_c, but the o that a caller has was
// rounded to bf16, and where a row sees few keys, dP - Delta is small against what that rounding does to Delta'.  So it
// sums r = sum_s P (dP - Delta') in fp32 beside its products -- Delta = Delta' + r, as the P of a row add up to 1 -- and ends
// with dQ = A1 - r A2, A2 = P K.  It leaves -lse log2(e) and -Delta to the keys kernel, in blocks of 64 rows that come
// with the tiles.  P and dS enter their products in bf16, as the tensor cores take them beside bf16 operands: 2^-9 of each
// term, which adds up like noise.
//
// What bounds it: per tile 512 clocks of exponentials (16 per SM and clock) against four products of 128 clocks;
// between them lies a chain of latencies (S out of TMEM, P into it, three barriers).  Two groups of eight warps take
// the tiles in turn, each with its own S and dP columns.  P and dS have columns of their own that serve both groups in
// turn, so a group's next S and dP are made while it still works on the ones before: the SM's 512 TMEM columns are full,
// and one CTA has the SM.
// Measured: 1 x 9217 tokens, 24 query and 8 key heads: 991 us for both, 0.58 us a tile; 4 of 257 to 9217: 1.63 ms.
// Against one kernel that makes all products once and adds dQ by atomics this makes S, dP and P twice; it buys
// results that repeat, and no 32-bit dQ in memory.
//
// Warps 0-7 and 8-15: the two groups, two threads per own row, 32 of a tile's 64 columns each.  Warp 16: the
// products of P and dS.  Warp 17: TMA.  Warp 18: S and dP.  (One warp adds to A1 and A2, so the order of the additions
// is fixed.)
#include "lasad_full.cuh"
#include "lasad_window_tma.cuh"
#include <type_traits>

namespace lasad {
namespace {

using namespace tcx;

constexpr int kRows = 128, kCols = 64, kStages = 4, kGroup = 256, kThreads = 2 * kGroup + 96;
constexpr int kTile = kCols * 128;                         // bytes of a passing tile
constexpr uint32_t kColX1 = 0, kColX2 = 32, kColS = 64, kColDP = 128, kGroupCols = 128, kColA1 = 320, kColA2 = 384;
constexpr uint32_t kColP = 448, kColDS = 480;
constexpr int kTmemCols = 512;

struct Smem {
    unsigned char y1[kStages][kTile];
    unsigned char y2[kStages][kTile];
    float stat[kStages][2][kCols];                         // keys: -lse log2(e) and -Delta of the tile's rows
    float part[2][kRows], rest[4][kRows];                  // queries: halves of Delta', quarters of r
    unsigned long long full[kStages], free[kStages];       // Y1 and Y2 have landed; their products have been made
    unsigned long long x_ready;                            // X1 and X2 are in TMEM (2 kGroup arrivals)
    unsigned long long s_full[2];                          // S and dP of a group's tile are there
    unsigned long long s_free[2];                          // ... and have been read (kGroup arrivals)
    unsigned long long p_ready[2];                         // P and dS of a group's tile are there (kGroup arrivals)
    unsigned long long p_free[2];                          // ... and their products have been made
    unsigned long long r_ready;                            // queries: Delta' is in part, then r in rest (2 kGroup arrivals)
    unsigned long long done, drain[2];
    uint32_t tmem_base;
    int abort_flag;
};

struct Params {
    int N, S, Hq, Hk, d;
    float scale, scale2;                                   // scale2 = scale log2(e)
    const int* offsets;
    const float* lse;                                      // queries: [Hq,N]
    float* stat;                                           // see packed_stat_at
    long long stat_blocks;                                 // of a head
    const __nv_bfloat16* x1;
    const __nv_bfloat16* x2;
    const __nv_bfloat16* o;                                // queries
    long long x1s[2], x2s[2], os[2];
    __nv_bfloat16* a1;
    __nv_bfloat16* a2;
    long long a1s[2], a2s[2];
    int* status;
    unsigned wait_limit;
};

// 32 channels of a row, or zeros.
__device__ __forceinline__ void half_row(const __nv_bfloat16* row, bool live, uint32_t (&r)[16])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (live) v = *reinterpret_cast<const uint4*>(row + 8 * i);
        r[4 * i] = v.x, r[4 * i + 1] = v.y, r[4 * i + 2] = v.z, r[4 * i + 3] = v.w;
    }
}

template <bool KEYS>
__global__ void __launch_bounds__(kThreads, 1)
packed_backward_tc_kernel(const __grid_constant__ CUtensorMap tm_y1, const __grid_constant__ CUtensorMap tm_y2, const Params p)
{
    extern __shared__ unsigned char smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    volatile int* abort_flag = &sm.abort_flag;
    const unsigned limit = p.wait_limit;
    // (of each sequence the CTAs with most tiles first: the first key tiles, the last query tiles)
    const int tiles = (int)region_tiles(p.N, p.S, kRows), heads = KEYS ? p.Hk : p.Hq, G = p.Hq / p.Hk;
    const int at = (int)(blockIdx.x / (unsigned)heads), h = blockIdx.x % (unsigned)heads;

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm.full[s], 1);
            mbar_init(&sm.free[s], 1);
        }
        mbar_init(&sm.x_ready, 2 * kGroup);
        for (int w = 0; w < 2; ++w) {
            mbar_init(&sm.s_full[w], 1);
            mbar_init(&sm.s_free[w], kGroup);
            mbar_init(&sm.p_ready[w], kGroup);
            mbar_init(&sm.p_free[w], 1);
            mbar_init(&sm.drain[w], 1);
        }
        mbar_init(&sm.r_ready, 2 * kGroup);
        mbar_init(&sm.done, 1);
        sm.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // (TMEM only after the kernel before has ended, the next kernel only after the TMEM: see the forward)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    // The CTA's rows r0 .. of its sequence of len tokens, which begin at row `start` of memory; rows: those that are to be
    // written (of what no sequence has, len is 0 and zeros are).
    int r0, len, rows, start, block0;
    {
        const Region r = region_of<kRows>(p.offsets, p.S, p.N, KEYS ? at : tiles - 1 - at);
        r0 = uniform(r.first), rows = uniform(r.len), len = uniform(r.owned ? r.len : 0), start = uniform(r.start);
        block0 = uniform(r.start / kStatRows + r.base - r.start / kRows);     // of the region's statistics
    }
    if (r0 >= rows) return;
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

    // the tiles that pass.  keys: the query tiles r0/64 .. of every head of the group; queries: the key tiles up to the diagonal
    int per = 0, n = 0;
    if (r0 < len) {
        per = KEYS ? (len + kCols - 1) / kCols - r0 / kCols : (min(r0 + kRows, len) + kCols - 1) / kCols;
        n = KEYS ? per * G : per;
    }
    // A walk over them: tile i is tile number `at` of head `head`.
    struct Walk {
        int at, head;
    };
    auto move = [&](Walk& w, int by) {
        w.at += by;
        while (KEYS && w.at >= per) w.at -= per, ++w.head;
    };
    auto first_of = [&](const Walk& w) { return (KEYS ? r0 : 0) + w.at * kCols; };

    if (warp == 17) {
        if (elect_one()) {
            int issued = 0;
            Walk w{0, KEYS ? h * G : h / G};
            for (; issued < n; ++issued, move(w, 1)) {
                const int s = issued % kStages;
                if (issued >= kStages && !mbar_wait(&sm.free[s], (issued / kStages - 1) & 1, limit, abort_flag, p.status)) break;
                mbar_arrive_expect_tx(&sm.full[s], 2 * kTile + (KEYS ? 8 * kCols : 0));
                tma_load_4d(sm.y1[s], &tm_y1, &sm.full[s], 0, w.head, start + first_of(w), 0);
                tma_load_4d(sm.y2[s], &tm_y2, &sm.full[s], 0, w.head, start + first_of(w), 0);
                if (KEYS)
                    bulk_load(sm.stat[s], p.stat + (w.head * p.stat_blocks + block0 + first_of(w) / kStatRows) * (2 * kStatRows),
                              8 * kCols, &sm.full[s]);
            }
            // leave only when every issued load has landed
            for (int j = max(0, issued - kStages); j < issued; ++j)
                for (unsigned it = 0; it < kDrainLimit; ++it)
                    if (mbar_try_wait(&sm.full[j % kStages], (j / kStages) & 1)) break;
        }
        __syncwarp();
    } else if (warp == 18) {
        // ===================== S and dP of every tile =====================
        const uint64_t dy1 = make_desc(smem_u32(sm.y1[0])), dy2 = make_desc(smem_u32(sm.y2[0]));
        constexpr uint64_t stage = kTile >> 4;
        constexpr uint32_t idesc = make_idesc(128, 64, 0, 0);      // X (tmem) x Y (K-major)
        bool ok = n > 0 && warp_wait(&sm.x_ready, 0, limit, abort_flag, p.status);
        for (int i = 0; ok && i < n; ++i) {
            const int s = i % kStages, w = i & 1;
            if (i >= 2 && !(ok = warp_wait(&sm.s_free[w], ((i >> 1) - 1) & 1, limit, abort_flag, p.status))) break;
            if (!(ok = warp_wait(&sm.full[s], (i / kStages) & 1, limit, abort_flag, p.status))) break;
            tc_fence_after();
            if (elect_one()) {
                const uint32_t at_s = tmem + kColS + w * kGroupCols, at_dp = tmem + kColDP + w * kGroupCols;
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) mma_ts(at_s, tmem + kColX1 + 8 * kk, dy1 + s * stage + 2 * kk, idesc, kk > 0);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) mma_ts(at_dp, tmem + kColX2 + 8 * kk, dy2 + s * stage + 2 * kk, idesc, kk > 0);
                mma_commit(&sm.s_full[w]);
            }
            __syncwarp();
        }
        // (no product may still run when the CTA's memory goes)
        if (elect_one()) {
            mma_commit(&sm.drain[0]);
            for (unsigned it = 0; it < kDrainLimit; ++it)
                if (mbar_try_wait(&sm.drain[0], 0)) break;
        }
        __syncwarp();
    } else if (warp == 16) {
        // ===================== what P and dS add to A2 and A1, tile after tile =====================
        const uint64_t dy1 = make_desc(smem_u32(sm.y1[0])), dy2 = make_desc(smem_u32(sm.y2[0]));
        constexpr uint64_t stage = kTile >> 4;
        constexpr uint32_t idesc = make_idesc(128, 64, 0, 1);      // P, dS (tmem) x Y (MN-major)
        bool ok = true;
        for (int i = 0; ok && i < n; ++i) {
            const int s = i % kStages, w = i & 1;
            if (!(ok = warp_wait(&sm.full[s], (i / kStages) & 1, limit, abort_flag, p.status))) break;
            if (!(ok = warp_wait(&sm.p_ready[w], (i >> 1) & 1, limit, abort_flag, p.status))) break;
            tc_fence_after();
            if (elect_one()) {
                // 16 passing rows: 8 columns of P or dS, 2048 bytes of Y
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    mma_ts(tmem + kColA2, tmem + kColP + 8 * kk, (KEYS ? dy2 : dy1) + s * stage + 128 * kk, idesc, i > 0 || kk > 0);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    mma_ts(tmem + kColA1, tmem + kColDS + 8 * kk, dy1 + s * stage + 128 * kk, idesc, i > 0 || kk > 0);
                mma_commit(&sm.p_free[w]);
                mma_commit(&sm.free[s]);
                if (i == n - 1) mma_commit(&sm.done);
            }
            __syncwarp();
        }
        if (elect_one()) {
            mma_commit(&sm.drain[1]);
            for (unsigned it = 0; it < kDrainLimit; ++it)
                if (mbar_try_wait(&sm.drain[1], 0)) break;
        }
        __syncwarp();
    } else {
        const int group = warp >> 3, c = (warp >> 2) & 1;         // c: which 32 of the columns
        const int row = (warp & 3) * 32 + lane, r = r0 + row, gt = tid & (kGroup - 1);
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const int rw0 = r0 + (warp & 3) * 32, rw1 = rw0 + 31;     // the warp's rows
        // X1 by group 0, X2 by group 1, half a row each (all loads first: they are in flight together)
        const bool mine = r < len && 32 * c < p.d;
        uint32_t xv[16], ov[16];
        const long long at_row = start + r;
        half_row((group == 0 ? p.x1 + at_row * p.x1s[0] + h * p.x1s[1] : p.x2 + at_row * p.x2s[0] + h * p.x2s[1]) + 32 * c, mine, xv);
        float row_lse = 0.0f, row_delta = 0.0f, rest[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (!KEYS) {
            if (group == 1) half_row(p.o + at_row * p.os[0] + h * p.os[1] + 32 * c, mine, ov);
            if (r < len) row_lse = minus_lse(p.lse[(long long)h * p.N + at_row]);
        }
        tmem_st16(lanes + (group == 0 ? kColX1 : kColX2) + 16 * c, xv);
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&sm.x_ready);

        bool ok = true;
        if (!KEYS && n > 0) {
            if (group == 1) {
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < 16; ++e) sum = fmaf(bf16_lo(xv[e]), bf16_lo(ov[e]), fmaf(bf16_hi(xv[e]), bf16_hi(ov[e]), sum));
                sm.part[c][row] = sum;
            }
            mbar_arrive(&sm.r_ready);
            ok = warp_wait(&sm.r_ready, 0, limit, abort_flag, p.status);
            if (r < len) row_delta = -(sm.part[0][row] + sm.part[1][row]);
        }
        Walk at_tile{0, 0};
        if (n > 0) move(at_tile, group);
        for (int i = group; ok && i < n; i += 2, move(at_tile, 2)) {
            const int s = i % kStages, c0 = first_of(at_tile);
            // (the tile's statistics; a group has every other tile, so it sees every phase of its places, and a
            // place's next phase needs this tile's products)
            if (KEYS && !(ok = warp_wait(&sm.full[s], (i / kStages) & 1, limit, abort_flag, p.status))) break;
            if (!(ok = warp_wait(&sm.s_full[group], (i >> 1) & 1, limit, abort_flag, p.status))) break;
            tc_fence_after();
            {
                // what the warp's rows and these 32 columns have to do with each other: 0 nothing, 1 part, 2 all
                const int s0 = c0 + 32 * c, s1 = s0 + 31;
                bool any, all;
                if (KEYS) {
                    any = s1 >= rw0 && s0 < len && rw0 < len;
                    all = s0 >= rw1 && s1 < len && rw1 < len;
                } else {
                    any = s0 <= rw1 && s0 < len && rw0 < len;
                    all = s1 <= rw0 && rw1 < len;
                }
                uint32_t pp[16], pd[16];
                if (any) {
                    uint32_t sv[32], dv[32];
                    tmem_ld32(lanes + kColS + group * kGroupCols + 32 * c, sv);
                    tmem_ld32(lanes + kColDP + group * kGroupCols + 32 * c, dv);
                    tmem_wait_ld();
                    tc_fence_before();
                    mbar_arrive(&sm.s_free[group]);
                    // MASKED: not all of the pairs count (what is masked may be NaN: its bits go)
                    auto elements = [&](auto masked) {
                        constexpr bool MASKED = decltype(masked)::value;
                        uint32_t bits = 0xffffffffu;
                        if (MASKED)
                            bits = r >= len ? 0u : KEYS ? bit_range(r - s0, len - 1 - s0) : bit_range(0, r - s0);
                        float4 ls = make_float4(row_lse, row_lse, row_lse, row_lse), de = make_float4(row_delta, row_delta, row_delta, row_delta);
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float x0, x1, g0 = __uint_as_float(dv[2 * e]), g1 = __uint_as_float(dv[2 * e + 1]);
                            if (KEYS && (e & 1) == 0) {
                                ls = *reinterpret_cast<const float4*>(&sm.stat[s][0][32 * c + 2 * e]);
                                de = *reinterpret_cast<const float4*>(&sm.stat[s][1][32 * c + 2 * e]);
                            }
                            fma2(__uint_as_float(sv[2 * e]), __uint_as_float(sv[2 * e + 1]), p.scale2, e & 1 ? ls.z : ls.x,
                                 e & 1 ? ls.w : ls.y, x0, x1);
                            x0 = ex2_approx(x0);
                            x1 = ex2_approx(x1);
                            add2(g0, g1, e & 1 ? de.z : de.x, e & 1 ? de.w : de.y);
                            mul2_pair(g0, g1, x0, x1);
                            if (MASKED) {
                                if (!((bits >> (2 * e)) & 1u)) x0 = g0 = 0.0f;
                                if (!((bits >> (2 * e + 1)) & 1u)) x1 = g1 = 0.0f;
                            }
                            if (!KEYS) add2(rest[(e & 1) * 2], rest[(e & 1) * 2 + 1], g0, g1);
                            pp[e] = pack_bf16(x0, x1);
                            pd[e] = pack_bf16(g0, g1);
                        }
                    };
                    if (all) elements(std::false_type{});
                    else elements(std::true_type{});
                } else {
                    tc_fence_before();
                    mbar_arrive(&sm.s_free[group]);
#pragma unroll
                    for (int e = 0; e < 16; ++e) pp[e] = pd[e] = 0u;
                }
                // The columns of P and dS serve both groups in turn: the products of the tile before, the other
                // group's, have been made.  (That group waits for these before its next ones, so neither can be two
                // phases ahead.)
                if (i > 0 && !(ok = warp_wait(&sm.p_free[group ^ 1], ((i - 1) >> 1) & 1, limit, abort_flag, p.status))) break;
                tc_fence_after();
                tmem_st16(lanes + kColP + 16 * c, pp);
                tmem_st16(lanes + kColDS + 16 * c, pd);
            }
            // rows past the sequence's end do not count, whatever they hold
            if (c0 + kCols > len) {
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
        float r_sum = 0.0f;
        if (!KEYS && ok && n > 0) {
            sm.rest[2 * group + c][row] = (rest[0] + rest[1]) + (rest[2] + rest[3]);
            mbar_arrive(&sm.r_ready);
            ok = warp_wait(&sm.r_ready, 1, limit, abort_flag, p.status);
            r_sum = (sm.rest[0][row] + sm.rest[1][row]) + (sm.rest[2][row] + sm.rest[3][row]);
        }
        // (zeros behind the sequence's end, up to the end of the last block)
        if (!KEYS && ok && group == 1 && r < (len + kStatRows - 1) / kStatRows * kStatRows)
            p.stat[(h * p.stat_blocks + block0 + r / kStatRows) * (2 * kStatRows) + kStatRows * c + r % kStatRows] =
                r >= len ? 0.0f : c == 0 ? row_lse : row_delta - r_sum;
        if (ok && n > 0) ok = warp_wait(&sm.done, 0, limit, abort_flag, p.status);
        tc_fence_after();
        // group 0: A1 (dK, dQ - what r takes away), times scale; group 1, keys: A2 (dV)
        if (ok && (KEYS || group == 0)) {
            const float f = group == 0 ? p.scale : 1.0f;
            __nv_bfloat16* out = group == 0 ? p.a1 + at_row * p.a1s[0] + h * p.a1s[1] : p.a2 + at_row * p.a2s[0] + h * p.a2s[1];
            {
                uint32_t a[32];
                if (n > 0) {
                    tmem_ld32(lanes + (group == 0 ? kColA1 : kColA2) + 32 * c, a);
                    tmem_wait_ld();
                    if (!KEYS) {
                        uint32_t pk[32];
                        tmem_ld32(lanes + kColA2 + 32 * c, pk);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) a[e] = __float_as_uint(fmaf(-r_sum, __uint_as_float(pk[e]), __uint_as_float(a[e])));
                    }
                }
                const bool live = r < rows && 32 * c < p.d;
#pragma unroll
                for (int e = 0; e < 32; ++e) a[e] = n == 0 || r >= len ? 0u : __float_as_uint(__uint_as_float(a[e]) * f);
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

void copy2(long long (&to)[2], const long long (&from)[2])
{
    to[0] = from[0], to[1] = from[1];
}

}  // namespace

cudaError_t launch_packed_backward_tc(const PackedArgs& a, cudaStream_t st)
{
    CUtensorMap mq, mg, mk, mv;
    if (!encode_packed_map(&mq, a.q, a.d, a.N, a.Hq, a.qs, kCols) || !encode_packed_map(&mg, a.dout, a.d, a.N, a.Hq, a.dos, kCols) ||
        !encode_packed_map(&mk, a.k, a.d, a.N, a.Hk, a.ks, kCols) || !encode_packed_map(&mv, a.v, a.d, a.N, a.Hk, a.vs, kCols))
        return cudaErrorInvalidValue;
    static bool done1[64], done2[64];
    const size_t smem = sizeof(Smem) + 1024;
    cudaError_t e = allow_dynamic_smem(packed_backward_tc_kernel<true>, smem, done1);
    if (e == cudaSuccess) e = allow_dynamic_smem(packed_backward_tc_kernel<false>, smem, done2);
    if (e != cudaSuccess) return e;
    const unsigned tiles = (unsigned)region_tiles(a.N, a.S, kRows);
    Params p{};
    p.N = a.N, p.S = a.S, p.Hq = a.Hq, p.Hk = a.Hk, p.d = a.d;
    p.scale = a.scale, p.scale2 = a.scale * kLog2e;
    p.offsets = a.offsets, p.lse = a.lse, p.stat = a.ws, p.stat_blocks = region_tiles(a.N, a.S, kStatRows);
    p.status = a.status, p.wait_limit = a.wait_limit;
    typedef const __nv_bfloat16* in;
    typedef __nv_bfloat16* out;
    p.x1 = static_cast<in>(a.q), p.x2 = static_cast<in>(a.dout), p.o = static_cast<in>(a.o), p.a1 = static_cast<out>(a.dq);
    copy2(p.x1s, a.qs), copy2(p.x2s, a.dos), copy2(p.os, a.os), copy2(p.a1s, a.dqs);
    e = launch_dependent(packed_backward_tc_kernel<false>, dim3(tiles * a.Hq), dim3(kThreads), smem, st, mk, mv, p);
    if (e != cudaSuccess) return e;
    p.x1 = static_cast<in>(a.k), p.x2 = static_cast<in>(a.v), p.a1 = static_cast<out>(a.dk), p.a2 = static_cast<out>(a.dv);
    copy2(p.x1s, a.ks), copy2(p.x2s, a.vs), copy2(p.a1s, a.dks), copy2(p.a2s, a.dvs);
    return launch_dependent(packed_backward_tc_kernel<true>, dim3(tiles * a.Hk), dim3(kThreads), smem, st, mq, mg, p);
}

}  // namespace lasad
