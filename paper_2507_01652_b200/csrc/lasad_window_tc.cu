// Window attention, forward, on the tensor cores (bf16):
//
//     S = Q K^T (tcgen05 128 x 128 x 64, smem x smem) ,  P = 2^(S c - m) with c = scale log2(e) ,
//     O += P V (128 x 64 x 128, P from TMEM) ,  l += rowsum(P) ,  o = O / l ,  lse = (m + log2 l) ln 2 .
//
// A CTA has 128 queries of one head and goes over the visible tiles of 64 keys only: from the
// window's edge to the diagonal and, where the window has left them, the tiles of the sinks (their
// last one cut to the 32-column blocks that hold any).  Two groups of four warps take the tiles in
// turn, each with S, P (written over S) and O columns of its own and its own maximum and sum per
// row, joined at the end; one thread has one row, so neither needs an exchange.  m is a lagging
// maximum: it moves, and O and l are scaled, only when a row's maximum has grown by more than 8
// (a factor 2^8, far inside the range of fp32 and bf16), which after the first tiles is rare.
// 32-column blocks that no row of a warp sees are skipped, and only blocks on an edge are masked.
//
// What bounds it: the exponentials, 16 per SM and clock: 512 clocks for a 128 x 64 tile whose
// products take 256.  Everything else a tile needs (its products, their way through TMEM, the maximum)
// is latency, some 1500 clocks of it, and has to pass under other tiles' exponentials: two CTAs of two
// groups share an SM (2 x 256 TMEM columns, 2 x 82 KB), four warps on each scheduler.  (One
// group of 128 x 128 tiles per CTA, two warps on a scheduler, took 1.9 times the exponentials' time.)
//
// Warps 0-3 and 4-7: the groups, rows 32 (w mod 4) .. + 31 (TMEM lane quadrant).  Warp 8: MMA issue.
// Warp 9: TMA.  All waits are bounded (see mbar_wait); a wait that gives up sets the status word and the
// CTA leaves through the normal exit with its copies landed and its TMEM freed.
#include "lasad_window_tma.cuh"

namespace lasad {
namespace {

using namespace tcx;

constexpr int kRows = 128, kCols = 64, kStages = 4, kThreads = 320;
constexpr int kTile = kCols * 128;                         // bytes of a key or value tile
constexpr uint32_t kColS = 0, kColO = 64, kGroupCols = 128;
constexpr int kTmemCols = 256;

struct Smem {
    unsigned char q[kRows * 128];              // the queries, then the output tile
    unsigned char k[kStages][kTile];           // (the other group's O at the end, 32-bit: both arrays, 64 KB)
    unsigned char v[kStages][kTile];
    float m[kRows], l[kRows];                  // the second group's, at the end
    unsigned long long q_full, full[kStages];   // Q; K and V of a tile have landed
    unsigned long long s_full[2];              // S of a group's tile is in TMEM (and all products before it are done)
    unsigned long long p_ready[2];             // P of a group's tile is (128 arrivals)
    unsigned long long done;                   // every product
    unsigned long long joined;                 // the second group's m, l, O are in shared memory (128 arrivals)
    unsigned long long st_ready;               // the output tile is in q (128 arrivals)
    unsigned long long drain;
    uint32_t tmem_base;
    int abort_flag;
};

struct Params {
    int B, T, Hq, Hk, window, sinks;
    float scale2;                // |scale| log2(e), at least 1e-37
    bool negate;                 // scale < 0
    const int* lengths;
    float* lse;
    int* status;
    unsigned wait_limit;
};

__global__ void __launch_bounds__(kThreads, 2)
window_forward_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                         const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_o, const Params p)
{
    extern __shared__ unsigned char smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    volatile int* abort_flag = &sm.abort_flag;
    const unsigned limit = p.wait_limit;
    // the last query tiles, which have the most key tiles, first
    const int tiles = (p.T + kRows - 1) / kRows, BH = p.B * p.Hq;
    const int qt = tiles - 1 - (int)(blockIdx.x / (unsigned)BH), bh = blockIdx.x % (unsigned)BH;
    const int b = bh / p.Hq, h = bh - b * p.Hq, hk = h / (p.Hq / p.Hk);
    const int q0 = qt * kRows;

    if (tid == 0) {
        mbar_init(&sm.q_full, 1);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm.full[s], 1);
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(&sm.s_full[w], 1);
            mbar_init(&sm.p_ready[w], kRows);
        }
        mbar_init(&sm.done, 1);
        mbar_init(&sm.joined, kRows);
        mbar_init(&sm.st_ready, kRows);
        mbar_init(&sm.drain, 1);
        sm.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // What this kernel reads may come from the one before it; its TMEM is taken only now, too, so that it
    // never holds columns that a late CTA of that kernel waits for, and the next kernel is let in
    // only when every CTA of this one has its own.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == 8) {
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
    // key tiles of this CTA: the sinks' that lie before the window's, then lo .. hi - 1
    const int hi = q0 >= len ? 0 : (min(q0 + kRows, len) + kCols - 1) / kCols;
    const int lo = min(hi, q0 >= p.window ? (q0 - p.window + 1) / kCols : 0);
    const int extra = min(lo, (p.sinks + kCols - 1) / kCols), n = hi == 0 ? 0 : extra + hi - lo;
    auto first_of = [&](int i) { return (i < extra ? i : lo + i - extra) * kCols; };
    auto blocks_of = [&](int i) { return i < extra && p.sinks - i * kCols <= 32 ? 1 : 2; };     // 32-column blocks

    if (warp == 9) {
        if (elect_one()) {
            int issued = 0;
            if (n > 0) {
                mbar_arrive_expect_tx(&sm.q_full, kRows * 128);
                tma_load_4d(sm.q, &tm_q, &sm.q_full, 0, h, q0, b);
            }
            for (; issued < n; ++issued) {
                const int s = issued % kStages;
                // (the place of tile j = issued - kStages is free with its group's next commit, the one of number j / 2 + 1)
                const int j = issued - kStages;
                // (a wait names a phase by its parity: the one before it has to be known to be over, so the first
                // two tiles wait for commit 0 as well; commit j / 2 + 2 cannot come before tile j + 4 is here)
                if (j >= 0 && j < 2 && !mbar_wait(&sm.s_full[j], 0, limit, abort_flag, p.status)) break;
                if (j >= 0 && !mbar_wait(&sm.s_full[j & 1], ((j >> 1) + 1) & 1, limit, abort_flag, p.status)) break;
                mbar_arrive_expect_tx(&sm.full[s], 2 * kTile);
                tma_load_4d(sm.k[s], &tm_k, &sm.full[s], 0, hk, first_of(issued), b);
                tma_load_4d(sm.v[s], &tm_v, &sm.full[s], 0, hk, first_of(issued), b);
            }
            if (mbar_wait(&sm.st_ready, 0, limit, abort_flag, p.status)) {
                tma_store_4d(&tm_o, sm.q, 0, h, q0, b);
                tma_store_commit();
                tma_store_wait_all();
            }
            // leave only when every issued load has landed
            if (n > 0)
                for (unsigned it = 0; it < kDrainLimit; ++it)
                    if (mbar_try_wait(&sm.q_full, 0)) break;
            for (int j = max(0, issued - kStages); j < issued; ++j)
                for (unsigned it = 0; it < kDrainLimit; ++it)
                    if (mbar_try_wait(&sm.full[j % kStages], (j / kStages) & 1)) break;
        }
        __syncwarp();
    } else if (warp == 8) {
        const uint64_t dq = make_desc(smem_u32(sm.q)), dk = make_desc(smem_u32(sm.k[0])), dv = make_desc(smem_u32(sm.v[0]));
        constexpr uint64_t stage = kTile >> 4;
        const uint32_t minus = p.negate ? 1u << 13 : 0u;          // (the descriptor's negation of A)
        constexpr uint32_t idesc_pv = make_idesc(128, 64, 0, 1);  // P (tmem) x V (MN-major)
        // (the elected lane) S of tile i
        auto scores = [&](int i) {
            const int s = i % kStages, w = i & 1;
            const uint32_t idesc = make_idesc(128, 32 * blocks_of(i), 0, 0) | minus;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
                mma_ss(tmem + kColS + w * kGroupCols, dq + 2 * kk, dk + s * stage + 2 * kk, idesc, kk > 0);
        };
        auto landed = [&](int i) { return warp_wait(&sm.full[i % kStages], (i / kStages) & 1, limit, abort_flag, p.status); };
        bool ok = n > 0 && warp_wait(&sm.q_full, 0, limit, abort_flag, p.status);
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
                const uint32_t at_p = tmem + kColS + w * kGroupCols, at_o = tmem + kColO + w * kGroupCols;
                const uint64_t at_v = dv + s * stage;
                mma_ts(at_o, at_p, at_v, idesc_pv, i > 1);               // 16 keys: 8 columns of P, 2048 bytes of V
                mma_ts(at_o, at_p + 8, at_v + 128, idesc_pv, 1);
                if (blocks_of(i) > 1) {                                  // keys 32-63 stand 32 columns on
                    mma_ts(at_o, at_p + 32, at_v + 256, idesc_pv, 1);
                    mma_ts(at_o, at_p + 40, at_v + 384, idesc_pv, 1);
                }
                // the group's next S, over this P (the products run in the order they were issued); with
                // it this tile's place is free
                if (i + 2 < n) scores(i + 2);
                mma_commit(&sm.s_full[w]);
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
        const int group = warp >> 2, row = (warp & 3) * 32 + lane, t = q0 + row;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16) + group * kGroupCols;
        const int tw0 = q0 + (warp & 3) * 32, tw1 = tw0 + 31;    // the warp's queries
        float m = -INFINITY, l[4] = {0.0f, 0.0f, 0.0f, 0.0f};     // (four sums: no long chain of additions)
        bool ok = true;
        for (int i = group; i < n; i += 2) {
            const int k0 = first_of(i), blocks = blocks_of(i);
            // what the warp sees of each block: 0 nothing, 1 part, 2 all
            int vis[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int s0 = k0 + 32 * c, s1 = s0 + 31;
                const bool any = c < blocks && s0 <= tw1 && s0 < len && (tw0 - s1 < p.window || s0 < p.sinks);
                const bool all = s1 <= tw0 && s1 < len && (tw1 - s0 < p.window || s1 < p.sinks);
                vis[c] = !any ? 0 : all ? 2 : 1;
            }
            if (!(ok = warp_wait(&sm.s_full[group], (i >> 1) & 1, limit, abort_flag, p.status))) break;
            tc_fence_after();
            uint32_t sv[2][32];
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (vis[c]) tmem_ld32(lanes + kColS + 32 * c, sv[c]);
            tmem_wait_ld();
            float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                if (vis[c] == 1) {
                    const uint32_t bits = seen_bits(t, k0 + 32 * c, p.window, p.sinks, len);
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (!((bits >> e) & 1u)) sv[c][e] = 0xff800000u;     // -infinity
                }
                if (vis[c])
#pragma unroll
                    for (int e = 0; e < 32; e += 2)
                        tops[(e >> 1) & 3] = max3(tops[(e >> 1) & 3], __uint_as_float(sv[c][e]), __uint_as_float(sv[c][e + 1]));
            }
            const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * p.scale2;
            const bool grow = top > m + 8.0f || (m == -INFINITY && top > m);
            if (i < 2) {
                m = top;
            } else if (__any_sync(0xffffffffu, grow)) {
                const float now = grow ? top : m, f = grow ? ex2_approx(m - now) : 1.0f;
                m = now;
#pragma unroll
                for (int e = 0; e < 4; ++e) l[e] *= f;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t o[16];
                    tmem_ld16(lanes + kColO + 16 * c, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                    tmem_st16(lanes + kColO + 16 * c, o);
                }
            }
            const float base = m == -INFINITY ? 0.0f : -m;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                if (c >= blocks) break;
                uint32_t pk[16];
                if (vis[c]) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float x0, x1;
                        fma2s(__uint_as_float(sv[c][2 * e]), __uint_as_float(sv[c][2 * e + 1]), p.scale2, base, x0, x1);
                        x0 = ex2_approx(x0);
                        x1 = ex2_approx(x1);
                        add2(l[(e & 1) * 2], l[(e & 1) * 2 + 1], x0, x1);
                        pk[e] = pack_bf16(x0, x1);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) pk[e] = 0u;
                }
                tmem_st16(lanes + kColS + 32 * c, pk);           // (over columns that this thread has read)
            }
            // values past the sequence's end do not count, whatever they are
            if (len < p.T && k0 + kCols > len) {
                if (row < kCols && k0 + row >= len) zero_row(sm.v[i % kStages] + row * 128);
                fence_proxy_async();
            }
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(&sm.p_ready[group]);
        }
        float sum = (l[0] + l[1]) + (l[2] + l[3]);
        if (ok && n > 0) ok = warp_wait(&sm.done, 0, limit, abort_flag, p.status);
        tc_fence_after();
        // 16-byte pieces of 32-bit rows, turned by the row so that eight rows use all banks
        float4* part = reinterpret_cast<float4*>(sm.k[0]) + row * 16;
        if (ok && group == 1 && n > 1) {
            sm.m[row] = m;
            sm.l[row] = sum;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t o[32];
                tmem_ld32(lanes + kColO + 32 * c, o);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    part[(8 * c + e) ^ (row & 7)] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]),
                                                                __uint_as_float(o[4 * e + 2]), __uint_as_float(o[4 * e + 3]));
            }
            tc_fence_before();
            mbar_arrive(&sm.joined);
        } else if (group == 0) {
            float f0 = 1.0f, f1 = 0.0f;
            if (ok && n > 1 && (ok = warp_wait(&sm.joined, 0, limit, abort_flag, p.status))) {
                const float m1 = sm.m[row], both = fmaxf(m, m1), base = both == -INFINITY ? 0.0f : both;
                f0 = ex2_approx(m - base);
                f1 = ex2_approx(m1 - base);
                sum = sum * f0 + sm.l[row] * f1;
                m = both;
            }
            if (ok) {
                const bool none = t >= len || sum == 0.0f;
                const float inv = none ? 0.0f : 1.0f / sum;
                if (p.lse && t < p.T)
                    p.lse[(long long)bh * p.T + t] = none ? -INFINITY : m * kLn2 + logf(sum);
                f0 *= inv;
                f1 *= inv;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t o[32];
                    if (n > 0) {
                        tmem_ld32(lanes + kColO + 32 * c, o);
                        tmem_wait_ld();
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float a[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) a[e] = none ? 0.0f : __uint_as_float(o[8 * k + e]) * f0;
                        if (n > 1 && !none) {
                            const float4 u = part[(8 * c + 2 * k) ^ (row & 7)], w = part[(8 * c + 2 * k + 1) ^ (row & 7)];
                            a[0] = fmaf(u.x, f1, a[0]), a[1] = fmaf(u.y, f1, a[1]), a[2] = fmaf(u.z, f1, a[2]), a[3] = fmaf(u.w, f1, a[3]);
                            a[4] = fmaf(w.x, f1, a[4]), a[5] = fmaf(w.y, f1, a[5]), a[6] = fmaf(w.z, f1, a[6]), a[7] = fmaf(w.w, f1, a[7]);
                        }
                        reinterpret_cast<uint4*>(sm.q + row * 128)[(4 * c + k) ^ (row & 7)] =
                            make_uint4(pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3]), pack_bf16(a[4], a[5]), pack_bf16(a[6], a[7]));
                    }
                }
                fence_proxy_async();
                tc_fence_before();
                mbar_arrive(&sm.st_ready);
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

}  // namespace

cudaError_t launch_window_forward_tc(const WindowArgs& a, cudaStream_t st)
{
    CUtensorMap mq, mk, mv, mo;
    if (!encode_rows_map(&mq, a.q, a.d, a.B, a.T, a.Hq, a.qs, kRows) || !encode_rows_map(&mk, a.k, a.d, a.B, a.T, a.Hk, a.ks, kCols) ||
        !encode_rows_map(&mv, a.v, a.d, a.B, a.T, a.Hk, a.vs, kCols) || !encode_rows_map(&mo, a.o, a.d, a.B, a.T, a.Hq, a.os, kRows))
        return cudaErrorInvalidValue;
    static bool done[64];
    const size_t smem = sizeof(Smem) + 1024;
    const cudaError_t e = allow_dynamic_smem(window_forward_tc_kernel, smem, done);
    if (e != cudaSuccess) return e;
    Params p{a.B, a.T, a.Hq, a.Hk, a.window, a.sinks, fmaxf(fabsf(a.scale) * kLog2e, 1e-37f), a.scale < 0.0f, a.lengths,
             a.lse, a.status, a.wait_limit};
    const unsigned grid = (unsigned)((a.T + kRows - 1) / kRows) * a.B * a.Hq;
    return launch_dependent(window_forward_tc_kernel, dim3(grid), dim3(kThreads), smem, st, mq, mk, mv, mo, p);
}

}  // namespace lasad
