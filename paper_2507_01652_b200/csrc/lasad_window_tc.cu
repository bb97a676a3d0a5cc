// Window attention, forward, on the tensor cores (bf16):
//
//     S = Q K^T (tcgen05 128 x 128 x 64, smem x smem) ,  P = 2^(S c - m) with c = scale log2(e) ,
//     O += P V (128 x 64 x 128, P from TMEM) ,  l += rowsum(P) ,  o = O / l ,  lse = (m + log2 l) ln 2 .
//
// A CTA has 128 queries of one head and goes over the visible key tiles only: the tiles from the
// window's edge to the diagonal and, where the window has left tile 0, the sinks' columns of that tile
// (rounded up to 32: products and exponentials are made for those columns alone).  One thread
// has one row, so the maximum and the sum need no exchange.  m is a lagging maximum: it moves, and O
// and l are scaled, only when a row's maximum has grown by more than 8 (a factor 2^8, far inside
// the range of fp32 and bf16), which after the first tiles is rare.  32-column blocks that no row
// of a warp sees are skipped, and only blocks on an edge are masked.
//
// What bounds it: the exponentials, 16 per SM and clock: 1024 clocks for a 128 x 128 tile whose
// products take 512.  So two CTAs share an SM (256 TMEM columns and 81 KB each) and one's products and
// loads run under the other's exponentials; S, P and O have columns of their own, so that the
// next tile's S is made while this one's P is.
//
// Warps 0-3: softmax, rows 32 w .. 32 w + 31 (TMEM lane quadrant w).  Warp 4: MMA issue.  Warp 5: TMA.
// All waits are bounded (see mbar_wait); a wait that gives up sets the status word and the CTA leaves
// through the normal exit with its copies landed and its TMEM freed.
#include "lasad_window_tma.cuh"

namespace lasad {
namespace {

using namespace tcx;

constexpr int kRows = 128, kStages = 2, kThreads = 192;
constexpr int kTileBytes128 = kRows * 128;
constexpr uint32_t kColS = 0, kColP = 128, kColO = 192;
constexpr int kTmemCols = 256;

struct Smem {
    unsigned char q[kTileBytes128];            // the queries, then the output tile
    unsigned char k[kStages][kTileBytes128];
    unsigned char v[kStages][kTileBytes128];
    unsigned long long q_full, k_full[kStages], v_full[kStages];
    unsigned long long k_free[kStages], v_free[kStages];   // the tile's products have been made
    unsigned long long s_full;                 // S of a tile is in TMEM
    unsigned long long s_free;                 // ... and has been read (128 arrivals)
    unsigned long long p_ready;                // P of a tile is in TMEM (128 arrivals)
    unsigned long long o_done;                 // P V of a tile has been added
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
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
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
            mbar_init(&sm.k_full[s], 1);
            mbar_init(&sm.v_full[s], 1);
            mbar_init(&sm.k_free[s], 1);
            mbar_init(&sm.v_free[s], 1);
        }
        mbar_init(&sm.s_full, 1);
        mbar_init(&sm.s_free, kRows);
        mbar_init(&sm.p_ready, kRows);
        mbar_init(&sm.o_done, 1);
        mbar_init(&sm.st_ready, kRows);
        mbar_init(&sm.drain, 1);
        sm.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // What this kernel reads may come from the one before it; its TMEM is taken only now, too, so that it
    // never holds columns that a late CTA of that kernel waits for, and the next kernel is let in
    // only when every CTA of this one has its own.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == 4) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem_base)),
                     "r"(kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tmem = sm.tmem_base;

    const int len = p.lengths ? max(0, min(p.lengths[b], p.T)) : p.T;
    // key tiles of this CTA: (the sinks' part of tile 0,) lo .. hi - 1
    const int hi = q0 >= len ? 0 : min(qt, (len - 1) / kRows) + 1;
    const int lo = min(hi, q0 >= p.window ? (q0 - p.window + 1) / kRows : 0);
    const int extra = p.sinks > 0 && lo > 0 ? 1 : 0;
    const int n = hi == 0 ? 0 : extra + hi - lo;
    auto tile_of = [&](int j) { return j < extra ? 0 : lo + j - extra; };
    auto blocks_of = [&](int j) { return j < extra ? (p.sinks + 31) / 32 : 4; };     // 32-column blocks

    if (warp == 5) {
        if (n > 0 && elect_one()) {
            mbar_arrive_expect_tx(&sm.q_full, kTileBytes128);
            tma_load_4d(sm.q, &tm_q, &sm.q_full, 0, h, q0, b);
            int issued = 0;
            for (; issued < n; ++issued) {
                const int s = issued % kStages;
                const unsigned parity = (issued / kStages - 1) & 1;
                if (issued >= kStages && !mbar_wait(&sm.k_free[s], parity, limit, abort_flag, p.status)) break;
                mbar_arrive_expect_tx(&sm.k_full[s], kTileBytes128);
                tma_load_4d(sm.k[s], &tm_k, &sm.k_full[s], 0, hk, tile_of(issued) * kRows, b);
                const bool ok = issued < kStages || mbar_wait(&sm.v_free[s], parity, limit, abort_flag, p.status);
                // (after a failed wait V's barrier is completed without a load, for the exit below)
                if (ok) {
                    mbar_arrive_expect_tx(&sm.v_full[s], kTileBytes128);
                    tma_load_4d(sm.v[s], &tm_v, &sm.v_full[s], 0, hk, tile_of(issued) * kRows, b);
                } else {
                    mbar_arrive(&sm.v_full[s]);
                    ++issued;
                    break;
                }
            }
            if (mbar_wait(&sm.st_ready, 0, limit, abort_flag, p.status)) {
                tma_store_4d(&tm_o, sm.q, 0, h, q0, b);
                tma_store_commit();
                tma_store_wait_all();
            }
            // leave only when every issued load has landed
            for (unsigned it = 0; it < kDrainLimit; ++it)
                if (mbar_try_wait(&sm.q_full, 0)) break;
            for (int j = max(0, issued - kStages); j < issued; ++j) {
                for (unsigned it = 0; it < kDrainLimit; ++it)
                    if (mbar_try_wait(&sm.k_full[j % kStages], (j / kStages) & 1)) break;
                for (unsigned it = 0; it < kDrainLimit; ++it)
                    if (mbar_try_wait(&sm.v_full[j % kStages], (j / kStages) & 1)) break;
            }
        } else if (n == 0 && elect_one()) {
            if (mbar_wait(&sm.st_ready, 0, limit, abort_flag, p.status)) {
                tma_store_4d(&tm_o, sm.q, 0, h, q0, b);
                tma_store_commit();
                tma_store_wait_all();
            }
        }
        __syncwarp();
    } else if (warp == 4) {
        const uint64_t dq = make_desc(smem_u32(sm.q));
        const uint64_t dk0 = make_desc(smem_u32(sm.k[0])), dk1 = make_desc(smem_u32(sm.k[1]));
        const uint64_t dv0 = make_desc(smem_u32(sm.v[0])), dv1 = make_desc(smem_u32(sm.v[1]));
        const uint32_t minus = p.negate ? 1u << 13 : 0u;          // (the descriptor's negation of A)
        constexpr uint32_t idesc_pv = make_idesc(128, 64, 0, 1);  // P (tmem) x V (MN-major)
        auto issue_s = [&](int j) {
            const int s = j % kStages;
            if (!warp_wait(&sm.k_full[s], (j / kStages) & 1, limit, abort_flag, p.status)) return false;
            tc_fence_after();
            if (elect_one()) {
                const uint32_t idesc = make_idesc(128, 32 * blocks_of(j), 0, 0) | minus;
                const uint64_t dk = s ? dk1 : dk0;
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) mma_ss(tmem + kColS, dq + 2 * kk, dk + 2 * kk, idesc, kk > 0);
                mma_commit(&sm.k_free[s]);
                mma_commit(&sm.s_full);
            }
            __syncwarp();
            return true;
        };
        bool ok = n > 0 && warp_wait(&sm.q_full, 0, limit, abort_flag, p.status) && issue_s(0);
        for (int j = 0; ok && j < n; ++j) {
            const int s = j % kStages;
            if (j + 1 < n) {
                if (!warp_wait(&sm.s_free, j & 1, limit, abort_flag, p.status) || !issue_s(j + 1)) break;
            }
            if (!warp_wait(&sm.v_full[s], (j / kStages) & 1, limit, abort_flag, p.status)) break;
            if (!warp_wait(&sm.p_ready, j & 1, limit, abort_flag, p.status)) break;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t dv = s ? dv1 : dv0;
                const int steps = 2 * blocks_of(j);
                for (int kk = 0; kk < steps; ++kk)       // 16 keys: 8 columns of P, 2048 bytes of V
                    mma_ts(tmem + kColO, tmem + kColP + 8 * kk, dv + 128 * kk, idesc_pv, j > 0 || kk > 0);
                mma_commit(&sm.v_free[s]);
                mma_commit(&sm.o_done);
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
        const int row = warp * 32 + lane, t = q0 + row;
        const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
        const int tw0 = q0 + warp * 32, tw1 = tw0 + 31;          // the warp's queries
        float m = -INFINITY, l[4] = {0.0f, 0.0f, 0.0f, 0.0f};     // (four sums: no long chain of additions)
        bool ok = true;
        for (int j = 0; j < n; ++j) {
            const int k0 = tile_of(j) * kRows, blocks = blocks_of(j);
            // what the warp sees of each block: 0 nothing, 1 part, 2 all
            int vis[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int s0 = k0 + 32 * c, s1 = s0 + 31;
                const bool any = c < blocks && s0 <= tw1 && s0 < len && (tw0 - s1 < p.window || s0 < p.sinks);
                const bool all = s1 <= tw0 && s1 < len && (tw1 - s0 < p.window || s1 < p.sinks);
                vis[c] = !any ? 0 : all ? 2 : 1;
            }
            if (!(ok = warp_wait(&sm.s_full, j & 1, limit, abort_flag, p.status))) break;
            tc_fence_after();
            uint32_t sv[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (vis[c]) tmem_ld32(lanes + kColS + 32 * c, sv[c]);
            tmem_wait_ld();
            tc_fence_before();
            mbar_arrive(&sm.s_free);
            float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
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
            // P of the tile before has been used, and O is complete up to it
            if (j > 0 && !(ok = warp_wait(&sm.o_done, (j - 1) & 1, limit, abort_flag, p.status))) break;
            tc_fence_after();
            const bool grow = top > m + 8.0f || (m == -INFINITY && top > m);
            if (j == 0) {
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
            for (int c = 0; c < 4; ++c) {
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
                tmem_st16(lanes + kColP + 16 * c, pk);
            }
            // values past the sequence's end do not count, whatever they are
            if (len < p.T && k0 + kRows > len) {
                if (!(ok = warp_wait(&sm.v_full[j % kStages], (j / kStages) & 1, limit, abort_flag, p.status))) break;
                if (k0 + row >= len) zero_row(sm.v[j % kStages] + row * 128);
                fence_proxy_async();
            }
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(&sm.p_ready);
        }
        if (ok && n > 0) ok = warp_wait(&sm.o_done, (n - 1) & 1, limit, abort_flag, p.status);
        if (ok) {
            tc_fence_after();
            const float sum = (l[0] + l[1]) + (l[2] + l[3]);
            const bool none = t >= len || sum == 0.0f;
            const float inv = none ? 0.0f : 1.0f / sum;
            if (p.lse && t < p.T)
                p.lse[(long long)bh * p.T + t] = none ? -INFINITY : m * kLn2 + logf(sum);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t o[32];
                if (n > 0) {
                    tmem_ld32(lanes + kColO + 32 * c, o);
                    tmem_wait_ld();
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        w[e] = none ? 0u : pack_bf16(__uint_as_float(o[8 * i + 2 * e]) * inv, __uint_as_float(o[8 * i + 2 * e + 1]) * inv);
                    reinterpret_cast<uint4*>(sm.q + row * 128)[(4 * c + i) ^ (row & 7)] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            fence_proxy_async();
            tc_fence_before();
            mbar_arrive(&sm.st_ready);
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 4) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

}  // namespace

cudaError_t launch_window_forward_tc(const WindowArgs& a, cudaStream_t st)
{
    CUtensorMap mq, mk, mv, mo;
    if (!encode_rows_map(&mq, a.q, a.d, a.B, a.T, a.Hq, a.qs, kRows) || !encode_rows_map(&mk, a.k, a.d, a.B, a.T, a.Hk, a.ks, kRows) ||
        !encode_rows_map(&mv, a.v, a.d, a.B, a.T, a.Hk, a.vs, kRows) || !encode_rows_map(&mo, a.o, a.d, a.B, a.T, a.Hq, a.os, kRows))
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
