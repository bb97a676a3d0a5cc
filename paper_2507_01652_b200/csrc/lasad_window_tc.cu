// Window attention, forward, on the tensor cores (bf16):
//
//     S = Q K^T (tcgen05 128 x 64 x 64, smem x smem) ,  P = 2^(S c - m) with c = scale log2(e) ,
//     O += P V (128 x 64 x 64, P from TMEM) ,  l += rowsum(P) ,  o = O / l ,  lse = (m + log2 l) ln 2 .
//
// A unit of work is 128 queries of one head, over the visible tiles of 64 keys only: from the
// window's edge to the diagonal and, where the window has left them, the tiles of the sinks.  One CTA per SM stays for the whole launch; in it three groups of
// warps take units on their own, one after another: four softmax warps and one that issues the
// products; one more warp asks for the tiles of all three.  One thread has one row, so its maximum and
// sum need no exchange.  m is a lagging maximum: it moves, and O and l are scaled, only when a row's
// maximum has grown by more than 8 (a factor 2^8, far inside the range of fp32 and bf16), which after
// the first tiles is rare.  32-column blocks that no row of a warp sees are skipped, and only blocks on
// an edge are masked.
//
// What bounds it: the exponentials, 16 per SM and clock, are 512 clocks for a 128 x 64 tile, and its
// products 320.  A tile costs each of its group's warps 460 instructions and its group about 2700 clocks, most of
// them latency (S out of TMEM, the maximum, P into TMEM, the barriers), so that three groups bring
// one every 900.  S, P and O have columns of their own (160 a group, 480 of the SM's 512): the next
// tile's S is made while this tile's exponentials run.  Measured: 1 x 9217 tokens, 24 query and 8 key
// heads, window 1536: 162 us; 64 x 577 tokens, 16 heads, window 144: 124 us (in a graph; alone in a cold
// cache 179 and 136).  (Two CTAs of two groups with P over S, so that a tile's products stood between two
// tiles' exponentials, cost 170 and 162 us where the step to this form brought 168 and 147; tiles of 128 keys do
// not fit the registers: 363 us for the first.)
//
// P is rounded to bf16 where it enters P V, as the tensor cores take it beside bf16 values: 2^-9 of each term,
// which adds up like noise (l sums the P that were not rounded).  Against 64 bits o is off by 0.21 % of its size,
// 0.16 of which is its own rounding to bf16.  P as a sum of two bf16 numbers would cost a second P V and 32 columns
// a group more than TMEM has; a caller who needs 32 bits has the CUDA-core kernel (LASAD_OPT_WINDOW_IMPL).
//
// All waits are bounded (see mbar_wait); a wait that gives up sets the status word and the CTA leaves
// through the normal exit with its copies landed and its TMEM freed.
#include "lasad_window_tma.cuh"

namespace lasad {
namespace {

using namespace tcx;

constexpr int kRows = 128, kCols = 64, kStages = 3, kGroups = 3;
constexpr int kSoftmaxWarps = 4 * kGroups, kThreads = 32 * (kSoftmaxWarps + kGroups + 1);
constexpr int kTile = kCols * 128;                         // bytes of a key or value tile
constexpr uint32_t kColS = 0, kColP = 64, kColO = 96, kGroupCols = 160;
constexpr int kTmemCols = 512;

struct Group {
    unsigned char q[kRows * 128];
    unsigned char k[kStages][kTile];
    unsigned char v[kStages][kTile];
};
struct Barriers {
    unsigned long long q_full, q_free;         // a unit's Q has landed; its last S has been made
    unsigned long long full[kStages], free[kStages];   // a tile's K and V have landed; its P V has been added
    unsigned long long s_full;                 // S of a tile is in TMEM
    unsigned long long s_free;                 // ... and has been read (128 arrivals)
    unsigned long long p_ready;                // P of a tile is in TMEM (128 arrivals)
    unsigned long long o_done;                 // P V of a tile has been added
    unsigned long long drain;
};
struct Smem {
    Group g[kGroups];
    Barriers bar[kGroups];
    uint32_t tmem_base;
    int abort_flag;
};

struct Params {
    int B, T, Hq, Hk, window, sinks, units;
    float scale2;                // |scale| log2(e), at least 1e-37
    bool negate;                 // scale < 0
    const int* lengths;
    __nv_bfloat16* o;
    long long os[3];
    int d;
    float* lse;
    int* status;
    unsigned wait_limit;
};

// One unit: its rows and its key tiles.
struct Unit {
    int b, h, hk, q0, len;
    int lo, extra, n;            // key tiles 0 .. extra - 1 (the sinks'), then lo .. lo + n - extra - 1
    // the last query tiles, which have the most key tiles, come first
    __device__ __forceinline__ void set(const Params& p, int u)
    {
        const int BH = p.B * p.Hq, tiles = (p.T + kRows - 1) / kRows;
        const int at = u / BH, bh = u - at * BH;
        b = bh / p.Hq;
        h = bh - b * p.Hq;
        hk = h / (p.Hq / p.Hk);
        q0 = (tiles - 1 - at) * kRows;
        len = p.lengths ? max(0, min(p.lengths[b], p.T)) : p.T;
        lo = extra = n = 0;
        if (q0 < len) {
            lo = q0 >= p.window ? (q0 - p.window + 1) / kCols : 0;
            extra = min(lo, (p.sinks + kCols - 1) / kCols);
            n = extra + (min(q0 + kRows, len) + kCols - 1) / kCols - lo;
        }
    }
    __device__ __forceinline__ int first_of(int i) const { return (i < extra ? i : lo + i - extra) * kCols; }
};

// A walk over the tiles of all units of a group (unit first, first + step, ..).
struct Walk {
    Unit u;
    int unit, step, i;
    bool live;
    __device__ __forceinline__ void find(const Params& p)
    {
        for (; unit < p.units; unit += step) {
            u.set(p, unit);
            if (u.n > 0) {
                live = true;
                return;
            }
        }
        live = false;
    }
    __device__ __forceinline__ void start(const Params& p, int first, int by)
    {
        unit = first;
        step = by;
        i = 0;
        find(p);
    }
    __device__ __forceinline__ void next(const Params& p)
    {
        if (!live || ++i < u.n) return;
        i = 0;
        unit += step;
        find(p);
    }
};

__global__ void __launch_bounds__(kThreads, 1)
window_forward_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                         const __grid_constant__ CUtensorMap tm_v, const Params p)
{
    extern __shared__ unsigned char smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    volatile int* abort_flag = &sm.abort_flag;
    const unsigned limit = p.wait_limit;

    if (tid == 0) {
        for (int g = 0; g < kGroups; ++g) {
            Barriers& bar = sm.bar[g];
            mbar_init(&bar.q_full, 1);
            mbar_init(&bar.q_free, 1);
            for (int s = 0; s < kStages; ++s) {
                mbar_init(&bar.full[s], 1);
                mbar_init(&bar.free[s], 1);
            }
            mbar_init(&bar.s_full, 1);
            mbar_init(&bar.s_free, kRows);
            mbar_init(&bar.p_ready, kRows);
            mbar_init(&bar.o_done, 1);
            mbar_init(&bar.drain, 1);
        }
        sm.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // What this kernel reads may come from the one before it; its TMEM is taken only now, too, so that it
    // never holds columns that a late CTA of that kernel waits for, and the next kernel is let in
    // only when every CTA of this one has its own.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == 0) {
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

    if (warp == kSoftmaxWarps + kGroups) {
        // ===================== the loads of all groups: one thread goes round them =====================
        if (elect_one()) {
            Walk walk[kGroups];
            int issued[kGroups], q[kGroups], left = 0;            // tiles, units asked for; groups with more to ask for
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                walk[g].start(p, g * gridDim.x + blockIdx.x, kGroups * gridDim.x);
                issued[g] = q[g] = 0;
                left += walk[g].live;
            }
            unsigned idle = 0;
            while (left > 0) {
                bool some = false;
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    Walk& w = walk[g];
                    if (!w.live) continue;
                    Barriers& bar = sm.bar[g];
                    const int s = issued[g] % kStages, round = issued[g] / kStages;
                    if (round > 0 && !mbar_test_wait(&bar.free[s], (round - 1) & 1)) continue;
                    if (w.i == 0) {
                        if (q[g] > 0 && !mbar_test_wait(&bar.q_free, (q[g] - 1) & 1)) continue;
                        mbar_arrive_expect_tx(&bar.q_full, kRows * 128);
                        tma_load_4d(sm.g[g].q, &tm_q, &bar.q_full, 0, w.u.h, w.u.q0, w.u.b);
                        ++q[g];
                    }
                    mbar_arrive_expect_tx(&bar.full[s], 2 * kTile);
                    tma_load_4d(sm.g[g].k[s], &tm_k, &bar.full[s], 0, w.u.hk, w.u.first_of(w.i), w.u.b);
                    tma_load_4d(sm.g[g].v[s], &tm_v, &bar.full[s], 0, w.u.hk, w.u.first_of(w.i), w.u.b);
                    ++issued[g];
                    w.next(p);
                    left -= !w.live;
                    some = true;
                }
                idle = some ? 0 : idle + 1;
                if (!some && ((idle & 63u) == 63u && *abort_flag)) break;
                if (idle > limit) {
                    *abort_flag = 1;
                    atomicExch(p.status, 1);
                    break;
                }
            }
            // leave only when every issued load has landed
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                for (int j = max(0, issued[g] - kStages); j < issued[g]; ++j)
                    for (unsigned it = 0; it < kDrainLimit; ++it)
                        if (mbar_try_wait(&sm.bar[g].full[j % kStages], (j / kStages) & 1)) break;
                if (q[g] > 0)
                    for (unsigned it = 0; it < kDrainLimit; ++it)
                        if (mbar_try_wait(&sm.bar[g].q_full, (q[g] - 1) & 1)) break;
            }
        }
        __syncwarp();
    } else if (warp >= kSoftmaxWarps) {
        // ===================== the products of group g =====================
        const int g = warp - kSoftmaxWarps;
        Barriers& bar = sm.bar[g];
        const uint32_t cols = tmem + g * kGroupCols;
        const uint64_t dq = make_desc(smem_u32(sm.g[g].q)), dk = make_desc(smem_u32(sm.g[g].k[0])), dv = make_desc(smem_u32(sm.g[g].v[0]));
        constexpr uint64_t stage = kTile >> 4;
        const uint32_t idesc_s = make_idesc(128, 64, 0, 0) | (p.negate ? 1u << 13 : 0u);   // (the descriptor's negation of A)
        constexpr uint32_t idesc_pv = make_idesc(128, 64, 0, 1);  // P (tmem) x V (MN-major)
        Walk walk;                                                // at the tile whose S comes next
        walk.start(p, g * gridDim.x + blockIdx.x, kGroups * gridDim.x);
        int units = 0;
        // S of tile number J
        auto scores = [&](int J) {
            const int s = J % kStages;
            if (walk.i == 0 && !warp_wait(&bar.q_full, units++ & 1, limit, abort_flag, p.status)) return false;
            if (!warp_wait(&bar.full[s], (J / kStages) & 1, limit, abort_flag, p.status)) return false;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) mma_ss(cols + kColS, dq + 2 * kk, dk + s * stage + 2 * kk, idesc_s, kk > 0);
                mma_commit(&bar.s_full);
                if (walk.i == walk.u.n - 1) mma_commit(&bar.q_free);
            }
            __syncwarp();
            return true;
        };
        bool first = true, ok = !walk.live || scores(0);          // first: tile J is its unit's first
        for (int J = 0; ok && walk.live; ++J) {
            const bool opens = first;
            walk.next(p);                                         // (now at tile J + 1)
            first = walk.i == 0;
            // S of tile J has been read: the next one may have its place (a new unit's waits for its Q: after
            // this unit's last P V)
            if (!(ok = warp_wait(&bar.s_free, J & 1, limit, abort_flag, p.status))) break;
            if (walk.live && !first && !(ok = scores(J + 1))) break;
            if (!(ok = warp_wait(&bar.p_ready, J & 1, limit, abort_flag, p.status))) break;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t at = dv + (J % kStages) * stage;
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)                    // 16 keys: 8 columns of P, 2048 bytes of V
                    mma_ts(cols + kColO, cols + kColP + 8 * kk, at + 128 * kk, idesc_pv, !opens || kk > 0);
                mma_commit(&bar.o_done);
                mma_commit(&bar.free[J % kStages]);
            }
            __syncwarp();
            if (walk.live && first && !(ok = scores(J + 1))) break;
        }
        // no product may still run when the CTA's memory goes
        if (elect_one()) {
            mma_commit(&bar.drain);
            for (unsigned it = 0; it < kDrainLimit; ++it)
                if (mbar_try_wait(&bar.drain, 0)) break;
        }
        __syncwarp();
    } else {
        // ===================== softmax warps of group g =====================
        const int g = warp >> 2, row = (warp & 3) * 32 + lane;
        const int first = g * gridDim.x + blockIdx.x, step = kGroups * gridDim.x;
        Barriers& bar = sm.bar[g];
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16) + g * kGroupCols;
        bool ok = true;
        int J = 0;                                                // the group's tiles so far
        Unit u;
        for (int unit = first; ok && unit < p.units; unit += step) {
            u.set(p, unit);
            const int t = u.q0 + row, tw0 = u.q0 + (warp & 3) * 32, tw1 = tw0 + 31;     // the warp's queries
            float m = -INFINITY, l[4] = {0.0f, 0.0f, 0.0f, 0.0f};     // (four sums: no long chain of additions)
            for (int i = 0; i < u.n; ++i, ++J) {
                const int k0 = u.first_of(i);
                // what the warp sees of each 32-column block: 0 nothing, 1 part, 2 all
                int vis[2] = {2, 2};
                const bool inside = k0 + kCols - 1 <= tw0 && k0 + kCols <= u.len && tw1 - k0 < p.window;
                if (!inside)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int s0 = k0 + 32 * c, s1 = s0 + 31;
                        const bool any = s0 <= tw1 && s0 < u.len && (tw0 - s1 < p.window || s0 < p.sinks);
                        const bool all = s1 <= tw0 && s1 < u.len && (tw1 - s0 < p.window || s1 < p.sinks);
                        vis[c] = !any ? 0 : all ? 2 : 1;
                    }
                if (!(ok = warp_wait(&bar.s_full, J & 1, limit, abort_flag, p.status))) break;
                tc_fence_after();
                uint32_t sv[2][32];
#pragma unroll
                for (int c = 0; c < 2; ++c) tmem_ld32(lanes + kColS + 32 * c, sv[c]);
                tmem_wait_ld();
                tc_fence_before();
                mbar_arrive(&bar.s_free);
                if (!inside) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        if (vis[c] != 2) {
                            const uint32_t bits = vis[c] ? seen_bits(t, k0 + 32 * c, p.window, p.sinks, u.len) : 0u;
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!((bits >> e) & 1u)) sv[c][e] = 0xff800000u;     // -infinity
                        }
                }
                float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 32; e += 2)
                        tops[(e >> 1) & 3] = max3(tops[(e >> 1) & 3], __uint_as_float(sv[c][e]), __uint_as_float(sv[c][e + 1]));
                const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * p.scale2;
                // P of the tile before has been used, and O is complete up to it
                if (J > 0 && !(ok = warp_wait(&bar.o_done, (J - 1) & 1, limit, abort_flag, p.status))) break;
                tc_fence_after();
                const bool grow = top > m + 8.0f || (m == -INFINITY && top > m);
                if (i == 0) {
                    m = top;
                } else if (__any_sync(0xffffffffu, grow)) {
                    // (every row of the warp moves to its maximum now, or its turn would come one by one: 25 % of
                    // the steps scaled where only rows that had grown moved)
                    const float now = fmaxf(m, top), f = now == m ? 1.0f : ex2_approx(m - now);
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
                if (u.len < p.T && k0 + kCols > u.len) {
                    if (row < kCols && k0 + row >= u.len) zero_row(sm.g[g].v[J % kStages] + row * 128);
                    fence_proxy_async();
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(&bar.p_ready);
            }
            if (!ok) break;
            const float sum = (l[0] + l[1]) + (l[2] + l[3]);
            if (u.n > 0 && !(ok = warp_wait(&bar.o_done, (J - 1) & 1, limit, abort_flag, p.status))) break;
            tc_fence_after();
            const bool none = t >= u.len || sum == 0.0f;
            const float inv = none ? 0.0f : 1.0f / sum;
            if (p.lse && t < p.T)
                p.lse[((long long)u.b * p.Hq + u.h) * p.T + t] = none ? -INFINITY : m * kLn2 + logf(sum);
            __nv_bfloat16* out = p.o + u.b * p.os[0] + (long long)t * p.os[1] + u.h * p.os[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t o[32];
                if (u.n > 0) {
                    tmem_ld32(lanes + kColO + 32 * c, o);
                    tmem_wait_ld();
                }
                if (t < p.T && 32 * c < p.d)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            w[e] = none ? 0u : pack_bf16(__uint_as_float(o[8 * k + 2 * e]) * inv, __uint_as_float(o[8 * k + 2 * e + 1]) * inv);
                        *reinterpret_cast<uint4*>(out + 32 * c + 8 * k) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
            }
            // (the next unit's first P V comes after its P, which these threads write after this)
            tc_fence_before();
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

}  // namespace

cudaError_t launch_window_forward_tc(const WindowArgs& a, cudaStream_t st)
{
    CUtensorMap mq, mk, mv;
    if (!encode_rows_map(&mq, a.q, a.d, a.B, a.T, a.Hq, a.qs, kRows) || !encode_rows_map(&mk, a.k, a.d, a.B, a.T, a.Hk, a.ks, kCols) ||
        !encode_rows_map(&mv, a.v, a.d, a.B, a.T, a.Hk, a.vs, kCols))
        return cudaErrorInvalidValue;
    static bool done[64];
    const size_t smem = sizeof(Smem) + 1024;
    const cudaError_t e = allow_dynamic_smem(window_forward_tc_kernel, smem, done);
    if (e != cudaSuccess) return e;
    Params p{a.B, a.T, a.Hq, a.Hk, a.window, a.sinks, (a.T + kRows - 1) / kRows * a.B * a.Hq,
             fmaxf(fabsf(a.scale) * kLog2e, 1e-37f), a.scale < 0.0f, a.lengths, static_cast<__nv_bfloat16*>(a.o),
             {a.os[0], a.os[1], a.os[2]}, a.d, a.lse, a.status, a.wait_limit};
    // one CTA per SM, fewer where there are fewer units than groups
    const int want = (p.units + kGroups - 1) / kGroups, grid = want < a.sms ? (p.units < a.sms ? p.units : a.sms) : a.sms;
    return launch_dependent(window_forward_tc_kernel, dim3(grid), dim3(kThreads), smem, st, mq, mk, mv, p);
}

}  // namespace lasad
