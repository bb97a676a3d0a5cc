// Causal attention over packed sequences, forward, on the tensor cores (bf16):
//
//     S = Q K^T (tcgen05 128 x 128 x 64, smem x smem) ,  P = 2^(S c - m) with c = scale log2(e) ,
//     O += P V (128 x 64 x 128, P from TMEM) ,  l += rowsum(P) ,  o = O / l ,  lse = (m + log2 l) ln 2 .
//
// A unit of work is 256 queries of one head of one sequence.  One CTA per SM stays for the whole launch and
// takes units one after another, the longest of a sequence first, rank and counter-rank in turn so that the long and the
// short ones even out.  Two groups of four warps have 128 queries each, one thread a row; both go over the
// same tiles of 128 keys, which are fetched once for the two (a tile for each group would be 43 bytes a
// clock and SM, more than L2 gives).  A warp per group issues its products, one more warp the loads.
// S, P and O of a group have TMEM columns of their own (128 + 64 + 64, the SM's 512 in all): the next tile's S
// is made while this tile's exponentials run.  Only the last tile of a group lies on the diagonal, and there
// a warp leaves out the 32-column blocks that none of its rows sees.
//
// m is a lagging maximum: it moves, and O and l are scaled, only when a row's maximum has grown by more than 8
// (a factor 2^8, far inside the range of fp32 and bf16), which after the first tiles is rare.
//
// P is rounded to bf16 where it enters P V, as the tensor cores take it beside bf16 values: 2^-9 of each term, which
// adds up like noise (l sums the P that were not rounded).
//
// All waits are bounded (see mbar_wait); a wait that gives up sets the status word and the CTA leaves through
// the normal exit with its copies landed and its TMEM freed.
#include "lasad_full.cuh"
#include "lasad_window_tma.cuh"

namespace lasad {
namespace {

using namespace tcx;

constexpr int kRows = 128, kCols = 128, kStages = 4, kGroups = 2, kUnit = kGroups * kRows;
constexpr int kSoftmaxWarps = 4 * kGroups, kThreads = 32 * (kSoftmaxWarps + 4);
constexpr int kTile = kCols * 128;                         // bytes of a tile of queries, keys or values
constexpr int kSoftmaxRegs = 216, kOtherRegs = 72;         // 2 x 128 x 216 + 128 x 72 = 384 x 168, the launch's own
constexpr uint32_t kColS = 0, kColP = 256, kColO = 384;    // + 128, 64, 64 columns per group
constexpr int kTmemCols = 512;

struct Smem {
    unsigned char q[2][kGroups][kTile];                    // of two units
    unsigned char k[kStages][kTile];
    unsigned char v[kStages][kTile];
    unsigned long long q_full[2], q_free[2];               // a unit's Q has landed; its last S has been made (both groups)
    unsigned long long full[kStages], free[kStages];       // a tile's K and V have landed; both groups are done with them
    unsigned long long s_full[kGroups];                    // S of a group's tile is in TMEM
    unsigned long long s_free[kGroups];                    // ... and has been read (128 arrivals)
    unsigned long long p_ready[kGroups];                   // P is in TMEM (128 arrivals)
    unsigned long long o_done[kGroups];                    // P V has been added
    unsigned long long drain[kGroups];
    uint32_t tmem_base;
    int abort_flag;
};

struct Params {
    int N, S, Hq, G, units;
    float scale2;                // |scale| log2(e), at least 1e-37
    bool negate;                 // scale < 0
    const int* offsets;
    __nv_bfloat16* o;
    long long os[2];
    int d;
    float* lse;
    int* status;
    unsigned wait_limit;
};

struct Unit {
    Region r;
    int h;
    int tiles0, tiles1, n;       // key tiles of each group, and of the unit
    __device__ __forceinline__ void set(const Params& p, int u)
    {
        const int at = u / p.Hq;
        h = u - at * p.Hq;
        r = region_of<kUnit>(p.offsets, p.S, p.N, (int)region_tiles(p.N, p.S, kUnit) - 1 - at);
        tiles0 = r.owned && r.first < r.len ? r.first / kCols + 1 : 0;
        tiles1 = r.owned && r.first + kRows < r.len ? tiles0 + 1 : 0;
        n = max(tiles0, tiles1);
    }
    __device__ __forceinline__ int tiles(int g) const { return g ? tiles1 : tiles0; }
};
// The i-th unit of a CTA (or one past the last).
__device__ __forceinline__ int unit_of(int i)
{
    const int n = gridDim.x, c = blockIdx.x;
    return i * n + ((i & 1) ? n - 1 - c : c);
}
__device__ __forceinline__ int rounds(const Params& p) { return (p.units + gridDim.x - 1) / gridDim.x; }

template <int N> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

__device__ __forceinline__ void load_tiles(const Params& p, Smem& sm, const CUtensorMap* tm_q, const CUtensorMap* tm_k,
                                           const CUtensorMap* tm_v)
{
    volatile int* abort_flag = &sm.abort_flag;
    int issued = 0, q = 0;                                 // tiles, units asked for
    bool ok = true;
    for (int i = 0; ok && i < rounds(p); ++i) {
        const int u = unit_of(i);
        if (u >= p.units) continue;
        Unit w;
        w.set(p, u);
        if (w.n == 0) continue;
        if (q >= 2 && !(ok = mbar_wait(&sm.q_free[q & 1], ((q >> 1) - 1) & 1, p.wait_limit, abort_flag, p.status))) break;
        const int row = w.r.start + w.r.first;
        mbar_arrive_expect_tx(&sm.q_full[q & 1], (w.tiles1 ? 2 : 1) * kTile);
        tma_load_4d(sm.q[q & 1][0], tm_q, &sm.q_full[q & 1], 0, w.h, row, 0);
        if (w.tiles1) tma_load_4d(sm.q[q & 1][1], tm_q, &sm.q_full[q & 1], 0, w.h, row + kRows, 0);
        ++q;
        const int hk = w.h / p.G;
        for (int j = 0; j < w.n; ++j, ++issued) {
            const int s = issued % kStages, round = issued / kStages;
            if (round > 0 && !(ok = mbar_wait(&sm.free[s], (round - 1) & 1, p.wait_limit, abort_flag, p.status))) break;
            mbar_arrive_expect_tx(&sm.full[s], 2 * kTile);
            tma_load_4d(sm.k[s], tm_k, &sm.full[s], 0, hk, w.r.start + j * kCols, 0);
            tma_load_4d(sm.v[s], tm_v, &sm.full[s], 0, hk, w.r.start + j * kCols, 0);
        }
    }
    // leave only when every issued load has landed
    for (int j = max(0, issued - kStages); j < issued; ++j)
        for (unsigned it = 0; it < kDrainLimit; ++it)
            if (mbar_try_wait(&sm.full[j % kStages], (j / kStages) & 1)) break;
    for (int j = max(0, q - 2); j < q; ++j)
        for (unsigned it = 0; it < kDrainLimit; ++it)
            if (mbar_try_wait(&sm.q_full[j & 1], (j >> 1) & 1)) break;
}

// Where a group stands: its units with tiles, their tiles, and the CTA's tiles (which choose the stage).
struct Walk {
    Unit w;
    int i, j, q, tile;           // round, tile of the unit, units so far, tiles of the CTA so far
    bool live;
    __device__ __forceinline__ void find(const Params& p)
    {
        for (; i < rounds(p); ++i) {
            const int u = unit_of(i);
            if (u >= p.units) continue;
            w.set(p, u);
            if (w.n > 0) {
                live = true;
                return;
            }
        }
        live = false;
    }
    __device__ __forceinline__ void start(const Params& p)
    {
        i = j = q = tile = 0;
        find(p);
    }
    __device__ __forceinline__ void next(const Params& p)
    {
        ++tile;
        if (++j < w.n) return;
        j = 0;
        ++q;
        ++i;
        find(p);
    }
};

__device__ __forceinline__ void issue_products(const Params& p, Smem& sm, int g, uint32_t tmem)
{
    volatile int* abort_flag = &sm.abort_flag;
    const unsigned limit = p.wait_limit;
    const uint32_t at_s = tmem + kColS + g * 128, at_p = tmem + kColP + g * 64, at_o = tmem + kColO + g * 64;
    const uint64_t dq = make_desc(smem_u32(sm.q[0][g])), dk = make_desc(smem_u32(sm.k[0])), dv = make_desc(smem_u32(sm.v[0]));
    constexpr uint64_t stage = kTile >> 4, next_q = kGroups * stage;
    const uint32_t idesc_s = make_idesc(128, 128, 0, 0) | (p.negate ? 1u << 13 : 0u);   // (the descriptor's negation of A)
    constexpr uint32_t idesc_pv = make_idesc(128, 64, 0, 1);   // P (tmem) x V (MN-major)
    Walk a;                                                // at the tile whose S comes next
    a.start(p);
    // To the next tile that the group has, past those that only the other one has (its Q and stages are let go
    // all the same, each after it has landed, so that no barrier is a phase ahead).
    auto skip = [&]() {
        while (a.live && a.j >= a.w.tiles(g)) {
            if (!warp_wait(&sm.full[a.tile % kStages], (a.tile / kStages) & 1, limit, abort_flag, p.status)) return false;
            if (a.j == 0 && !warp_wait(&sm.q_full[a.q & 1], (a.q >> 1) & 1, limit, abort_flag, p.status)) return false;
            if (elect_one()) {
                mbar_arrive(&sm.free[a.tile % kStages]);
                if (a.j == 0) mbar_arrive(&sm.q_free[a.q & 1]);
            }
            __syncwarp();
            a.next(p);
        }
        return true;
    };
    auto scores = [&]() {
        const int s = a.tile % kStages;
        if (a.j == 0 && !warp_wait(&sm.q_full[a.q & 1], (a.q >> 1) & 1, limit, abort_flag, p.status)) return false;
        if (!warp_wait(&sm.full[s], (a.tile / kStages) & 1, limit, abort_flag, p.status)) return false;
        tc_fence_after();
        if (elect_one()) {
            const uint64_t q = dq + (a.q & 1) * next_q;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) mma_ss(at_s, q + 2 * kk, dk + s * stage + 2 * kk, idesc_s, kk > 0);
            mma_commit(&sm.s_full[g]);
            if (a.j == a.w.tiles(g) - 1) mma_commit(&sm.q_free[a.q & 1]);
        }
        __syncwarp();
        return true;
    };
    bool ok = skip() && (!a.live || scores());
    for (int J = 0; ok && a.live; ++J) {
        const int s = a.tile % kStages;
        const bool opens = a.j == 0;
        a.next(p);                                         // (now at the tile of J + 1, or past some that are not the group's)
        // S of tile J has been read: the next one may have its place
        if (!(ok = warp_wait(&sm.s_free[g], J & 1, limit, abort_flag, p.status))) break;
        // (also a new unit's: its Q has a place of its own, and its stage does not wait for this tile's)
        const bool now = a.live && a.j < a.w.tiles(g);
        if (now && !(ok = scores())) break;
        if (!(ok = warp_wait(&sm.p_ready[g], J & 1, limit, abort_flag, p.status))) break;
        tc_fence_after();
        if (elect_one()) {
            const uint64_t v = dv + s * stage;
#pragma unroll
            for (int kk = 0; kk < 8; ++kk)                 // 16 keys: 8 columns of P, 2048 bytes of V
                mma_ts(at_o, at_p + 8 * kk, v + 128 * kk, idesc_pv, !opens || kk > 0);
            mma_commit(&sm.o_done[g]);
            mma_commit(&sm.free[s]);
        }
        __syncwarp();
        if (!now && !(ok = skip() && (!a.live || scores()))) break;
    }
    // no product may still run when the CTA's memory goes
    if (elect_one()) {
        mma_commit(&sm.drain[g]);
        for (unsigned it = 0; it < kDrainLimit; ++it)
            if (mbar_try_wait(&sm.drain[g], 0)) break;
    }
    __syncwarp();
}

__device__ __forceinline__ void softmax_rows(const Params& p, Smem& sm, int g, int quad, int lane, uint32_t tmem)
{
    volatile int* abort_flag = &sm.abort_flag;
    const unsigned limit = p.wait_limit;
    const int row = quad * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
    const uint32_t at_s = lanes + kColS + g * 128, at_p = lanes + kColP + g * 64, at_o = lanes + kColO + g * 64;
    bool ok = true;
    int J = 0, tile = 0;                                   // the group's tiles so far, and the CTA's
    for (int i = 0; ok && i < rounds(p); ++i) {
        const int u = unit_of(i);
        if (u >= p.units) continue;
        Unit w;
        w.set(p, u);
        const int n = w.tiles(g), t = w.r.first + g * kRows + row;     // the thread's query
        float m = -INFINITY, l[4] = {0.0f, 0.0f, 0.0f, 0.0f};          // (four sums: no long chain of additions)
        for (int j = 0; j < n; ++j, ++J) {
            // what the warp sees of each 32-column block: 0 nothing, 1 part, 2 all
            const bool diagonal = j == n - 1;
            if (!(ok = warp_wait(&sm.s_full[g], J & 1, limit, abort_flag, p.status))) break;
            tc_fence_after();
            uint32_t sv[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(at_s + 32 * c, sv[c]);
            tmem_wait_ld();
            tc_fence_before();
            mbar_arrive(&sm.s_free[g]);
            if (diagonal) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint32_t bits = c < quad ? 0xffffffffu : c > quad ? 0u : 0xffffffffu >> (31 - lane);
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (!((bits >> e) & 1u)) sv[c][e] = 0xff800000u;     // -infinity
                }
            }
            float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int e = 0; e < 32; e += 2) tops[c] = max3(tops[c], __uint_as_float(sv[c][e]), __uint_as_float(sv[c][e + 1]));
            const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * p.scale2;
            // P of the tile before has been used, and O is complete up to it
            if (J > 0 && !(ok = warp_wait(&sm.o_done[g], (J - 1) & 1, limit, abort_flag, p.status))) break;
            tc_fence_after();
            const bool grow = top > m + 8.0f || (m == -INFINITY && top > m);
            if (j == 0) {
                m = top;
            } else if (__any_sync(0xffffffffu, grow)) {
                // (every row of the warp moves to its maximum now, or its turn would come one by one)
                const float now = fmaxf(m, top), f = now == m ? 1.0f : ex2_approx(m - now);
                m = now;
#pragma unroll
                for (int e = 0; e < 4; ++e) l[e] *= f;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t o[16];
                    tmem_ld16(at_o + 16 * c, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                    tmem_st16(at_o + 16 * c, o);
                }
            }
            const float base = m == -INFINITY ? 0.0f : -m;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t pk[16];
                if (!diagonal || c <= quad) {
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
                tmem_st16(at_p + 16 * c, pk);
            }
            // values past the sequence's end do not count, whatever they are
            if ((j + 1) * kCols > w.r.len) {
                if (j * kCols + row >= w.r.len) zero_row(sm.v[(tile + j) % kStages] + row * 128);
                fence_proxy_async();
            }
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(&sm.p_ready[g]);
        }
        if (!ok) break;
        tile += w.n;
        const float sum = (l[0] + l[1]) + (l[2] + l[3]);
        if (n > 0 && !(ok = warp_wait(&sm.o_done[g], (J - 1) & 1, limit, abort_flag, p.status))) break;
        tc_fence_after();
        const bool none = n == 0 || sum == 0.0f, live = t < w.r.len;
        const float inv = none ? 0.0f : 1.0f / sum;
        if (p.lse && live) p.lse[(long long)w.h * p.N + w.r.start + t] = none ? -INFINITY : m * kLn2 + logf(sum);
        __nv_bfloat16* out = p.o + (long long)(w.r.start + t) * p.os[0] + w.h * p.os[1];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint32_t o[32];
            if (n > 0) {
                tmem_ld32(at_o + 32 * c, o);
                tmem_wait_ld();
            }
            if (live && 32 * c < p.d)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[e] = none ? 0u : pack_bf16(__uint_as_float(o[8 * k + 2 * e]) * inv, __uint_as_float(o[8 * k + 2 * e + 1]) * inv);
                    *reinterpret_cast<uint4*>(out + 32 * c + 8 * k) = make_uint4(x[0], x[1], x[2], x[3]);
                }
        }
        // (the next unit's first P V comes after its P, which these threads write after this)
        tc_fence_before();
    }
}

__global__ void __launch_bounds__(kThreads, 1)
packed_forward_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                         const __grid_constant__ CUtensorMap tm_v, const Params p)
{
    extern __shared__ unsigned char smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;

    if (tid == 0) {
        for (int s = 0; s < 2; ++s) {
            mbar_init(&sm.q_full[s], 1);
            mbar_init(&sm.q_free[s], kGroups);
        }
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm.full[s], 1);
            mbar_init(&sm.free[s], kGroups);
        }
        for (int g = 0; g < kGroups; ++g) {
            mbar_init(&sm.s_full[g], 1);
            mbar_init(&sm.s_free[g], kRows);
            mbar_init(&sm.p_ready[g], kRows);
            mbar_init(&sm.o_done[g], 1);
            mbar_init(&sm.drain[g], 1);
        }
        sm.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // (TMEM only after the kernel before has ended, the next kernel only after the TMEM: see the window's forward)
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

    if (warp >= kSoftmaxWarps) {
        regs_down<kOtherRegs>();
        if (warp == kSoftmaxWarps) {
            if (elect_one()) load_tiles(p, sm, &tm_q, &tm_k, &tm_v);
            __syncwarp();
        } else if (warp <= kSoftmaxWarps + kGroups) {
            issue_products(p, sm, warp - kSoftmaxWarps - 1, tmem);
        }
    } else {
        regs_up<kSoftmaxRegs>();
        softmax_rows(p, sm, warp >> 2, warp & 3, lane, tmem);
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

// [N,H,d] with element strides of (token, head) -> the rows map's (d, h, t, b) with one batch element
bool encode_packed(CUtensorMap* map, const void* base, int d, int N, int H, const long long (&s)[2], int rows)
{
    const long long strides[3] = {0, s[0], s[1]};
    return encode_rows_map(map, base, d, 1, N, H, strides, rows);
}

}  // namespace

cudaError_t launch_packed_forward_tc(const PackedArgs& a, cudaStream_t st)
{
    CUtensorMap mq, mk, mv;
    if (!encode_packed(&mq, a.q, a.d, a.N, a.Hq, a.qs, kRows) || !encode_packed(&mk, a.k, a.d, a.N, a.Hk, a.ks, kCols) ||
        !encode_packed(&mv, a.v, a.d, a.N, a.Hk, a.vs, kCols))
        return cudaErrorInvalidValue;
    static bool done[64];
    const size_t smem = sizeof(Smem) + 1024;
    const cudaError_t e = allow_dynamic_smem(packed_forward_tc_kernel, smem, done);
    if (e != cudaSuccess) return e;
    Params p{a.N, a.S, a.Hq, a.Hq / a.Hk, (int)region_tiles(a.N, a.S, kUnit) * a.Hq, fmaxf(fabsf(a.scale) * kLog2e, 1e-37f),
             a.scale < 0.0f, a.offsets, static_cast<__nv_bfloat16*>(a.o), {a.os[0], a.os[1]}, a.d, a.lse, a.status, a.wait_limit};
    return launch_dependent(packed_forward_tc_kernel, dim3(p.units < a.sms ? p.units : a.sms), dim3(kThreads), smem, st, mq, mk, mv, p);
}

}  // namespace lasad
