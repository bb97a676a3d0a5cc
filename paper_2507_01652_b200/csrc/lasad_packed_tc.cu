// Causal attention over packed sequences, forward, on the tensor cores (bf16):
//
//     S = Q K^T (tcgen05 128 x 64 x 64, smem x smem) ,  P = 2^(S c - m) with c = scale log2(e) ,
//     O += P V (128 x 64 x 64, P from TMEM) ,  l += rowsum(P) ,  o = O / l ,  lse = (m + log2 l) ln 2 .
//
// A unit of work is 256 queries of one head of one sequence.  One CTA per SM stays for the whole launch and
// takes units one after another, the longest of a sequence first: it is launched with one, and asks the hardware for
// the next CTA that has not begun (clusterlaunchcontrol), which leaves nothing in memory that two launches could
// share.  Two groups of four warps have 128 queries each, one thread a row; both go over the same tiles of 64
// keys, which are fetched once for the two.  A warp per group issues its products, one the loads, one finds the units.
//
// What bounds it: the exponentials (16 per SM and clock: 512 clocks for a 128 x 64 tile, its products 256).  So what a group
// does beside them is kept short, and lies under the other group's.  S and P of a group have two places
// each (2 x 64 and 2 x 32 TMEM columns, 64 for O, the SM's 512 for both groups): S of the next tile is there before
// this tile's P is.  A tile is one wait and one arrival for a thread: the products of P come ahead of the S that
// takes the same places' turn, so S being there says that P's place is free.  And the maximum is not waited for:
// P is formed with the m that the row has, its maximum beside it; only where that has grown by more than 8 (a factor
// 2^8, far inside the range of fp32 and bf16; after the first tiles rare) m moves, O and l are scaled and P is formed
// again, behind a wait for the first one's stores.
//
// Measured: 1 x 9217 tokens, 24 query and 8 key heads: 421 to 424 us, 617 TFLOP/s of the pairs that count, the pipe of the
// exponentials issuing on 56 % of the clocks; 64 sequences of 1 to 577 tokens, 16 and 4 heads: 61.5 us (d = 32, at d = 64's
// width: 421 and 60).  With clocks read in the loop (which slows it a little) a group alone takes 1290 clocks for a tile,
// 740 of them from the scores to P, the two groups together 1775 to 1800 for two tiles: they meet in the exponentials, also
// when one is made to start late (424 to 450 us).  Tried on that case, where a form without the care for empty rows and
// for rows behind the sequence's end took 418: 128-key tiles 421, with a quarter of the exponentials as polynomials 412 (tiles of 64 with an
// eighth, a quarter, three eighths: 429, 419, 444); sixteen warps on even and odd tiles 417; three groups 450 (and 83
// instead of 61 us on the short sequences); S issued right behind the product 429; masked and other tiles as two
// bodies 443; a short rolled body 462.
//
// P is rounded to bf16 where it enters P V, as the tensor cores take it beside bf16 values: 2^-9 of each term, which
// adds up like noise (l sums the P that were not rounded).
//
// All waits are bounded (see mbar_wait); a wait that gives up sets the status word and the CTA leaves through
// the normal exit with its copies landed and its TMEM freed.
#include "lasad_full.cuh"
#include "lasad_window_tma.cuh"

#include <cfloat>

namespace lasad {
namespace {

using namespace tcx;

constexpr int kRows = 128, kCols = 64, kStages = 8, kGroups = 2, kUnit = kGroups * kRows;
constexpr int kSoftmaxWarps = 4 * kGroups, kThreads = 32 * (kSoftmaxWarps + 4);
constexpr int kQTile = kRows * 128, kTile = kCols * 128;   // bytes of a tile of queries, and of keys or values
constexpr int kSoftmaxRegs = 216, kOtherRegs = 72;         // 2 x 128 x 216 + 128 x 72 = 384 x 168, the launch's own
constexpr uint32_t kGroupCols = 256, kColS = 0, kColP = 128, kColO = 192;
constexpr int kTmemCols = 512;

struct Unit {
    int start, len;              // of the sequence (or of rows that nobody has)
    int first, h;                // the unit's first row in it, and its head (-1: no more units)
    int tiles[kGroups];          // key tiles of each group
};
struct Smem {
    unsigned char q[2][kGroups][kQTile];                   // of two units
    unsigned char k[kStages][kTile];
    unsigned char v[kStages][kTile];
    uint4 answer;                                          // to the request for a unit
    Unit unit[2];
    unsigned long long answered;
    unsigned long long u_full[2], u_free[2];               // a unit is there; every role has read it
    unsigned long long q_full[2], q_free[2];               // a unit's Q has landed; its last S has been made (both groups)
    unsigned long long full[kStages], free[kStages];       // a tile's K and V have landed; both groups are done with them
    unsigned long long s_full[kGroups][2];                 // S of a tile is in TMEM, and its P's place is free
    unsigned long long p_ready[kGroups][2];                // S has been read and P is in TMEM (4 warps)
    // P V has been added: of even and odd tiles, as a warp that has seen S of tile J knows of tile J - 2's product and not of
    // the next one's (a barrier's parity tells only two neighbouring phases apart)
    unsigned long long o_done[kGroups][2];
    unsigned long long drain[kGroups];
    uint32_t tmem_base;
    int abort_flag;
};
constexpr int kReaders = 1 + kGroups + kSoftmaxWarps;      // of a unit: loads, products, softmax warps

struct Params {
    int N, S, Hq, G;
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

template <int N> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// Asks for a CTA of this launch that has not begun to be cancelled, so that its work can be done here.
__device__ __forceinline__ void ask_for_cta(void* answer, void* bar)
{
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(answer)),
                 "r"(smem_u32(bar))
                 : "memory");
}
// Its number, or -1 where none was left (then no more may be asked for).
__device__ __forceinline__ int cta_of(const void* answer)
{
    unsigned some, x;
    asm volatile(
        "{\n\t.reg .b128 a;\n\t.reg .pred p;\n\t.reg .b32 y, z, w;\n\t"
        "ld.shared.b128 a, [%2];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n\t"
        "selp.u32 %0, 1, 0, p;\n\tmov.u32 %1, 0;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, y, z, w}, a;\n\t}"
        : "=r"(some), "=r"(x)
        : "r"(smem_u32(answer))
        : "memory");
    return some ? (int)x : -1;
}

// Hands the CTA's units to the others (one thread).
__device__ __forceinline__ void find_units(const Params& p, Smem& sm)
{
    volatile int* abort_flag = &sm.abort_flag;
    int u = blockIdx.x, given = 0, asked = 0;
    for (;;) {
        Unit w;
        w.h = -1;
        if (u >= 0) {
            const int at = u / p.Hq;
            const Region r = region_of<kUnit>(p.offsets, p.S, p.N, (int)region_tiles(p.N, p.S, kUnit) - 1 - at);
            w.start = r.start, w.len = r.len, w.first = r.first;
            if (r.first < r.len) w.h = u - at * p.Hq;
            w.tiles[0] = r.owned ? (min(r.first + kRows, r.len) + kCols - 1) / kCols : 0;
            w.tiles[1] = r.owned && r.first + kRows < r.len ? (min(r.first + kUnit, r.len) + kCols - 1) / kCols : 0;
        }
        if (u < 0 || w.h >= 0) {
            const int s = given & 1;
            if (given >= 2 && !mbar_wait(&sm.u_free[s], ((given >> 1) - 1) & 1, p.wait_limit, abort_flag, p.status)) return;
            sm.unit[s] = w;
            mbar_arrive(&sm.u_full[s]);
            ++given;
        }
        if (u < 0) return;
        mbar_arrive_expect_tx(&sm.answered, 16);
        ask_for_cta(&sm.answer, &sm.answered);
        // (not given up: the answer comes without anyone's help, and would be written into memory that is gone)
        bool ok = false;
        for (unsigned it = 0; !ok && it < kDrainLimit; ++it) ok = mbar_try_wait(&sm.answered, asked & 1);
        if (!ok) {
            *abort_flag = 1;
            atomicExch(p.status, 1);
            return;
        }
        ++asked;
        u = cta_of(&sm.answer);
        fence_proxy_async();                               // (read before the next answer is written)
    }
}
// The next of them (`taken` so far); false where a wait gave up.  Whole warps read it, or one thread.
template <bool WARP> __device__ __forceinline__ bool next_unit(const Params& p, Smem& sm, int& taken, Unit& w)
{
    const int s = taken & 1, parity = (taken >> 1) & 1;
    volatile int* abort_flag = &sm.abort_flag;
    if (!(WARP ? warp_wait(&sm.u_full[s], parity, p.wait_limit, abort_flag, p.status)
               : mbar_wait(&sm.u_full[s], parity, p.wait_limit, abort_flag, p.status)))
        return false;
    w = sm.unit[s];
    if (WARP) {
        // (values that all lanes have, in a form that the compiler knows to be such)
        w.start = uniform(w.start), w.len = uniform(w.len), w.first = uniform(w.first), w.h = uniform(w.h);
        w.tiles[0] = uniform(w.tiles[0]), w.tiles[1] = uniform(w.tiles[1]);
        __syncwarp();
        if (elect_one()) mbar_arrive(&sm.u_free[s]);
        __syncwarp();
    } else {
        mbar_arrive(&sm.u_free[s]);
    }
    ++taken;
    return true;
}

__device__ __forceinline__ void load_tiles(const Params& p, Smem& sm, const CUtensorMap* tm_q, const CUtensorMap* tm_k,
                                           const CUtensorMap* tm_v)
{
    volatile int* abort_flag = &sm.abort_flag;
    int issued = 0, q = 0, taken = 0;                      // tiles, units asked for
    Unit w;
    while (next_unit<false>(p, sm, taken, w) && w.h >= 0) {
        const int n = max(w.tiles[0], w.tiles[1]);
        if (n == 0) continue;
        if (q >= 2 && !mbar_wait(&sm.q_free[q & 1], ((q >> 1) - 1) & 1, p.wait_limit, abort_flag, p.status)) break;
        const int row = w.start + w.first;
        mbar_arrive_expect_tx(&sm.q_full[q & 1], (w.tiles[1] ? 2 : 1) * kQTile);
        tma_load_4d(sm.q[q & 1][0], tm_q, &sm.q_full[q & 1], 0, w.h, row, 0);
        if (w.tiles[1]) tma_load_4d(sm.q[q & 1][1], tm_q, &sm.q_full[q & 1], 0, w.h, row + kRows, 0);
        ++q;
        const int hk = w.h / p.G;
        bool ok = true;
        for (int j = 0; j < n; ++j, ++issued) {
            const int s = issued % kStages, round = issued / kStages;
            if (round > 0 && !(ok = mbar_wait(&sm.free[s], (round - 1) & 1, p.wait_limit, abort_flag, p.status))) break;
            mbar_arrive_expect_tx(&sm.full[s], 2 * kTile);
            tma_load_4d(sm.k[s], tm_k, &sm.full[s], 0, hk, w.start + j * kCols, 0);
            tma_load_4d(sm.v[s], tm_v, &sm.full[s], 0, hk, w.start + j * kCols, 0);
        }
        if (!ok) break;
    }
    // leave only when every issued load has landed
    for (int j = max(0, issued - kStages); j < issued; ++j)
        for (unsigned it = 0; it < kDrainLimit; ++it)
            if (mbar_try_wait(&sm.full[j % kStages], (j / kStages) & 1)) break;
    for (int j = max(0, q - 2); j < q; ++j)
        for (unsigned it = 0; it < kDrainLimit; ++it)
            if (mbar_try_wait(&sm.q_full[j & 1], (j >> 1) & 1)) break;
}

__device__ __forceinline__ void issue_products(const Params& p, Smem& sm, int g, uint32_t tmem)
{
    volatile int* abort_flag = &sm.abort_flag;
    const unsigned limit = p.wait_limit;
    const uint32_t cols = tmem + g * kGroupCols;
    const uint64_t dq = make_desc(smem_u32(sm.q[0][g])), dk = make_desc(smem_u32(sm.k[0])), dv = make_desc(smem_u32(sm.v[0]));
    constexpr uint64_t stage = kTile >> 4, next_q = kGroups * (kQTile >> 4);
    const uint32_t idesc_s = make_idesc(128, 64, 0, 0) | (p.negate ? 1u << 13 : 0u);   // (the descriptor's negation of A)
    constexpr uint32_t idesc_pv = make_idesc(128, 64, 0, 1);   // P (tmem) x V (MN-major)
    // Where the next S stands: tile j of its unit (mine of its n tiles are the group's), tile number `tile` of the CTA's
    Unit w;
    int taken = 0, q = -1, j = 0, mine = 0, n = 0, tile = 0;
    // To the group's next tile, past those that only the other group has: their stages (and a unit's Q where the group
    // has none of it) are let go all the same, each after it has landed, so that no barrier is a phase ahead.
    // While a product is still owed (the softmax warps then wait for this warp) nothing may be waited for that comes only
    // after it: tiles kStages further on, or a unit after the next.
    enum { kTileThere, kOwedFirst, kEnd, kGaveUp };
    auto reach = [&](bool owed) {
        for (bool crossed = false;; crossed = true) {
            if (j < mine) return kTileThere;
            if (owed && (crossed || n - j > kStages / 2)) return kOwedFirst;
            for (; j < n; ++j, ++tile) {
                if (!warp_wait(&sm.full[tile % kStages], (tile / kStages) & 1, limit, abort_flag, p.status)) return kGaveUp;
                if (mine == 0 && j == 0 && !warp_wait(&sm.q_full[q & 1], (q >> 1) & 1, limit, abort_flag, p.status)) return kGaveUp;
                if (elect_one()) {
                    mbar_arrive(&sm.free[tile % kStages]);
                    if (mine == 0 && j == 0) mbar_arrive(&sm.q_free[q & 1]);
                }
                __syncwarp();
            }
            if (!next_unit<true>(p, sm, taken, w)) return kGaveUp;
            if (w.h < 0) return kEnd;
            j = 0;
            mine = g ? w.tiles[1] : w.tiles[0];
            n = max(w.tiles[0], w.tiles[1]);
            q += n > 0;
        }
    };
    // S of the group's tile number J
    auto scores = [&](int J) {
        const int s = tile % kStages;
        if (j == 0 && !warp_wait(&sm.q_full[q & 1], (q >> 1) & 1, limit, abort_flag, p.status)) return false;
        if (!warp_wait(&sm.full[s], (tile / kStages) & 1, limit, abort_flag, p.status)) return false;
        tc_fence_after();
        if (elect_one()) {
            const uint64_t at_q = dq + (q & 1) * next_q;
            const uint32_t to = cols + kColS + 64 * (J & 1);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) mma_ss(to, at_q + 2 * kk, dk + s * stage + 2 * kk, idesc_s, kk > 0);
            mma_commit(&sm.s_full[g][J & 1]);
            if (j == mine - 1) mma_commit(&sm.q_free[q & 1]);
        }
        __syncwarp();
        return true;
    };
    // Up to two scores ahead of the product of P that comes next: that one's stage and whether it opens a unit, and the
    // other's.
    int stage0 = 0, stage1 = 0, made = 0;
    bool opens0 = false, opens1 = false, live = true, ok = true;
    for (int J = 0; ok; ++J) {
        while (ok && live && made - J < 2) {
            const int at = reach(made > J);
            if (at == kOwedFirst) break;
            live = at == kTileThere;
            ok = at != kGaveUp;
            if (!live) break;
            if (made == J) stage0 = tile % kStages, opens0 = j == 0;
            else stage1 = tile % kStages, opens1 = j == 0;
            if (!(ok = scores(made))) break;
            ++made, ++j, ++tile;
        }
        if (!ok || made == J) break;
        if (!(ok = warp_wait(&sm.p_ready[g][J & 1], (J >> 1) & 1, limit, abort_flag, p.status))) break;
        tc_fence_after();
        if (elect_one()) {
            const uint64_t v = dv + stage0 * stage;
            const uint32_t from = cols + kColP + 32 * (J & 1);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)                 // 16 keys: 8 columns of P, 2048 bytes of V
                mma_ts(cols + kColO, from + 8 * kk, v + 128 * kk, idesc_pv, !opens0 || kk > 0);
            mma_commit(&sm.o_done[g][J & 1]);
            mma_commit(&sm.free[stage0]);
        }
        __syncwarp();
        stage0 = stage1, opens0 = opens1;
    }
    // no product may still run when the CTA's memory goes
    if (elect_one()) {
        mma_commit(&sm.drain[g]);
        for (unsigned it = 0; it < kDrainLimit; ++it)
            if (mbar_try_wait(&sm.drain[g], 0)) break;
    }
    __syncwarp();
}

// P = 2^(S scale2 + base) of 64 scores into TMEM, their sum added to l; returns the largest score.
__device__ __forceinline__ float exponentials(const uint32_t (&sv)[2][32], float scale2, float base, uint32_t at_p, float (&l)[4])
{
    float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        uint32_t pk[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float s0 = __uint_as_float(sv[c][2 * e]), s1 = __uint_as_float(sv[c][2 * e + 1]);
            float x0, x1;
            tops[e & 3] = max3(tops[e & 3], s0, s1);
            fma2s(s0, s1, scale2, base, x0, x1);
            x0 = ex2_approx(x0);
            x1 = ex2_approx(x1);
            add2(l[(e & 1) * 2], l[(e & 1) * 2 + 1], x0, x1);
            pk[e] = pack_bf16(x0, x1);
        }
        tmem_st16(at_p + 16 * c, pk);
    }
    return fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
}

__device__ __forceinline__ void softmax_rows(const Params& p, Smem& sm, int g, int quad, int lane, uint32_t tmem)
{
    volatile int* abort_flag = &sm.abort_flag;
    const unsigned limit = p.wait_limit;
    const int row = quad * 32 + lane;
    const uint32_t cols = tmem + ((uint32_t)(quad * 32) << 16) + g * kGroupCols, at_o = cols + kColO;
    bool ok = true;
    int J = 0, tile = 0, taken = 0;                        // the group's tiles so far, and the CTA's
    Unit w;
    while (ok && next_unit<true>(p, sm, taken, w) && w.h >= 0) {
        const int n = g ? w.tiles[1] : w.tiles[0], q0 = w.first + g * kRows, t = q0 + row;     // the thread's query
        float m = -INFINITY, l[4] = {0.0f, 0.0f, 0.0f, 0.0f};          // (four sums: no long chain of additions)
        for (int j = 0; j < n; ++j, ++J) {
            const uint32_t at_s = cols + kColS + 64 * (J & 1), at_p = cols + kColP + 32 * (J & 1);
            const int ahead = q0 + quad * 32 - j * kCols;  // of the warp's first row over the tile's first key
            if (!(ok = warp_wait(&sm.s_full[g][J & 1], (J >> 1) & 1, limit, abort_flag, p.status))) break;
            tc_fence_after();
            if (ahead <= -32) {
                // no row of the warp sees any of them
                uint32_t none[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) none[e] = 0u;
                tmem_st16(at_p, none);
                tmem_st16(at_p + 16, none);
            } else {
                uint32_t sv[2][32];
                tmem_ld32(at_s, sv[0]);
                tmem_ld32(at_s + 32, sv[1]);
                tmem_wait_ld();
                if (ahead < kCols - 1) {                   // the diagonal: a row sees ahead + lane + 1 keys
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const uint32_t bits = bit_range(0, ahead + lane - 32 * c);
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (!((bits >> e) & 1u)) sv[c][e] = 0xff800000u;     // -infinity
                    }
                }
                float now = m, keep[4] = {l[0], l[1], l[2], l[3]}, top = -INFINITY;
                // A row's first m is its first tile's maximum.  (Rows behind the sequence's end hold what another one has, and must
                // not decide when these move: nothing grows over theirs.)
                if (j == 0) {
                    float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int e = 0; e < 32; e += 2)
                            tops[(e >> 1) & 3] = max3(tops[(e >> 1) & 3], __uint_as_float(sv[c][e]), __uint_as_float(sv[c][e + 1]));
                    m = now = t < w.len ? fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * p.scale2 : INFINITY;
                }
                top = exponentials(sv, p.scale2, m == -INFINITY ? 0.0f : -m, at_p, l) * p.scale2;
                if (__any_sync(0xffffffffu, top > m + 8.0f || (m == -INFINITY && top > m))) {
                    // (P is written again below, to the same columns: stores are in no order until they are waited for)
                    tmem_wait_st();
                    // (every row of the warp moves to its maximum now, or its turn would come one by one)
                    now = fmaxf(m, top);
                    const float f = now == m ? 1.0f : ex2_approx(m - now);
                    m = now;
#pragma unroll
                    for (int e = 0; e < 4; ++e) l[e] = keep[e] * f;
                    // O is complete up to the tile before
                    if (!(ok = warp_wait(&sm.o_done[g][(J - 1) & 1], ((J - 1) >> 1) & 1, limit, abort_flag, p.status))) break;
                    tc_fence_after();
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t o[16];
                        tmem_ld16(at_o + 16 * c, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                        tmem_st16(at_o + 16 * c, o);
                    }
                    // (a row of the warp may still have seen nothing but -infinity: no -infinity + infinity.  One minimum here
                    // instead of a comparison and a selection: 421 instead of 424 us on the long case above.)
                    exponentials(sv, p.scale2, fminf(-m, FLT_MAX), at_p, l);
                }
            }
            // values past the sequence's end do not count, whatever they are
            if ((j + 1) * kCols > w.len) {
                if (row < kCols && j * kCols + row >= w.len) zero_row(sm.v[(tile + j) % kStages] + row * 128);
                fence_proxy_async();
            }
            tmem_wait_st();
            tc_fence_before();
            // (one arrival for the warp: 32 of them are made one after another)
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.p_ready[g][J & 1]);
        }
        if (!ok) break;
        tile += max(w.tiles[0], w.tiles[1]);
        const float sum = (l[0] + l[1]) + (l[2] + l[3]);
        if (n > 0 && !(ok = warp_wait(&sm.o_done[g][(J - 1) & 1], ((J - 1) >> 1) & 1, limit, abort_flag, p.status))) break;
        tc_fence_after();
        const bool none = n == 0 || sum == 0.0f, live = t < w.len;
        const float inv = none ? 0.0f : 1.0f / sum;
        if (p.lse && live) p.lse[(long long)w.h * p.N + w.start + t] = none ? -INFINITY : m * kLn2 + logf(sum);
        __nv_bfloat16* out = p.o + (long long)(w.start + t) * p.os[0] + w.h * p.os[1];
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
            mbar_init(&sm.u_full[s], 1);
            mbar_init(&sm.u_free[s], kReaders);
            mbar_init(&sm.q_full[s], 1);
            mbar_init(&sm.q_free[s], kGroups);
        }
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm.full[s], 1);
            mbar_init(&sm.free[s], kGroups);
        }
        for (int g = 0; g < kGroups; ++g) {
            for (int s = 0; s < 2; ++s) {
                mbar_init(&sm.s_full[g][s], 1);
                mbar_init(&sm.p_ready[g][s], 4);
                mbar_init(&sm.o_done[g][s], 1);
            }
            mbar_init(&sm.drain[g], 1);
        }
        mbar_init(&sm.answered, 1);
        sm.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // (TMEM only after the kernel before has ended: see the window's forward.  The next kernel is not let in early: its CTAs
    // would take the places of this one's that have not begun.)
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
    const uint32_t tmem = (uint32_t)uniform((int)sm.tmem_base);

    if (warp >= kSoftmaxWarps) {
        regs_down<kOtherRegs>();
        if (warp == kSoftmaxWarps) {
            if (elect_one()) load_tiles(p, sm, &tm_q, &tm_k, &tm_v);
            __syncwarp();
        } else if (warp == kSoftmaxWarps + 1) {
            if (elect_one()) find_units(p, sm);
            __syncwarp();
        } else {
            issue_products(p, sm, warp - kSoftmaxWarps - 2, tmem);
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

}  // namespace

cudaError_t launch_packed_forward_tc(const PackedArgs& a, cudaStream_t st)
{
    CUtensorMap mq, mk, mv;
    if (!encode_packed_map(&mq, a.q, a.d, a.N, a.Hq, a.qs, kRows) || !encode_packed_map(&mk, a.k, a.d, a.N, a.Hk, a.ks, kCols) ||
        !encode_packed_map(&mv, a.v, a.d, a.N, a.Hk, a.vs, kCols))
        return cudaErrorInvalidValue;
    static bool done[64];
    const size_t smem = sizeof(Smem) + 1024;
    const cudaError_t e = allow_dynamic_smem(packed_forward_tc_kernel, smem, done);
    if (e != cudaSuccess) return e;
    Params p{a.N, a.S, a.Hq, a.Hq / a.Hk, fmaxf(fabsf(a.scale) * kLog2e, 1e-37f),
             a.scale < 0.0f, a.offsets, static_cast<__nv_bfloat16*>(a.o), {a.os[0], a.os[1]}, a.d, a.lse, a.status, a.wait_limit};
    return launch_dependent(packed_forward_tc_kernel, dim3((unsigned)region_tiles(a.N, a.S, kUnit) * a.Hq), dim3(kThreads), smem, st, mq, mk, mv, p);
}

}  // namespace lasad
