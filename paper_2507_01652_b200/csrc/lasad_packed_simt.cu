// Causal attention over packed sequences on CUDA cores in fp32:
//
//     o_t = sum_{s <= t} p_ts v_s ,   p_ts = e^(scale q_t.k_s - lse_t)   over the tokens s of t's own sequence,
//
// and its gradient, with Delta_t = do_t.o_t,
//
//     dv_s = sum_{t >= s} p_ts do_t ,  ds_ts = scale p_ts (do_t.v_s - Delta_t) ,  dq_t = sum_s ds_ts k_s ,  dk_s = sum_t ds_ts q_t .
//
// This is the path of fp32 tensors (their products have no place on tensor cores that round their operands)
// and, by option, of bf16 ones.  Tiles of 64 queries by 64 keys of one sequence stand in shared memory;
// the forward keeps the running maximum and sum of each row.  The gradient goes over query tiles (dq, and
// Delta for the other) and over key tiles (dk, dv, each key head's CTA over all of its query heads):
// no atomics, so results repeat bit for bit.  The longest tiles of a sequence come first.
//
// No unit is near its limit: two CTAs an SM wait for shared memory and for a tile's rows (1 x 2049 tokens, 24 query and 8 key
// heads, d = 64: issue slots 60 to 65 %, multiply-adds 49 to 53 %, shared memory 45 to 66 % in the three kernels).  1 x 9217:
// 7.99 ms, 33 TFLOP/s of the pairs that count, and 26.9 ms for the gradient, 24 (34 with what it makes twice: two products
// forward, seven in the two passes of the gradient).  A CTA that has an SM to itself takes 3.8 us for a tile forward at d = 32 and 6.2 at d = 64 (12 and 20 in
// the gradient's two kernels together), so 3 sequences of up to 256 tokens, four tiles in turn, take 18 and 55 us.
#include "lasad_full.cuh"
#include "lasad_simt_tile.cuh"

namespace lasad {
namespace {

using namespace simt;

template <typename T> __device__ __forceinline__ const T* rows_of(const void* p, const long long (&s)[2], int start, int h)
{
    return static_cast<const T*>(p) + start * s[0] + h * s[1];
}
template <typename T> __device__ __forceinline__ T* rows_of(void* p, const long long (&s)[2], int start, int h)
{
    return static_cast<T*>(p) + start * s[0] + h * s[1];
}

template <int D> struct SmemFwd { Tile<D> q, k, v; Scores p; };

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) packed_forward_simt_kernel(const PackedArgs a)
{
    extern __shared__ __align__(16) unsigned char raw[];
    SmemFwd<D>& sm = *reinterpret_cast<SmemFwd<D>*>(raw);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int at = blockIdx.x / (unsigned)a.Hq, h = blockIdx.x - (unsigned)at * a.Hq, hk = h / (a.Hq / a.Hk);
    pdl_wait();
    const Region r = region_of<kTile>(a.offsets, a.S, a.N, (int)region_tiles(a.N, a.S, kTile) - 1 - at);
    const int q0 = r.first, len = r.len;
    if (q0 >= len) return;
    const int seen = r.owned ? min(q0 + kTile, len) : 0;           // keys that any of the rows sees
    load_tile<T, D>(sm.q, rows_of<T>(a.q, a.qs, r.start, h), a.qs[0], q0, r.owned ? len : 0);
    float m[4], l[4], o[4][D / 16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = -INFINITY, l[i] = 0.0f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) o[i][c] = 0.0f;
    }
    const float scale2 = a.scale * kLog2e;
    for (int k0 = 0; k0 < seen; k0 += kTile) {
        __syncthreads();
        load_tile<T, D>(sm.k, rows_of<T>(a.k, a.ks, r.start, hk), a.ks[0], k0, len);
        load_tile<T, D>(sm.v, rows_of<T>(a.v, a.vs, r.start, hk), a.vs[0], k0, len);
        __syncthreads();
        float s[4][4];
        dot_tile<D>(sm.q, sm.k, ty, tx, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = q0 + ty * 4 + i;
            float top = -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                s[i][c] = k0 + tx + 16 * c <= t && t < len ? s[i][c] * scale2 : -INFINITY;
                top = fmaxf(top, s[i][c]);
            }
#pragma unroll
            for (int k = 8; k >= 1; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
            const float now = fmaxf(m[i], top), base = now == -INFINITY ? 0.0f : now;   // nothing but infinities yet
            const float keep = exp2f(m[i] - base);
            float sum = 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float p = exp2f(s[i][c] - base);
                sm.p.x[ty * 4 + i][tx + 16 * c] = p;
                sum += p;
            }
#pragma unroll
            for (int k = 8; k >= 1; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
            l[i] = fmaf(l[i], keep, sum);
            m[i] = now;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) o[i][c] *= keep;
        }
        __syncwarp();                    // a row of p is written and read by the same half warp
        add_rows<D>(sm.p, sm.v, ty, tx, o);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = q0 + ty * 4 + i;
        if (t >= len) continue;
        const float inv = l[i] > 0.0f || l[i] != l[i] ? 1.0f / l[i] : 0.0f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) o[i][c] *= inv;
        store_cols<T, D>(rows_of<T>(a.o, a.os, r.start + t, h), tx, o[i]);
        if (tx == 0 && a.lse)
            a.lse[(long long)h * a.N + r.start + t] = m[i] == -INFINITY && l[i] == 0.0f ? -INFINITY : m[i] * (1.0f / kLog2e) + logf(l[i]);
    }
}

template <int D> struct SmemBwd { Tile<D> q, g, k, v; Scores p, s; float lse[kTile], delta[kTile]; };

// p and ds of one tile of 64 queries and 64 keys, into shared memory; a thread's part of sum_s p (dP - Delta) in rest
template <int D>
__device__ __forceinline__ void gradient_scores(SmemBwd<D>& sm, const PackedArgs& a, int q0, int k0, int len, int ty, int tx, float (&rest)[4])
{
    float s[4][4], d[4][4];
    dot_tile<D>(sm.q, sm.k, ty, tx, s);
    dot_tile<D>(sm.g, sm.v, ty, tx, d);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = q0 + ty * 4 + i;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int col = tx + 16 * c;
            const bool sees = k0 + col <= t && t < len;
            const float p = sees ? exp2f(fmaf(s[i][c] * a.scale, kLog2e, sm.lse[ty * 4 + i])) : 0.0f;
            const float ds = sees ? p * (d[i][c] + sm.delta[ty * 4 + i]) : 0.0f;
            rest[i] += ds;
            sm.p.x[ty * 4 + i][col] = p;
            sm.s.x[ty * 4 + i][col] = ds * a.scale;
        }
    }
}
template <typename T, int D>
__device__ __forceinline__ void load_queries(SmemBwd<D>& sm, const PackedArgs& a, const Region& r, int h, int q0)
{
    load_tile<T, D>(sm.q, rows_of<T>(a.q, a.qs, r.start, h), a.qs[0], q0, r.len);
    load_tile<T, D>(sm.g, rows_of<T>(a.dout, a.dos, r.start, h), a.dos[0], q0, r.len);
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) packed_dq_simt_kernel(const PackedArgs a)
{
    extern __shared__ __align__(16) unsigned char raw[];
    SmemBwd<D>& sm = *reinterpret_cast<SmemBwd<D>*>(raw);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int at = blockIdx.x / (unsigned)a.Hq, h = blockIdx.x - (unsigned)at * a.Hq, hk = h / (a.Hq / a.Hk);
    const int number = (int)region_tiles(a.N, a.S, kTile) - 1 - at;
    pdl_wait();
    const Region r = region_of<kTile>(a.offsets, a.S, a.N, number);
    const int q0 = r.first, len = r.len;
    if (q0 >= len) return;
    // The o of a bf16 caller was rounded, and where a row sees few keys dP - Delta is small against what that does to
    // Delta' = do.o: so the sum r of P (dP - Delta') over the row, which is Delta - Delta', is taken off again.
    constexpr bool ROUNDED = sizeof(T) == 2;
    float dq[4][D / 16], pk[4][D / 16], rest[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < D / 16; ++c) dq[i][c] = pk[i][c] = 0.0f;
    if (r.owned) {
        load_queries<T, D>(sm, a, r, h, q0);
        __syncthreads();
        // Delta: four threads have a row
        const int row = threadIdx.x / 4, part = threadIdx.x % 4;
        float sum = 0.0f;
        if (q0 + row < len) {
            const T* o = rows_of<const T>(const_cast<const void*>(a.o), a.os, r.start + q0 + row, h);
#pragma unroll
            for (int c = 0; c < D / 4; ++c) sum = fmaf(sm.g.x[row][part * (D / 4) + c], io<T>::load(o + part * (D / 4) + c), sum);
        }
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if (part == 0) {
            const float lse = q0 + row < len ? minus_lse(a.lse[(long long)h * a.N + r.start + q0 + row]) : 0.0f;
            sm.lse[row] = lse;
            sm.delta[row] = -sum;
            float* stat = a.ws + packed_stat_at(a, h, number);
            stat[row] = lse;
            if (!ROUNDED) stat[kStatRows + row] = -sum;
        }
        for (int k0 = 0; k0 < min(q0 + kTile, len); k0 += kTile) {
            __syncthreads();
            load_tile<T, D>(sm.k, rows_of<T>(a.k, a.ks, r.start, hk), a.ks[0], k0, len);
            load_tile<T, D>(sm.v, rows_of<T>(a.v, a.vs, r.start, hk), a.vs[0], k0, len);
            __syncthreads();
            gradient_scores<D>(sm, a, q0, k0, len, ty, tx, rest);
            __syncwarp();
            add_rows<D>(sm.s, sm.k, ty, tx, dq);
            if (ROUNDED) add_rows<D>(sm.p, sm.k, ty, tx, pk);
        }
        if (ROUNDED) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int k = 8; k >= 1; k >>= 1) rest[i] += __shfl_xor_sync(0xffffffffu, rest[i], k);
#pragma unroll
                for (int c = 0; c < D / 16; ++c) dq[i][c] = fmaf(-rest[i] * a.scale, pk[i][c], dq[i][c]);
                if (tx == 0) a.ws[packed_stat_at(a, h, number) + kStatRows + ty * 4 + i] = sm.delta[ty * 4 + i] - rest[i];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = q0 + ty * 4 + i;
        if (t < len) store_cols<T, D>(rows_of<T>(a.dq, a.dqs, r.start + t, h), tx, dq[i]);
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) packed_dkdv_simt_kernel(const PackedArgs a)
{
    extern __shared__ __align__(16) unsigned char raw[];
    SmemBwd<D>& sm = *reinterpret_cast<SmemBwd<D>*>(raw);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int at = blockIdx.x / (unsigned)a.Hk, hk = blockIdx.x - (unsigned)at * a.Hk, G = a.Hq / a.Hk;
    pdl_wait();
    const Region r = region_of<kTile>(a.offsets, a.S, a.N, at);
    const int k0 = r.first, len = r.len;
    if (k0 >= len) return;
    float dk[4][D / 16], dv[4][D / 16];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < D / 16; ++c) dk[i][c] = dv[i][c] = 0.0f;
    if (r.owned) {
        load_tile<T, D>(sm.k, rows_of<T>(a.k, a.ks, r.start, hk), a.ks[0], k0, len);
        load_tile<T, D>(sm.v, rows_of<T>(a.v, a.vs, r.start, hk), a.vs[0], k0, len);
        const int qtiles = (len - k0 + kTile - 1) / kTile;
        for (int n = 0; n < qtiles * G; ++n) {
            const int h = hk * G + n / qtiles, q0 = k0 + (n % qtiles) * kTile;
            __syncthreads();
            load_queries<T, D>(sm, a, r, h, q0);
            if (threadIdx.x < kTile) {
                const float* stat = a.ws + packed_stat_at(a, h, r.base + q0 / kTile);
                sm.lse[threadIdx.x] = stat[threadIdx.x];
                sm.delta[threadIdx.x] = stat[kStatRows + threadIdx.x];
            }
            __syncthreads();
            float unused[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            gradient_scores<D>(sm, a, q0, k0, len, ty, tx, unused);
            __syncthreads();
            add_cols<D>(sm.p, sm.g, ty, tx, dv);
            add_cols<D>(sm.s, sm.q, ty, tx, dk);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int s = k0 + ty * 4 + i;
        if (s >= len) continue;
        store_cols<T, D>(rows_of<T>(a.dk, a.dks, r.start + s, hk), tx, dk[i]);
        store_cols<T, D>(rows_of<T>(a.dv, a.dvs, r.start + s, hk), tx, dv[i]);
    }
}

static_assert(kTile == kStatRows, "the statistics' blocks are the tiles");

template <typename T, int D>
cudaError_t forward_t(const PackedArgs& a, cudaStream_t st)
{
    static bool done[64];
    const cudaError_t e = tcx::allow_dynamic_smem(packed_forward_simt_kernel<T, D>, sizeof(SmemFwd<D>), done);
    if (e != cudaSuccess) return e;
    const unsigned tiles = (unsigned)region_tiles(a.N, a.S, kTile);
    return launch_dependent(packed_forward_simt_kernel<T, D>, dim3(tiles * a.Hq), dim3(kThreads), sizeof(SmemFwd<D>), st, a);
}
template <typename T, int D>
cudaError_t backward_t(const PackedArgs& a, cudaStream_t st)
{
    static bool done1[64], done2[64];
    cudaError_t e = tcx::allow_dynamic_smem(packed_dq_simt_kernel<T, D>, sizeof(SmemBwd<D>), done1);
    if (e == cudaSuccess) e = tcx::allow_dynamic_smem(packed_dkdv_simt_kernel<T, D>, sizeof(SmemBwd<D>), done2);
    const unsigned tiles = (unsigned)region_tiles(a.N, a.S, kTile);
    if (e == cudaSuccess)
        e = launch_dependent(packed_dq_simt_kernel<T, D>, dim3(tiles * a.Hq), dim3(kThreads), sizeof(SmemBwd<D>), st, a);
    if (e == cudaSuccess)
        e = launch_dependent(packed_dkdv_simt_kernel<T, D>, dim3(tiles * a.Hk), dim3(kThreads), sizeof(SmemBwd<D>), st, a);
    return e;
}

}  // namespace

cudaError_t launch_packed_forward_simt(const PackedArgs& a, cudaStream_t st)
{
    if (a.bf16) return a.d == 64 ? forward_t<__nv_bfloat16, 64>(a, st) : forward_t<__nv_bfloat16, 32>(a, st);
    return a.d == 64 ? forward_t<float, 64>(a, st) : forward_t<float, 32>(a, st);
}
cudaError_t launch_packed_backward_simt(const PackedArgs& a, cudaStream_t st)
{
    if (a.bf16) return a.d == 64 ? backward_t<__nv_bfloat16, 64>(a, st) : backward_t<__nv_bfloat16, 32>(a, st);
    return a.d == 64 ? backward_t<float, 64>(a, st) : backward_t<float, 32>(a, st);
}

}  // namespace lasad
