// Attention over a sliding window with visible first tokens, on CUDA cores in fp32:
//
//     o_t = sum_{s in V(t)} p_ts v_s ,  p_ts = e^(scale q_t.k_s - lse_t) ,  V(t) = { s <= t : t - s < W or s < S } ,
//
// and its gradient, with Delta_t = do_t.o_t,
//
//     dv_s = sum_t p_ts do_t ,  ds_ts = scale p_ts (do_t.v_s - Delta_t) ,  dq_t = sum_s ds_ts k_s ,  dk_s = sum_t ds_ts q_t .
//
// This is the path of fp32 tensors (their products have no place on tensor cores that round their
// operands) and, by option, of bf16 ones.  Tiles of 64 queries by 64 keys stand in shared memory
// as fp32; a thread has a 4 x 4 piece of the scores, so 64 multiply-adds feed on eight 16-byte
// reads.  The forward is one pass over the visible tiles with the running maximum and sum of each
// row; no tile outside the window is touched.  The gradient runs over key tiles (dk, dv: each key
// head's CTA goes over all of its query heads) and over query tiles (dq) in two launches: nothing
// is accumulated by atomics, so results repeat bit for bit.
#include "lasad_simt_tile.cuh"

namespace lasad {
namespace {

using namespace simt;

// The visible key tiles of queries q0..q0+63: those of the sinks, then those of the windows.
struct KeyTiles {
    int sink_end, lo, hi;
    __device__ __forceinline__ KeyTiles(const WindowArgs& a, int q0, int len)
    {
        const int last = min(q0 + kTile, len) - 1;                 // the last query with keys (maybe < q0)
        hi = last < q0 ? 0 : last / kTile + 1;
        lo = q0 >= a.window ? (q0 - a.window + 1) / kTile : 0;
        sink_end = min(hi, (a.sinks + kTile - 1) / kTile);
    }
    __device__ __forceinline__ int first() const { return hi == 0 ? 0 : sink_end > 0 ? 0 : lo; }
    __device__ __forceinline__ int after(int j) const { return j + 1 < sink_end ? j + 1 : max(j + 1, lo); }
};

template <int D> struct SmemFwd { Tile<D> q, k, v; Scores p; };

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) window_forward_simt_kernel(const WindowArgs a)
{
    extern __shared__ __align__(16) unsigned char raw[];
    SmemFwd<D>& sm = *reinterpret_cast<SmemFwd<D>*>(raw);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int tiles = (a.T + kTile - 1) / kTile, bh = blockIdx.x / tiles, b = bh / a.Hq, h = bh - b * a.Hq;
    const int q0 = (tiles - 1 - (int)(blockIdx.x - (unsigned)bh * tiles)) * kTile, hk = h / (a.Hq / a.Hk);
    pdl_wait();
    const int len = a.lengths ? min(a.lengths[b], a.T) : a.T;
    load_tile<T, D>(sm.q, static_cast<const T*>(a.q) + b * a.qs[0] + h * a.qs[2], a.qs[1], q0, len);
    float m[4], l[4], o[4][D / 16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = -INFINITY, l[i] = 0.0f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) o[i][c] = 0.0f;
    }
    const float scale2 = a.scale * kLog2e;
    const KeyTiles kt(a, q0, len);
    for (int j = kt.first(); j < kt.hi; j = kt.after(j)) {
        __syncthreads();
        load_tile<T, D>(sm.k, static_cast<const T*>(a.k) + b * a.ks[0] + hk * a.ks[2], a.ks[1], j * kTile, len);
        load_tile<T, D>(sm.v, static_cast<const T*>(a.v) + b * a.vs[0] + hk * a.vs[2], a.vs[1], j * kTile, len);
        __syncthreads();
        float s[4][4];
        dot_tile<D>(sm.q, sm.k, ty, tx, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = q0 + ty * 4 + i;
            float top = -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                s[i][c] = window_sees(t, j * kTile + tx + 16 * c, a.window, a.sinks, len) ? s[i][c] * scale2 : -INFINITY;
                top = fmaxf(top, s[i][c]);
            }
#pragma unroll
            for (int k = 8; k >= 1; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
            const float now = fmaxf(m[i], top), base = now == -INFINITY ? 0.0f : now;   // nothing visible yet
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
        if (t >= a.T) continue;
        const float inv = l[i] > 0.0f || l[i] != l[i] ? 1.0f / l[i] : 0.0f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) o[i][c] *= inv;
        store_cols<T, D>(static_cast<T*>(a.o) + b * a.os[0] + t * a.os[1] + h * a.os[2], tx, o[i]);
        if (tx == 0 && a.lse)
            a.lse[((long long)b * a.Hq + h) * a.T + t] = m[i] == -INFINITY && l[i] == 0.0f ? -INFINITY : m[i] * (1.0f / kLog2e) + logf(l[i]);
    }
}

template <int D> struct SmemBwd { Tile<D> q, g, k, v; Scores p, s; float lse[kTile], delta[kTile]; };

// p and ds of one tile of 64 queries and 64 keys, into shared memory; only pairs of the window, or
// (all = true) of the sinks too
template <int D>
__device__ __forceinline__ void gradient_scores(SmemBwd<D>& sm, const WindowArgs& a, int q0, int k0, int len, bool all,
                                                int ty, int tx)
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
            const bool sees = window_sees(t, k0 + col, a.window, all ? a.sinks : 0, len);
            const float p = sees ? exp2f((s[i][c] * a.scale - sm.lse[ty * 4 + i]) * kLog2e) : 0.0f;
            sm.p.x[ty * 4 + i][col] = p;
            sm.s.x[ty * 4 + i][col] = sees ? p * (d[i][c] + sm.delta[ty * 4 + i]) * a.scale : 0.0f;
        }
    }
}
template <typename T, int D>
__device__ __forceinline__ void load_queries(SmemBwd<D>& sm, const WindowArgs& a, int b, int h, int q0, int len)
{
    load_tile<T, D>(sm.q, static_cast<const T*>(a.q) + b * a.qs[0] + h * a.qs[2], a.qs[1], q0, len);
    load_tile<T, D>(sm.g, static_cast<const T*>(a.dout) + b * a.dos[0] + h * a.dos[2], a.dos[1], q0, len);
    if (threadIdx.x < kTile) {
        const int t = q0 + threadIdx.x;
        const long long at = ((long long)b * a.Hq + h) * a.T + t;
        sm.lse[threadIdx.x] = t < len ? a.lse[at] : 0.0f;
        sm.delta[threadIdx.x] = t < len ? a.ws[window_stat_at(a.T, (long long)b * a.Hq + h, t) + kPrepRows] : 0.0f;   // -Delta
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) window_dkdv_simt_kernel(const WindowArgs a)
{
    extern __shared__ __align__(16) unsigned char raw[];
    SmemBwd<D>& sm = *reinterpret_cast<SmemBwd<D>*>(raw);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int tiles = (a.T + kTile - 1) / kTile, bh = blockIdx.x / tiles, b = bh / a.Hk, hk = bh - b * a.Hk;
    const int k0 = (int)(blockIdx.x - (unsigned)bh * tiles) * kTile, G = a.Hq / a.Hk;
    pdl_wait();
    const int len = a.lengths ? min(a.lengths[b], a.T) : a.T;
    float dk[4][D / 16], dv[4][D / 16];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < D / 16; ++c) dk[i][c] = dv[i][c] = 0.0f;
    // queries k0 .. k0 + 63 + W - 1
    const long long last = min((long long)k0 + kTile + a.window - 1, (long long)len);
    const int qtiles = k0 >= len ? 0 : (int)((last + kTile - 1) / kTile) - k0 / kTile;
    load_tile<T, D>(sm.k, static_cast<const T*>(a.k) + b * a.ks[0] + hk * a.ks[2], a.ks[1], k0, len);
    load_tile<T, D>(sm.v, static_cast<const T*>(a.v) + b * a.vs[0] + hk * a.vs[2], a.vs[1], k0, len);
    for (int n = 0; n < qtiles * G; ++n) {
        const int h = hk * G + n / qtiles, q0 = k0 + (n % qtiles) * kTile;
        __syncthreads();
        load_queries<T, D>(sm, a, b, h, q0, len);
        __syncthreads();
        gradient_scores<D>(sm, a, q0, k0, len, false, ty, tx);
        __syncthreads();
        add_cols<D>(sm.p, sm.g, ty, tx, dv);
        add_cols<D>(sm.s, sm.q, ty, tx, dk);
    }
    const int sinks = min(a.sinks, a.T), chunks = (a.T + kPrepRows - 1) / kPrepRows;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int s = k0 + ty * 4 + i;
        if (s >= a.T) continue;
        if (s < sinks && a.window < len) {      // the sums of launch_window_prep: chunks with a row past the window, before the end
            const float* sums = a.ws + window_stat_floats(a) + ((long long)bh * chunks * sinks + s) * 2 * D;
            for (int c = a.window / kPrepRows; c < (len + kPrepRows - 1) / kPrepRows; ++c) {
                const float* w = sums + (long long)c * sinks * 2 * D;
#pragma unroll
                for (int e = 0; e < D / 16; ++e) {
                    dk[i][e] += w[tx * (D / 16) + e];
                    dv[i][e] += w[D + tx * (D / 16) + e];
                }
            }
        }
        store_cols<T, D>(static_cast<T*>(a.dk) + b * a.dks[0] + s * a.dks[1] + hk * a.dks[2], tx, dk[i]);
        store_cols<T, D>(static_cast<T*>(a.dv) + b * a.dvs[0] + s * a.dvs[1] + hk * a.dvs[2], tx, dv[i]);
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) window_dq_simt_kernel(const WindowArgs a)
{
    extern __shared__ __align__(16) unsigned char raw[];
    SmemBwd<D>& sm = *reinterpret_cast<SmemBwd<D>*>(raw);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int tiles = (a.T + kTile - 1) / kTile, bh = blockIdx.x / tiles, b = bh / a.Hq, h = bh - b * a.Hq;
    const int q0 = (tiles - 1 - (int)(blockIdx.x - (unsigned)bh * tiles)) * kTile, hk = h / (a.Hq / a.Hk);
    pdl_wait();
    const int len = a.lengths ? min(a.lengths[b], a.T) : a.T;
    load_queries<T, D>(sm, a, b, h, q0, len);
    float dq[4][D / 16];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < D / 16; ++c) dq[i][c] = 0.0f;
    const KeyTiles kt(a, q0, len);
    for (int j = kt.first(); j < kt.hi; j = kt.after(j)) {
        __syncthreads();
        load_tile<T, D>(sm.k, static_cast<const T*>(a.k) + b * a.ks[0] + hk * a.ks[2], a.ks[1], j * kTile, len);
        load_tile<T, D>(sm.v, static_cast<const T*>(a.v) + b * a.vs[0] + hk * a.vs[2], a.vs[1], j * kTile, len);
        __syncthreads();
        gradient_scores<D>(sm, a, q0, j * kTile, len, true, ty, tx);
        __syncwarp();
        add_rows<D>(sm.s, sm.k, ty, tx, dq);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = q0 + ty * 4 + i;
        if (t < a.T) store_cols<T, D>(static_cast<T*>(a.dq) + b * a.dqs[0] + t * a.dqs[1] + h * a.dqs[2], tx, dq[i]);
    }
}

template <typename T, int D>
cudaError_t forward_t(const WindowArgs& a, cudaStream_t st)
{
    static bool done[64];
    cudaError_t e = tcx::allow_dynamic_smem(window_forward_simt_kernel<T, D>, sizeof(SmemFwd<D>), done);
    if (e != cudaSuccess) return e;
    const unsigned tiles = (a.T + kTile - 1) / kTile;
    return launch_dependent(window_forward_simt_kernel<T, D>, dim3(tiles * a.B * a.Hq), dim3(kThreads), sizeof(SmemFwd<D>), st, a);
}
template <typename T, int D>
cudaError_t backward_t(const WindowArgs& a, cudaStream_t st)
{
    static bool done1[64], done2[64];
    cudaError_t e = tcx::allow_dynamic_smem(window_dkdv_simt_kernel<T, D>, sizeof(SmemBwd<D>), done1);
    if (e == cudaSuccess) e = tcx::allow_dynamic_smem(window_dq_simt_kernel<T, D>, sizeof(SmemBwd<D>), done2);
    const unsigned tiles = (a.T + kTile - 1) / kTile;
    if (e == cudaSuccess)
        e = launch_dependent(window_dkdv_simt_kernel<T, D>, dim3(tiles * a.B * a.Hk), dim3(kThreads), sizeof(SmemBwd<D>), st, a);
    if (e == cudaSuccess)
        e = launch_dependent(window_dq_simt_kernel<T, D>, dim3(tiles * a.B * a.Hq), dim3(kThreads), sizeof(SmemBwd<D>), st, a);
    return e;
}

}  // namespace

cudaError_t launch_window_forward_simt(const WindowArgs& a, cudaStream_t st)
{
    if (a.bf16) return a.d == 64 ? forward_t<__nv_bfloat16, 64>(a, st) : forward_t<__nv_bfloat16, 32>(a, st);
    return a.d == 64 ? forward_t<float, 64>(a, st) : forward_t<float, 32>(a, st);
}
cudaError_t launch_window_backward_simt(const WindowArgs& a, cudaStream_t st)
{
    const cudaError_t e = launch_window_prep(a, true, st);
    if (e != cudaSuccess) return e;
    if (a.bf16) return a.d == 64 ? backward_t<__nv_bfloat16, 64>(a, st) : backward_t<__nv_bfloat16, 32>(a, st);
    return a.d == 64 ? backward_t<float, 64>(a, st) : backward_t<float, 32>(a, st);
}

}  // namespace lasad
