// What the gradient of the window attention needs beside its products:
//
//     Delta_t = sum_c do_tc o_tc        (per query head; the tensor-core kernels form it themselves),
//
// and, for the sinks (tokens s < S, visible to every later query), the gradients from the queries
// that see s only because it is a sink, t >= s + W:
//
//     dv_s += sum_t p_ts do_t ,  dk_s += sum_t ds_ts q_t ,  p = e^(scale q.k - lse),  ds = scale p (do.v - Delta) .
//
// Those queries are up to the whole sequence for a few keys: a key tile's own loop would be T / W
// times as long for the sinks' tile as for any other.  Here the rows are read once anyway, so each
// CTA (kPrepRows tokens of the query heads of one key head) leaves one sum per sink, and the
// key tile's epilogue adds the sums of the CTAs in order.  Bound by device memory: o and do, and q
// where there are sinks.
#include "lasad_mixers.cuh"
#include "lasad_tc_ptx.cuh"

namespace lasad {
namespace {

template <typename T, int N>
__device__ __forceinline__ void load_piece(const T* p, float (&v)[N])
{
    if constexpr (sizeof(T) == 2) {
        static_assert(N == 8, "");
        const uint4 r = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = tcx::bf16_lo(w[i]), v[2 * i + 1] = tcx::bf16_hi(w[i]);
    } else {
        static_assert(N == 4, "");
        const float4 r = *reinterpret_cast<const float4*>(p);
        v[0] = r.x, v[1] = r.y, v[2] = r.z, v[3] = r.w;
    }
}

constexpr int kWarps = 8, kAhead = 3;

template <typename T, int D, bool DELTA>
__global__ void __launch_bounds__(32 * kWarps) window_prep_kernel(const WindowArgs a)
{
    constexpr int N = sizeof(T) == 2 ? 8 : 4, LANES = D / N, ROWS = 32 / LANES;
    __shared__ float part[kWarps][2][D];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % LANES, mine = lane / LANES;
    const int chunks = (a.T + kPrepRows - 1) / kPrepRows;
    const int chunk = blockIdx.x % chunks, bh = blockIdx.x / chunks, b = bh / a.Hk, hk = bh - b * a.Hk;
    const int G = a.Hq / a.Hk, t0 = chunk * kPrepRows, rows = min(kPrepRows, a.T - t0);
    pdl_wait();
    const int len = a.lengths ? a.lengths[b] : a.T;
    const T* o = static_cast<const T*>(a.o) + b * a.os[0] + sub * N;
    const T* g = static_cast<const T*>(a.dout) + b * a.dos[0] + sub * N;
    const T* q = static_cast<const T*>(a.q) + b * a.qs[0] + sub * N;
    // (kAhead rows of each lane group at a time: their loads are in flight together)
    for (int r0 = 0; DELTA && r0 < rows * G; r0 += kWarps * ROWS * kAhead) {
        float ov[kAhead][N], gv[kAhead][N];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int r = min(r0 + (i * kWarps + warp) * ROWS + mine, rows * G - 1), t = t0 + r / G, h = hk * G + r % G;
            load_piece<T, N>(o + t * a.os[1] + h * a.os[2], ov[i]);
            load_piece<T, N>(g + t * a.dos[1] + h * a.dos[2], gv[i]);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int r = r0 + (i * kWarps + warp) * ROWS + mine, t = t0 + r / G, h = hk * G + r % G;
            float d = 0.0f;
#pragma unroll
            for (int e = 0; e < N; ++e) d = fmaf(ov[i][e], gv[i][e], d);
#pragma unroll
            for (int k = LANES / 2; k >= 1; k >>= 1) d += __shfl_xor_sync(0xffffffffu, d, k);
            // (a row past its sequence's end counts for nothing, whatever stands in o and do)
            if (r < rows * G && sub == 0)
                a.ws[window_stat_at(a.T, (long long)b * a.Hq + h, t) + kPrepRows] = t < len ? -d : 0.0f;
        }
    }
    const int sinks = min(a.sinks, a.T);
    if (sinks == 0 || t0 + rows <= a.window || t0 >= len) return;   // (uniform over the CTA)
    if (DELTA) __syncthreads();                                     // what the CTA's rows have left
    float* sums = a.ws + window_stat_floats(a) + ((long long)bh * chunks + chunk) * sinks * 2 * D;
    constexpr float kLog2e = 1.4426950408889634f;
    for (int s = blockIdx.y; s < sinks; s += gridDim.y) {
        float kv[N], vv[N], dk[N], dv[N];
        load_piece<T, N>(static_cast<const T*>(a.k) + b * a.ks[0] + s * a.ks[1] + hk * a.ks[2] + sub * N, kv);
        load_piece<T, N>(static_cast<const T*>(a.v) + b * a.vs[0] + s * a.vs[1] + hk * a.vs[2] + sub * N, vv);
#pragma unroll
        for (int e = 0; e < N; ++e) dk[e] = dv[e] = 0.0f;
        const int lo = max(0, s + a.window - t0), hi = min(rows, len - t0);   // rows lo..hi-1 see s as a sink only
        const int n = max(0, hi - lo) * G;
        for (int r0 = 0; r0 < n; r0 += kWarps * ROWS * kAhead) {
            float qv[kAhead][N], gv[kAhead][N], ls[kAhead], de[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int r = min(r0 + (i * kWarps + warp) * ROWS + mine, n - 1), t = t0 + lo + r / G, h = hk * G + r % G;
                load_piece<T, N>(q + t * a.qs[1] + h * a.qs[2], qv[i]);
                load_piece<T, N>(g + t * a.dos[1] + h * a.dos[2], gv[i]);
                const long long bhq = (long long)b * a.Hq + h;
                ls[i] = a.lse[bhq * a.T + t];
                de[i] = a.ws[window_stat_at(a.T, bhq, t) + kPrepRows];      // -Delta
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                float x = 0.0f, y = 0.0f;
#pragma unroll
                for (int e = 0; e < N; ++e) x = fmaf(qv[i][e], kv[e], x), y = fmaf(gv[i][e], vv[e], y);
#pragma unroll
                for (int k = LANES / 2; k >= 1; k >>= 1) {
                    x += __shfl_xor_sync(0xffffffffu, x, k);
                    y += __shfl_xor_sync(0xffffffffu, y, k);
                }
                if (r0 + (i * kWarps + warp) * ROWS + mine < n) {
                    const float p = exp2f((x * a.scale - ls[i]) * kLog2e), ds = p * (y + de[i]) * a.scale;
#pragma unroll
                    for (int e = 0; e < N; ++e) dk[e] = fmaf(ds, qv[i][e], dk[e]), dv[e] = fmaf(p, gv[i][e], dv[e]);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
#pragma unroll
            for (int k = 16; k >= LANES; k >>= 1) {
                dk[e] += __shfl_xor_sync(0xffffffffu, dk[e], k);
                dv[e] += __shfl_xor_sync(0xffffffffu, dv[e], k);
            }
            if (mine == 0) part[warp][0][sub * N + e] = dk[e], part[warp][1][sub * N + e] = dv[e];
        }
        __syncthreads();
        if (threadIdx.x < 2 * D) {
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) v += part[w][threadIdx.x / D][threadIdx.x % D];
            sums[s * 2 * D + threadIdx.x] = v;
        }
        __syncthreads();
    }
}

template <bool DELTA> cudaError_t launch_prep(const WindowArgs& a, cudaStream_t st)
{
    const unsigned n = (unsigned)((a.T + kPrepRows - 1) / kPrepRows) * a.B * a.Hk;
    auto kernel = a.bf16 ? (a.d == 64 ? window_prep_kernel<__nv_bfloat16, 64, DELTA> : window_prep_kernel<__nv_bfloat16, 32, DELTA>)
                         : (a.d == 64 ? window_prep_kernel<float, 64, DELTA> : window_prep_kernel<float, 32, DELTA>);
    // (the sums alone: a CTA per sink as well; with Delta the CTA that has formed it goes over all sinks)
    return launch_dependent(kernel, dim3(n, DELTA ? 1 : (unsigned)(a.sinks < a.T ? a.sinks : a.T)), dim3(32 * kWarps), 0, st, a);
}

}  // namespace

size_t window_workspace_bytes(const WindowArgs& a)
{
    const size_t chunks = (a.T + kPrepRows - 1) / kPrepRows, sinks = a.sinks < a.T ? a.sinks : a.T;
    return (window_stat_floats(a) + (size_t)a.B * a.Hk * chunks * sinks * 2 * a.d) * sizeof(float);
}

cudaError_t launch_window_prep(const WindowArgs& a, bool delta, cudaStream_t st)
{
    return delta ? launch_prep<true>(a, st) : launch_prep<false>(a, st);
}

}  // namespace lasad
