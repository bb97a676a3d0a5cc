// Norm of every head's queries and keys and their rotation by position, in one pass, with the gradient:
//
//     y = R (w * x r) ,  r = 1 / sqrt(mean(x^2) + eps) ,
//
// R turns each pair of channels by (position x frequency); on a grid the first half of the pairs
// goes by the token's row and the other half by its column, and tokens before the grid are not
// turned.  With u = R^T dy, xn = x r and the means over one head's channels
//
//     dw = sum over tokens and heads of u * xn ,   dx = r (w * u - xn mean(w * u * xn)) .
//
// Bound by device memory: x in and y out (x, dy in and dx out).  A head's channels lie in the
// 16-byte pieces of d / 8 (bf16) or d / 4 (fp32) neighbouring lanes, so the sums are three or four
// shuffles, and a warp works on one token: its angles are read once and serve all of the heads.
#include "lasad_mixers.cuh"
#include "lasad_tc_ptx.cuh"

namespace lasad {
namespace {

constexpr int kRopeWarps = 8;

template <typename T> struct piece;      // the 16 bytes of one lane
template <> struct piece<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void get(const uint4& r, float (&v)[8])
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = tcx::bf16_lo(w[i]), v[2 * i + 1] = tcx::bf16_hi(w[i]);
    }
    static __device__ __forceinline__ uint4 put(const float (&v)[8])
    {
        return make_uint4(tcx::pack_bf16(v[0], v[1]), tcx::pack_bf16(v[2], v[3]), tcx::pack_bf16(v[4], v[5]),
                          tcx::pack_bf16(v[6], v[7]));
    }
};
template <> struct piece<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void get(const uint4& r, float (&v)[4])
    {
        v[0] = __uint_as_float(r.x), v[1] = __uint_as_float(r.y), v[2] = __uint_as_float(r.z), v[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ uint4 put(const float (&v)[4])
    {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};

// cos and sin of one lane's channels at one position.  Channel 2m and 2m + 1 are a pair (HALF: m
// and m + D / 2), so a lane has N / 2 (N) pairs, all of them of the row or all of the column.
template <typename T, int D, bool HALF>
struct Turn {
    static constexpr int N = piece<T>::N, LANES = D / N, PAIRS = HALF ? N : N / 2;
    float c[PAIRS], s[PAIRS];
    __device__ __forceinline__ void at(const RopeArgs& a, long long i, int sub)
    {
        int m = HALF ? (sub % (LANES / 2)) * N : sub * (N / 2);   // the lane's first pair
        long long row = i;
        int width = D / 2;
        if (a.grid_w > 0) {
            const long long j = i - a.prefix_len;
            if (j < 0) {
#pragma unroll
                for (int p = 0; p < PAIRS; ++p) c[p] = 1.0f, s[p] = 0.0f;
                return;
            }
            const long long r = j <= 0x7fffffffLL ? (long long)((unsigned)j / (unsigned)a.grid_w) : j / a.grid_w;
            width = D / 4;
            row = m < width ? r : j - r * a.grid_w;
            m = m < width ? m : m - width;
        }
        // (positions that come from device memory are not known to the host: they end at the table's edge)
        row = row < 0 ? 0 : row < a.table_rows ? row : a.table_rows - 1;
        const float* t = a.table + (row * width + m) * 2;
#pragma unroll
        for (int p = 0; p < PAIRS; p += 2) {
            const float4 f = *reinterpret_cast<const float4*>(t + 2 * p);
            c[p] = f.x, s[p] = f.y, c[p + 1] = f.z, s[p + 1] = f.w;
        }
    }
    // v <- R v (back: R^T v)
    __device__ __forceinline__ void apply(float (&v)[N], int sub, bool back) const
    {
        if (HALF) {
            const float sign = (sub < LANES / 2) != back ? -1.0f : 1.0f;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float o = __shfl_xor_sync(0xffffffffu, v[e], LANES / 2);
                v[e] = fmaf(sign * s[e % PAIRS], o, v[e] * c[e % PAIRS]);
            }
        } else {
#pragma unroll
            for (int p = 0; p < N / 2; ++p) {
                const float sn = back ? -s[p] : s[p], x0 = v[2 * p], x1 = v[2 * p + 1];
                v[2 * p] = fmaf(x0, c[p], -x1 * sn);
                v[2 * p + 1] = fmaf(x0, sn, x1 * c[p]);
            }
        }
    }
};

template <int LANES>
__device__ __forceinline__ float sum_over(float x)
{
#pragma unroll
    for (int o = LANES / 2; o >= 1; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

template <int N>
__device__ __forceinline__ void load_weight(const float* w, int sub, float (&v)[N])
{
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = w ? w[sub * N + e] : 1.0f;
}

// A warp takes token blockIdx.x * kRopeWarps + its number and the head groups of slice blockIdx.y
// of its `slices` (a group: the 32 / LANES heads of one access; the q groups come first).
template <typename T, int D, bool HALF>
__global__ void __launch_bounds__(32 * kRopeWarps) rope_forward_kernel(const RopeArgs a, int per_slice)
{
    typedef piece<T> P;
    constexpr int N = P::N, LANES = D / N, HEADS = 32 / LANES, AHEAD = 4;
    const int lane = threadIdx.x & 31, sub = lane % LANES, mine = lane / LANES;
    const long long token = (long long)blockIdx.x * kRopeWarps + (threadIdx.x >> 5);
    pdl_wait();
    if (token >= (long long)a.B * a.T) return;
    const int b = (int)(token / a.T), t = (int)(token - (long long)b * a.T);
    Turn<T, D, HALF> turn;
    turn.at(a, (a.pos ? (long long)a.pos[b] : a.t0) + t, sub);
    const int gq = (a.Hq + HEADS - 1) / HEADS, gk = (a.Hk + HEADS - 1) / HEADS;
    const int g0 = blockIdx.y * per_slice, g1 = min(g0 + per_slice, gq + gk);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const int lo = w ? max(g0, gq) - gq : min(g0, gq), hi = w ? max(g1, gq) - gq : min(g1, gq);
        const int H = w ? a.Hk : a.Hq;
        if (lo >= hi) continue;
        const T* in = static_cast<const T*>(a.in[w]) + b * a.s[w][0][0] + t * a.s[w][0][1] + sub * N;
        T* out = static_cast<T*>(const_cast<void*>(a.out[w])) + b * a.s[w][1][0] + t * a.s[w][1][1] + sub * N;
        float wt[N];
        load_weight<N>(a.weight[w], sub, wt);
        for (int g = lo; g < hi; g += AHEAD) {
            uint4 r[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int h = (g + k) * HEADS + mine;
                r[k] = make_uint4(0, 0, 0, 0);
                if (g + k < hi && h < H) r[k] = *reinterpret_cast<const uint4*>(in + h * a.s[w][0][2]);
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (g + k >= hi) break;
                const int h = (g + k) * HEADS + mine;
                float v[N], ss = 0.0f;
                P::get(r[k], v);
#pragma unroll
                for (int e = 0; e < N; ++e) ss = fmaf(v[e], v[e], ss);
                const float n = rsqrtf(fmaf(sum_over<LANES>(ss), 1.0f / D, a.eps));
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] *= n * wt[e];
                turn.apply(v, sub, false);
                if (h < H) *reinterpret_cast<uint4*>(out + h * a.s[w][1][2]) = P::put(v);
            }
        }
    }
}

// The gradient: each warp goes over tokens (and, with few tokens, over one slice of the head
// groups) and keeps its lanes' sums of dw in registers; the CTA's sums go to ws[cta][q, k][D].
template <typename T, int D, bool HALF>
__global__ void __launch_bounds__(32 * kRopeWarps) rope_backward_kernel(const RopeArgs a, int per_slice, int slices)
{
    typedef piece<T> P;
    constexpr int N = P::N, LANES = D / N, HEADS = 32 / LANES, AHEAD = 2;
    __shared__ float part[kRopeWarps][2][D];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % LANES, mine = lane / LANES;
    const int gq = (a.Hq + HEADS - 1) / HEADS, gk = (a.Hk + HEADS - 1) / HEADS;
    pdl_wait();
    float dw[2][N];
#pragma unroll
    for (int e = 0; e < N; ++e) dw[0][e] = dw[1][e] = 0.0f;
    const long long units = (long long)a.B * a.T * slices, step = (long long)gridDim.x * kRopeWarps;
    for (long long u = (long long)blockIdx.x * kRopeWarps + warp; u < units; u += step) {
        const long long token = u / slices;
        const int slice = (int)(u - token * slices);
        const int b = (int)(token / a.T), t = (int)(token - (long long)b * a.T);
        Turn<T, D, HALF> turn;
        turn.at(a, (a.pos ? (long long)a.pos[b] : a.t0) + t, sub);
        const int g0 = slice * per_slice, g1 = min(g0 + per_slice, gq + gk);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int lo = w ? max(g0, gq) - gq : min(g0, gq), hi = w ? max(g1, gq) - gq : min(g1, gq);
            const int H = w ? a.Hk : a.Hq;
            if (lo >= hi) continue;
            const T* in = static_cast<const T*>(a.in[w]) + b * a.s[w][0][0] + t * a.s[w][0][1] + sub * N;
            const T* dy = static_cast<const T*>(a.dout[w]) + b * a.s[w][2][0] + t * a.s[w][2][1] + sub * N;
            T* dx = static_cast<T*>(a.din[w]) + b * a.s[w][3][0] + t * a.s[w][3][1] + sub * N;
            float wt[N];
            load_weight<N>(a.weight[w], sub, wt);
            for (int g = lo; g < hi; g += AHEAD) {
                uint4 rx[AHEAD], rd[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    const int h = (g + k) * HEADS + mine;
                    rx[k] = rd[k] = make_uint4(0, 0, 0, 0);
                    if (g + k < hi && h < H) {
                        rx[k] = *reinterpret_cast<const uint4*>(in + h * a.s[w][0][2]);
                        rd[k] = *reinterpret_cast<const uint4*>(dy + h * a.s[w][2][2]);
                    }
                }
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    if (g + k >= hi) break;
                    const int h = (g + k) * HEADS + mine;
                    float x[N], d[N], ss = 0.0f, dot = 0.0f;
                    P::get(rx[k], x);
                    P::get(rd[k], d);
                    turn.apply(d, sub, true);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        ss = fmaf(x[e], x[e], ss);
                        dot = fmaf(d[e] * wt[e], x[e], dot);
                    }
                    const float n = rsqrtf(fmaf(sum_over<LANES>(ss), 1.0f / D, a.eps));
                    const float m = sum_over<LANES>(dot) * (1.0f / D) * n * n;
                    // a head past the last one has x = dy = 0 and adds nothing (with eps = 0 its n is not finite)
                    if (h < H) {
                        float o[N];
#pragma unroll
                        for (int e = 0; e < N; ++e) {
                            dw[w][e] = fmaf(d[e], x[e] * n, dw[w][e]);
                            o[e] = n * fmaf(-x[e], m, d[e] * wt[e]);
                        }
                        *reinterpret_cast<uint4*>(dx + h * a.s[w][3][2]) = P::put(o);
                    }
                }
            }
        }
    }
    if (!a.ws) return;
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            float v = dw[w][e];
#pragma unroll
            for (int o = 16; o >= LANES; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (mine == 0) part[warp][w][sub * N + e] = v;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += 32 * kRopeWarps) {
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < kRopeWarps; ++k) v += part[k][i / D][i % D];
        a.ws[(long long)blockIdx.x * 2 * D + i] = v;
    }
}

// dw: the CTAs' sums in a fixed order.  One warp per channel.
__global__ void __launch_bounds__(256) rope_dw_kernel(const float* ws, int ctas, int D, float* dwq, float* dwk)
{
    pdl_wait();
    const int i = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (i >= 2 * D) return;
    float* to = i < D ? dwq : dwk;
    float v = 0.0f;
#pragma unroll 8
    for (int k = lane; k < ctas; k += 32) v += ws[(long long)k * 2 * D + i];
    v = sum_over<32>(v);
    if (lane == 0 && to) to[i < D ? i : i - D] = v;
}

int heads_per_access(const RopeArgs& a) { return 32 * (a.bf16 ? 8 : 4) / a.d; }
int head_groups(const RopeArgs& a)
{
    const int n = heads_per_access(a);
    return (a.Hq + n - 1) / n + (a.Hk + n - 1) / n;
}
// Head groups of one warp: all of a token's, unless that leaves fewer than about 32 warps per SM.
int groups_per_slice(const RopeArgs& a, int sms)
{
    const int groups = head_groups(a);
    const long long want = 32LL * sms, tokens = (long long)a.B * a.T;
    const long long slices = tokens >= want ? 1 : (want + tokens - 1) / tokens;
    return slices >= groups ? 1 : (int)((groups + slices - 1) / slices);
}
int backward_ctas(const RopeArgs& a, int sms)
{
    const int per = groups_per_slice(a, sms), slices = (head_groups(a) + per - 1) / per;
    const long long units = (long long)a.B * a.T * slices, ctas = (units + kRopeWarps - 1) / kRopeWarps;
    return (int)(ctas < 4LL * sms ? ctas : 4LL * sms);
}

template <typename T, int D, bool HALF>
cudaError_t forward_t(const RopeArgs& a, int sms, cudaStream_t st)
{
    const int per = groups_per_slice(a, sms), slices = (head_groups(a) + per - 1) / per;
    const long long blocks = ((long long)a.B * a.T + kRopeWarps - 1) / kRopeWarps;
    return launch_dependent(rope_forward_kernel<T, D, HALF>, dim3((unsigned)blocks, slices), dim3(32 * kRopeWarps), 0, st, a, per);
}
template <typename T, int D, bool HALF>
cudaError_t backward_t(const RopeArgs& a, int sms, cudaStream_t st)
{
    const int per = groups_per_slice(a, sms), slices = (head_groups(a) + per - 1) / per, ctas = backward_ctas(a, sms);
    const cudaError_t e =
        launch_dependent(rope_backward_kernel<T, D, HALF>, dim3(ctas), dim3(32 * kRopeWarps), 0, st, a, per, slices);
    if (e != cudaSuccess || !a.ws) return e;
    return launch_dependent(rope_dw_kernel, dim3(2 * D / 8), dim3(256), 0, st, a.ws, ctas, D, a.dw[0], a.dw[1]);
}

#define LASAD_ROPE_DISPATCH(fn)                                                                                      \
    (a.bf16 ? a.d == 64 ? (a.half ? fn<__nv_bfloat16, 64, true>(a, sms, st) : fn<__nv_bfloat16, 64, false>(a, sms, st)) \
                        : (a.half ? fn<__nv_bfloat16, 32, true>(a, sms, st) : fn<__nv_bfloat16, 32, false>(a, sms, st)) \
            : a.d == 64 ? (a.half ? fn<float, 64, true>(a, sms, st) : fn<float, 64, false>(a, sms, st))                 \
                        : (a.half ? fn<float, 32, true>(a, sms, st) : fn<float, 32, false>(a, sms, st)))

}  // namespace

size_t rope_workspace_bytes(const RopeArgs& a, int sms) { return (size_t)backward_ctas(a, sms) * 2 * a.d * sizeof(float); }
int rope_backward_launches(const RopeArgs& a) { return a.ws ? 2 : 1; }
cudaError_t launch_rope_forward(const RopeArgs& a, int sms, cudaStream_t st) { return LASAD_ROPE_DISPATCH(forward_t); }
cudaError_t launch_rope_backward(const RopeArgs& a, int sms, cudaStream_t st) { return LASAD_ROPE_DISPATCH(backward_t); }

}  // namespace lasad
