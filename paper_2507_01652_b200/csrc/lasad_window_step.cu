// One generated token against a ring cache of the window attention.  A sequence keeps S + W slots:
// token i stands in slot i (i < S, the sinks) or S + (i - S) mod W, so the slots in use are always
// the sinks and the last W other tokens -- what the token at position i sees -- and their order
// does not matter to a softmax.  The call puts the token's own k and v into its slot and returns
//
//     o = sum_n e^(scale q.k_n) v_n / sum_n e^(scale q.k_n)    over the slots in use.
//
// Bound by reading the cache once.  A key row lies in the 16-byte pieces of d / 8 (bf16) or d / 4
// (fp32) lanes; all query heads that share the key head (up to eight at a time) work on the row
// while it is in registers.  Every group of lanes keeps its own running maximum and sum over its
// rows; they are joined once, by shuffles, shared memory, and, where few sequences leave SMs idle
// and the slots are cut over several CTAs, by the last CTA of a (sequence, key head) to finish.
#include "lasad_mixers.cuh"
#include "lasad_tc_ptx.cuh"

namespace lasad {
namespace {

constexpr int kStepWarps = 4;
constexpr float kLog2e = 1.4426950408889634f;

template <typename T> struct row_piece;
template <> struct row_piece<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void get(const uint4& r, float (&v)[8])
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = tcx::bf16_lo(w[i]), v[2 * i + 1] = tcx::bf16_hi(w[i]);
    }
};
template <> struct row_piece<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void get(const uint4& r, float (&v)[4])
    {
        v[0] = __uint_as_float(r.x), v[1] = __uint_as_float(r.y), v[2] = __uint_as_float(r.z), v[3] = __uint_as_float(r.w);
    }
};

// Joins (m2, l2, o2) into (m, l, o): the same softmax over two sets of rows.  Maxima are in powers of two.
template <int N>
__device__ __forceinline__ void join(float& m, float& l, float (&o)[N], float m2, float l2, const float (&o2)[N])
{
    const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
    const float f = exp2f(m - base), f2 = exp2f(m2 - base);
    m = top;
    l = l * f + l2 * f2;
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = o[e] * f + o2[e] * f2;
}

// grid: (splits, Hk * head chunks, B).  GB: query heads of one CTA.
template <typename T, int D, int GB>
__global__ void __launch_bounds__(32 * kStepWarps) window_step_kernel(const WindowArgs a, int per_split)
{
    typedef row_piece<T> P;
    constexpr int N = P::N, LANES = D / N, ROWS = 32 / LANES, AHEAD = 4;   // rows of one access of a warp; accesses in flight
    __shared__ float part[kStepWarps][GB][D + 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % LANES, mine = lane / LANES;
    const int G = a.Hq / a.Hk, hchunks = (G + GB - 1) / GB;
    const int hk = blockIdx.y / hchunks, g0 = (blockIdx.y - hk * hchunks) * GB, b = blockIdx.z;
    const int heads = min(GB, G - g0), h0 = hk * G + g0;
    pdl_wait();
    const int pos = a.pos[b];
    const int S = a.sinks, W = a.window;
    // slots in use, 0 .. n - 1, and the token's own
    const int n = pos < 0 ? 0 : pos < S + W ? pos + 1 : S + W;
    const int own = pos < S ? pos : S + (pos - S) % W;
    const int lo = blockIdx.x * per_split, hi = min(lo + per_split, n);
    const T* knew = static_cast<const T*>(a.k) + b * a.ks[0] + hk * a.ks[2] + sub * N;
    const T* vnew = static_cast<const T*>(a.v) + b * a.vs[0] + hk * a.vs[2] + sub * N;
    T* kc = static_cast<T*>(a.kc) + b * a.kcs[0] + hk * a.kcs[2] + sub * N;
    T* vc = static_cast<T*>(a.vc) + b * a.vcs[0] + hk * a.vcs[2] + sub * N;
    float q[GB][N], o[GB][N], m[GB], l[GB];
#pragma unroll
    for (int g = 0; g < GB; ++g) {
        uint4 r = make_uint4(0, 0, 0, 0);
        if (g < heads) r = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + b * a.qs[0] + (h0 + g) * a.qs[2] + sub * N);
        P::get(r, q[g]);
        m[g] = -INFINITY, l[g] = 0.0f;
#pragma unroll
        for (int e = 0; e < N; ++e) q[g][e] *= a.scale * kLog2e, o[g][e] = 0.0f;
    }
    for (int r0 = lo; r0 < hi; r0 += kStepWarps * ROWS * AHEAD) {
        uint4 rk[AHEAD], rv[AHEAD];
        bool live[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int r = r0 + (i * kStepWarps + warp) * ROWS + mine;
            live[i] = r < hi;
            rk[i] = rv[i] = make_uint4(0, 0, 0, 0);
            if (live[i]) {
                const bool fresh = r == own;         // (its slot may not hold it yet)
                rk[i] = *reinterpret_cast<const uint4*>(fresh ? knew : kc + r * a.kcs[1]);
                rv[i] = *reinterpret_cast<const uint4*>(fresh ? vnew : vc + r * a.vcs[1]);
                if (fresh && g0 == 0) {
                    *reinterpret_cast<uint4*>(kc + r * a.kcs[1]) = rk[i];
                    *reinterpret_cast<uint4*>(vc + r * a.vcs[1]) = rv[i];
                }
            }
        }
        float x[AHEAD][GB];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            float k[N];
            P::get(rk[i], k);
#pragma unroll
            for (int g = 0; g < GB; ++g) {
                float s = 0.0f;
#pragma unroll
                for (int e = 0; e < N; ++e) s = fmaf(q[g][e], k[e], s);
#pragma unroll
                for (int w = LANES / 2; w >= 1; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
                x[i][g] = live[i] ? s : -INFINITY;
            }
        }
#pragma unroll
        for (int g = 0; g < GB; ++g) {
            float top = m[g];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) top = fmaxf(top, x[i][g]);
            const float base = top == -INFINITY ? 0.0f : top, keep = exp2f(m[g] - base);
            m[g] = top;
            l[g] *= keep;
#pragma unroll
            for (int e = 0; e < N; ++e) o[g][e] *= keep;
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                x[i][g] = exp2f(x[i][g] - base);
                l[g] += x[i][g];
            }
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            float v[N];
            P::get(rv[i], v);
#pragma unroll
            for (int g = 0; g < GB; ++g)
#pragma unroll
                for (int e = 0; e < N; ++e) o[g][e] = fmaf(x[i][g], v[e], o[g][e]);
        }
    }
    // the groups of lanes of the warp, then the warps
#pragma unroll
    for (int g = 0; g < GB; ++g) {
#pragma unroll
        for (int w = LANES; w < 32; w <<= 1) {
            float o2[N];
            const float m2 = __shfl_xor_sync(0xffffffffu, m[g], w), l2 = __shfl_xor_sync(0xffffffffu, l[g], w);
#pragma unroll
            for (int e = 0; e < N; ++e) o2[e] = __shfl_xor_sync(0xffffffffu, o[g][e], w);
            join<N>(m[g], l[g], o[g], m2, l2, o2);
        }
        if (mine == 0) {
#pragma unroll
            for (int e = 0; e < N; ++e) part[warp][g][sub * N + e] = o[g][e];
            if (sub == 0) part[warp][g][D] = m[g], part[warp][g][D + 1] = l[g];
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < heads * D; i += 32 * kStepWarps) {
        const int g = i / D, c = i - g * D;
        float mm = -INFINITY, ll = 0.0f, oo[1] = {0.0f};
#pragma unroll
        for (int w = 0; w < kStepWarps; ++w) {
            const float o2[1] = {part[w][g][c]};
            join<1>(mm, ll, oo, part[w][g][D], part[w][g][D + 1], o2);
        }
        if (gridDim.x == 1) {
            const float v = ll > 0.0f || ll != ll ? oo[0] / ll : 0.0f;
            io<T>::store(static_cast<T*>(a.o) + b * a.os[0] + (h0 + g) * a.os[2] + c, v);
        } else {
            float* w = a.ws + (((long long)b * a.Hq + h0 + g) * gridDim.x + blockIdx.x) * (D + 2);
            w[c] = oo[0];
            if (c == 0) w[D] = mm, w[D + 1] = ll;
        }
    }
}

// Joins the splits' parts: one warp per (sequence, head).
template <typename T, int D>
__global__ void __launch_bounds__(128) window_step_join_kernel(const WindowArgs a, int splits)
{
    pdl_wait();
    const int row = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (row >= a.B * a.Hq) return;
    const int b = row / a.Hq, h = row - b * a.Hq;
    const float* w = a.ws + (long long)row * splits * (D + 2);
    float top = -INFINITY;
    for (int s = lane; s < splits; s += 32) top = fmaxf(top, w[s * (D + 2) + D]);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float base = top == -INFINITY ? 0.0f : top;
    float l = 0.0f, o[D / 32];
#pragma unroll
    for (int e = 0; e < D / 32; ++e) o[e] = 0.0f;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const float* p = w + s * (D + 2);
        const float f = exp2f(p[D] - base);
        l = fmaf(p[D + 1], f, l);
#pragma unroll
        for (int e = 0; e < D / 32; ++e) o[e] = fmaf(p[lane + 32 * e], f, o[e]);
    }
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
        io<T>::store(static_cast<T*>(a.o) + b * a.os[0] + h * a.os[2] + lane + 32 * e, l > 0.0f || l != l ? o[e] / l : 0.0f);
}

// The prefill's keys and values into the ring: slot n gets the last token of the sequence that
// belongs there; slots that no token has reached are left as they are.
template <typename T, int D>
__global__ void __launch_bounds__(256) window_store_kernel(const WindowArgs a)
{
    constexpr int N = row_piece<T>::N, LANES = D / N;
    pdl_wait();
    const long long per = (long long)a.Hk * LANES, slots = a.sinks + (long long)a.window;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int b = blockIdx.y;
    if (i >= slots * per) return;
    const int slot = (int)(i / per), x = (int)(i - slot * per), h = x / LANES, c = (x - h * LANES) * N;
    const int len = a.lengths ? min(a.lengths[b], a.T) : a.T;
    if (slot >= len) return;                     // (the slots fill in order)
    const int t = slot < a.sinks ? slot : slot + (len - 1 - slot) / a.window * a.window;
    *reinterpret_cast<uint4*>(static_cast<T*>(a.kc) + b * a.kcs[0] + slot * a.kcs[1] + h * a.kcs[2] + c) =
        *reinterpret_cast<const uint4*>(static_cast<const T*>(a.k) + b * a.ks[0] + t * a.ks[1] + h * a.ks[2] + c);
    *reinterpret_cast<uint4*>(static_cast<T*>(a.vc) + b * a.vcs[0] + slot * a.vcs[1] + h * a.vcs[2] + c) =
        *reinterpret_cast<const uint4*>(static_cast<const T*>(a.v) + b * a.vs[0] + t * a.vs[1] + h * a.vs[2] + c);
}

// Query heads of one CTA: the group that shares a key head, up to eight.
int heads_per_cta(const WindowArgs& a)
{
    const int G = a.Hq / a.Hk;
    return G == 1 ? 1 : G == 2 ? 2 : G <= 4 ? 4 : 8;
}

template <typename T, int D>
cudaError_t step_t(const WindowArgs& a, cudaStream_t st)
{
    const int GB = heads_per_cta(a), G = a.Hq / a.Hk, splits = window_step_splits(a);
    const long long slots = a.sinks + (long long)a.window;
    const int per = (int)((slots + splits - 1) / splits);
    const dim3 grid(splits, a.Hk * ((G + GB - 1) / GB), a.B);
    auto kernel = GB == 1 ? window_step_kernel<T, D, 1> : GB == 2 ? window_step_kernel<T, D, 2>
                : GB == 4 ? window_step_kernel<T, D, 4> : window_step_kernel<T, D, 8>;
    const cudaError_t e = launch_dependent(kernel, grid, dim3(32 * kStepWarps), 0, st, a, per);
    if (e != cudaSuccess || splits == 1) return e;
    return launch_dependent(window_step_join_kernel<T, D>, dim3((unsigned)((a.B * a.Hq + 3) / 4)), dim3(128), 0, st, a, splits);
}

}  // namespace

int window_step_splits(const WindowArgs& a)
{
    const int GB = heads_per_cta(a), G = a.Hq / a.Hk;
    const long long ctas = (long long)a.B * a.Hk * ((G + GB - 1) / GB), slots = a.sinks + (long long)a.window;
    long long splits = (4LL * a.sms + ctas - 1) / ctas;
    const long long most = (slots + 63) / 64;
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    const long long per = (slots + splits - 1) / splits;
    return (int)((slots + per - 1) / per);
}
size_t window_step_workspace_bytes(const WindowArgs& a)
{
    const int splits = window_step_splits(a);
    return splits == 1 ? 0 : (size_t)a.B * a.Hq * splits * (a.d + 2) * sizeof(float);
}

cudaError_t launch_window_step(const WindowArgs& a, cudaStream_t st)
{
    if (a.bf16) return a.d == 64 ? step_t<__nv_bfloat16, 64>(a, st) : step_t<__nv_bfloat16, 32>(a, st);
    return a.d == 64 ? step_t<float, 64>(a, st) : step_t<float, 32>(a, st);
}

cudaError_t launch_window_store(const WindowArgs& a, cudaStream_t st)
{
    const long long lanes = (a.sinks + (long long)a.window) * a.Hk * (a.d / (a.bf16 ? 8 : 4));
    auto kernel = a.bf16 ? (a.d == 64 ? window_store_kernel<__nv_bfloat16, 64> : window_store_kernel<__nv_bfloat16, 32>)
                         : (a.d == 64 ? window_store_kernel<float, 64> : window_store_kernel<float, 32>);
    return launch_dependent(kernel, dim3((unsigned)((lanes + 255) / 256), a.B), dim3(256), 0, st, a);
}

}  // namespace lasad
