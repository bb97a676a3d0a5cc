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
// rows; they are joined once, by shuffles, and, where several warps have a (sequence, key head), in
// shared memory.  Who has one goes by how many there are: with 16 and more per SM a warp each (nothing
// is shared, and a CTA's warps are independent: 256 sequences x 20 heads, 55 MB of keys and values, 16.3 us;
// with a CTA each 27 us); with fewer a CTA of eight warps each, and with fewer than SMs a cluster of up to
// eight CTAs, whose parts the first one joins (2 x 24 heads of 8 key heads, 4097 slots: 14.6 us; parts in memory and
// a second launch that joins them: 17 us).
#include "lasad_mixers.cuh"
#include "lasad_tc_ptx.cuh"

namespace lasad {
namespace {

constexpr int kStepWarps = 8, kMaxCluster = 8;      // of a CTA that has one unit; of a unit
constexpr int kSoloWarps = 4, kSoloCtas = 6;        // of a CTA whose warps have a unit each; on an SM
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
    static __device__ __forceinline__ uint4 put(const float (&v)[8])
    {
        return make_uint4(tcx::pack_bf16(v[0], v[1]), tcx::pack_bf16(v[2], v[3]), tcx::pack_bf16(v[4], v[5]), tcx::pack_bf16(v[6], v[7]));
    }
};
template <> struct row_piece<float> {
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

template <int V> struct Int { static constexpr int value = V; };

// Reads the same place of the shared memory of the cluster's CTA number `rank`.
__device__ __forceinline__ float of_rank(const float* p, int rank)
{
    float x;
    asm volatile("{\n\t.reg .b32 r;\n\tmapa.shared::cluster.u32 r, %1, %2;\n\tld.shared::cluster.f32 %0, [r];\n\t}"
                 : "=f"(x)
                 : "r"(tcx::smem_u32(p)), "r"(rank)
                 : "memory");
    return x;
}

// Joins (m2, l2, o2) into (m, l, o): the same softmax over two sets of rows.  Maxima are in powers of two.
template <int N>
__device__ __forceinline__ void join(float& m, float& l, float (&o)[N], float m2, float l2, const float (&o2)[N])
{
    const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
    const float f = tcx::ex2_approx(m - base), f2 = tcx::ex2_approx(m2 - base);
    m = top;
    l = l * f + l2 * f2;
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = o[e] * f + o2[e] * f2;
}

// Accesses of a warp in flight, per tensor (and as many of the next rows): what the registers of GB
// query heads leave room for, with many warps on an SM (SOLO) or eight.
template <int GB, bool SOLO> struct ahead { static constexpr int value = SOLO ? (GB == 1 ? 3 : GB <= 4 ? 2 : 1) : GB == 1 ? 6 : GB <= 3 ? 4 : GB == 4 ? 3 : GB == 6 ? 2 : 1; };

// A unit is a sequence, a key head and up to GB of its query heads.  SOLO: a warp has a unit; else a CTA
// has one, or its cluster (blockIdx.x = unit * cluster + rank) with per_cta slots for each CTA.
template <typename T, int D, int GB, bool SOLO>
__global__ void __launch_bounds__(32 * (SOLO ? kSoloWarps : kStepWarps), SOLO && GB == 1 ? kSoloCtas : 1) window_step_kernel(const WindowArgs a, int cluster, int per_cta)
{
    typedef row_piece<T> P;
    constexpr int N = P::N, LANES = D / N, ROWS = 32 / LANES, AHEAD = ahead<GB, SOLO>::value;   // ROWS: of one access of a warp
    constexpr int WARPS = SOLO ? 1 : kStepWarps;                                          // warps of a unit in this CTA
    __shared__ float part[SOLO ? 1 : kStepWarps][GB][D + 2];
    __shared__ float whole[GB][D + 2];                               // the CTA's part of its cluster's result
    const int lane = threadIdx.x & 31, warp = SOLO ? 0 : threadIdx.x >> 5, sub = lane % LANES, mine = lane / LANES;
    const int G = a.Hq / a.Hk, hchunks = (G + GB - 1) / GB, per_b = a.Hk * hchunks;
    const int unit = SOLO ? blockIdx.x * kSoloWarps + (threadIdx.x >> 5) : blockIdx.x / cluster;
    const int rank = SOLO ? 0 : blockIdx.x - unit * cluster;
    pdl_wait();
    if (SOLO && unit >= a.B * per_b) return;
    const int b = unit / per_b, y = unit - b * per_b, hk = y / hchunks, g0 = (y - hk * hchunks) * GB;
    const int heads = min(GB, G - g0), h0 = hk * G + g0;
    const int pos = a.pos[b];
    const int S = a.sinks, W = a.window;
    // slots in use, 0 .. n - 1, and the token's own
    const int n = pos < 0 ? 0 : pos < S + W ? pos + 1 : S + W;
    const int own = pos < S ? pos : S + (pos - S) % W;
    const int lo = SOLO ? 0 : rank * per_cta, hi = SOLO ? n : min(lo + per_cta, n);
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
    // n accesses' rows: a dot product per query head, the running maximum once, then the values
    auto take = [&](auto& rk, auto& rv, int first, int end, int skip, auto count) {
        constexpr int C = decltype(count)::value;
        float x[C][GB];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const bool live = first + i * WARPS * ROWS < end && first + i * WARPS * ROWS != skip;
            float k[N];
            P::get(rk[i], k);
#pragma unroll
            for (int g = 0; g < GB; ++g) {
                float s = 0.0f;
#pragma unroll
                for (int e = 0; e < N; ++e) s = fmaf(q[g][e], k[e], s);
#pragma unroll
                for (int w = LANES / 2; w >= 1; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
                x[i][g] = live ? s : -INFINITY;
            }
        }
#pragma unroll
        for (int g = 0; g < GB; ++g) {
            float top = m[g];
#pragma unroll
            for (int i = 0; i < C; ++i) top = fmaxf(top, x[i][g]);
            const float base = top == -INFINITY ? 0.0f : top, keep = tcx::ex2_approx(m[g] - base);
            m[g] = top;
            l[g] *= keep;
#pragma unroll
            for (int e = 0; e < N; ++e) o[g][e] *= keep;
#pragma unroll
            for (int i = 0; i < C; ++i) {
                x[i][g] = tcx::ex2_approx(x[i][g] - base);
                l[g] += x[i][g];
            }
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float v[N];
            P::get(rv[i], v);
#pragma unroll
            for (int g = 0; g < GB; ++g)
#pragma unroll
                for (int e = 0; e < N; ++e) o[g][e] = fmaf(x[i][g], v[e], o[g][e]);
        }
    };
    // rows first, first + WARPS * ROWS, ..; the token's own slot may not hold it yet: it comes by itself
    const long long kstep = WARPS * ROWS * a.kcs[1], vstep = WARPS * ROWS * a.vcs[1];
    int row = lo + warp * ROWS + mine;
    const T* kp = kc + row * a.kcs[1];
    const T* vp = vc + row * a.vcs[1];
    auto load = [&](uint4 (&tk)[AHEAD], uint4 (&tv)[AHEAD], int first) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i, kp += kstep, vp += vstep) {
            const int r = first + i * WARPS * ROWS;
            tk[i] = tv[i] = make_uint4(0, 0, 0, 0);
            if (r < hi && r != own) {
                tk[i] = *reinterpret_cast<const uint4*>(kp);
                tv[i] = *reinterpret_cast<const uint4*>(vp);
            }
        }
    };
    constexpr int STEP = WARPS * ROWS * AHEAD;
    uint4 rk[2][AHEAD], rv[2][AHEAD];
    load(rk[0], rv[0], row);
    if (own >= lo && own < hi && warp == 0) {        // (uniform over the warp)
        uint4 ok[1] = {make_uint4(0, 0, 0, 0)}, ov[1] = {make_uint4(0, 0, 0, 0)};
        if (mine == 0) {
            ok[0] = *reinterpret_cast<const uint4*>(knew);
            ov[0] = *reinterpret_cast<const uint4*>(vnew);
            if (g0 == 0) {
                *reinterpret_cast<uint4*>(kc + own * a.kcs[1]) = ok[0];
                *reinterpret_cast<uint4*>(vc + own * a.vcs[1]) = ov[0];
            }
        }
        take(ok, ov, mine, 1, -1, Int<1>());       // (lane group 0 alone)
    }
    for (int r0 = lo; r0 < hi; r0 += 2 * STEP, row += 2 * STEP) {     // (uniform; the next rows come in under these ones' arithmetic)
        load(rk[1], rv[1], row + STEP);
        take(rk[0], rv[0], row, hi, own, Int<AHEAD>());
        load(rk[0], rv[0], row + 2 * STEP);
        if (r0 + STEP < hi) take(rk[1], rv[1], row + STEP, hi, own, Int<AHEAD>());
    }
    // the groups of lanes of the warp
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
            if (SOLO) {
                if (g < heads) {
                    const float inv = l[g] > 0.0f || l[g] != l[g] ? 1.0f / l[g] : 0.0f;
                    T* out = static_cast<T*>(a.o) + b * a.os[0] + (h0 + g) * a.os[2] + sub * N;
                    float r[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) r[e] = o[g][e] * inv;
                    *reinterpret_cast<uint4*>(out) = P::put(r);
                }
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) part[warp][g][sub * N + e] = o[g][e];
                if (sub == 0) part[warp][g][D] = m[g], part[warp][g][D + 1] = l[g];
            }
        }
    }
    if (SOLO) return;
    __syncthreads();
    // the warps of the CTA
    for (int i = threadIdx.x; i < heads * D; i += 32 * kStepWarps) {
        const int g = i / D, c = i - g * D;
        float mm = -INFINITY, ll = 0.0f, oo[1] = {0.0f};
#pragma unroll
        for (int w = 0; w < kStepWarps; ++w) {
            const float o2[1] = {part[w][g][c]};
            join<1>(mm, ll, oo, part[w][g][D], part[w][g][D + 1], o2);
        }
        if (cluster == 1) {
            io<T>::store(static_cast<T*>(a.o) + b * a.os[0] + (h0 + g) * a.os[2] + c, ll > 0.0f || ll != ll ? oo[0] / ll : 0.0f);
        } else {
            whole[g][c] = oo[0];
            if (c == 0) whole[g][D] = mm, whole[g][D + 1] = ll;
        }
    }
    if (cluster == 1) return;
    // the CTAs of the cluster, by the first one; the others stay until it has read their parts
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (rank == 0)
        for (int i = threadIdx.x; i < heads * D; i += 32 * kStepWarps) {
            const int g = i / D, c = i - g * D;
            float m2[kMaxCluster], l2[kMaxCluster], o2[kMaxCluster][1];    // (all asked for before the first is used)
#pragma unroll
            for (int w = 0; w < kMaxCluster; ++w) {
                m2[w] = -INFINITY, l2[w] = o2[w][0] = 0.0f;
                if (w < cluster) m2[w] = of_rank(&whole[g][D], w), l2[w] = of_rank(&whole[g][D + 1], w), o2[w][0] = of_rank(&whole[g][c], w);
            }
            float mm = -INFINITY, ll = 0.0f, oo[1] = {0.0f};
#pragma unroll
            for (int w = 0; w < kMaxCluster; ++w) join<1>(mm, ll, oo, m2[w], l2[w], o2[w]);
            io<T>::store(static_cast<T*>(a.o) + b * a.os[0] + (h0 + g) * a.os[2] + c, ll > 0.0f || ll != ll ? oo[0] / ll : 0.0f);
        }
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
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

template <typename T, int D, int GB>
cudaError_t step_g(const WindowArgs& a, cudaStream_t st)
{
    const int G = a.Hq / a.Hk;
    const long long units = (long long)a.B * a.Hk * ((G + GB - 1) / GB), slots = a.sinks + (long long)a.window;
    if (units >= 16LL * a.sms)
        return launch_dependent(window_step_kernel<T, D, GB, true>, dim3((unsigned)((units + kSoloWarps - 1) / kSoloWarps)),
                                dim3(32 * kSoloWarps), 0, st, a, 1, 0);
    // CTAs of a unit: as long as the SMs have room and a CTA keeps 64 slots
    int cluster = 1;
    while (cluster < kMaxCluster && units * cluster * 2 <= a.sms && slots >= 128LL * cluster) cluster *= 2;
    const int per = (int)((slots + cluster - 1) / cluster);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * cluster));
    cfg.blockDim = dim3(32 * kStepWarps);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, window_step_kernel<T, D, GB, false>, a, cluster, per);
}
template <typename T, int D>
cudaError_t step_t(const WindowArgs& a, cudaStream_t st)
{
    // query heads of one unit: the group that shares a key head, up to eight
    const int G = a.Hq / a.Hk;
    switch (G) {
        case 1: return step_g<T, D, 1>(a, st);
        case 2: return step_g<T, D, 2>(a, st);
        case 3: return step_g<T, D, 3>(a, st);
        case 4: return step_g<T, D, 4>(a, st);
        case 5:
        case 6: return step_g<T, D, 6>(a, st);
        default: return step_g<T, D, 8>(a, st);
    }
}

}  // namespace

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
