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
// Bound by device memory: x in and y out (x, dy in and dx out).  A head's channels lie in d / 8 (bf16)
// or d / 4 (fp32) neighbouring lanes, so the sums are three or four shuffles, and a warp works on
// one token: its angles are read once and serve all of the heads.  Two pairs at a time go through
// the packed arithmetic: without it the kernels were bound by the instructions they issue.
#include "lasad_mixers.cuh"
#include "lasad_tc_ptx.cuh"

namespace lasad {
namespace {

constexpr int kRopeWarps = 8;
constexpr int kForwardAhead = 3, kBackwardAhead = 3;        // accesses of a warp in flight (twice as many in the gradient)
constexpr int kBackwardCtas = 2;                              // CTAs of the gradient that share an SM (registers)

typedef unsigned long long pairf;        // two fp32 numbers, for the packed arithmetic of sm_100
__device__ __forceinline__ pairf mk(float a, float b)
{
    pairf r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float lo(pairf p)
{
    return __uint_as_float((uint32_t)p);
}
__device__ __forceinline__ float hi(pairf p)
{
    return __uint_as_float((uint32_t)(p >> 32));
}
__device__ __forceinline__ pairf mul(pairf a, pairf b)
{
    pairf r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ pairf fma(pairf a, pairf b, pairf c)
{
    pairf r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// What one lane has of a head: the first channels of P pairs in x0 and their partners in x1, two pairs
// to a number.  Adjacent pairs (2m, 2m + 1) come in one access of 16 bytes; pairs (m, m + D / 2) in
// two of 8, so that the partners are in one lane and the rotation needs no exchange.
template <typename T, bool HALF> struct Lane;
template <bool HALF> struct Lane<__nv_bfloat16, HALF> {
    static constexpr int P = 4;
    uint32_t r[4];
    template <int D> __device__ __forceinline__ void load(const __nv_bfloat16* head, int sub)
    {
        if (HALF) {
            const uint2 a = *reinterpret_cast<const uint2*>(head + sub * 4), b = *reinterpret_cast<const uint2*>(head + D / 2 + sub * 4);
            r[0] = a.x, r[1] = a.y, r[2] = b.x, r[3] = b.y;
        } else {
            const uint4 a = *reinterpret_cast<const uint4*>(head + sub * 8);
            r[0] = a.x, r[1] = a.y, r[2] = a.z, r[3] = a.w;
        }
    }
    __device__ __forceinline__ void none() { r[0] = r[1] = r[2] = r[3] = 0; }
    __device__ __forceinline__ void get(pairf (&x0)[2], pairf (&x1)[2]) const
    {
        using namespace tcx;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (HALF) {
                x0[i] = mk(bf16_lo(r[i]), bf16_hi(r[i]));
                x1[i] = mk(bf16_lo(r[2 + i]), bf16_hi(r[2 + i]));
            } else {
                x0[i] = mk(bf16_lo(r[2 * i]), bf16_lo(r[2 * i + 1]));
                x1[i] = mk(bf16_hi(r[2 * i]), bf16_hi(r[2 * i + 1]));
            }
    }
    template <int D> static __device__ __forceinline__ void store(__nv_bfloat16* head, int sub, const pairf (&x0)[2], const pairf (&x1)[2])
    {
        using namespace tcx;
        if (HALF) {
            *reinterpret_cast<uint2*>(head + sub * 4) = make_uint2(pack_bf16(lo(x0[0]), hi(x0[0])), pack_bf16(lo(x0[1]), hi(x0[1])));
            *reinterpret_cast<uint2*>(head + D / 2 + sub * 4) = make_uint2(pack_bf16(lo(x1[0]), hi(x1[0])), pack_bf16(lo(x1[1]), hi(x1[1])));
        } else {
            *reinterpret_cast<uint4*>(head + sub * 8) = make_uint4(pack_bf16(lo(x0[0]), lo(x1[0])), pack_bf16(hi(x0[0]), hi(x1[0])),
                                                                   pack_bf16(lo(x0[1]), lo(x1[1])), pack_bf16(hi(x0[1]), hi(x1[1])));
        }
    }
};
template <bool HALF> struct Lane<float, HALF> {
    static constexpr int P = 2;
    float2 a, b;
    template <int D> __device__ __forceinline__ void load(const float* head, int sub)
    {
        if (HALF) {
            a = *reinterpret_cast<const float2*>(head + sub * 2), b = *reinterpret_cast<const float2*>(head + D / 2 + sub * 2);
        } else {
            const float4 v = *reinterpret_cast<const float4*>(head + sub * 4);
            a = make_float2(v.x, v.z), b = make_float2(v.y, v.w);
        }
    }
    __device__ __forceinline__ void none() { a = b = make_float2(0.0f, 0.0f); }
    __device__ __forceinline__ void get(pairf (&x0)[1], pairf (&x1)[1]) const { x0[0] = mk(a.x, a.y), x1[0] = mk(b.x, b.y); }
    template <int D> static __device__ __forceinline__ void store(float* head, int sub, const pairf (&x0)[1], const pairf (&x1)[1])
    {
        if (HALF) {
            *reinterpret_cast<float2*>(head + sub * 2) = make_float2(lo(x0[0]), hi(x0[0]));
            *reinterpret_cast<float2*>(head + D / 2 + sub * 2) = make_float2(lo(x1[0]), hi(x1[0]));
        } else {
            *reinterpret_cast<float4*>(head + sub * 4) = make_float4(lo(x0[0]), lo(x1[0]), hi(x0[0]), hi(x1[0]));
        }
    }
};

// Where consecutive tokens stand: the table rows of their two halves of pairs.  One division per
// run of tokens (a 64-bit one is a hundred instructions), then steps.
struct Place {
    long long j;          // index on the grid (negative before it), or the position itself without a grid
    int row, col;
    __device__ __forceinline__ void set(const RopeArgs& a, long long i)
    {
        j = a.grid_w > 0 ? i - a.prefix_len : i;
        row = col = 0;
        if (a.grid_w > 0 && j > 0) {
            const long long r = j <= 0x7fffffffLL ? (long long)((unsigned)j / (unsigned)a.grid_w) : j / a.grid_w;
            row = (int)(r < 0x7fffffffLL ? r : 0x7fffffffLL);
            col = (int)(j - r * a.grid_w);
        }
    }
    __device__ __forceinline__ void next(const RopeArgs& a)
    {
        if (a.grid_w > 0 && j >= 0 && ++col == a.grid_w) col = 0, row = row < 0x7fffffff ? row + 1 : row;
        ++j;
    }
};

// cos and sin of a lane's pairs, sub * P .. sub * P + P - 1, at one place.  (P divides D / 4: they are
// all of the row or all of the column.)
template <int D, int P>
__device__ __forceinline__ void angles(const RopeArgs& a, const Place& at, int sub, pairf (&c)[P / 2], pairf (&s)[P / 2])
{
    int m = sub * P, width = D / 2, row;
    if (a.grid_w > 0) {
        if (at.j < 0) {
#pragma unroll
            for (int p = 0; p < P / 2; ++p) c[p] = mk(1.0f, 1.0f), s[p] = mk(0.0f, 0.0f);
            return;
        }
        width = D / 4;
        row = m < width ? at.row : at.col;
        m = m < width ? m : m - width;
    } else {
        row = at.j < 0 ? 0 : at.j < a.table_rows ? (int)at.j : a.table_rows - 1;
    }
    // (positions that come from device memory are not known to the host: they end at the table's edge)
    row = min(row, a.table_rows - 1);
    const float* t = a.table + ((long long)row * width + m) * 2;
#pragma unroll
    for (int p = 0; p < P / 2; ++p) {
        const float4 f = *reinterpret_cast<const float4*>(t + 4 * p);
        c[p] = mk(f.x, f.z), s[p] = mk(f.y, f.w);
    }
}

template <int LANES>
__device__ __forceinline__ float sum_over(float x)
{
#pragma unroll
    for (int o = LANES / 2; o >= 1; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// The weights of a lane's pairs (ones where there are none).
template <int D, int P, bool HALF>
__device__ __forceinline__ void load_weight(const float* w, int sub, pairf (&w0)[P / 2], pairf (&w1)[P / 2])
{
#pragma unroll
    for (int p = 0; p < P / 2; ++p) {
        const int m = sub * P + 2 * p, step = HALF ? 1 : 2, at = HALF ? m : 2 * m, by = HALF ? D / 2 : 1;
        w0[p] = w ? mk(w[at], w[at + step]) : mk(1.0f, 1.0f);
        w1[p] = w ? mk(w[at + by], w[at + step + by]) : mk(1.0f, 1.0f);
    }
}

// 1 / sqrt(x), the hardware's approximation (relative error about 2^-22)
__device__ __forceinline__ float rsqrt_approx(float x)
{
    float y;
    asm("rsqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A warp's unit is a token and, with few tokens, one slice of its head groups, `per` of them (a group:
// the 32 / LANES heads of one access; the q groups come first).  The weights are folded into the
// angles once per token, so a head costs its sum of squares and one rotation.  (One short unit per
// warp and many warps.  64 x 577 tokens, 16 and 4 heads, bf16, in a graph: 42.6 us, bound by the latency of its
// loads (40 % of the stalls; 62 % of the issue slots in use, memory at two thirds of its rate).  Warps that stay for
// several tokens, four or eight CTAs an SM: 59.5 and 49.5.  One, two, four or five accesses of a warp in flight in
// the place of three: 50.1, 41.7, 44.7, 46.4.)
template <typename T, int D, bool HALF>
__global__ void __launch_bounds__(32 * kRopeWarps) rope_forward_kernel(const RopeArgs a, int per, int slices)
{
    typedef Lane<T, HALF> L;
    constexpr int P = L::P, LANES = D / 2 / P, HEADS = 32 / LANES, AHEAD = kForwardAhead;
    const int lane = threadIdx.x & 31, sub = lane % LANES, mine = lane / LANES;
    const unsigned u = blockIdx.x * kRopeWarps + (threadIdx.x >> 5), token = slices == 1 ? u : u / slices;
    pdl_wait();
    if (token >= (unsigned)(a.B * a.T)) return;
    const int b = (int)(token / (unsigned)a.T), t = (int)(token - (unsigned)b * a.T);
    Place at;
    at.set(a, (a.pos ? (long long)a.pos[b] : a.t0) + t);
    pairf c[P / 2], s[P / 2];
    angles<D, P>(a, at, sub, c, s);
    const int gq = (a.Hq + HEADS - 1) / HEADS, gk = (a.Hk + HEADS - 1) / HEADS;
    const int g0 = (u - token * slices) * per, g1 = min(g0 + per, gq + gk);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const int from = w ? max(g0, gq) - gq : min(g0, gq), to = w ? max(g1, gq) - gq : min(g1, gq);
        if (from >= to) continue;
        const long long si = a.s[w][0][2], so = a.s[w][1][2];
        const T* in = static_cast<const T*>(a.in[w]) + b * a.s[w][0][0] + t * a.s[w][0][1] + (from * HEADS + mine) * si;
        T* out = static_cast<T*>(const_cast<void*>(a.out[w])) + b * a.s[w][1][0] + t * a.s[w][1][1] + (from * HEADS + mine) * so;
        pairf w0[P / 2], w1[P / 2], c0[P / 2], c1[P / 2], s0[P / 2], s1[P / 2];
        load_weight<D, P, HALF>(a.weight[w], sub, w0, w1);
#pragma unroll
        for (int p = 0; p < P / 2; ++p) {
            c0[p] = mul(c[p], w0[p]), s0[p] = mul(s[p], w0[p]);
            c1[p] = mul(c[p], w1[p]), s1[p] = mul(mul(s[p], w1[p]), mk(-1.0f, -1.0f));
        }
        int left = (w ? a.Hk : a.Hq) - from * HEADS - mine;   // the lane's heads still to come are 0, HEADS, 2 HEADS .. < left
        for (int g = from; g < to; g += AHEAD) {
            L r[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (g + k < to && k * HEADS < left) r[k].template load<D>(in + k * HEADS * si, sub);
                else r[k].none();
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (g + k >= to) break;
                pairf x0[P / 2], x1[P / 2], y0[P / 2], y1[P / 2];
                r[k].get(x0, x1);
                pairf ss = fma(x1[0], x1[0], mul(x0[0], x0[0]));
#pragma unroll
                for (int p = 1; p < P / 2; ++p) ss = fma(x1[p], x1[p], fma(x0[p], x0[p], ss));
                const float f = rsqrt_approx(fmaf(sum_over<LANES>(lo(ss) + hi(ss)), 1.0f / D, a.eps));
                const pairf ff = mk(f, f);
#pragma unroll
                for (int p = 0; p < P / 2; ++p) {
                    y0[p] = mul(fma(x1[p], s1[p], mul(x0[p], c0[p])), ff);
                    y1[p] = mul(fma(x0[p], s0[p], mul(x1[p], c1[p])), ff);
                }
                if (k * HEADS < left) L::template store<D>(out + k * HEADS * so, sub, y0, y1);
            }
            in += AHEAD * HEADS * si;
            out += AHEAD * HEADS * so;
            left -= AHEAD * HEADS;
        }
    }
}

// The gradient: a warp goes over a run of consecutive tokens (and, with few tokens, over one slice of
// their head groups) with its lanes' sums of dw in registers; the CTA's sums go to ws[cta][q, k][D].
template <typename T, int D, bool HALF>
__global__ void __launch_bounds__(32 * kRopeWarps, kBackwardCtas) rope_backward_kernel(const RopeArgs a, int per, int slices, int run)
{
    typedef Lane<T, HALF> L;
    constexpr int P = L::P, LANES = D / 2 / P, HEADS = 32 / LANES, AHEAD = kBackwardAhead;
    __shared__ float part[kRopeWarps][2][D];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % LANES, mine = lane / LANES;
    const int gq = (a.Hq + HEADS - 1) / HEADS, gk = (a.Hk + HEADS - 1) / HEADS;
    pdl_wait();
    pairf w0[2][P / 2], w1[2][P / 2], d0[2][P / 2], d1[2][P / 2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        load_weight<D, P, HALF>(a.weight[w], sub, w0[w], w1[w]);
#pragma unroll
        for (int p = 0; p < P / 2; ++p) d0[w][p] = d1[w][p] = mk(0.0f, 0.0f);
    }
    const unsigned u = blockIdx.x * kRopeWarps + warp, tokens = (unsigned)(a.B * a.T);
    unsigned token = u / slices;
    const int g0 = (u - token * slices) * per, g1 = min(g0 + per, gq + gk);
    token *= run;
    const unsigned end = min(token + run, tokens);
    int b = (int)(token / (unsigned)a.T), t = (int)(token - (unsigned)b * a.T);
    Place at;
    bool first = true;
    for (; token < end; ++token) {
        if (first || t == a.T) {
            if (t == a.T) t = 0, ++b;
            first = false;
            at.set(a, (a.pos ? (long long)a.pos[b] : a.t0) + t);
        }
        pairf c[P / 2], s[P / 2];
        angles<D, P>(a, at, sub, c, s);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int from = w ? max(g0, gq) - gq : min(g0, gq), to = w ? max(g1, gq) - gq : min(g1, gq);
            if (from >= to) continue;
            const long long si = a.s[w][0][2] * HEADS, sd = a.s[w][2][2] * HEADS, so = a.s[w][3][2] * HEADS;
            const int h0 = from * HEADS + mine;
            const T* in = static_cast<const T*>(a.in[w]) + b * a.s[w][0][0] + t * a.s[w][0][1] + h0 * a.s[w][0][2];
            const T* dy = static_cast<const T*>(a.dout[w]) + b * a.s[w][2][0] + t * a.s[w][2][1] + h0 * a.s[w][2][2];
            T* dx = static_cast<T*>(a.din[w]) + b * a.s[w][3][0] + t * a.s[w][3][1] + h0 * a.s[w][3][2];
            int left = (w ? a.Hk : a.Hq) - h0;
            for (int g = from; g < to; g += AHEAD) {
                L rx[AHEAD], rd[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k, in += si, dy += sd) {
                    if (g + k < to && k * HEADS < left) {
                        rx[k].template load<D>(in, sub);
                        rd[k].template load<D>(dy, sub);
                    } else {
                        rx[k].none();
                        rd[k].none();
                    }
                }
#pragma unroll
                for (int k = 0; k < AHEAD; ++k, dx += so) {
                    if (g + k >= to) break;
                    pairf x0[P / 2], x1[P / 2], y0[P / 2], y1[P / 2], u0[P / 2], u1[P / 2];
                    rx[k].get(x0, x1);
                    rd[k].get(y0, y1);
                    pairf ss = mk(0.0f, 0.0f), dot = ss;
                    const pairf minus = mk(-1.0f, -1.0f);
#pragma unroll
                    for (int p = 0; p < P / 2; ++p) {
                        u0[p] = fma(y1[p], s[p], mul(y0[p], c[p]));                 // R^T dy
                        u1[p] = fma(mul(y0[p], s[p]), minus, mul(y1[p], c[p]));
                        y0[p] = mul(u0[p], w0[w][p]);                              // w * u
                        y1[p] = mul(u1[p], w1[w][p]);
                        ss = fma(x1[p], x1[p], fma(x0[p], x0[p], ss));
                        dot = fma(y1[p], x1[p], fma(y0[p], x0[p], dot));
                    }
                    const float n = rsqrt_approx(fmaf(sum_over<LANES>(lo(ss) + hi(ss)), 1.0f / D, a.eps));
                    const float m = sum_over<LANES>(lo(dot) + hi(dot)) * (-1.0f / D) * n * n;
                    // a head past the last one has x = dy = 0 and adds nothing (with eps = 0 its n is not finite)
                    if (k * HEADS < left) {
                        const pairf nn = mk(n, n), mm = mk(m, m);
#pragma unroll
                        for (int p = 0; p < P / 2; ++p) {
                            d0[w][p] = fma(mul(x0[p], nn), u0[p], d0[w][p]);
                            d1[w][p] = fma(mul(x1[p], nn), u1[p], d1[w][p]);
                            y0[p] = mul(fma(x0[p], mm, y0[p]), nn);
                            y1[p] = mul(fma(x1[p], mm, y1[p]), nn);
                        }
                        L::template store<D>(dx, sub, y0, y1);
                    }
                }
                left -= AHEAD * HEADS;
            }
        }
        ++t;
        at.next(a);
    }
    if (!a.ws) return;
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int e = 0; e < 2 * P; ++e) {
            const pairf d = e < P ? d0[w][e / 2] : d1[w][(e - P) / 2];
            float v = e & 1 ? hi(d) : lo(d);
#pragma unroll
            for (int o = 16; o >= LANES; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            const int m = sub * P + (e < P ? e : e - P), which = e < P ? 0 : 1;
            if (mine == 0) part[warp][w][HALF ? m + which * (D / 2) : 2 * m + which] = v;
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
// How the work is cut.  Fewer tokens than warps that run at a time: slices of the head groups.  The
// gradient's warps go over runs of tokens, one run for each warp that runs at a time.
struct Cut { int per, slices, run, ctas; };
Cut cut(const RopeArgs& a, bool backward, int sms)
{
    const int groups = head_groups(a);
    const long long warps = (long long)sms * kRopeWarps * (backward ? kBackwardCtas : 4), tokens = (long long)a.B * a.T;
    long long slices = tokens >= warps ? 1 : (warps + tokens - 1) / tokens;
    if (slices > groups) slices = groups;
    const int per = (int)((groups + slices - 1) / slices), n = (groups + per - 1) / per;
    const long long run = !backward || tokens * n <= warps ? 1 : (tokens * n + warps - 1) / warps, runs = (tokens + run - 1) / run;
    return {per, n, (int)run, (int)((runs * n + kRopeWarps - 1) / kRopeWarps)};
}

template <typename T, int D, bool HALF>
cudaError_t forward_t(const RopeArgs& a, int sms, cudaStream_t st)
{
    const Cut c = cut(a, false, sms);
    return launch_dependent(rope_forward_kernel<T, D, HALF>, dim3(c.ctas), dim3(32 * kRopeWarps), 0, st, a, c.per, c.slices);
}
template <typename T, int D, bool HALF>
cudaError_t backward_t(const RopeArgs& a, int sms, cudaStream_t st)
{
    const Cut c = cut(a, true, sms);
    const cudaError_t e =
        launch_dependent(rope_backward_kernel<T, D, HALF>, dim3(c.ctas), dim3(32 * kRopeWarps), 0, st, a, c.per, c.slices, c.run);
    if (e != cudaSuccess || !a.ws) return e;
    return launch_dependent(rope_dw_kernel, dim3(2 * D / 8), dim3(256), 0, st, a.ws, c.ctas, D, a.dw[0], a.dw[1]);
}

#define LASAD_ROPE_DISPATCH(fn)                                                                                      \
    (a.bf16 ? a.d == 64 ? (a.half ? fn<__nv_bfloat16, 64, true>(a, sms, st) : fn<__nv_bfloat16, 64, false>(a, sms, st)) \
                        : (a.half ? fn<__nv_bfloat16, 32, true>(a, sms, st) : fn<__nv_bfloat16, 32, false>(a, sms, st)) \
            : a.d == 64 ? (a.half ? fn<float, 64, true>(a, sms, st) : fn<float, 64, false>(a, sms, st))                 \
                        : (a.half ? fn<float, 32, true>(a, sms, st) : fn<float, 32, false>(a, sms, st)))

}  // namespace

size_t rope_workspace_bytes(const RopeArgs& a, int sms) { return (size_t)cut(a, true, sms).ctas * 2 * a.d * sizeof(float); }
int rope_backward_launches(const RopeArgs& a) { return a.ws ? 2 : 1; }
cudaError_t launch_rope_forward(const RopeArgs& a, int sms, cudaStream_t st) { return LASAD_ROPE_DISPATCH(forward_t); }
cudaError_t launch_rope_backward(const RopeArgs& a, int sms, cudaStream_t st) { return LASAD_ROPE_DISPATCH(backward_t); }

}  // namespace lasad
