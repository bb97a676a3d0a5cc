// Gated linear recurrence with the spatial rule: for every channel
//
//     h_t = a_t h_{t-1} + b_t ,   a_t = 1 on the last token of a grid row, lambda_t elsewhere,
//     b_t = (1 - lambda_t) x_t (tied) or x_t ,   y_t = h_t ,
//
// which is the SAD recurrence (Section 3.4) with one state per channel, and its gradient
//
//     g_t = dy_t + a_{t+1} g_{t+1} ,  dx_t = gain_t g_t ,  dlambda_t = [a_t = lambda_t] g_t h_{t-1} - [tied] g_t x_t .
//
// A span of tokens maps h to A h + H with A the product of its a_t; spans compose, so a chunk of
// 128 tokens is cut over 16 slots of 8 tokens: every thread forms (A, H) of 8 tokens of two
// neighbouring channels in registers, the slots' pairs meet in shared memory once per chunk, and
// each thread runs its 8 tokens again from the state that the slots before it leave.  The gradient
// needs h_{t-1}: the forward keeps h before each chunk in 32 bits (4 bytes per 128 tokens) and the
// backward forms the rest again from x and lambda, which it reads anyway.  Both passes are bound
// by device memory: x, lambda and y, and x, lambda, dy, dx and dlambda, each move once.
//
// A CTA walks one tile of channels of one sequence.  Where that gives too few CTAs the sequence is
// cut into segments: a first launch forms each segment's (A, H) (of the backward: the same pair of
// the reversed recurrence), and the second, a programmatic dependent, starts each segment from the
// composition of those before it.  No CTA ever waits for another one.
#include "lasad_mixers.cuh"
#include "lasad_tc_ptx.cuh"

namespace lasad {
namespace {

constexpr int kSlots = 16, kTok = kScanChunk / kSlots;

// lambda = sigmoid(z) and 1 - lambda, each to full relative precision: the smaller of the two is
// e^-|z| / (1 + e^-|z|), never a difference.  (No clamp: infinities and NaN come out as they should.)
__device__ __forceinline__ void gate_of(float z, bool logits, float& lam, float& rest)
{
    if (logits) {
        const float t = tcx::ex2_approx(fabsf(z) * -1.4426950408889634f);
        const float big = __fdividef(1.0f, 1.0f + t), small = t * big;
        lam = z < 0.0f ? small : big;
        rest = z < 0.0f ? big : small;
    } else {
        lam = z;
        rest = 1.0f - z;
    }
}

// VEC neighbouring channels in one access (VEC = 2 needs pairs that are aligned to a pair)
template <typename T, int VEC> struct pack;
template <> struct pack<__nv_bfloat16, 2> {
    typedef uint32_t raw;
    static __device__ __forceinline__ void get(raw r, float (&v)[2]) { v[0] = tcx::bf16_lo(r); v[1] = tcx::bf16_hi(r); }
    static __device__ __forceinline__ raw put(const float (&v)[2]) { return tcx::pack_bf16(v[0], v[1]); }
};
template <> struct pack<__nv_bfloat16, 1> {
    typedef unsigned short raw;
    static __device__ __forceinline__ void get(raw r, float (&v)[1]) { v[0] = __uint_as_float((uint32_t)r << 16); }
    static __device__ __forceinline__ raw put(const float (&v)[1]) { return __bfloat16_as_ushort(__float2bfloat16_rn(v[0])); }
};
template <> struct pack<float, 2> {
    typedef float2 raw;
    static __device__ __forceinline__ void get(raw r, float (&v)[2]) { v[0] = r.x; v[1] = r.y; }
    static __device__ __forceinline__ raw put(const float (&v)[2]) { return make_float2(v[0], v[1]); }
};
template <> struct pack<float, 1> {
    typedef float raw;
    static __device__ __forceinline__ void get(raw r, float (&v)[1]) { v[0] = r; }
    static __device__ __forceinline__ raw put(const float (&v)[1]) { return v[0]; }
};

// LC lanes of VEC channels make a tile; a CTA has LC * kSlots threads.
template <typename T, int VEC, int LC, bool LOGITS, bool SUMMARY>
__global__ void __launch_bounds__(LC * kSlots) scan_forward_kernel(const ScanArgs a)
{
    typedef pack<T, VEC> P;
    typedef typename P::raw raw;
    __shared__ float2 pair[2][kSlots][LC * VEC];   // (A, H) of every slot, two chunks in turn
    __shared__ float next[2][LC * VEC];            // h after the chunk
    const int lane = threadIdx.x % LC, slot = threadIdx.x / LC;
    const int tiles = (a.C + LC * VEC - 1) / (LC * VEC);
    const int b = blockIdx.x / tiles, c0 = (blockIdx.x - b * tiles) * LC * VEC + lane * VEC;
    const int seg = blockIdx.y, chunks = (a.T + kScanChunk - 1) / kScanChunk;
    const int first = seg * a.seg_chunks, end = min(first + a.seg_chunks, chunks);
    const bool in = c0 < a.C;                      // (VEC = 2 only where C is even)
    const T* x = static_cast<const T*>(a.x) + b * a.xs[0] + c0;
    const T* z = static_cast<const T*>(a.gate) + b * a.gs[0] + c0;
    T* y = static_cast<T*>(a.y) + b * a.ys[0] + c0;
    pdl_wait();

    raw rx[kTok], rz[kTok];
    auto load = [&](int chunk) {
        const int t0 = chunk * kScanChunk + slot * kTok;
#pragma unroll
        for (int t = 0; t < kTok; ++t)
            if (in && chunk < end && t0 + t < a.T) {
                rx[t] = *reinterpret_cast<const raw*>(x + (long long)(t0 + t) * a.xs[1]);
                rz[t] = *reinterpret_cast<const raw*>(z + (long long)(t0 + t) * a.gs[1]);
            }
    };
    load(first);
    // the state at the segment's first token: h_in through the segments before it
    float h0[VEC], total[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
        h0[v] = !SUMMARY && a.h_in && in ? a.h_in[(long long)b * a.C + c0 + v] : 0.0f;
        total[v] = 1.0f;
    }
    if (!SUMMARY && in) {
        const float* w = a.ws + (long long)b * a.segs * 2 * a.C + c0;
#pragma unroll 4
        for (int s = 0; s < seg; ++s, w += 2 * a.C)
#pragma unroll
            for (int v = 0; v < VEC; ++v) h0[v] = fmaf(w[v], h0[v], w[a.C + v]);
    }
    for (int chunk = first; chunk < end; ++chunk) {
        const int buf = chunk & 1, t0 = chunk * kScanChunk + slot * kTok;
        float ca[kTok][VEC], cb[kTok][VEC], A[VEC], H[VEC];
        RowWalk row(a.t0 + t0, a.grid_w, a.prefix_len);
#pragma unroll
        for (int v = 0; v < VEC; ++v) A[v] = 1.0f, H[v] = 0.0f;
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            const bool ends = row.step(), live = in && t0 + t < a.T;
            float xv[VEC], zv[VEC];
            P::get(rx[t], xv);
            P::get(rz[t], zv);
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                float lam, rest;
                gate_of(zv[v], LOGITS, lam, rest);
                ca[t][v] = ends || !live ? 1.0f : lam;
                cb[t][v] = !live ? 0.0f : a.tied ? rest * xv[v] : xv[v];
                A[v] *= ca[t][v];
                H[v] = fmaf(ca[t][v], H[v], cb[t][v]);
            }
        }
        load(chunk + 1);
#pragma unroll
        for (int v = 0; v < VEC; ++v) pair[buf][slot][lane * VEC + v] = make_float2(A[v], H[v]);
        __syncthreads();
        // h before this slot (the chunk's own start came through `next` at the same barrier)
        float h[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) h[v] = chunk == first ? h0[v] : next[buf][lane * VEC + v];
        if (!SUMMARY && slot == 0 && a.saved && in)
#pragma unroll
            for (int v = 0; v < VEC; ++v) a.saved[((long long)b * chunks + chunk) * a.C + c0 + v] = h[v];
        for (int s = 0; s < slot; ++s)
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                const float2 m = pair[buf][s][lane * VEC + v];
                h[v] = fmaf(m.x, h[v], m.y);
                if (SUMMARY && slot == kSlots - 1) total[v] *= m.x;
            }
        if (slot == kSlots - 1)
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                const float after = fmaf(A[v], h[v], H[v]);
                if (SUMMARY) total[v] *= A[v];
                next[buf ^ 1][lane * VEC + v] = after;
                if (chunk == end - 1 && in) {
                    if (SUMMARY) {
                        float* w = a.ws + ((long long)b * a.segs + seg) * 2 * a.C + c0 + v;
                        w[0] = total[v];
                        w[a.C] = after;
                    } else if (end == chunks && a.h_out) {
                        a.h_out[(long long)b * a.C + c0 + v] = after;
                    }
                }
            }
        if (!SUMMARY && in)
#pragma unroll
            for (int t = 0; t < kTok; ++t) {
                if (t0 + t < a.T) {
#pragma unroll
                    for (int v = 0; v < VEC; ++v) h[v] = fmaf(ca[t][v], h[v], cb[t][v]);
                    *reinterpret_cast<raw*>(y + (long long)(t0 + t) * a.ys[1]) = P::put(h);
                }
            }
    }
}

// The same walk from the end.  With u_t = a_t g_t the reversed recurrence u_t = a_t (u_{t+1} + dy_t)
// has the forward's products A, so a slot's spans in both directions are (A, H) and (A, Q).
// SUMMARY: only (A, Q) of a whole segment, from lambda and dy.
template <typename T, int VEC, int LC, bool LOGITS, bool SUMMARY>
__global__ void __launch_bounds__(LC * kSlots) scan_backward_kernel(const ScanArgs a)
{
    typedef pack<T, VEC> P;
    typedef typename P::raw raw;
    __shared__ float2 pair[2][kSlots][LC * VEC];   // (A, Q) of every slot
    __shared__ float fwd[2][kSlots][LC * VEC];     // H of every slot
    __shared__ float next[2][LC * VEC];            // u before the chunk
    const int lane = threadIdx.x % LC, slot = threadIdx.x / LC;
    const int tiles = (a.C + LC * VEC - 1) / (LC * VEC);
    const int b = blockIdx.x / tiles, c0 = (blockIdx.x - b * tiles) * LC * VEC + lane * VEC;
    const int chunks = (a.T + kScanChunk - 1) / kScanChunk;
    const int seg = SUMMARY ? blockIdx.y + 1 : blockIdx.y;      // (nothing comes before segment 0: it needs no summary)
    const int first = seg * a.seg_chunks, end = min(first + a.seg_chunks, chunks);
    const bool in = c0 < a.C;
    const T* x = static_cast<const T*>(a.x) + b * a.xs[0] + c0;
    const T* z = static_cast<const T*>(a.gate) + b * a.gs[0] + c0;
    const T* dy = static_cast<const T*>(a.dy) + b * a.ys[0] + c0;
    T* dx = static_cast<T*>(a.dx) + b * a.dxs[0] + c0;
    T* dg = static_cast<T*>(a.dgate) + b * a.dgs[0] + c0;
    pdl_wait();

    raw rx[kTok], rz[kTok], rd[kTok];
    float hs[VEC];                                 // h before the chunk
    auto load = [&](int chunk) {
        const int t0 = chunk * kScanChunk + slot * kTok;
#pragma unroll
        for (int t = 0; t < kTok; ++t)
            if (in && chunk >= first && t0 + t < a.T) {
                if (!SUMMARY) rx[t] = *reinterpret_cast<const raw*>(x + (long long)(t0 + t) * a.xs[1]);
                rz[t] = *reinterpret_cast<const raw*>(z + (long long)(t0 + t) * a.gs[1]);
                rd[t] = *reinterpret_cast<const raw*>(dy + (long long)(t0 + t) * a.ys[1]);
            }
        if (!SUMMARY && in && chunk >= first)
#pragma unroll
            for (int v = 0; v < VEC; ++v) hs[v] = a.saved[((long long)b * chunks + chunk) * a.C + c0 + v];
    };
    load(end - 1);
    float u0[VEC], total[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
        u0[v] = !SUMMARY && a.dh_out && in ? a.dh_out[(long long)b * a.C + c0 + v] : 0.0f;
        total[v] = 1.0f;
    }
    if (!SUMMARY && in) {
#pragma unroll 4
        for (int s = a.segs - 1; s > seg; --s) {
            const float* w = a.ws + ((long long)b * a.segs + s) * 2 * a.C + c0;
#pragma unroll
            for (int v = 0; v < VEC; ++v) u0[v] = fmaf(w[v], u0[v], w[a.C + v]);
        }
    }
    for (int chunk = end - 1; chunk >= first; --chunk) {
        const int buf = chunk & 1, t0 = chunk * kScanChunk + slot * kTok;
        float la[kTok][VEC], A[VEC], H[VEC], Q[VEC], h[VEC];
        float xv[SUMMARY ? 1 : kTok][VEC], rest[SUMMARY ? 1 : kTok][VEC], dv[kTok][VEC];
        unsigned ends = 0;
        RowWalk row(a.t0 + t0, a.grid_w, a.prefix_len);
#pragma unroll
        for (int v = 0; v < VEC; ++v) A[v] = 1.0f, H[v] = 0.0f, Q[v] = 0.0f, h[v] = hs[v];
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            const bool e = row.step(), live = in && t0 + t < a.T;
            if (e) ends |= 1u << t;
            float zv[VEC];
            P::get(rz[t], zv);
            P::get(rd[t], dv[t]);
            if (!SUMMARY) P::get(rx[t], xv[t]);
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                float lam, r;
                gate_of(zv[v], LOGITS, lam, r);
                la[t][v] = live ? lam : 1.0f;
                if (!live) dv[t][v] = 0.0f;
                const float ca = e ? 1.0f : la[t][v];
                A[v] *= ca;
                if (!SUMMARY) {
                    rest[t][v] = r;
                    if (!live) xv[t][v] = 0.0f, rest[t][v] = 0.0f;
                    H[v] = fmaf(ca, H[v], a.tied ? rest[t][v] * xv[t][v] : xv[t][v]);
                }
            }
        }
#pragma unroll
        for (int t = kTok - 1; t >= 0; --t)
#pragma unroll
            for (int v = 0; v < VEC; ++v) Q[v] = ((ends >> t) & 1u ? 1.0f : la[t][v]) * (Q[v] + dv[t][v]);
        load(chunk - 1);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            pair[buf][slot][lane * VEC + v] = make_float2(A[v], Q[v]);
            if (!SUMMARY) fwd[buf][slot][lane * VEC + v] = H[v];
        }
        __syncthreads();
        float u[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) u[v] = chunk == end - 1 ? u0[v] : next[buf][lane * VEC + v];
        for (int s = kSlots - 1; s > slot; --s)
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                const float2 m = pair[buf][s][lane * VEC + v];
                u[v] = fmaf(m.x, u[v], m.y);
                if (SUMMARY && slot == 0) total[v] *= m.x;
            }
        if (!SUMMARY)
            for (int s = 0; s < slot; ++s)
#pragma unroll
                for (int v = 0; v < VEC; ++v)
                    h[v] = fmaf(pair[buf][s][lane * VEC + v].x, h[v], fwd[buf][s][lane * VEC + v]);
        if (slot == 0)
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                const float before = fmaf(A[v], u[v], Q[v]);
                if (SUMMARY) total[v] *= A[v];
                next[buf ^ 1][lane * VEC + v] = before;
                if (chunk == first && in) {
                    if (SUMMARY) {
                        float* w = a.ws + ((long long)b * a.segs + seg) * 2 * a.C + c0 + v;
                        w[0] = total[v];
                        w[a.C] = before;
                    } else if (first == 0 && a.dh_in) {
                        a.dh_in[(long long)b * a.C + c0 + v] = before;
                    }
                }
            }
        if (!SUMMARY && in) {
            float prev[kTok][VEC];
#pragma unroll
            for (int t = 0; t < kTok; ++t)
#pragma unroll
                for (int v = 0; v < VEC; ++v) {
                    prev[t][v] = h[v];
                    h[v] = fmaf((ends >> t) & 1u ? 1.0f : la[t][v], h[v], a.tied ? rest[t][v] * xv[t][v] : xv[t][v]);
                }
#pragma unroll
            for (int t = kTok - 1; t >= 0; --t) {
                float ox[VEC], og[VEC];
#pragma unroll
                for (int v = 0; v < VEC; ++v) {
                    const float g = u[v] + dv[t][v];
                    const bool e = (ends >> t) & 1u;
                    u[v] = (e ? 1.0f : la[t][v]) * g;
                    ox[v] = a.tied ? rest[t][v] * g : g;
                    float d = (e ? 0.0f : prev[t][v]) - (a.tied ? xv[t][v] : 0.0f);
                    if (LOGITS) d *= rest[t][v] * la[t][v];      // the derivative of the sigmoid
                    og[v] = d * g;
                }
                if (t0 + t < a.T) {
                    *reinterpret_cast<raw*>(dx + (long long)(t0 + t) * a.dxs[1]) = P::put(ox);
                    *reinterpret_cast<raw*>(dg + (long long)(t0 + t) * a.dgs[1]) = P::put(og);
                }
            }
        }
    }
}

// One token: h <- a h + b, y = h.  Bound by the state, 8 bytes per channel.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) scan_step_kernel(const ScanArgs a)
{
    typedef pack<T, VEC> P;
    typedef typename P::raw raw;
    pdl_wait();
    const unsigned per = (unsigned)(a.C / VEC);
    const long long n = (long long)blockIdx.x * 256 + threadIdx.x;
    if (n >= (long long)a.B * per) return;
    const int b = (int)(n / per), c = (int)(n - (long long)b * per) * VEC;
    const long long i = a.pos ? (long long)a.pos[b] : a.t0;
    RowWalk row(i, a.grid_w, a.prefix_len);
    const bool ends = row.step();
    float x[VEC], z[VEC], h[VEC];
    P::get(*reinterpret_cast<const raw*>(static_cast<const T*>(a.x) + b * a.xs[0] + c), x);
    P::get(*reinterpret_cast<const raw*>(static_cast<const T*>(a.gate) + b * a.gs[0] + c), z);
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
        float lam, rest;
        gate_of(z[v], a.logits, lam, rest);
        h[v] = fmaf(ends ? 1.0f : lam, a.h_in[(long long)b * a.C + c + v], a.tied ? rest * x[v] : x[v]);
        a.h_out[(long long)b * a.C + c + v] = h[v];
    }
    *reinterpret_cast<raw*>(static_cast<T*>(a.y) + b * a.ys[0] + c) = P::put(h);
}

// Whether every access to pairs of channels is aligned to a pair.
bool pairs_ok(const ScanArgs& a)
{
    const uintptr_t size = a.bf16 ? 4 : 8;
    const void* ptrs[] = {a.x, a.gate, a.y, a.dy, a.dx, a.dgate};
    for (const void* p : ptrs)
        if (reinterpret_cast<uintptr_t>(p) % size) return false;
    const long long* strides[] = {a.xs, a.gs, a.ys, a.dxs, a.dgs};
    for (const long long* s : strides)
        if ((s[0] & 1) || (s[1] & 1)) return false;
    return (a.C & 1) == 0;
}

template <typename T, int VEC, int LC>
cudaError_t forward_t(const ScanArgs& a, cudaStream_t st)
{
    const unsigned tiles = (unsigned)((a.C + LC * VEC - 1) / (LC * VEC)) * a.B;
    cudaError_t e = cudaSuccess;
    if (a.segs > 1)
        e = launch_dependent(a.logits ? scan_forward_kernel<T, VEC, LC, true, true> : scan_forward_kernel<T, VEC, LC, false, true>,
                             dim3(tiles, a.segs - 1), dim3(LC * kSlots), 0, st, a);
    if (e != cudaSuccess) return e;
    return launch_dependent(a.logits ? scan_forward_kernel<T, VEC, LC, true, false> : scan_forward_kernel<T, VEC, LC, false, false>,
                            dim3(tiles, a.segs), dim3(LC * kSlots), 0, st, a);
}
template <typename T, int VEC, int LC>
cudaError_t backward_t(const ScanArgs& a, cudaStream_t st)
{
    const unsigned tiles = (unsigned)((a.C + LC * VEC - 1) / (LC * VEC)) * a.B;
    cudaError_t e = cudaSuccess;
    if (a.segs > 1)
        e = launch_dependent(a.logits ? scan_backward_kernel<T, VEC, LC, true, true> : scan_backward_kernel<T, VEC, LC, false, true>,
                             dim3(tiles, a.segs - 1), dim3(LC * kSlots), 0, st, a);
    if (e != cudaSuccess) return e;
    return launch_dependent(a.logits ? scan_backward_kernel<T, VEC, LC, true, false> : scan_backward_kernel<T, VEC, LC, false, false>,
                            dim3(tiles, a.segs), dim3(LC * kSlots), 0, st, a);
}

}  // namespace

// How a call's work is cut.  Tiles are 16 lanes wide; a sequence is cut into segments until there
// are about four CTAs per SM.
void scan_plan(ScanArgs& a, int sms)
{
    const int width = 16 * 2;
    const long long tiles = (long long)a.B * ((a.C + width - 1) / width);
    const int chunks = (a.T + kScanChunk - 1) / kScanChunk;
    long long segs = tiles >= sms ? 1 : (4LL * sms + tiles - 1) / tiles;
    if (segs > chunks) segs = chunks;
    a.seg_chunks = (int)((chunks + segs - 1) / segs);
    a.segs = (chunks + a.seg_chunks - 1) / a.seg_chunks;
}
size_t scan_workspace_bytes(const ScanArgs& a) { return a.segs > 1 ? (size_t)a.B * a.segs * 2 * a.C * sizeof(float) : 0; }
int scan_launches(const ScanArgs& a) { return a.segs > 1 ? 2 : 1; }

cudaError_t launch_scan_forward(const ScanArgs& a, cudaStream_t st)
{
    if (pairs_ok(a)) return a.bf16 ? forward_t<__nv_bfloat16, 2, 16>(a, st) : forward_t<float, 2, 16>(a, st);
    return a.bf16 ? forward_t<__nv_bfloat16, 1, 32>(a, st) : forward_t<float, 1, 32>(a, st);
}
cudaError_t launch_scan_backward(const ScanArgs& a, cudaStream_t st)
{
    if (pairs_ok(a)) return a.bf16 ? backward_t<__nv_bfloat16, 2, 16>(a, st) : backward_t<float, 2, 16>(a, st);
    return a.bf16 ? backward_t<__nv_bfloat16, 1, 32>(a, st) : backward_t<float, 1, 32>(a, st);
}
cudaError_t launch_scan_step(const ScanArgs& a, cudaStream_t st)
{
    const bool pairs = pairs_ok(a);
    const long long n = (long long)a.B * (pairs ? a.C / 2 : a.C);
    const dim3 grid((unsigned)((n + 255) / 256));
    if (pairs)
        return launch_dependent(a.bf16 ? scan_step_kernel<__nv_bfloat16, 2> : scan_step_kernel<float, 2>, grid, dim3(256), 0, st, a);
    return launch_dependent(a.bf16 ? scan_step_kernel<__nv_bfloat16, 1> : scan_step_kernel<float, 1>, grid, dim3(256), 0, st, a);
}

}  // namespace lasad
