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
// backward forms the rest again from x and lambda, which it reads anyway.  What neither pass can do without
// is the memory: x, lambda and y, and x, lambda, dy, dx and dlambda, each moved once.  What bounds them now is
// the instructions around each element and the latency between them at 12 to 24 warps an SM: 8 x 9216 x 1536
// in bf16, forward 145 us and gradient 283 (1 x 9217 x 1536: 35 and 53), has device memory at half of its rate
// and 62 to 66 % of the issue slots in use; the exponentials and shared memory are below 40 % of theirs.
//
// A CTA walks one tile of channels of one sequence.  Where that gives too few CTAs the sequence is
// cut into segments: a first launch forms each segment's (A, H) (of the backward: the same pair of
// the reversed recurrence), and the second, a programmatic dependent, starts each segment from the
// composition of those before it.  No CTA ever waits for another one.
#include "lasad_mixers.cuh"
#include "lasad_tc_ptx.cuh"
#include "lasad_tc_tma.cuh"

namespace lasad {
namespace {

constexpr int kSlots = 16, kTok = kScanChunk / kSlots;

// VEC neighbouring channels as one number: pairs use the packed fp32 arithmetic of sm_100, which
// halves the instructions (the kernels are near the issue rate at full memory speed).
template <int VEC> struct num;
template <> struct num<1> {
    float v;
    static __device__ __forceinline__ num all(float x) { return {x}; }
    __device__ __forceinline__ float get(int) const { return v; }
    __device__ __forceinline__ void set(int, float x) { v = x; }
};
template <> struct num<2> {
    unsigned long long v;
    static __device__ __forceinline__ num of(float a, float b)
    {
        num r;
        asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
        return r;
    }
    static __device__ __forceinline__ num all(float x) { return of(x, x); }
    __device__ __forceinline__ float get(int i) const
    {
        float a, b;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
        return i ? b : a;
    }
    __device__ __forceinline__ void set(int i, float x) { *this = i ? of(get(0), x) : of(x, get(1)); }
};
__device__ __forceinline__ num<1> operator*(num<1> a, num<1> b) { return {a.v * b.v}; }
__device__ __forceinline__ num<1> operator+(num<1> a, num<1> b) { return {a.v + b.v}; }
__device__ __forceinline__ num<1> fma(num<1> a, num<1> b, num<1> c) { return {fmaf(a.v, b.v, c.v)}; }
__device__ __forceinline__ num<2> operator*(num<2> a, num<2> b)
{
    num<2> r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ num<2> operator+(num<2> a, num<2> b)
{
    num<2> r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ num<2> fma(num<2> a, num<2> b, num<2> c)
{
    num<2> r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// VEC channels in memory (VEC = 2 needs pairs that are aligned to a pair)
template <typename T, int VEC> struct pack;
template <> struct pack<__nv_bfloat16, 2> {
    typedef uint32_t raw;
    static __device__ __forceinline__ raw all(float x) { return tcx::pack_bf16(x, x); }
    static __device__ __forceinline__ num<2> get(raw r) { return num<2>::of(tcx::bf16_lo(r), tcx::bf16_hi(r)); }
    static __device__ __forceinline__ raw put(num<2> v) { return tcx::pack_bf16(v.get(0), v.get(1)); }
};
template <> struct pack<__nv_bfloat16, 1> {
    typedef unsigned short raw;
    static __device__ __forceinline__ raw all(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }
    static __device__ __forceinline__ num<1> get(raw r) { return {__uint_as_float((uint32_t)r << 16)}; }
    static __device__ __forceinline__ raw put(num<1> v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v.v)); }
};
template <> struct pack<float, 2> {
    typedef float2 raw;
    static __device__ __forceinline__ raw all(float x) { return make_float2(x, x); }
    static __device__ __forceinline__ num<2> get(raw r) { return num<2>::of(r.x, r.y); }
    static __device__ __forceinline__ raw put(num<2> v) { return make_float2(v.get(0), v.get(1)); }
};
template <> struct pack<float, 1> {
    typedef float raw;
    static __device__ __forceinline__ raw all(float x) { return x; }
    static __device__ __forceinline__ num<1> get(raw r) { return {r}; }
    static __device__ __forceinline__ raw put(num<1> v) { return v.v; }
};

// VEC floats of a state
template <int VEC>
__device__ __forceinline__ num<VEC> load_state(const float* p)
{
    num<VEC> r = num<VEC>::all(0.0f);
#pragma unroll
    for (int v = 0; v < VEC; ++v) r.set(v, p[v]);
    return r;
}
template <int VEC>
__device__ __forceinline__ void store_state(float* p, num<VEC> x)
{
#pragma unroll
    for (int v = 0; v < VEC; ++v) p[v] = x.get(v);
}

// lambda = sigmoid(z) = 1 / (1 + t) and 1 - lambda = t / (1 + t) with t = e^-z, neither as a difference: both
// have the relative error of t, about (|z| + 4) 2^-23 (the exponent's rounding and that of the hardware's power
// and reciprocal), however small they are.  The exponent ends at 126, where lambda is 2^-126 and the products
// stay finite; a NaN passes through.
template <bool LOGITS, int VEC>
__device__ __forceinline__ void gate_of(num<VEC> z, num<VEC>& lam, num<VEC>& rest)
{
    if (LOGITS) {
        const num<VEC> e = z * num<VEC>::all(-1.4426950408889634f);
        num<VEC> t = e;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            float x;
            asm("min.NaN.f32 %0, %1, 0f42fc0000;" : "=f"(x) : "f"(e.get(v)));
            t.set(v, tcx::ex2_approx(x));
        }
        const num<VEC> s = t + num<VEC>::all(1.0f);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            float x;
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(x) : "f"(s.get(v)));
            lam.set(v, x);
        }
        rest = t * lam;
    } else {
        lam = z;
        rest = fma(z, num<VEC>::all(-1.0f), num<VEC>::all(1.0f));
    }
}

// Which of a slot's kTok tokens end a grid row, for slots that are visited some tokens further on, or
// back, each time.
struct RowEnds {
    long long j;         // grid index of the slot's first token (negative before the grid)
    int w, by, col, step;    // col = j mod w where j >= 0; by: tokens to the next visit
    __device__ __forceinline__ RowEnds(long long i, int grid_w, int prefix_len, int tokens)
        : j(i - prefix_len), w(grid_w), by(tokens), col(0), step(0)
    {
        if (w > 0) {
            step = by % w;
            if (j >= 0) col = (int)(j % w);
        }
    }
    __device__ __forceinline__ unsigned mask() const
    {
        if (w <= 0) return 0u;
        unsigned m = 0;
        const long long first = j >= 0 ? w - 1 - col : w - 1 - j;
        for (int e = first < kTok ? (int)first : kTok; e < kTok; e += min(w, kTok)) m |= 1u << e;
        return m;
    }
    __device__ __forceinline__ void forward()
    {
        const bool on = j >= 0;
        j += by;
        if (w <= 0) return;
        if (on) {
            col = col < w - step ? col + step : col - (w - step);      // (a sum may pass 2^31)
        } else if (j >= 0) {
            col = (int)(j % w);
        }
    }
    __device__ __forceinline__ void back()
    {
        j -= by;
        if (w <= 0 || j < 0) return;
        col -= step;
        if (col < 0) col += w;
    }
};

// What a CTA has to do: chunks first .. end - 1 of the channels from c on, of batch element b.  The first
// a.whole tiles are whole sequences, the others are cut into a.segs segments (see scan_plan).
struct Work {
    int b, c, seg, segs, first, end, cut, cuts, width;
    // summary: the first segment that a summary is made of, or -1 (not a summary: every tile's work)
    __device__ __forceinline__ Work(const ScanArgs& a, int summary, int chunks, int w) : width(w)
    {
        const int per = (a.C + w - 1) / w;
        int at = blockIdx.x, tile;
        cuts = a.B * per - a.whole;
        if (summary < 0 && at < a.whole) {
            tile = at;
            seg = cut = 0;
            segs = 1;
        } else {
            if (summary < 0) at -= a.whole;
            seg = at / cuts;
            cut = at - seg * cuts;
            seg += max(summary, 0);
            tile = a.whole + cut;
            segs = a.segs;
        }
        b = tile / per;
        c = (tile - b * per) * w;
        first = segs == 1 ? 0 : seg * a.seg_chunks;
        end = segs == 1 ? chunks : min(first + a.seg_chunks, chunks);
    }
    // (A, H) or (A, Q) of segment s of this CTA's tile: 2 x width floats.  The last segment of a walk has nothing
    // behind it and no summary: its place (forward the last one, backward the first) has a copy of the state that the
    // walk starts from, from which every segment of the second launch starts.  So the state at the walk's end, which
    // one of them stores, may have the memory of the state at its start.
    __device__ __forceinline__ float* span(const ScanArgs& a, int s) const
    {
        return a.ws + ((long long)s * cuts + cut) * 2 * width;
    }
};

// How a tile of NA tensors comes into shared memory: rows of the tile's channels, kTok rows to a slot,
// and 64 bytes between slots, so that the two slots of a warp (16 lanes of pairs) use different
// banks.  A warp copies the rows of its own slots, so a chunk's arrival is a matter of the warp alone.
// WIDE: 16-byte asynchronous copies, one chunk ahead (pointers, strides and C in whole 16 bytes).
// Otherwise every lane fetches its own channels; right for any alignment, and slower.
template <typename T, int VEC, int LC, int NA, bool WIDE>
struct Stage {
    typedef typename pack<T, VEC>::raw raw;
    static constexpr int kRow = LC * VEC * (int)sizeof(T), kSlot = kTok * kRow + 64, kArray = kSlots * kSlot;
    static constexpr int kBytes = 2 * NA * kArray;                 // two chunks
    static constexpr int kPieces = kRow / 16, kRows = 32 / LC * kTok, kCopies = kRows * kPieces / 32;
    unsigned char* mem;
    const T* src[NA];        // WIDE: the lane's first piece of the warp's first row; else the lane's channels there
    long long stride[NA];
    int row, piece;          // WIDE: of the lane's first copy
    int gap;                 // tokens from a slot to the next
    bool in;
    __device__ __forceinline__ Stage(unsigned char* m, int lane32, int warp, int g) : mem(m), gap(g)
    {
        static_assert(kTok % (32 / kPieces) == 0 || !WIDE, "");
        row = lane32 / kPieces;
        piece = lane32 % kPieces;
        mem += warp * (32 / LC) * kSlot;
    }
    // base: the CTA's first channel at the warp's first token of the first chunk
    __device__ __forceinline__ void tensor(int n, const void* base, long long str, int c_tile, int C)
    {
        const int lane = threadIdx.x % LC, sub = (threadIdx.x & 31) / LC;
        stride[n] = str;
        if (WIDE) {
            const int c = piece * (16 / (int)sizeof(T));
            src[n] = static_cast<const T*>(base) + row * str + c;
            in = c_tile + c < C;
        } else {
            src[n] = static_cast<const T*>(base) + (long long)sub * gap * str + lane * VEC;
            in = c_tile + lane * VEC < C;
        }
    }
    // rows: tokens from the warp's first one to the end of the sequence
    __device__ __forceinline__ void fetch(int buf, int rows)
    {
#pragma unroll
        for (int n = 0; n < NA; ++n) {
            unsigned char* to = mem + (buf * NA + n) * kArray;
            if (WIDE) {
#pragma unroll
                for (int k = 0; k < kCopies; ++k) {
                    const int slot = k * (32 / kPieces) / kTok, t = k * (32 / kPieces) % kTok, at = slot * gap + t;
                    const bool live = in && row + at < rows;
                    const uint32_t dst = tcx::smem_u32(to + slot * kSlot + (row + t) * kRow + piece * 16);
                    const T* from = live ? src[n] + at * stride[n] : src[n];
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(from), "r"(live ? 16 : 0) : "memory");
                }
            } else {
                const int lane = threadIdx.x % LC, sub = (threadIdx.x & 31) / LC;
#pragma unroll
                for (int t = 0; t < kTok; ++t)
                    if (in && sub * gap + t < rows)
                        reinterpret_cast<raw*>(to + sub * kSlot + t * kRow)[lane] = *reinterpret_cast<const raw*>(src[n] + t * stride[n]);
            }
        }
        if (WIDE) asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ void move(int tokens)
    {
#pragma unroll
        for (int n = 0; n < NA; ++n) src[n] += tokens * stride[n];
    }
    __device__ __forceinline__ void landed(bool last)
    {
        if (WIDE) {
            if (last) asm volatile("cp.async.wait_group 0;" ::: "memory");
            else asm volatile("cp.async.wait_group 1;" ::: "memory");
        }
        __syncwarp();
    }
    // the thread's channels of token t of its slot
    __device__ __forceinline__ raw get(int buf, int n, int t) const
    {
        const int lane = threadIdx.x % LC, sub = (threadIdx.x & 31) / LC;
        return reinterpret_cast<const raw*>(mem + (buf * NA + n) * kArray + sub * kSlot + t * kRow)[lane];
    }
};

// The wait for the launch before.  The next launch is let in early only by a summary whose launch behind it
// has no whole tiles: CTAs that come while others still run spread over the SMs as places fall free, and the
// whole walk then goes at the pace of the fullest SM (one after another in a graph: 4 x 2304 x 1536 forward 35 against
// 30 us, 10 x 2304 x 1536, cut in its last round, 63 against 48; the summaries' own early release: forward and gradient
// of 1 x 9217 x 1536 87.3 against 88.1).
template <bool SUMMARY> __device__ __forceinline__ void wait_for(const ScanArgs& a)
{
    if (SUMMARY && a.whole == 0) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// LC lanes of VEC channels make a tile; a CTA has LC * kSlots threads.
// SUMMARY: only (A, H) of a whole segment.  A slot then has a run of the segment's tokens, not a part of every
// chunk, and the slots meet once at the end.
template <typename T, int VEC, int LC, bool WIDE, bool LOGITS, bool TIED, bool SUMMARY>
__global__ void __launch_bounds__(LC * kSlots, LC == 16 ? 3 : 1) scan_forward_kernel(const ScanArgs a)
{
    typedef pack<T, VEC> P;
    typedef typename P::raw raw;
    typedef num<VEC> N;
    struct Span { N A, H; };
    extern __shared__ __align__(16) unsigned char mem[];
    __shared__ Span span[2][kSlots][LC];           // of every slot, two chunks in turn
    __shared__ N next[2][LC];                      // h after the chunk
    const int lane = threadIdx.x % LC, slot = threadIdx.x / LC, warp = threadIdx.x >> 5;
    const int chunks = (a.T + kScanChunk - 1) / kScanChunk;
    const Work wk(a, SUMMARY ? 0 : -1, chunks, LC * VEC);
    const int b = wk.b, tile0 = wk.c, c0 = tile0 + lane * VEC, first = wk.first, end = wk.end;
    const bool in = c0 < a.C;                      // (VEC = 2 only where C is even)
    const int run = SUMMARY ? (end - first) * kTok : kTok, by = SUMMARY ? kTok : kScanChunk;   // a slot's tokens; to its next visit
    const int w0 = first * kScanChunk + warp * (32 / LC) * run, t0 = first * kScanChunk + slot * run;
    Stage<T, VEC, LC, 2, WIDE> st(mem, threadIdx.x & 31, warp, run);
    st.tensor(0, static_cast<const T*>(a.x) + b * a.xs[0] + tile0 + w0 * a.xs[1], a.xs[1], tile0, a.C);
    st.tensor(1, static_cast<const T*>(a.gate) + b * a.gs[0] + tile0 + w0 * a.gs[1], a.gs[1], tile0, a.C);
    T* y = static_cast<T*>(a.y) + b * a.ys[0] + c0 + t0 * a.ys[1];
    const long long state = (long long)b * a.C + c0;
    RowEnds rows(a.t0 + t0, a.grid_w, a.prefix_len, by);
    int rest_rows = a.T - w0, left = a.T - t0;     // tokens from the warp's, the slot's first one to the end
    wait_for<SUMMARY>(a);
    st.fetch(first & 1, rest_rows);
    // the state at the segment's first token: h_in through the segments before it
    N h0 = N::all(0.0f), total = N::all(1.0f);
    if (!SUMMARY && in) {
        if (wk.segs > 1) h0 = load_state<VEC>(wk.span(a, wk.segs - 1) + lane * VEC);
        else if (a.h_in) h0 = load_state<VEC>(a.h_in + state);
#pragma unroll 4
        for (int s = 0; s < wk.seg; ++s) {
            const float* w = wk.span(a, s) + lane * VEC;
            h0 = fma(load_state<VEC>(w), h0, load_state<VEC>(w + LC * VEC));
        }
    }
    for (int chunk = first; chunk < end; ++chunk) {
        const int buf = chunk & 1;
        // the next chunk comes in under this one's arithmetic (its buffer was read before the last barrier)
        if (chunk + 1 < end) {
            if (SUMMARY) __syncwarp();             // (there is no barrier: the warp's own lanes have read it)
            st.move(by);
            st.fetch(buf ^ 1, rest_rows - by);
        }
        st.landed(chunk + 1 == end);
        N ca[kTok], cb[kTok];
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            N rest;
            const N xv = P::get(st.get(buf, 0, t));
            gate_of<LOGITS>(P::get(st.get(buf, 1, t)), ca[t], rest);
            cb[t] = TIED ? rest * xv : xv;
        }
        const unsigned ends = rows.mask();
        if (ends)
#pragma unroll
            for (int t = 0; t < kTok; ++t)
                if ((ends >> t) & 1u) ca[t] = N::all(1.0f);
        if (left < kTok)                           // a token past the end changes nothing
#pragma unroll
            for (int t = 0; t < kTok; ++t)
                if (t >= left) ca[t] = N::all(1.0f), cb[t] = N::all(0.0f);
        N A = ca[0], H = cb[0];
#pragma unroll
        for (int t = 1; t < kTok; ++t) {
            A = A * ca[t];
            H = fma(ca[t], H, cb[t]);
        }
        if constexpr (SUMMARY) {
            h0 = fma(A, h0, H);
            total = total * A;
            rest_rows -= by;
            left -= by;
            rows.forward();
            continue;
        }
        span[buf][slot][lane] = {A, H};
        __syncthreads();
        // h before this slot (the chunk's own start came through `next` at the same barrier)
        N h = chunk == first ? h0 : next[buf][lane];
        if (slot == 0 && a.saved && in)
            store_state<VEC>(a.saved + ((long long)b * chunks + chunk) * a.C + c0, h);
#pragma unroll 5
        for (int s = 0; s < slot; ++s) {
            const Span m = span[buf][s][lane];
            h = fma(m.A, h, m.H);
        }
        if (slot == kSlots - 1) {
            const N after = fma(A, h, H);
            next[buf ^ 1][lane] = after;
            if (chunk == chunks - 1 && in && a.h_out) store_state<VEC>(a.h_out + state, after);
        }
        if (in)
#pragma unroll
            for (int t = 0; t < kTok; ++t) {
                h = fma(ca[t], h, cb[t]);
                if (t < left) *reinterpret_cast<raw*>(y + t * a.ys[1]) = P::put(h);
            }
        y += kScanChunk * a.ys[1];
        rest_rows -= by;
        left -= by;
        rows.forward();
    }
    if constexpr (SUMMARY) {
        span[0][slot][lane] = {total, h0};
        __syncthreads();
        if (slot == 0 && in) {
            for (int s = 1; s < kSlots; ++s) {
                const Span m = span[0][s][lane];
                h0 = fma(m.A, h0, m.H);
                total = total * m.A;
            }
            float* w = wk.span(a, wk.seg) + lane * VEC;
            store_state<VEC>(w, total);
            store_state<VEC>(w + LC * VEC, h0);
            if (wk.seg == 0) store_state<VEC>(wk.span(a, wk.segs - 1) + lane * VEC, a.h_in ? load_state<VEC>(a.h_in + state) : N::all(0.0f));
        }
    }
}

// The same walk from the end.  With u_t = a_t g_t the reversed recurrence u_t = a_t (u_{t+1} + dy_t)
// has the forward's products A, so a slot's spans in both directions are (A, H) and (A, Q).
// SUMMARY: only (A, Q) of a whole segment, from lambda and dy.
template <typename T, int VEC, int LC, bool WIDE, bool LOGITS, bool TIED, bool SUMMARY>
__global__ void __launch_bounds__(LC * kSlots, LC != 16 ? 1 : sizeof(T) == 2 ? 2 : 1) scan_backward_kernel(const ScanArgs a)
{
    typedef pack<T, VEC> P;
    typedef typename P::raw raw;
    typedef num<VEC> N;
    struct Span { N A, X; };
    extern __shared__ __align__(16) unsigned char mem[];
    __shared__ Span back[2][kSlots][LC];           // (A, Q) of every slot
    __shared__ N fwd[SUMMARY ? 1 : 2][kSlots][LC]; // H
    __shared__ N next[2][LC];                      // u before the chunk
    const int lane = threadIdx.x % LC, slot = threadIdx.x / LC, warp = threadIdx.x >> 5;
    const int chunks = (a.T + kScanChunk - 1) / kScanChunk;
    const Work wk(a, SUMMARY ? 1 : -1, chunks, LC * VEC);       // (nothing comes before segment 0: it needs no summary)
    const int b = wk.b, tile0 = wk.c, c0 = tile0 + lane * VEC, first = wk.first, end = wk.end;
    const bool in = c0 < a.C;
    const int run = SUMMARY ? (end - first) * kTok : kTok, by = SUMMARY ? kTok : kScanChunk;
    const int last = SUMMARY ? first * kScanChunk + run - kTok : (end - 1) * kScanChunk;       // slot 0's first visit
    const int w0 = last + warp * (32 / LC) * run, t0 = last + slot * run;
    Stage<T, VEC, LC, SUMMARY ? 2 : 3, WIDE> st(mem, threadIdx.x & 31, warp, run);
    st.tensor(0, static_cast<const T*>(a.gate) + b * a.gs[0] + tile0 + w0 * a.gs[1], a.gs[1], tile0, a.C);
    st.tensor(1, static_cast<const T*>(a.dy) + b * a.ys[0] + tile0 + w0 * a.ys[1], a.ys[1], tile0, a.C);
    if constexpr (!SUMMARY) st.tensor(2, static_cast<const T*>(a.x) + b * a.xs[0] + tile0 + w0 * a.xs[1], a.xs[1], tile0, a.C);
    T* dx = static_cast<T*>(a.dx) + b * a.dxs[0] + c0 + t0 * a.dxs[1];
    T* dg = static_cast<T*>(a.dgate) + b * a.dgs[0] + c0 + t0 * a.dgs[1];
    const float* saved = a.saved + ((long long)b * chunks + end - 1) * a.C + c0;
    const long long state = (long long)b * a.C + c0;
    RowEnds rows(a.t0 + t0, a.grid_w, a.prefix_len, by);
    int rest_rows = a.T - w0, left = a.T - t0;
    wait_for<SUMMARY>(a);
    st.fetch((end - 1) & 1, rest_rows);
    N u0 = N::all(0.0f), total = N::all(1.0f), hs = N::all(0.0f);      // hs: h before the chunk
    if (!SUMMARY && in) {
        hs = load_state<VEC>(saved);
        if (wk.segs > 1) u0 = load_state<VEC>(wk.span(a, 0) + lane * VEC);
        else if (a.dh_out) u0 = load_state<VEC>(a.dh_out + state);
#pragma unroll 4
        for (int s = wk.segs - 1; s > wk.seg; --s) {
            const float* w = wk.span(a, s) + lane * VEC;
            u0 = fma(load_state<VEC>(w), u0, load_state<VEC>(w + LC * VEC));
        }
    }
    for (int chunk = end - 1; chunk >= first; --chunk) {
        const int buf = chunk & 1;
        N h = hs;
        if (chunk > first) {
            __syncwarp();                          // (dy of the chunk before this one has been read)
            st.move(-by);
            st.fetch(buf ^ 1, rest_rows + by);
            saved -= a.C;
            if (!SUMMARY && in) hs = load_state<VEC>(saved);
        }
        st.landed(chunk == first);
        N ca[kTok], rest[kTok], xv[SUMMARY ? 1 : kTok];
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            gate_of<LOGITS>(P::get(st.get(buf, 0, t)), ca[t], rest[t]);
            if constexpr (!SUMMARY) xv[t] = P::get(st.get(buf, 2, t));
        }
        const unsigned ends = rows.mask();
        if (ends)
#pragma unroll
            for (int t = 0; t < kTok; ++t)
                if ((ends >> t) & 1u) ca[t] = N::all(1.0f);
        if (left < kTok)                           // a token past the end changes nothing (its dy is 0 below)
#pragma unroll
            for (int t = 0; t < kTok; ++t)
                if (t >= left) {
                    ca[t] = N::all(1.0f), rest[t] = N::all(0.0f);
                    if constexpr (!SUMMARY) xv[t] = N::all(0.0f);
                }
        auto grad = [&](int t) { return t < left ? P::get(st.get(buf, 1, t)) : N::all(0.0f); };
        N A = ca[0], H = N::all(0.0f), Q = N::all(0.0f);
#pragma unroll
        for (int t = 1; t < kTok; ++t) A = A * ca[t];
        if constexpr (!SUMMARY)
#pragma unroll
            for (int t = 0; t < kTok; ++t) H = fma(ca[t], H, TIED ? rest[t] * xv[t] : xv[t]);
#pragma unroll
        for (int t = kTok - 1; t >= 0; --t) Q = ca[t] * (Q + grad(t));
        if constexpr (SUMMARY) {
            u0 = fma(A, u0, Q);
            total = total * A;
            rest_rows += by;
            left += by;
            rows.back();
            continue;
        }
        back[buf][slot][lane] = {A, Q};
        if (!SUMMARY) fwd[buf][slot][lane] = H;
        __syncthreads();
        N u = chunk == end - 1 ? u0 : next[buf][lane];
#pragma unroll 5
        for (int s = kSlots - 1; s > slot; --s) {
            const Span m = back[buf][s][lane];
            u = fma(m.A, u, m.X);
        }
        if (!SUMMARY)
#pragma unroll 5
            for (int s = 0; s < slot; ++s) h = fma(back[buf][s][lane].A, h, fwd[buf][s][lane]);
        if (slot == 0) {
            const N before = fma(A, u, Q);
            next[buf ^ 1][lane] = before;
            if (chunk == 0 && in && a.dh_in) store_state<VEC>(a.dh_in + state, before);
        }
        if constexpr (!SUMMARY) {
            // dlambda_t = g_t f_t, f_t = h_{t-1} - x_t (tied): f_t takes x_t's place
            const N minus = N::all(-1.0f);
#pragma unroll
            for (int t = 0; t < kTok; ++t) {
                const N prev = h;
                h = fma(ca[t], h, TIED ? rest[t] * xv[t] : xv[t]);
                N f = TIED ? fma(xv[t], minus, prev) : prev;
                if (LOGITS) f = f * (rest[t] * ca[t]);             // the derivative of the sigmoid
                if (ends && ((ends >> t) & 1u)) {
                    // a row's last token does not pass h on through lambda; ca is 1 there, and lambda is formed
                    // again from the gate (not as 1 - rest, which has lost it where lambda is small)
                    f = TIED ? xv[t] * minus : N::all(0.0f);
                    if (LOGITS) {
                        N lam, same;
                        gate_of<true>(P::get(st.get(buf, 0, t)), lam, same);
                        f = f * (rest[t] * lam);
                    }
                }
                xv[t] = f;
            }
            if (in)
#pragma unroll
                for (int t = kTok - 1; t >= 0; --t) {
                    const N g = u + grad(t);
                    u = ca[t] * g;
                    if (t < left) {
                        *reinterpret_cast<raw*>(dx + t * a.dxs[1]) = P::put(TIED ? rest[t] * g : g);
                        *reinterpret_cast<raw*>(dg + t * a.dgs[1]) = P::put(xv[t] * g);
                    }
                }
            dx -= kScanChunk * a.dxs[1];
            dg -= kScanChunk * a.dgs[1];
        }
        rest_rows += by;
        left += by;
        rows.back();
    }
    if constexpr (SUMMARY) {
        back[0][slot][lane] = {total, u0};
        __syncthreads();
        if (slot == kSlots - 1 && in) {
            for (int s = kSlots - 2; s >= 0; --s) {
                const Span m = back[0][s][lane];
                u0 = fma(m.A, u0, m.X);
                total = total * m.A;
            }
            float* w = wk.span(a, wk.seg) + lane * VEC;
            store_state<VEC>(w, total);
            store_state<VEC>(w + LC * VEC, u0);
            if (wk.seg == wk.segs - 1) store_state<VEC>(wk.span(a, 0) + lane * VEC, a.dh_out ? load_state<VEC>(a.dh_out + state) : N::all(0.0f));
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
    typedef num<VEC> N;
    const N x = P::get(*reinterpret_cast<const raw*>(static_cast<const T*>(a.x) + b * a.xs[0] + c));
    const N z = P::get(*reinterpret_cast<const raw*>(static_cast<const T*>(a.gate) + b * a.gs[0] + c));
    N lam, rest;
    if (a.logits) gate_of<true>(z, lam, rest);
    else gate_of<false>(z, lam, rest);
    const N h = fma(ends ? N::all(1.0f) : lam, load_state<VEC>(a.h_in + (long long)b * a.C + c), a.tied ? rest * x : x);
    store_state<VEC>(a.h_out + (long long)b * a.C + c, h);
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

// Whether every tensor that is read has rows of whole 16-byte pieces.
bool wide_ok(const ScanArgs& a)
{
    const long long per = a.bf16 ? 8 : 4;
    const void* ptrs[] = {a.x, a.gate, a.dy};
    for (const void* p : ptrs)
        if (reinterpret_cast<uintptr_t>(p) % 16) return false;
    const long long* strides[] = {a.xs, a.gs, a.ys};
    for (int i = 0; i < (a.dy ? 3 : 2); ++i)
        if (strides[i][0] % per || strides[i][1] % per) return false;
    return a.C % per == 0;
}

template <typename T, int VEC, int LC, bool WIDE, bool LOGITS, bool TIED, bool SUMMARY>
cudaError_t launch_one(const ScanArgs& a, dim3 grid, cudaStream_t st)
{
    static bool done[2][64];
    const size_t bytes = Stage<T, VEC, LC, 2, WIDE>::kBytes, bytes3 = Stage<T, VEC, LC, SUMMARY ? 2 : 3, WIDE>::kBytes;
    if (a.dy) {
        const cudaError_t e = tcx::allow_dynamic_smem(scan_backward_kernel<T, VEC, LC, WIDE, LOGITS, TIED, SUMMARY>, bytes3, done[1]);
        return e != cudaSuccess ? e : launch_dependent(scan_backward_kernel<T, VEC, LC, WIDE, LOGITS, TIED, SUMMARY>, grid,
                                                       dim3(LC * kSlots), bytes3, st, a);
    }
    const cudaError_t e = tcx::allow_dynamic_smem(scan_forward_kernel<T, VEC, LC, WIDE, LOGITS, TIED, SUMMARY>, bytes, done[0]);
    return e != cudaSuccess ? e : launch_dependent(scan_forward_kernel<T, VEC, LC, WIDE, LOGITS, TIED, SUMMARY>, grid,
                                                   dim3(LC * kSlots), bytes, st, a);
}
template <typename T, int VEC, int LC, bool WIDE, bool LOGITS, bool TIED>
cudaError_t launch_t(const ScanArgs& a, cudaStream_t st)
{
    const int tiles = (a.C + LC * VEC - 1) / (LC * VEC) * a.B, cuts = tiles - a.whole;
    if (a.segs > 1) {
        const cudaError_t e = launch_one<T, VEC, LC, WIDE, LOGITS, TIED, true>(a, dim3(cuts * (a.segs - 1)), st);
        if (e != cudaSuccess) return e;
    }
    return launch_one<T, VEC, LC, WIDE, LOGITS, TIED, false>(a, dim3(a.whole + cuts * a.segs), st);
}
template <typename T, int VEC, int LC, bool WIDE>
cudaError_t launch_v(const ScanArgs& a, cudaStream_t st)
{
    if (a.logits) return a.tied ? launch_t<T, VEC, LC, WIDE, true, true>(a, st) : launch_t<T, VEC, LC, WIDE, true, false>(a, st);
    return a.tied ? launch_t<T, VEC, LC, WIDE, false, true>(a, st) : launch_t<T, VEC, LC, WIDE, false, false>(a, st);
}
// Pairs of channels, 16 lanes of them, and 16-byte copies where the memory allows them; single
// channels, 32 lanes, elsewhere.
cudaError_t launch(const ScanArgs& a, cudaStream_t st)
{
    if (pairs_ok(a) && wide_ok(a)) return a.bf16 ? launch_v<__nv_bfloat16, 2, 16, true>(a, st) : launch_v<float, 2, 16, true>(a, st);
    return a.bf16 ? launch_v<__nv_bfloat16, 1, 32, false>(a, st) : launch_v<float, 1, 32, false>(a, st);
}

}  // namespace

// How a call's work is cut.  A tile is 32 channels of one sequence, `slots` the CTAs that run at a time.
// A segment's summary reads two streams once more, of the forward's three and the backward's five, in a
// launch before, so a cut has to bring three CTAs in the place of one (backward: two).  (us below: launches one after
// another in a graph, bf16 unless said, cut against whole.)
//   - So few tiles, and eight chunks or more: all are cut, into as many segments as there are slots for.
//     Forward and gradient: 1 x 9217 x 1536 35.5 and 53 against 89 and 146, 1 x 1024 x 1536 7.4 and 11.5 against 11.1 and
//     18.1.  Two segments: 4 x 2304 x 1536 forward 31.6 against 30.4, 3 x 2304 x 1536 gradient 36.6 against 38.7.  Four
//     chunks (1 x 512 x 1536): 6.1 and 7.2 against 6.3 and 9.8 (left whole: one launch).
//   - A last round of tiles that leaves a quarter of the SMs or more idle: that round is cut.  Gradient of 8 x
//     2304 x 1536 (88 of 384 tiles) 78 against 85, of 4 x 2304 x 1536 in fp32 (44 of 192) 65 against 83; forward of
//     10 x 2304 x 1536 (36 of 480) 48 against 57, of 8 x 2304 x 1536 in fp32 61 against 67; with 132 of 576 left (12 x
//     2304 x 1536, forward) 61 against 58.
//   - After four whole rounds one round more is a fifth of the time at most: no cut.  Forward 38, 47, 57 x 1152 x 1536
//     82.7, 100.6, 120.4 against 83.6, 101.1, 119.7; what it leaves is the gradient's, 25 and 32 x 1152 x 1536 110 and
//     140 against 118 and 143, in fp32 13 and 16 x 1152 x 1536 101 and 121 against 108 and 129.
// The rule counts the slots of the 16-byte kernel for the single-channel one as well, which has twice the threads and one
// CTA an SM: how much workspace a call needs is asked before its pointers' alignment is known.  Cut against whole
// there: 1 x 9217 x 1535 forward 100 against 163, gradient 133 against 240, 10 x 2304 x 1535 forward 156 against 169; where
// its fewer slots make the cut a second round, 3 x 2304 x 1535, 62 against 46 and 82 against 66.
void scan_plan(ScanArgs& a, bool backward, int sms)
{
    const long long tiles = (long long)a.B * ((a.C + 31) / 32);
    const int chunks = (a.T + kScanChunk - 1) / kScanChunk;
    const long long slots = (long long)sms * (a.bf16 ? backward ? 2 : 3 : backward ? 1 : 2);
    long long whole = tiles, segs = 1;
    if (chunks < 8) {
    } else if (tiles * (backward ? 2 : 3) <= slots) {
        whole = 0;
    } else if (tiles > slots && tiles < 4 * slots && tiles % slots * 4 <= 3 * sms) {
        whole = tiles - tiles % slots;
    }
    if (whole < tiles) {
        segs = slots / (tiles - whole);
        if (segs > chunks) segs = chunks;
        a.seg_chunks = (int)((chunks + segs - 1) / segs);
        segs = (chunks + a.seg_chunks - 1) / a.seg_chunks;
    }
    if (segs == 1) whole = tiles;
    a.whole = (int)whole;
    a.segs = (int)segs;
}
size_t scan_workspace_bytes(const ScanArgs& a)
{
    const size_t tiles = (size_t)a.B * ((a.C + 31) / 32);
    return a.segs > 1 ? (tiles - a.whole) * a.segs * 2 * 32 * sizeof(float) : 0;
}
int scan_launches(const ScanArgs& a) { return a.segs > 1 ? 2 : 1; }

cudaError_t launch_scan_forward(const ScanArgs& a, cudaStream_t st) { return launch(a, st); }     // (a.dy is null)
cudaError_t launch_scan_backward(const ScanArgs& a, cudaStream_t st) { return launch(a, st); }
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
