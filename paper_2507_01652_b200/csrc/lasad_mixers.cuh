// Arguments and launchers of the operators that stand beside LASAD in a hybrid stack: the gated
// linear recurrence (scan), the norm and rotation of queries and keys (rope) and attention over a
// sliding window (window).  The host fills these from the C structs of lasad.h.
#pragma once
#include "lasad_common.cuh"

namespace lasad {

// Launches as a programmatic dependent of the kernel before it in the stream: its CTAs may take
// SMs as they become free, and every kernel launched this way runs pdl_wait() before it touches
// device memory.
template <typename... P, typename... A>
inline cudaError_t launch_dependent(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

#ifdef __CUDACC__
// (It does not let the next launch in early: its CTAs would spread over the SMs as places fall free, and take
// turns with the ones that still run.  Launches one after another in a graph: gradient of the norm and rotation with its
// forward, 8 x 4096 x 24, 184 us, let in early 193; one recurrence step 2.1 against 2.6.)
__device__ __forceinline__ void pdl_wait()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// The column of token i in its grid row, for a walk over consecutive tokens: a token before the
// grid has a negative one, and the last of a row is the one whose column is `last`.  Without a
// grid `last` is a value that no walk of 2^30 tokens reaches.
struct RowWalk {
    int col, last;
    __device__ __forceinline__ RowWalk(long long i, int grid_w, int prefix_len)
    {
        last = grid_w > 0 ? grid_w - 1 : 0x7fffffff;
        const long long j = i - prefix_len;
        if (grid_w <= 0) col = 0;
        else if (j < 0) col = j < -(1LL << 30) ? -(1 << 30) : (int)j;
        else if (j <= 0x7fffffffLL) col = (int)((unsigned)j % (unsigned)grid_w);
        else col = (int)(j % grid_w);
    }
    __device__ __forceinline__ bool step()   // whether this token ends its row; moves to the next one
    {
        const bool end = col == last;
        col = end ? 0 : col + 1;
        return end;
    }
};
#endif

// ---- scan ------------------------------------------------------------------------------------
constexpr int kScanChunk = 128;   // tokens between two saved states

struct ScanArgs {
    int B, T, C;
    int grid_w, prefix_len;
    long long t0;
    bool bf16, tied, logits;
    long long xs[2], gs[2], ys[2], dxs[2], dgs[2];   // element strides of (batch, token); ys is dy's too
    const void* x;
    const void* gate;
    const float* h_in;     // [B,C] or null
    void* y;
    float* h_out;          // [B,C] or null
    float* saved;          // [B, chunks, C] or null: h before each chunk
    const void* dy;        // null in the forward
    const float* dh_out;   // [B,C] or null
    void* dx;
    void* dgate;
    float* dh_in;          // [B,C] or null
    const int* pos;        // step only: [B] or null (t0 for all)
    // how the work is cut (scan_plan)
    int whole, segs, seg_chunks;
    float* ws;             // the segments' summaries when segs > 1
};
void scan_plan(ScanArgs& a, bool backward, int sms);
size_t scan_workspace_bytes(const ScanArgs& a);
int scan_launches(const ScanArgs& a);
cudaError_t launch_scan_forward(const ScanArgs& a, cudaStream_t st);
cudaError_t launch_scan_backward(const ScanArgs& a, cudaStream_t st);
cudaError_t launch_scan_step(const ScanArgs& a, cudaStream_t st);

// ---- rope ------------------------------------------------------------------------------------
struct RopeArgs {
    int B, T, Hq, Hk, d;
    int grid_w, prefix_len;
    long long t0;
    bool bf16, half;
    float eps;
    int table_rows;
    long long s[2][4][3];        // [q, k][in, out, dout, din] element strides of (batch, token, head)
    const void* in[2];
    const void* out[2];          // forward: written
    const void* dout[2];
    void* din[2];
    const float* weight[2];      // [d] or null
    const float* table;          // [rows, pairs, 2]
    const int* pos;              // [B] or null
    float* dw[2];                // [d] or null
    float* ws;                   // partial sums of dw
};
size_t rope_workspace_bytes(const RopeArgs& a, int sms);
int rope_backward_launches(const RopeArgs& a);
cudaError_t launch_rope_forward(const RopeArgs& a, int sms, cudaStream_t st);
cudaError_t launch_rope_backward(const RopeArgs& a, int sms, cudaStream_t st);

// ---- window ----------------------------------------------------------------------------------
struct WindowArgs {
    int B, T, Hq, Hk, d;
    int window, sinks;
    bool bf16;
    float scale;
    long long qs[3], ks[3], vs[3], os[3], dos[3], dqs[3], dks[3], dvs[3];
    const void* q;
    const void* k;
    const void* v;
    void* o;
    float* lse;                  // [B,Hq,T] or null
    const int* lengths;          // [B] or null (T for all)
    const void* dout;
    void* dq;
    void* dk;
    void* dv;
    float* ws;
    // step and store: the ring cache (strides of batch, slot, head)
    void* kc;
    void* vc;
    long long kcs[3], vcs[3];
    const int* pos;
    int sms;
    int* status;
    unsigned wait_limit;
};
constexpr int kMaxSinks = 128;

#ifdef __CUDACC__
// Whether token t sees token s of a sequence of n tokens.
__device__ __forceinline__ bool window_sees(int t, int s, int window, int sinks, int n)
{
    return s <= t && t < n && (t - s < window || s < sinks);
}
#endif

// The backward's workspace: what it needs of each row, and the gradients of the sinks' keys and values
// from the queries whose window has left them, in sums over kPrepRows rows (see lasad_window_prep.cu).
// Of kPrepRows rows of a query head at a time first -lse log2(e), then -Delta (a block is 512 bytes
// on a 16-byte boundary, which a bulk copy can take); behind them the sums [B,Hk,ceil(T/kPrepRows),sinks,2,d].
constexpr int kPrepRows = 64;
__host__ __device__ inline long long window_stat_at(int T, long long bh, int t)
{
    return (bh * ((T + kPrepRows - 1) / kPrepRows) + t / kPrepRows) * (2 * kPrepRows) + t % kPrepRows;
}
__host__ __device__ inline size_t window_stat_floats(const WindowArgs& a) { return (size_t)window_stat_at(a.T, (long long)a.B * a.Hq, 0); }
size_t window_workspace_bytes(const WindowArgs& a);
// Fills the workspace (delta), or the sums alone from what stands there of the rows.
cudaError_t launch_window_prep(const WindowArgs& a, bool delta, cudaStream_t st);
cudaError_t launch_window_forward_tc(const WindowArgs& a, cudaStream_t st);      // bf16
// (two launches, with launch_window_prep between them where a window leaves a sink)
cudaError_t launch_window_backward_tc(const WindowArgs& a, cudaStream_t st);
inline int window_backward_tc_launches(const WindowArgs& a) { return a.sinks > 0 && a.window < a.T ? 3 : 2; }
cudaError_t launch_window_forward_simt(const WindowArgs& a, cudaStream_t st);
cudaError_t launch_window_backward_simt(const WindowArgs& a, cudaStream_t st);   // three launches
// One token against the ring cache.
cudaError_t launch_window_step(const WindowArgs& a, cudaStream_t st);
cudaError_t launch_window_store(const WindowArgs& a, cudaStream_t st);

}  // namespace lasad
