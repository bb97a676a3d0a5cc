// Host side of the operators beside LASAD: argument validation and launches.
#include "lasad_ctx.cuh"
#include "lasad_mixers.cuh"

#include <algorithm>
#include <cmath>
#include <initializer_list>

namespace {

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool all16(std::initializer_list<const void*> ps)
{
    for (const void* p : ps)
        if (!aligned(p, 16)) return false;
    return true;
}
int fail(lasad_ctx* ctx, cudaError_t e)
{
    ctx->last_cuda_error = (int)e;
    return LASAD_ERR_CUDA;
}
int launched(lasad_ctx* ctx, cudaError_t e, int launches)
{
    if (e != cudaSuccess) return fail(ctx, e);
    ctx->launches += launches;
    return LASAD_OK;
}
int on_device(const lasad_ctx* ctx)
{
    int current = -1;
    return cudaGetDevice(&current) == cudaSuccess && current == ctx->device ? LASAD_OK : LASAD_ERR_INVALID_ARG;
}
// Strides of (batch, token, head): whole 16 bytes, none that lets two elements share memory.
bool strides_ok(const int64_t* s, int64_t esz, int B, int T, int H, int d)
{
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0 || (s[i] * esz) % 16 != 0) return false;
    return (s[0] > 0 || B == 1) && (s[1] > 0 || T == 1) && (s[2] >= d || H == 1);
}
// A first position that leaves room for T tokens, and for the chunk behind the last one, in 64 bits.
bool first_ok(int64_t t0) { return t0 >= 0 && t0 <= (int64_t)1 << 62; }
void copy3(long long (&to)[3], const int64_t* from)
{
    for (int i = 0; i < 3; ++i) to[i] = from[i];
}

// ---- scan ------------------------------------------------------------------------------------
int scan_args(lasad_ctx* ctx, const lasad_scan_params* p, bool step, bool backward, lasad::ScanArgs& a)
{
    if (!ctx || !p) return LASAD_ERR_INVALID_ARG;
    if (p->B <= 0 || p->C <= 0 || (!step && p->T <= 0) || p->grid_w < 0 || p->prefix_len < 0 ||
        !first_ok(p->t0) || p->reserved != 0 || (p->flags & ~(LASAD_SCAN_TIED | LASAD_SCAN_LOGITS)) ||
        (p->dtype != LASAD_F32 && p->dtype != LASAD_BF16))
        return LASAD_ERR_INVALID_ARG;
    const int64_t* strides[] = {p->x_stride, p->gate_stride, p->y_stride, p->dx_stride, p->dgate_stride};
    for (int i = 0; i < (backward ? 5 : 3); ++i) {
        const int64_t* s = strides[i];
        if (s[0] < 0 || (s[0] == 0 && p->B > 1)) return LASAD_ERR_INVALID_ARG;
        if (!step && (s[1] < 0 || (s[1] < p->C && p->T > 1))) return LASAD_ERR_INVALID_ARG;
    }
    if (p->B > 65535 || (int64_t)p->B * p->C > 0x7fffffffLL || (!step && p->T > (1 << 30))) return LASAD_ERR_UNSUPPORTED;
    if (on_device(ctx) != LASAD_OK) return LASAD_ERR_INVALID_ARG;
    a.B = p->B, a.T = step ? 1 : p->T, a.C = p->C;
    a.grid_w = p->grid_w, a.prefix_len = p->prefix_len, a.t0 = p->t0;
    a.bf16 = p->dtype == LASAD_BF16, a.tied = p->flags & LASAD_SCAN_TIED, a.logits = p->flags & LASAD_SCAN_LOGITS;
    for (int i = 0; i < 2; ++i) {
        if (step && i == 1) break;
        a.xs[i] = p->x_stride[i], a.gs[i] = p->gate_stride[i], a.ys[i] = p->y_stride[i];
        if (backward) a.dxs[i] = p->dx_stride[i], a.dgs[i] = p->dgate_stride[i];
    }
    if (!step) lasad::scan_plan(a, backward, ctx->sm_count);
    return LASAD_OK;
}
bool scan_aligned(const lasad::ScanArgs& a, std::initializer_list<const void*> data, std::initializer_list<const void*> states)
{
    for (const void* p : data)
        if (!aligned(p, a.bf16 ? 2 : 4)) return false;
    for (const void* p : states)
        if (!aligned(p, 4)) return false;
    return true;
}

// ---- rope ------------------------------------------------------------------------------------
int rope_args(lasad_ctx* ctx, const lasad_rope_params* p, bool backward, bool has_pos, lasad::RopeArgs& a)
{
    if (!ctx || !p) return LASAD_ERR_INVALID_ARG;
    if (p->B <= 0 || p->T <= 0 || p->Hq <= 0 || p->Hk <= 0 || p->d <= 0 || p->grid_w < 0 || p->prefix_len < 0 ||
        !first_ok(p->t0) || p->table_rows <= 0 || p->reserved != 0 || (p->flags & ~LASAD_ROPE_HALF) || !(p->eps >= 0.0f) ||
        !std::isfinite(p->eps) || (p->dtype != LASAD_F32 && p->dtype != LASAD_BF16))
        return LASAD_ERR_INVALID_ARG;
    const int64_t* strides[2][4] = {{p->q_stride, p->q_out_stride, p->dq_out_stride, p->dq_stride},
                                    {p->k_stride, p->k_out_stride, p->dk_out_stride, p->dk_stride}};
    for (int w = 0; w < 2; ++w)
        for (int i = 0; i < 4; ++i) {
            if (i == 1 ? backward : i > 1 && !backward) continue;
            if (!strides_ok(strides[w][i], p->dtype == LASAD_F32 ? 4 : 2, p->B, p->T, w ? p->Hk : p->Hq, p->d))
                return LASAD_ERR_INVALID_ARG;
            copy3(a.s[w][i], strides[w][i]);
        }
    if (!has_pos) {     // the largest index into the table
        int64_t last = p->t0 + p->T - 1;
        if (p->grid_w > 0) {
            const int64_t w = p->grid_w, first = std::max<int64_t>(p->t0 - p->prefix_len, 0), j = last - p->prefix_len;
            // (tokens of one grid row: its number or the last one's column; of several: a row's last column is among theirs)
            last = j < 0 ? 0 : std::max(j / w, first / w == j / w ? j % w : w - 1);
        }
        if (last >= p->table_rows) return LASAD_ERR_INVALID_ARG;
    }
    if ((p->d != 32 && p->d != 64) || (int64_t)p->B * p->T > (1 << 30)) return LASAD_ERR_UNSUPPORTED;
    // (units of a launch are counted in 32 bits)
    if (p->B > 65535 || (int64_t)p->B * p->T * ((int64_t)p->Hq + p->Hk) > 0x7fffffffLL) return LASAD_ERR_UNSUPPORTED;
    if (on_device(ctx) != LASAD_OK) return LASAD_ERR_INVALID_ARG;
    a.B = p->B, a.T = p->T, a.Hq = p->Hq, a.Hk = p->Hk, a.d = p->d;
    a.grid_w = p->grid_w, a.prefix_len = p->prefix_len, a.t0 = p->t0;
    a.bf16 = p->dtype == LASAD_BF16, a.half = p->flags & LASAD_ROPE_HALF;
    a.eps = p->eps, a.table_rows = p->table_rows;
    return LASAD_OK;
}

// ---- window ----------------------------------------------------------------------------------
enum { kForward, kBackward, kStep, kStore };
int window_args(lasad_ctx* ctx, const lasad_window_params* p, int what, lasad::WindowArgs& a)
{
    if (!ctx || !p) return LASAD_ERR_INVALID_ARG;
    const int T = what == kStep ? 1 : p->T;
    if (p->B <= 0 || T <= 0 || p->Hq <= 0 || p->Hk <= 0 || p->d <= 0 || p->Hq % p->Hk != 0 || p->window <= 0 ||
        p->sinks < 0 || p->reserved != 0 || !std::isfinite(p->scale) || (p->dtype != LASAD_F32 && p->dtype != LASAD_BF16))
        return LASAD_ERR_INVALID_ARG;
    const int64_t esz = p->dtype == LASAD_F32 ? 4 : 2;
    const int64_t slots = (int64_t)p->sinks + p->window;
    struct { const int64_t* s; long long* to; int n, H; bool used; } all[] = {
        {p->q_stride, a.qs, T, p->Hq, what != kStore},
        {p->k_stride, a.ks, T, p->Hk, true},
        {p->v_stride, a.vs, T, p->Hk, true},
        {p->o_stride, a.os, T, p->Hq, what != kStore},
        {p->do_stride, a.dos, T, p->Hq, what == kBackward},
        {p->dq_stride, a.dqs, T, p->Hq, what == kBackward},
        {p->dk_stride, a.dks, T, p->Hk, what == kBackward},
        {p->dv_stride, a.dvs, T, p->Hk, what == kBackward},
        {p->k_cache_stride, a.kcs, slots > 1 ? 2 : 1, p->Hk, what == kStep || what == kStore},
        {p->v_cache_stride, a.vcs, slots > 1 ? 2 : 1, p->Hk, what == kStep || what == kStore},
    };
    for (auto& t : all) {
        if (!t.used) continue;
        int64_t s[3] = {t.s[0], t.s[1], t.s[2]};
        if (what == kStep && t.s != p->k_cache_stride && t.s != p->v_cache_stride) s[1] = 0;
        if (!strides_ok(s, esz, p->B, t.n, t.H, p->d)) return LASAD_ERR_INVALID_ARG;
        for (int i = 0; i < 3; ++i) t.to[i] = s[i];
    }
    if ((p->d != 32 && p->d != 64) || p->sinks > lasad::kMaxSinks || p->B > 65535 ||
        ((what == kStep || what == kStore) && p->window > (1 << 30)))
        return LASAD_ERR_UNSUPPORTED;
    if ((int64_t)p->B * p->Hq * ((T + 31) / 32) > 0x7fffffffLL || T > (1 << 30) || p->Hk > 65535)
        return LASAD_ERR_UNSUPPORTED;
    if (what == kStore && slots * p->Hk > (1LL << 34)) return LASAD_ERR_UNSUPPORTED;
    if (on_device(ctx) != LASAD_OK) return LASAD_ERR_INVALID_ARG;
    a.B = p->B, a.T = T, a.Hq = p->Hq, a.Hk = p->Hk, a.d = p->d;
    a.sinks = p->sinks;
    // a window longer than the sequence hides nothing more than one of its length
    a.window = (what == kForward || what == kBackward) && p->window > T ? T : p->window;
    a.bf16 = p->dtype == LASAD_BF16;
    a.scale = p->scale;
    a.sms = ctx->sm_count;
    a.status = ctx->d_status;
    a.wait_limit = ctx->wait_limit;
    return LASAD_OK;
}

// 1: CUDA cores, 2: tensor cores (LASAD_OPT_WINDOW_IMPL)
int window_impl(const lasad_ctx* ctx, const lasad::WindowArgs& a)
{
    if (ctx->opt_window_impl == 0) return a.bf16 ? 2 : 1;
    return ctx->opt_window_impl == 2 && !a.bf16 ? LASAD_ERR_UNSUPPORTED : ctx->opt_window_impl;
}

}  // namespace

extern "C" {

int64_t lasad_scan_workspace(lasad_ctx* ctx, const lasad_scan_params* p)
{
    lasad::ScanArgs a{};
    const int rc = scan_args(ctx, p, false, false, a);
    if (rc != LASAD_OK) return rc;
    const size_t forward = lasad::scan_workspace_bytes(a);
    lasad::scan_plan(a, true, ctx->sm_count);
    return (int64_t)std::max(forward, lasad::scan_workspace_bytes(a));
}

int lasad_scan_forward(lasad_ctx* ctx, const lasad_scan_params* p, const void* x, const void* gate, const float* h_in,
                       void* y, float* h_out, float* saved, void* workspace, void* cuda_stream)
{
    lasad::ScanArgs a{};
    const int rc = scan_args(ctx, p, false, false, a);
    if (rc != LASAD_OK) return rc;
    if (!x || !gate || !y || (!workspace && lasad::scan_workspace_bytes(a))) return LASAD_ERR_INVALID_ARG;
    if (!scan_aligned(a, {x, gate, y}, {h_in, h_out, saved}) || !aligned(workspace, 16)) return LASAD_ERR_INVALID_ARG;
    a.x = x, a.gate = gate, a.h_in = h_in, a.y = y, a.h_out = h_out, a.saved = saved;
    a.ws = static_cast<float*>(workspace);
    return launched(ctx, lasad::launch_scan_forward(a, static_cast<cudaStream_t>(cuda_stream)), lasad::scan_launches(a));
}

int lasad_scan_backward(lasad_ctx* ctx, const lasad_scan_params* p, const void* x, const void* gate, const float* saved,
                        const void* dy, const float* dh_out, void* dx, void* dgate, float* dh_in, void* workspace,
                        void* cuda_stream)
{
    lasad::ScanArgs a{};
    const int rc = scan_args(ctx, p, false, true, a);
    if (rc != LASAD_OK) return rc;
    if (!x || !gate || !saved || !dy || !dx || !dgate || (!workspace && lasad::scan_workspace_bytes(a)))
        return LASAD_ERR_INVALID_ARG;
    if (!scan_aligned(a, {x, gate, dy, dx, dgate}, {saved, dh_out, dh_in}) || !aligned(workspace, 16))
        return LASAD_ERR_INVALID_ARG;
    a.x = x, a.gate = gate, a.saved = const_cast<float*>(saved), a.dy = dy, a.dh_out = dh_out;
    a.dx = dx, a.dgate = dgate, a.dh_in = dh_in, a.ws = static_cast<float*>(workspace);
    return launched(ctx, lasad::launch_scan_backward(a, static_cast<cudaStream_t>(cuda_stream)), lasad::scan_launches(a));
}

int lasad_scan_step(lasad_ctx* ctx, const lasad_scan_params* p, const void* x, const void* gate, const float* h_in,
                    void* y, float* h_out, const int32_t* pos, void* cuda_stream)
{
    lasad::ScanArgs a{};
    const int rc = scan_args(ctx, p, true, false, a);
    if (rc != LASAD_OK) return rc;
    if (!x || !gate || !h_in || !y || !h_out) return LASAD_ERR_INVALID_ARG;
    if (!scan_aligned(a, {x, gate, y}, {h_in, h_out, pos})) return LASAD_ERR_INVALID_ARG;
    a.x = x, a.gate = gate, a.h_in = h_in, a.y = y, a.h_out = h_out, a.pos = pos;
    return launched(ctx, lasad::launch_scan_step(a, static_cast<cudaStream_t>(cuda_stream)), 1);
}

int lasad_qk_norm_rope(lasad_ctx* ctx, const lasad_rope_params* p, const void* q, const void* k, const float* table,
                       const float* q_weight, const float* k_weight, const int32_t* pos, void* q_out, void* k_out,
                       void* cuda_stream)
{
    lasad::RopeArgs a{};
    const int rc = rope_args(ctx, p, false, pos != nullptr, a);
    if (rc != LASAD_OK) return rc;
    if (!q || !k || !table || !q_out || !k_out) return LASAD_ERR_INVALID_ARG;
    if (!all16({q, k, table, q_out, k_out}) || !aligned(q_weight, 4) || !aligned(k_weight, 4) || !aligned(pos, 4))
        return LASAD_ERR_INVALID_ARG;
    a.in[0] = q, a.in[1] = k, a.out[0] = q_out, a.out[1] = k_out, a.table = table;
    a.weight[0] = q_weight, a.weight[1] = k_weight, a.pos = pos;
    return launched(ctx, lasad::launch_rope_forward(a, ctx->sm_count, static_cast<cudaStream_t>(cuda_stream)), 1);
}

int64_t lasad_qk_norm_rope_workspace(lasad_ctx* ctx, const lasad_rope_params* p)
{
    lasad::RopeArgs a{};
    const int rc = rope_args(ctx, p, true, true, a);
    return rc != LASAD_OK ? rc : (int64_t)lasad::rope_workspace_bytes(a, ctx->sm_count);
}

int lasad_qk_norm_rope_backward(lasad_ctx* ctx, const lasad_rope_params* p, const void* q, const void* k,
                                const float* table, const float* q_weight, const float* k_weight, const int32_t* pos,
                                const void* dq_out, const void* dk_out, void* dq, void* dk, float* dq_weight,
                                float* dk_weight, void* workspace, void* cuda_stream)
{
    lasad::RopeArgs a{};
    const int rc = rope_args(ctx, p, true, pos != nullptr, a);
    if (rc != LASAD_OK) return rc;
    const bool sums = dq_weight || dk_weight;
    if (!q || !k || !table || !dq_out || !dk_out || !dq || !dk || (sums && !workspace)) return LASAD_ERR_INVALID_ARG;
    if (!all16({q, k, table, dq_out, dk_out, dq, dk, workspace})) return LASAD_ERR_INVALID_ARG;
    if (!aligned(q_weight, 4) || !aligned(k_weight, 4) || !aligned(pos, 4) || !aligned(dq_weight, 4) || !aligned(dk_weight, 4))
        return LASAD_ERR_INVALID_ARG;
    a.in[0] = q, a.in[1] = k, a.dout[0] = dq_out, a.dout[1] = dk_out, a.din[0] = dq, a.din[1] = dk, a.table = table;
    a.weight[0] = q_weight, a.weight[1] = k_weight, a.pos = pos, a.dw[0] = dq_weight, a.dw[1] = dk_weight;
    a.ws = sums ? static_cast<float*>(workspace) : nullptr;
    return launched(ctx, lasad::launch_rope_backward(a, ctx->sm_count, static_cast<cudaStream_t>(cuda_stream)),
                    lasad::rope_backward_launches(a));
}

int lasad_window_attention(lasad_ctx* ctx, const lasad_window_params* p, const void* q, const void* k, const void* v,
                           const int32_t* lengths, void* o, float* lse, void* cuda_stream)
{
    lasad::WindowArgs a{};
    const int rc = window_args(ctx, p, kForward, a);
    if (rc != LASAD_OK) return rc;
    if (!q || !k || !v || !o || !all16({q, k, v, o}) || !aligned(lengths, 4) || !aligned(lse, 4)) return LASAD_ERR_INVALID_ARG;
    a.q = q, a.k = k, a.v = v, a.o = o, a.lse = lse, a.lengths = lengths;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int impl = window_impl(ctx, a);
    if (impl < 0) return impl;
    return launched(ctx, impl == 2 ? lasad::launch_window_forward_tc(a, st) : lasad::launch_window_forward_simt(a, st), 1);
}

int64_t lasad_window_attention_workspace(lasad_ctx* ctx, const lasad_window_params* p)
{
    lasad::WindowArgs a{};
    const int rc = window_args(ctx, p, kBackward, a);
    return rc != LASAD_OK ? rc : (int64_t)lasad::window_workspace_bytes(a);
}

int lasad_window_attention_backward(lasad_ctx* ctx, const lasad_window_params* p, const void* q, const void* k,
                                    const void* v, const void* o, const float* lse, const void* d_o,
                                    const int32_t* lengths, void* dq, void* dk, void* dv, void* workspace,
                                    void* cuda_stream)
{
    lasad::WindowArgs a{};
    const int rc = window_args(ctx, p, kBackward, a);
    if (rc != LASAD_OK) return rc;
    if (!q || !k || !v || !o || !lse || !d_o || !dq || !dk || !dv || !workspace) return LASAD_ERR_INVALID_ARG;
    if (!all16({q, k, v, o, d_o, dq, dk, dv, workspace}) || !aligned(lengths, 4) || !aligned(lse, 4))
        return LASAD_ERR_INVALID_ARG;
    a.q = q, a.k = k, a.v = v, a.o = const_cast<void*>(o), a.lse = const_cast<float*>(lse), a.dout = d_o;
    a.lengths = lengths, a.dq = dq, a.dk = dk, a.dv = dv, a.ws = static_cast<float*>(workspace);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int impl = window_impl(ctx, a);
    if (impl < 0) return impl;
    return impl == 2 ? launched(ctx, lasad::launch_window_backward_tc(a, st), lasad::window_backward_tc_launches(a))
                     : launched(ctx, lasad::launch_window_backward_simt(a, st), 3);
}

int lasad_window_attention_step(lasad_ctx* ctx, const lasad_window_params* p, const void* q, const void* k,
                                const void* v, void* k_cache, void* v_cache, const int32_t* pos, void* o,
                                void* cuda_stream)
{
    lasad::WindowArgs a{};
    const int rc = window_args(ctx, p, kStep, a);
    if (rc != LASAD_OK) return rc;
    if (!q || !k || !v || !k_cache || !v_cache || !pos || !o) return LASAD_ERR_INVALID_ARG;
    if (!all16({q, k, v, k_cache, v_cache, o}) || !aligned(pos, 4)) return LASAD_ERR_INVALID_ARG;
    a.q = q, a.k = k, a.v = v, a.kc = k_cache, a.vc = v_cache, a.pos = pos, a.o = o;
    return launched(ctx, lasad::launch_window_step(a, static_cast<cudaStream_t>(cuda_stream)), 1);
}

int lasad_window_cache_store(lasad_ctx* ctx, const lasad_window_params* p, const void* k, const void* v,
                             const int32_t* lengths, void* k_cache, void* v_cache, void* cuda_stream)
{
    lasad::WindowArgs a{};
    const int rc = window_args(ctx, p, kStore, a);
    if (rc != LASAD_OK) return rc;
    if (!k || !v || !k_cache || !v_cache || !all16({k, v, k_cache, v_cache}) || !aligned(lengths, 4))
        return LASAD_ERR_INVALID_ARG;
    a.k = k, a.v = v, a.kc = k_cache, a.vc = v_cache, a.lengths = lengths;
    return launched(ctx, lasad::launch_window_store(a, static_cast<cudaStream_t>(cuda_stream)), 1);
}

}  // extern "C"
