// Host side of the operators of a layer that attends to whole sequences: argument validation and launches.
#include "lasad_ctx.cuh"
#include "lasad_full.cuh"

#include <cmath>
#include <initializer_list>

namespace {

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool all(std::initializer_list<const void*> ps, uintptr_t n)
{
    for (const void* p : ps)
        if (!aligned(p, n)) return false;
    return true;
}
int launched(lasad_ctx* ctx, cudaError_t e, int launches)
{
    if (e != cudaSuccess) {
        ctx->last_cuda_error = (int)e;
        return LASAD_ERR_CUDA;
    }
    ctx->launches += launches;
    return LASAD_OK;
}
bool on_device(const lasad_ctx* ctx)
{
    int current = -1;
    return cudaGetDevice(&current) == cudaSuccess && current == ctx->device;
}
// Whether runs of `size` elements at these strides share no memory, one dimension inside another: sorted by stride, each steps
// over all that the ones before it span.  (Layouts that interleave in another way are refused with those that overlap.)
template <int NDIM> bool apart(const int64_t* stride, const int (&extent)[NDIM], int size)
{
    int order[NDIM], n = 0;
    for (int i = 0; i < NDIM; ++i) {
        if (extent[i] < 2) continue;
        int at = n++;
        for (; at > 0 && stride[order[at - 1]] > stride[i]; --at) order[at] = order[at - 1];
        order[at] = i;
    }
    __int128 span = size;
    for (int i = 0; i < n; ++i) {
        if (stride[order[i]] < span) return false;
        span += (__int128)stride[order[i]] * (extent[order[i]] - 1);
    }
    return true;
}
// Strides of (row, head): whole 16 bytes, none that repeats a row; those of an output lead to no element twice.
bool rows_ok(const int64_t* s, int64_t esz, int N, int H, int d, bool output, long long (&to)[2])
{
    for (int i = 0; i < 2; ++i) {
        if (s[i] < 0 || s[i] % (16 / esz) != 0) return false;
        to[i] = s[i];
    }
    if (output) return apart(s, {N, H}, d);
    return (s[0] > 0 || N == 1) && (s[1] >= d || H == 1);
}
bool heads_ok(int Hq, int Hk, int d) { return Hq > 0 && Hk > 0 && d > 0 && Hq % Hk == 0; }
bool dtype_ok(int dtype) { return dtype == LASAD_F32 || dtype == LASAD_BF16; }

int packed_args(lasad_ctx* ctx, const lasad_packed_params* p, bool backward, lasad::PackedArgs& a)
{
    if (!ctx || !p) return LASAD_ERR_INVALID_ARG;
    if (p->N <= 0 || p->S <= 0 || !heads_ok(p->Hq, p->Hk, p->d) || p->reserved != 0 || !std::isfinite(p->scale) || !dtype_ok(p->dtype))
        return LASAD_ERR_INVALID_ARG;
    struct { const int64_t* s; long long (&to)[2]; int H; } tensors[] = {
        {p->q_stride, a.qs, p->Hq}, {p->k_stride, a.ks, p->Hk}, {p->v_stride, a.vs, p->Hk}, {p->o_stride, a.os, p->Hq},
        {p->do_stride, a.dos, p->Hq}, {p->dq_stride, a.dqs, p->Hq}, {p->dk_stride, a.dks, p->Hk}, {p->dv_stride, a.dvs, p->Hk}};
    for (int i = 0; i < (backward ? 8 : 4); ++i)
        if (!rows_ok(tensors[i].s, p->dtype == LASAD_F32 ? 4 : 2, p->N, tensors[i].H, p->d, i == (backward ? 5 : 3) || i > 5, tensors[i].to))
            return LASAD_ERR_INVALID_ARG;
    if ((p->d != 32 && p->d != 64) || p->N > (1 << 30) || p->S > 65535) return LASAD_ERR_UNSUPPORTED;
    // (the tiles of all heads are counted in 32 bits)
    if (lasad::region_tiles(p->N, p->S, lasad::kStatRows) * p->Hq > 0x7fffffffLL) return LASAD_ERR_UNSUPPORTED;
    if (!on_device(ctx)) return LASAD_ERR_INVALID_ARG;
    a.N = p->N, a.S = p->S, a.Hq = p->Hq, a.Hk = p->Hk, a.d = p->d;
    a.bf16 = p->dtype == LASAD_BF16;
    a.scale = p->scale;
    a.sms = ctx->sm_count;
    a.status = ctx->d_status;
    a.wait_limit = ctx->wait_limit;
    return LASAD_OK;
}

// 1: CUDA cores, 2: tensor cores (LASAD_OPT_WINDOW_IMPL)
int packed_impl(const lasad_ctx* ctx, const lasad::PackedArgs& a)
{
    if (ctx->opt_window_impl == 0) return a.bf16 ? 2 : 1;
    return ctx->opt_window_impl == 2 && !a.bf16 ? LASAD_ERR_UNSUPPORTED : ctx->opt_window_impl;
}

// Strides in bytes of (page, head, slot), with the rules of rows_ok.
bool pages_ok(const int64_t* s, const lasad_paged_params* p, bool output, long long (&to)[3])
{
    for (int i = 0; i < 3; ++i) {
        if (s[i] < 0 || s[i] % 16 != 0) return false;
        to[i] = s[i];
    }
    if (output) return apart(s, {p->pages, p->Hk, p->page}, p->d);
    return (s[0] > 0 || p->pages == 1) && (s[1] >= p->d || p->Hk == 1) && s[2] >= p->d;
}
// Whether a head's last slot of the last page begins less than 2^32 - 1 times 16 bytes behind its first of the first.
bool places_fit(const int64_t* s, const lasad_paged_params* p)
{
    const int64_t limit = 0xffffffffLL * 16;
    return s[0] < limit && s[2] < limit && (p->pages - 1) * (s[0] / 16) + (p->page - 1) * (s[2] / 16) < 0xffffffffLL;
}
int paged_args(lasad_ctx* ctx, const lasad_paged_params* p, bool append, bool queries, bool packed, bool turn, lasad::PagedArgs& a)
{
    if (!ctx || !p) return LASAD_ERR_INVALID_ARG;
    if (p->B <= 0 || !heads_ok(p->Hq, p->Hk, p->d) || !dtype_ok(p->dtype) || p->pages <= 0 || p->table_pages <= 0 || p->page <= 0)
        return LASAD_ERR_INVALID_ARG;
    if (append && (p->N <= 0 || (!packed && p->N != p->B) || p->grid_w < 0 || p->prefix_len < 0 || (p->flags & ~LASAD_ROPE_HALF) ||
                   (turn && p->table_rows <= 0)))
        return LASAD_ERR_INVALID_ARG;
    if (!append && !std::isfinite(p->scale)) return LASAD_ERR_INVALID_ARG;
    const int64_t esz = p->dtype == LASAD_F32 ? 4 : 2;
    const int rows = append ? p->N : p->B;
    if (!pages_ok(p->k_pages_stride, p, append, a.kps) || !pages_ok(p->v_pages_stride, p, append, a.vps)) return LASAD_ERR_INVALID_ARG;
    if (append && (!rows_ok(p->k_stride, esz, rows, p->Hk, p->d, false, a.ks) || !rows_ok(p->v_stride, esz, rows, p->Hk, p->d, false, a.vs)))
        return LASAD_ERR_INVALID_ARG;
    if (queries && (!rows_ok(p->q_stride, esz, rows, p->Hq, p->d, false, a.qs) ||
                    !rows_ok(p->o_stride, esz, rows, p->Hq, p->d, true, append ? a.qos : a.os)))
        return LASAD_ERR_INVALID_ARG;
    if ((p->d != 32 && p->d != 64) || (p->page != 16 && p->page != 32 && p->page != 64 && p->page != 128) || p->B > 65535 ||
        (int64_t)p->table_pages * p->page > (1 << 30))
        return LASAD_ERR_UNSUPPORTED;
    // (places in the pool are counted in 16 bytes and 32 bits)
    if (!append && !(places_fit(p->k_pages_stride, p) && places_fit(p->v_pages_stride, p))) return LASAD_ERR_UNSUPPORTED;
    // (the units of a launch are counted in 32 bits)
    if (append ? p->N > (1 << 30) || 2 * ((int64_t)p->N / p->page + 2LL * p->B) * p->Hk + (int64_t)p->N * p->Hq > 0x7fffffffLL
               : (int64_t)p->B * p->Hq * 256 > 0x7fffffffLL)
        return LASAD_ERR_UNSUPPORTED;
    if (!on_device(ctx)) return LASAD_ERR_INVALID_ARG;
    a.B = p->B, a.N = p->N, a.Hq = p->Hq, a.Hk = p->Hk, a.d = p->d;
    a.page = p->page, a.pages = p->pages, a.table_pages = p->table_pages;
    a.bf16 = p->dtype == LASAD_BF16;
    a.grid_w = p->grid_w, a.prefix_len = p->prefix_len, a.table_rows = p->table_rows, a.half = p->flags & LASAD_ROPE_HALF;
    a.scale = p->scale;
    a.sms = ctx->sm_count;
    if (!append) a.splits = lasad::paged_splits(a);
    return LASAD_OK;
}

}  // namespace

extern "C" {

int lasad_packed_attention(lasad_ctx* ctx, const lasad_packed_params* p, const void* q, const void* k, const void* v,
                           const int32_t* offsets, void* o, float* lse, void* cuda_stream)
{
    lasad::PackedArgs a{};
    const int rc = packed_args(ctx, p, false, a);
    if (rc != LASAD_OK) return rc;
    if (!q || !k || !v || !offsets || !o || !all({q, k, v, o}, 16) || !all({offsets, lse}, 4)) return LASAD_ERR_INVALID_ARG;
    a.q = q, a.k = k, a.v = v, a.o = o, a.lse = lse, a.offsets = offsets;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int impl = packed_impl(ctx, a);
    if (impl < 0) return impl;
    return launched(ctx, impl == 2 ? lasad::launch_packed_forward_tc(a, st) : lasad::launch_packed_forward_simt(a, st), 1);
}

int64_t lasad_packed_attention_workspace(lasad_ctx* ctx, const lasad_packed_params* p)
{
    lasad::PackedArgs a{};
    const int rc = packed_args(ctx, p, true, a);
    return rc != LASAD_OK ? rc : (int64_t)lasad::packed_workspace_bytes(a);
}

int lasad_packed_attention_backward(lasad_ctx* ctx, const lasad_packed_params* p, const void* q, const void* k,
                                    const void* v, const void* o, const float* lse, const void* d_o,
                                    const int32_t* offsets, void* dq, void* dk, void* dv, void* workspace,
                                    void* cuda_stream)
{
    lasad::PackedArgs a{};
    const int rc = packed_args(ctx, p, true, a);
    if (rc != LASAD_OK) return rc;
    if (!q || !k || !v || !o || !lse || !d_o || !offsets || !dq || !dk || !dv || !workspace) return LASAD_ERR_INVALID_ARG;
    if (!all({q, k, v, o, d_o, dq, dk, dv, workspace}, 16) || !all({offsets, lse}, 4)) return LASAD_ERR_INVALID_ARG;
    a.q = q, a.k = k, a.v = v, a.o = const_cast<void*>(o), a.lse = const_cast<float*>(lse), a.dout = d_o, a.offsets = offsets;
    a.dq = dq, a.dk = dk, a.dv = dv, a.ws = static_cast<float*>(workspace);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int impl = packed_impl(ctx, a);
    if (impl < 0) return impl;
    return launched(ctx, impl == 2 ? lasad::launch_packed_backward_tc(a, st) : lasad::launch_packed_backward_simt(a, st), 2);
}

int lasad_paged_append(lasad_ctx* ctx, const lasad_paged_params* p, const void* k, const void* v, const void* q,
                       const float* table, const int32_t* offsets, const int32_t* pos, const int32_t* block_table,
                       void* k_pages, void* v_pages, float* k_scales, float* v_scales, void* q_out, void* cuda_stream)
{
    lasad::PagedArgs a{};
    const int rc = paged_args(ctx, p, true, q != nullptr, offsets != nullptr, table != nullptr, a);
    if (rc != LASAD_OK) return rc;
    if (!k || !v || !pos || !block_table || !k_pages || !v_pages || !k_scales || !v_scales || !q != !q_out) return LASAD_ERR_INVALID_ARG;
    if (!all({k, v, q, q_out, table, k_pages, v_pages}, 16) || !all({offsets, pos, block_table, k_scales, v_scales}, 4))
        return LASAD_ERR_INVALID_ARG;
    a.k = k, a.v = v, a.q = q, a.q_out = q_out, a.table = table, a.offsets = offsets, a.pos = pos, a.block_table = block_table;
    a.kp = static_cast<unsigned char*>(k_pages), a.vp = static_cast<unsigned char*>(v_pages), a.kscale = k_scales, a.vscale = v_scales;
    return launched(ctx, lasad::launch_paged_append(a, static_cast<cudaStream_t>(cuda_stream)), 1);
}

int64_t lasad_paged_attention_workspace(lasad_ctx* ctx, const lasad_paged_params* p)
{
    lasad::PagedArgs a{};
    const int rc = paged_args(ctx, p, false, true, false, false, a);
    return rc != LASAD_OK ? rc : (int64_t)lasad::paged_workspace_bytes(a);
}

int lasad_paged_attention(lasad_ctx* ctx, const lasad_paged_params* p, const void* q, const void* k_pages,
                          const void* v_pages, const float* k_scales, const float* v_scales, const int32_t* block_table,
                          const int32_t* pos, void* o, float* lse, void* workspace, void* cuda_stream)
{
    lasad::PagedArgs a{};
    const int rc = paged_args(ctx, p, false, true, false, false, a);
    if (rc != LASAD_OK) return rc;
    if (!q || !k_pages || !v_pages || !k_scales || !v_scales || !block_table || !pos || !o ||
        (!workspace && lasad::paged_workspace_bytes(a)))
        return LASAD_ERR_INVALID_ARG;
    if (!all({q, k_pages, v_pages, o, workspace}, 16) || !all({k_scales, v_scales, block_table, pos, lse}, 4)) return LASAD_ERR_INVALID_ARG;
    a.q = q, a.o = o, a.lse = lse, a.pos = pos, a.block_table = block_table, a.ws = static_cast<float*>(workspace);
    a.kp = static_cast<unsigned char*>(const_cast<void*>(k_pages)), a.vp = static_cast<unsigned char*>(const_cast<void*>(v_pages));
    a.kscale = const_cast<float*>(k_scales), a.vscale = const_cast<float*>(v_scales);
    return launched(ctx, lasad::launch_paged_attention(a, static_cast<cudaStream_t>(cuda_stream)), lasad::paged_attention_launches(a));
}

}  // extern "C"
