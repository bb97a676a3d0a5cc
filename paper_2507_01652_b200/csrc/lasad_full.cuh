// Arguments and launchers of the operators of a layer that attends to whole sequences: causal attention over
// packed sequences, appending to a paged cache in 8 bits, and attention of one token per sequence over it.
// The host fills these from the C structs of lasad.h.
#pragma once
#include "lasad_mixers.cuh"

namespace lasad {

// ---- packed sequences --------------------------------------------------------------------------
struct PackedArgs {
    int N, S, Hq, Hk, d;         // tokens in memory, sequences
    bool bf16;
    float scale;
    long long qs[2], ks[2], vs[2], os[2], dos[2], dqs[2], dks[2], dvs[2];   // element strides of (token, head)
    const void* q;
    const void* k;
    const void* v;
    void* o;
    float* lse;                  // [Hq,N] or null
    const int* offsets;          // [S + 1]
    const void* dout;
    void* dq;
    void* dk;
    void* dv;
    float* ws;
    int sms;
    int* status;
    unsigned wait_limit;
};

// Tiles of `rows` tokens of every sequence, numbered without a table: the memory is cut at every offset into
// S + 2 regions (what lies before the first and behind the last sequence, which nobody owns, and the
// sequences), and region r starts at number start / rows + r.  That leaves room for each one's tiles
// (floor((a + n) / rows) - floor(a / rows) + 1 >= ceil(n / rows)); numbers without a tile have no rows.
__host__ __device__ inline long long region_tiles(long long N, long long S, int rows) { return N / rows + S + 2; }

#ifdef __CUDACC__
// Offsets are device data that nobody has checked: whatever stands there, no region leaves 0 .. N.
struct Region {
    int start, len;              // its first token in memory, its tokens
    int first;                   // of the tile, counted in the region
    int base;                    // the number of the region's first tile
    bool owned;                  // by a sequence
};
__device__ __forceinline__ int region_edge(const int* offsets, int S, int N, int r)
{
    return r == 0 ? 0 : r == S + 2 ? N : max(0, min(offsets[r - 1], N));
}
template <int ROWS>
__device__ __forceinline__ Region region_of(const int* offsets, int S, int N, int number)
{
    int lo = 0, hi = S + 2;      // the last region that starts at or before `number`
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (region_edge(offsets, S, N, mid) / ROWS + mid <= number) lo = mid;
        else hi = mid;
    }
    Region r;
    r.start = region_edge(offsets, S, N, lo);
    r.len = max(0, region_edge(offsets, S, N, lo + 1) - r.start);
    r.base = r.start / ROWS + lo;
    r.first = (number - r.base) * ROWS;
    r.owned = lo > 0 && lo <= S;
    return r;
}
// What a row's scores are moved by in the gradient, -lse log2(e).  A row that has seen nothing but scores of -infinity is empty,
// and so are its weights: no -infinity + infinity.
__device__ __forceinline__ float minus_lse(float lse) { return lse == -INFINITY ? lse : lse * -1.4426950408889634f; }
#endif

// The gradient's workspace: of each row -lse log2(e) and -Delta, Delta_t = do_t.o_t, in blocks of 64 rows of a
// tile and query head (first 64 of the one, then 64 of the other).
constexpr int kStatRows = 64;
__host__ __device__ inline long long packed_stat_at(const PackedArgs& a, int h, long long tile)
{
    return ((long long)h * region_tiles(a.N, a.S, kStatRows) + tile) * (2 * kStatRows);
}
inline size_t packed_workspace_bytes(const PackedArgs& a) { return (size_t)packed_stat_at(a, a.Hq, 0) * sizeof(float); }
cudaError_t launch_packed_forward_tc(const PackedArgs& a, cudaStream_t st);       // bf16
cudaError_t launch_packed_backward_tc(const PackedArgs& a, cudaStream_t st);      // two launches
cudaError_t launch_packed_forward_simt(const PackedArgs& a, cudaStream_t st);
cudaError_t launch_packed_backward_simt(const PackedArgs& a, cudaStream_t st);   // two launches

// ---- paged cache in 8 bits ---------------------------------------------------------------------
struct PagedArgs {
    int B, N, Hq, Hk, d;         // sequences, new tokens in memory
    int page, pages, table_pages;     // tokens of a page, pages of the pool, entries of a sequence
    bool bf16;
    unsigned char* kp;
    unsigned char* vp;
    long long kps[3], vps[3];    // strides in bytes of (page, head, slot)
    float* kscale;               // [pages,Hk]
    float* vscale;
    const int* block_table;      // [B,table_pages]
    const int* pos;              // [B]
    // append
    const int* offsets;          // [B + 1] or null: one token per sequence
    const void* k;
    const void* v;
    const void* q;               // or null
    void* q_out;
    long long ks[2], vs[2], qs[2], qos[2];    // element strides of (token, head); attention: of (sequence, head)
    const float* table;          // [rows, pairs, 2] or null: no rotation
    int table_rows, grid_w, prefix_len;
    bool half;
    // attention
    void* o;
    long long os[2];
    float* lse;                  // [B,Hq] or null
    float scale;
    float* ws;
    int splits;
    int sms;
};
constexpr int kScaleLow = -40, kScaleHigh = 40;     // exponents of a page's scale
cudaError_t launch_paged_append(const PagedArgs& a, cudaStream_t st);
// Into how many parts a sequence's tokens are cut, from the sizes alone.
int paged_splits(const PagedArgs& a);
size_t paged_workspace_bytes(const PagedArgs& a);
cudaError_t launch_paged_attention(const PagedArgs& a, cudaStream_t st);
inline int paged_attention_launches(const PagedArgs& a) { return a.splits > 1 ? 2 : 1; }

}  // namespace lasad
