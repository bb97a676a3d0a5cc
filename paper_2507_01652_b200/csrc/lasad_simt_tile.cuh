// Tiles of the attention kernels that work on CUDA cores in fp32: 64 queries by 64 keys stand in shared memory,
// a thread of the 256 has a 4 x 4 piece of the scores and 4 x D / 16 of a result.
#pragma once
#include "lasad_mixers.cuh"
#include "lasad_tc_tma.cuh"

namespace lasad {
namespace simt {

constexpr int kTile = 64, kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

template <int D> struct Tile { float x[kTile][D + 4]; };    // rows 16 bytes apart mod 128: no bank conflicts
struct Scores { float x[kTile][kTile + 4]; };

// rows r0.. of one head; rows past n are zero
template <typename T, int D>
__device__ __forceinline__ void load_tile(Tile<D>& to, const T* base, long long stride, int r0, int n)
{
    constexpr int N = 16 / sizeof(T), PER = D / N;
    for (int i = threadIdx.x; i < kTile * PER; i += kThreads) {
        const int r = i / PER, c = (i - r * PER) * N;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r0 + r < n) v = *reinterpret_cast<const uint4*>(base + (long long)(r0 + r) * stride + c);
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<uint4*>(&to.x[r][c]) = v;
        } else {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                to.x[r][c + 2 * k] = __uint_as_float(w[k] << 16);
                to.x[r][c + 2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
            }
        }
    }
}

// acc[i][j] = sum_c a[ty*4+i][c] b[tx+16j][c]
template <int D>
__device__ __forceinline__ void dot_tile(const Tile<D>& a, const Tile<D>& b, int ty, int tx, float (&acc)[4][4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0.0f;
#pragma unroll 4
    for (int c = 0; c < D; c += 4) {
        float4 u[4], w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = *reinterpret_cast<const float4*>(&a.x[ty * 4 + i][c]);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = *reinterpret_cast<const float4*>(&b.x[tx + 16 * j][c]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[i][j] += u[i].x * w[j].x + u[i].y * w[j].y + u[i].z * w[j].z + u[i].w * w[j].w;
    }
}

// A thread's columns of a D-wide accumulator: tx * (D / 16)...
template <int D>
__device__ __forceinline__ void load_cols(const float* row, int tx, float (&v)[D / 16])
{
    if constexpr (D == 64) {
        const float4 r = *reinterpret_cast<const float4*>(row + tx * 4);
        v[0] = r.x, v[1] = r.y, v[2] = r.z, v[3] = r.w;
    } else {
        const float2 r = *reinterpret_cast<const float2*>(row + tx * 2);
        v[0] = r.x, v[1] = r.y;
    }
}
// acc[i][:] += sum_k s[ty*4+i][k] v[k][:]        (rows of s)
template <int D>
__device__ __forceinline__ void add_rows(const Scores& s, const Tile<D>& v, int ty, int tx, float (&acc)[4][D / 16])
{
#pragma unroll 4
    for (int k = 0; k < kTile; k += 4) {
        float4 u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = *reinterpret_cast<const float4*>(&s.x[ty * 4 + i][k]);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            float w[D / 16];
            load_cols<D>(v.x[k + kk], tx, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = kk == 0 ? u[i].x : kk == 1 ? u[i].y : kk == 2 ? u[i].z : u[i].w;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) acc[i][c] = fmaf(p, w[c], acc[i][c]);
            }
        }
    }
}
// acc[i][:] += sum_k s[k][ty*4+i] v[k][:]        (columns of s)
template <int D>
__device__ __forceinline__ void add_cols(const Scores& s, const Tile<D>& v, int ty, int tx, float (&acc)[4][D / 16])
{
#pragma unroll 8
    for (int k = 0; k < kTile; ++k) {
        const float4 u = *reinterpret_cast<const float4*>(&s.x[k][ty * 4]);
        const float p[4] = {u.x, u.y, u.z, u.w};
        float w[D / 16];
        load_cols<D>(v.x[k], tx, w);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < D / 16; ++c) acc[i][c] = fmaf(p[i], w[c], acc[i][c]);
    }
}
template <typename T, int D>
__device__ __forceinline__ void store_cols(T* row, int tx, const float (&v)[D / 16])
{
#pragma unroll
    for (int c = 0; c < D / 16; ++c) io<T>::store(row + tx * (D / 16) + c, v[c]);
}

}  // namespace simt
}  // namespace lasad
