// Tile staging and products shared by the fp32-pipe attention kernels.
//
// 256 threads as a 16 x 16 grid (ty = tid / 16, tx = tid % 16) own a 4 x 4
// micro tile each of a 64 x 64 tile; both operands of a product sit in shared
// memory with the summation index slowest, so that one step of a thread is
// two 16-byte shared loads and 16 FMAs.  Rows of 68 floats keep the loads
// 16-byte aligned and the stores of a warp on different banks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attention.h"
#include "ptx.cuh"

namespace gs {
namespace simt {

constexpr int kThreads = 256;
constexpr int T = 64;           // tile edge
constexpr int KC = 32;          // channels staged per step of a score product
constexpr int LD = T + 4;

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename E>
__device__ __forceinline__ E from_f(float x);
template <>
__device__ __forceinline__ float from_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Channels d0 .. d0 + 31 of 64 rows into dst[channel][row]; `row` is this
// thread's row tid % 64 (null: zeros).
template <typename E>
__device__ __forceinline__ void stage_t(float* dst, const E* row, int d0, int width) {
    const int r = threadIdx.x & (T - 1);
    const int dg = (threadIdx.x >> 6) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int d = d0 + dg + e;
        dst[(dg + e) * LD + r] = (row && d < width) ? to_f(row[d]) : 0.f;
    }
}

// Channels c0 .. c0 + 63 of 64 rows into dst[row][channel]; `row` is this
// thread's row tid / 4 (null: zeros).
template <typename E>
__device__ __forceinline__ void stage_n(float* dst, const E* row, int c0, int width) {
    const int r = threadIdx.x >> 2;
    const int cg = (threadIdx.x & 3) * 16;
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
        float4 x;
        float* f = &x.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = c0 + cg + e + i;
            f[i] = (row && c < width) ? to_f(row[c]) : 0.f;
        }
        *reinterpret_cast<float4*>(dst + r * LD + cg + e) = x;
    }
}

// acc[i][j] += sum_k a[k][4 ty + i] b[k][4 tx + j], k < steps.
template <int steps>
__device__ __forceinline__ void mac(float (&acc)[4][4], const float* a, const float* b) {
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll 8
    for (int k = 0; k < steps; ++k) {
        const float4 x = *reinterpret_cast<const float4*>(a + k * LD + ty * 4);
        const float4 y = *reinterpret_cast<const float4*>(b + k * LD + tx * 4);
        const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xs[i], ys[j], acc[i][j]);
    }
}

// acc = (rows of a) . (rows of b) over `width` channels, staged KC at a time
// through as and bs (KC x LD floats each).
template <typename E>
__device__ __forceinline__ void scores(float (&acc)[4][4], float* as, float* bs, const E* arow,
                                       const E* brow, int width) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
    for (int d0 = 0; d0 < width; d0 += KC) {
        __syncthreads();
        stage_t(as, arow, d0, width);
        stage_t(bs, brow, d0, width);
        __syncthreads();
        mac<KC>(acc, as, bs);
    }
}

// The thread's 4 x 4 tile into w[4 tx + j][4 ty + i] (the summation index of
// the next product slowest).
__device__ __forceinline__ void put_t(float* w, const float (&x)[4][4]) {
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(w + (tx * 4 + j) * LD + ty * 4) =
            make_float4(x[0][j], x[1][j], x[2][j], x[3][j]);
}

// acc[u] += w^T x for the 64-channel groups u of x, whose rows are staged
// through xs (64 x LD floats).
template <int NB, typename E>
__device__ __forceinline__ void accumulate(float (&acc)[NB][4][4], const float* w, float* xs,
                                           const E* xrow, int width) {
#pragma unroll
    for (int u = 0; u < NB; ++u) {
        if (u * T < width) {
            __syncthreads();
            stage_n(xs, xrow, u * T, width);
            __syncthreads();
            mac<T>(acc[u], w, xs);
        }
    }
}

template <typename E>
__device__ __forceinline__ const E* base(const Arr& a, int b, int h) {
    return reinterpret_cast<const E*>(a.p) + b * a.sb + h * a.sh;
}

// Row r = m G + g of key head j, or null past the first `rows` of them.
template <typename E>
__device__ __forceinline__ const E* query_row(const Arr& a, const AttnParams& p, int b, int j,
                                              int64_t r, int64_t rows) {
    if (r >= rows) return nullptr;
    const int64_t m = r / p.G;
    const int h = j * p.G + static_cast<int>(r - m * p.G);
    return base<E>(a, b, h) + m * a.sr;
}

template <typename E>
__device__ __forceinline__ const E* key_row(const Arr& a, int b, int j, int64_t n, int kl) {
    return n < kl ? base<E>(a, b, j) + n * a.sr : nullptr;
}

// Writes scale x the thread's channels of rows 4 ty + i, whose base pointers
// are rows[i] (null: not written).
template <int NB, typename E>
__device__ __forceinline__ void put_rows(const float (&acc)[NB][4][4], E* const (&rows)[4],
                                         const float (&scale)[4], int width) {
    const int tx = threadIdx.x & 15;
#pragma unroll
    for (int u = 0; u < NB; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int c = u * T + tx * 4 + e;
                if (rows[i] && c < width) rows[i][c] = from_f<E>(acc[u][i][e] * scale[i]);
            }
}

}  // namespace simt
}  // namespace gs
