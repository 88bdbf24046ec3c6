// Tile staging and products shared by the fp32-pipe attention kernels.
//
// 256 threads as a 16 x 16 grid (ty = tid / 16, tx = tid % 16) own a 4 x 4
// micro tile each of a 64 x 64 tile; both operands of a product sit in shared
// memory with the summation index slowest, so that one step of a thread is
// two 16-byte shared loads and 16 FMAs.  Rows that are written transposed
// have their 16-byte groups permuted by the summation index (column r of row
// k lies at r ^ 4 ((k / 4) % 8)), which puts a warp's stores on 32 banks.
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

// Channels d .. d + 3 of a row (null, or past the width: zeros); `vec`: rows
// start on the boundary of four elements.
template <typename E>
__device__ __forceinline__ float4 load4(const E* row, int d, int width, bool vec) {
    if (!row || d >= width) return make_float4(0.f, 0.f, 0.f, 0.f);
    if (vec && d + 4 <= width) {
        if constexpr (sizeof(E) == 4) {
            return *reinterpret_cast<const float4*>(row + d);
        } else {
            const uint2 w = *reinterpret_cast<const uint2*>(row + d);
            const E* e = reinterpret_cast<const E*>(&w);
            return make_float4(to_f(e[0]), to_f(e[1]), to_f(e[2]), to_f(e[3]));
        }
    }
    return make_float4(to_f(row[d]), d + 1 < width ? to_f(row[d + 1]) : 0.f,
                       d + 2 < width ? to_f(row[d + 2]) : 0.f, d + 3 < width ? to_f(row[d + 3]) : 0.f);
}

// Permutation of the columns of row k.
__device__ __forceinline__ int permuted(int k, int r) { return r ^ (k & 28); }

// acc[i][j] += sum_k a[k][4 ty + i] b[k][CW tx + j], k < steps; a has
// permuted rows, b as well if PERM_B; rows of b are 16 CW long.
template <int steps, bool PERM_B, int CW>
__device__ __forceinline__ void mac(float (&acc)[4][CW], const float* a, const float* b) {
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll 2
    for (int k0 = 0; k0 < steps; k0 += 4) {
        const int ra = permuted(k0, ty * 4), rb = PERM_B ? permuted(k0, tx * CW) : tx * CW;
#pragma unroll
        for (int k = k0; k < k0 + 4; ++k) {
            const float4 x = *reinterpret_cast<const float4*>(a + k * T + ra);
            struct alignas(4 * CW) {
                float e[CW];
            } y;
            y = *reinterpret_cast<const decltype(y)*>(b + k * 16 * CW + rb);
            const float xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < CW; ++j) acc[i][j] = fmaf(xs[i], y.e[j], acc[i][j]);
        }
    }
}

// Channels 4 (tid % 8) .. of the thread's rows tid / 8 and tid / 8 + 32 into
// dst[channel][row].
__device__ __forceinline__ void put_channels(float* dst, const float4 (&x)[2]) {
    const int c = (threadIdx.x & 7) * 4, r = threadIdx.x >> 3;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int at = permuted(c, r + 32 * i);
        dst[c * T + at] = x[i].x;
        dst[(c + 1) * T + at] = x[i].y;
        dst[(c + 2) * T + at] = x[i].z;
        dst[(c + 3) * T + at] = x[i].w;
    }
}

// acc = (rows of a) . (rows of b) over `width` channels, KC at a time through
// as and bs (KC x T floats each).  arow, brow: the thread's rows tid / 8 and
// tid / 8 + 32.  Reads start before the barrier that frees the buffers.
template <typename E>
__device__ __forceinline__ void scores(float (&acc)[4][4], float* as, float* bs, const E* const (&arow)[2],
                                       const E* const (&brow)[2], int width, bool vec) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
    for (int d0 = 0; d0 < width; d0 += KC) {
        const int d = d0 + (threadIdx.x & 7) * 4;
        float4 x[2], y[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            x[i] = load4(arow[i], d, width, vec);
            y[i] = load4(brow[i], d, width, vec);
        }
        __syncthreads();
        put_channels(as, x);
        put_channels(bs, y);
        __syncthreads();
        mac<KC, true, 4>(acc, as, bs);
    }
}

// The thread's 4 x 4 tile into w[4 tx + j][4 ty + i] (the summation index of
// the next product slowest).
__device__ __forceinline__ void put_t(float* w, const float (&x)[4][4]) {
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(w + (tx * 4 + j) * T + permuted(tx * 4, ty * 4)) =
            make_float4(x[0][j], x[1][j], x[2][j], x[3][j]);
}

// Channels of an accumulator of a 64-row tile: NB groups of 16 CW, thread tx
// holding CW of each (CW = 2: one group of 32 channels).
// acc[u] += w^T x for the groups u of x, whose rows are staged through xs
// (T x 16 CW floats).  xrow: the thread's rows tid / 16 + 16 i.
template <int NB, int CW, typename E>
__device__ __forceinline__ void accumulate(float (&acc)[NB][4][CW], const float* w, float* xs,
                                           const E* const (&xrow)[4], int width, bool vec) {
    constexpr int W = 16 * CW, kLanes = W / 4;   // of the 16 lanes of a row, four channels each
    const int r = threadIdx.x >> 4, lane = threadIdx.x & 15, c = lane * 4;
#pragma unroll
    for (int u = 0; u < NB; ++u) {
        if (u * W < width) {
            float4 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (lane < kLanes) x[i] = load4(xrow[i], u * W + c, width, vec);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (lane < kLanes) *reinterpret_cast<float4*>(xs + (r + 16 * i) * W + c) = x[i];
            __syncthreads();
            mac<T, false, CW>(acc[u], w, xs);
        }
    }
}

template <typename E>
__device__ __forceinline__ const E* base(const Arr& a, int b, int h) {
    return reinterpret_cast<const E*>(a.p) + b * a.sb + h * a.sh;
}

// Token of row r = m G + g of a key head: no division for heads with their own
// keys, a 32-bit one up to 2^32 rows.
__device__ __forceinline__ int64_t row_token(const AttnParams& p, int64_t r) {
    if (p.G == 1) return r;
    if (r >> 32 == 0) return static_cast<uint32_t>(r) / static_cast<uint32_t>(p.G);
    return r / p.G;
}

// Row r = m G + g of key head j, or null past the first `rows` of them.
template <typename E>
__device__ __forceinline__ const E* query_row(const Arr& a, const AttnParams& p, int b, int j,
                                              int64_t r, int64_t rows) {
    if (r >= rows) return nullptr;
    const int64_t m = row_token(p, r);
    const int h = j * p.G + static_cast<int>(r - m * p.G);
    return base<E>(a, b, h) + m * a.sr;
}

template <typename E>
__device__ __forceinline__ const E* key_row(const Arr& a, int b, int j, int64_t n, int kl) {
    return n < kl ? base<E>(a, b, j) + n * a.sr : nullptr;
}

// The thread's rows of a staged tile that starts at row `first`: with N = 2
// (channels transposed) tid / 8 + 32 i, with N = 4 tid / 16 + 16 i.
template <int N, typename E>
__device__ __forceinline__ void query_rows(const E* (&to)[N], const Arr& a, const AttnParams& p, int b, int j,
                                           int64_t first, int64_t rows) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        to[i] = query_row<E>(a, p, b, j, first + threadIdx.x / (4 * N) + T / N * i, rows);
}
template <int N, typename E>
__device__ __forceinline__ void key_rows(const E* (&to)[N], const Arr& a, int b, int j, int64_t first, int kl) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        to[i] = key_row<E>(a, b, j, first + threadIdx.x / (4 * N) + T / N * i, kl);
}

// Writes scale x the thread's channels of rows 4 ty + i, whose base pointers
// are rows[i] (null: not written).
template <int NB, int CW, typename E>
__device__ __forceinline__ void put_rows(const float (&acc)[NB][4][CW], E* const (&rows)[4],
                                         const float (&scale)[4], int width) {
    const int tx = threadIdx.x & 15;
#pragma unroll
    for (int u = 0; u < NB; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < CW; ++e) {
                const int c = (u * 16 + tx) * CW + e;
                if (rows[i] && c < width) rows[i][c] = from_f<E>(acc[u][i][e] * scale[i]);
            }
}

}  // namespace simt
}  // namespace gs
