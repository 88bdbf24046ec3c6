// Rows into and out of the 4-bit cache (include/gauss_sum/attention_cache.h).
//
// A lane takes eight channels of a row: one 32-bit word of its codes; eight
// lanes take a group, whose least and largest value three shuffles give.  Both
// kernels read and write every byte once and are bound by that.  A block
// takes the rows of a run of tokens of one problem, all heads, keys or values;
// each lane has kRows rows on their way before it works on the first.
#include <algorithm>

#include "attention_cache.h"
#include "attention_simt.cuh"

namespace gs {
namespace {

using simt::from_f;
using simt::to_f;

constexpr int kThreads = 256;
constexpr int kRows = 4;

template <typename E>
struct alignas(16) Eight {
    E e[8];
};

template <typename E>
__device__ __forceinline__ void load8(float (&x)[8], const E* src, int c0, int width, bool vec) {
    if (vec) {
        const Eight<E> w = *reinterpret_cast<const Eight<E>*>(src + c0);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = to_f(w.e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = c0 + i < width ? to_f(src[c0 + i]) : 0.f;
    }
}

template <typename E>
__device__ __forceinline__ void store8(E* dst, const float (&x)[8], int c0, int width, bool vec) {
    if (vec) {
        Eight<E> w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w.e[i] = from_f<E>(x[i]);
        *reinterpret_cast<Eight<E>*>(dst + c0) = w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c0 + i < width) dst[c0 + i] = from_f<E>(x[i]);
    }
}

// Where a block and its lanes are: problem, side (keys or values), and for
// every row of it the row index m, the head and the token.
struct Place {
    int b, ql, kl;
    bool values;
    int first, items;     // row of the block's first item; items: (row, head) pairs
    int lanes, lane, row0, rows;   // lanes of a row, this one's, its first item, items at a time
};

__device__ __forceinline__ Place place(const CacheRows& r) {
    Place p;
    const int tiles = (r.M + r.block_tokens - 1) / r.block_tokens;
    p.b = static_cast<int>(blockIdx.x / tiles);
    const int tile = static_cast<int>(blockIdx.x - static_cast<unsigned>(p.b) * tiles);
    p.values = blockIdx.y != 0;
    p.kl = r.k_len ? min(max(r.k_len[p.b], 0), static_cast<int>(r.c.N)) : static_cast<int>(r.c.N);
    p.ql = r.q_len ? min(max(r.q_len[p.b], 0), r.M) : r.M;
    if (r.all) p.ql = p.kl;                       // row m is token m
    p.first = tile * r.block_tokens;
    p.items = min(r.block_tokens, r.M - p.first) * r.heads;
    const int words = p.values ? r.c.vw : r.c.kw;
    p.lanes = words <= 1 ? 4 : words <= 2 ? 8 : words <= 4 ? 16 : 32;
    p.lane = threadIdx.x & (p.lanes - 1);
    p.rows = kThreads / p.lanes;
    p.row0 = threadIdx.x / p.lanes;
    return p;
}

// Address of block `token / 16` of a page and head.
__device__ __forceinline__ char* block_of(const CacheParams& c, int page, int head, int token) {
    const int in_page = c.shift >= 0 ? token & (c.tokens - 1) : token % c.tokens;
    return c.data + page * c.sp + head * c.sh + static_cast<int64_t>(in_page >> 4) * c.block_bytes;
}

// Offsets in a block of row r: its codes and its groups.
__device__ __forceinline__ int codes_at(const CacheParams& c, bool values, int r) {
    return values ? 256 * c.kw + r * 16 * c.vw : r * 16 * c.kw;
}
__device__ __forceinline__ int groups_at(const CacheParams& c, bool values, int r) {
    return 256 * (c.kw + c.vw) + (values ? 64 * c.kg + r * 4 * c.vg : r * 4 * c.kg);
}

__device__ __forceinline__ float floor_bf16(float x) {
    const uint32_t w = __float_as_uint(x), low = w & 0xffffu;
    return __uint_as_float(w - low + ((w >> 31) && low ? 0x10000u : 0u));
}

template <typename E>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(const __grid_constant__ CacheRows r) {
    pdl_wait();
    const Place p = place(r);
    const CacheParams& c = r.c;
    const int width = p.values ? c.C : c.D, words = p.values ? c.vw : c.kw;
    const Arr& in = p.values ? r.v : r.k;
    const bool vec = p.values ? r.vec_v : r.vec_k;
    const int c0 = p.lane * 8, j = p.lane >> 2, t = p.lane & 3;
    const bool on = c0 < width, word_on = j < words;
    for (int u0 = 0; u0 < p.items; u0 += kRows * p.rows) {
        float x[kRows][8];
        char* block[kRows];
        int row[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int u = u0 + p.row0 + i * p.rows;
            const int mt = r.heads == 1 ? u : static_cast<int>(__umulhi(static_cast<unsigned>(u), r.head_magic));
            const int h = u - mt * r.heads, m = p.first + mt;
            const int token = m < p.ql ? m - p.ql + p.kl : -1;
            block[i] = nullptr;
            row[i] = token & 15;
            if (u < p.items && token >= 0) {
                const int page = cache_page(c, p.b, token);
                if (page != kNoPage) {
                    block[i] = block_of(c, page, h, token);
                    const E* src = reinterpret_cast<const E*>(in.p) + p.b * in.sb + m * in.sr + h * in.sh;
                    if (on) load8(x[i], src, c0, width, vec);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            float least = INFINITY, most = -INFINITY;
            bool fine = true;
            if (block[i] && on) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (c0 + e < width) {
                        fine = fine && fabsf(x[i][e]) <= 3.402823466e38f;
                        least = fminf(least, x[i][e]);
                        most = fmaxf(most, x[i][e]);
                    }
            }
#pragma unroll
            for (int d = 1; d < 8; d *= 2) {      // (a row of four lanes has one half group)
                const float l = __shfl_xor_sync(~0u, least, d), g = __shfl_xor_sync(~0u, most, d);
                if (d < p.lanes) {
                    least = fminf(least, l);
                    most = fmaxf(most, g);
                }
            }
            const unsigned votes = __ballot_sync(~0u, fine);
            const unsigned group = (p.lanes == 4 ? 0xfu : 0xffu) << (threadIdx.x & (p.lanes == 4 ? 28 : 24));
            fine = (votes & group) == group;
            if (!block[i] || !word_on) continue;
            const float low = floor_bf16(least);
            float s = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(__fsub_rn(most, low), 15.f)));
            if (s < 0x1p-126f) s = 0.f;
            fine = fine && s <= 3.402823466e38f;       // (not NaN either; a word without channels: NaN)
            const float inv = s > 0.f ? __fdiv_rn(1.f, s) : 0.f;
            uint32_t word = 0;
            if (fine && on) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    // The product is within 2^-22 of the quotient; the remainder, which
                    // is exact, moves a code that this puts on the wrong side.
                    const float y = __fsub_rn(x[i][e], low);
                    float q = rintf(__fmul_rn(y, inv));
                    const float twice = 2.f * fmaf(-q, s, y);
                    const bool odd = static_cast<int>(q) & 1;
                    if (twice > s || (twice == s && odd)) q += 1.f;
                    if (twice < -s || (twice == -s && odd)) q -= 1.f;
                    q = s > 0.f ? fminf(fmaxf(q, 0.f), 15.f) : 0.f;
                    if (c0 + e < width) word |= static_cast<uint32_t>(q) << (4 * e);
                }
            }
            char* codes = block[i] + codes_at(c, p.values, row[i]);
            if (p.values) {
                uint16_t* to = reinterpret_cast<uint16_t*>(codes);
                to[2 * t * words + j] = static_cast<uint16_t>(word);
                to[(2 * t + 1) * words + j] = static_cast<uint16_t>(word >> 16);
            } else {
                reinterpret_cast<uint32_t*>(codes)[t * words + j] = word;
            }
            if (on && (p.lane & 7) == 0)
                reinterpret_cast<uint32_t*>(block[i] + groups_at(c, p.values, row[i]))[p.lane >> 3] =
                    fine ? (__float_as_uint(s) >> 16) | (__float_as_uint(low) & 0xffff0000u) : kNanGroup;
        }
    }
}

template <typename E>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const __grid_constant__ CacheRows r) {
    pdl_wait();
    const Place p = place(r);
    const CacheParams& c = r.c;
    const Arr& out = p.values ? r.v : r.k;
    if (!out.p) return;
    const int width = p.values ? c.C : c.D, words = p.values ? c.vw : c.kw;
    const bool vec = p.values ? r.vec_v : r.vec_k;
    const int c0 = p.lane * 8, j = p.lane >> 2, t = p.lane & 3;
    const bool on = c0 < width;
    if (r.all && p.first >= p.kl) return;
    for (int u0 = 0; u0 < p.items; u0 += kRows * p.rows) {
        uint32_t word[kRows], group[kRows];
        E* to[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int u = u0 + p.row0 + i * p.rows;
            const int mt = r.heads == 1 ? u : static_cast<int>(__umulhi(static_cast<unsigned>(u), r.head_magic));
            const int h = u - mt * r.heads, m = p.first + mt;
            const int token = m < p.ql ? m - p.ql + p.kl : -1;
            const bool in = token >= 0;
            word[i] = group[i] = 0;
            to[i] = nullptr;
            if (u >= p.items || !on || (r.all && !in)) continue;
            to[i] = reinterpret_cast<E*>(out.p) + p.b * out.sb + m * out.sr + h * out.sh;
            if (!in) continue;
            const int page = cache_page(c, p.b, token);
            group[i] = kNanGroup;
            if (page == kNoPage) continue;
            const char* block = block_of(c, page, r.head0 + h, token);
            const char* codes = block + codes_at(c, p.values, token & 15);
            if (p.values) {
                const uint16_t* from = reinterpret_cast<const uint16_t*>(codes);
                word[i] = from[2 * t * words + j] | static_cast<uint32_t>(from[(2 * t + 1) * words + j]) << 16;
            } else {
                word[i] = reinterpret_cast<const uint32_t*>(codes)[t * words + j];
            }
            group[i] = reinterpret_cast<const uint32_t*>(block + groups_at(c, p.values, token & 15))[p.lane >> 3];
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (!to[i]) continue;
            const float s = __uint_as_float(group[i] << 16), low = __uint_as_float(group[i] & 0xffff0000u);
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = fmaf(s, static_cast<float>((word[i] >> (4 * e)) & 15u), low);
            store8(to[i], x, c0, width, vec);
        }
    }
}

// Whether rows start on 16-byte boundaries and are whole vectors of eight.
bool eights(const Arr& a, int B, int M, int heads, int width, int es) {
    return width % 8 == 0 && reinterpret_cast<uintptr_t>(a.p) % 16 == 0 && (B == 1 || a.sb * es % 16 == 0) &&
           (M == 1 || a.sr * es % 16 == 0) && (heads == 1 || a.sh * es % 16 == 0);
}

// Tokens of a block: kRows rows for every lane, fewer until each SM has two
// blocks.
cudaError_t plan(CacheRows& r, InType t, int sms, dim3* grid) {
    const int es = t == InType::F32 ? 4 : 2;
    r.vec_k = eights(r.k, r.B, r.M, r.heads, r.c.D, es);
    r.vec_v = eights(r.v, r.B, r.M, r.heads, r.c.C, es);
    r.head_magic = r.heads > 1 ? static_cast<unsigned>(((uint64_t(1) << 32) + r.heads - 1) / r.heads) : 0u;
    const int words = std::max(r.c.kw, r.c.vw);
    const int rows = kThreads / (words <= 1 ? 4 : words <= 2 ? 8 : words <= 4 ? 16 : 32);
    int tokens = std::max(1, std::min(r.M, kRows * rows / r.heads));
    const auto blocks = [&](int n) { return static_cast<int64_t>(r.B) * ((r.M + n - 1) / n); };
    while (tokens > 1 && tokens * r.heads > rows && blocks(tokens) < sms) tokens = (tokens + 1) / 2;
    r.block_tokens = tokens;
    if (blocks(tokens) >= int64_t(1) << 31) return cudaErrorInvalidConfiguration;
    *grid = dim3(static_cast<unsigned>(blocks(tokens)), 2);
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_cache_write(CacheRows r, InType t, int sms, cudaStream_t s) {
    dim3 grid;
    const cudaError_t e = plan(r, t, sms, &grid);
    if (e != cudaSuccess) return e;
    note_launches(1);
    if (t == InType::F32) return launch_kernel(cache_write_kernel<float>, grid, kThreads, 0, s, r);
    if (t == InType::F16) return launch_kernel(cache_write_kernel<__half>, grid, kThreads, 0, s, r);
    return launch_kernel(cache_write_kernel<__nv_bfloat16>, grid, kThreads, 0, s, r);
}

cudaError_t launch_cache_read(CacheRows r, InType t, int sms, cudaStream_t s) {
    dim3 grid;
    const cudaError_t e = plan(r, t, sms, &grid);
    if (e != cudaSuccess) return e;
    note_launches(1);
    if (t == InType::F32) return launch_kernel(cache_read_kernel<float>, grid, kThreads, 0, s, r);
    if (t == InType::F16) return launch_kernel(cache_read_kernel<__half>, grid, kThreads, 0, s, r);
    return launch_kernel(cache_read_kernel<__nv_bfloat16>, grid, kThreads, 0, s, r);
}

}  // namespace gs
