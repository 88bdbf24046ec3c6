// Attention of few query rows over the 4-bit cache (single tokens, drafts).
//
// Every byte of the cache is read once, and a value takes about a dozen bits
// of HBM time, so what counts is how few instructions a code needs on its way
// into a product:
//
//   A nibble is a denormal fp16 number where it lies: x & 0x000f000f is a pair
//   of codes times 2^-24, x & 0x00f000f0 a pair times 2^-20.  With the factor 16
//   in the other operand, and steps and least values applied to the sums,
//
//     S_n   = sum_i s_ni (q_i . u_ni) + m_ni sum q_i                     (groups i)
//     out   = sum_n (p_n s_ni) (u_ni - 8) + sum_n p_n (m_ni + 8 s_ni)    (channels of group i)
//
//   are two products of the codes u alone, which are exact, and a few fp32
//   operations per pair and group.  The values' codes are centred, one fp16
//   addition a pair: the sum over many keys would otherwise be a hundred times
//   its result, and the roundings of p s, and the products' own accumulation
//   (which cuts rather than rounds), with it (relative error of 1501 keys of
//   32 channels, fp32: 4.3e-5 without).
//
// The products are mma.sync m16n8k16 with the codes as the 16-row operand in
// registers: S^T has keys as rows and queries as columns, out^T channels as rows.
// (There is no shared-memory operand to feed: tcgen05 would want the codes
// expanded to 16 bits and written to shared memory or TMEM first, which costs
// 128 bytes a clock of an SM's shared memory more than HBM delivers.  At the 0.5
// m16n8k16 a clock and SM that this card does, 8 rows take a third of the tensor pipe's
// time under the HBM time of a block.)  p s goes from the layout of a result to
// that of an operand by movmatrix.
//
// Queries are scaled by a power of two per row to fp16 (exact down to 2^-28 of
// the row's largest); fp32 queries, and p s of such calls, are two fp16 numbers
// each (SPLIT).  p s 2^-E is rounded to fp16, E the exponent of the largest |m|
// or s that the warp has seen (p itself is scaled): it keeps fp16's 11 bits down to 2^-22 of the largest value
// and vanishes below 2^-32 of it.  The running maximum lags by up to 2^6.
//
// A warp takes pairs of blocks, 32 tokens, by itself: a ring of bulk copies in its own
// shared memory, no barrier between warps until their results are joined at
// the end (and those of the splits by attn_join_kernel).
#include <algorithm>

#include "attention_cache.h"
#include "attention_simt.cuh"

namespace gs {
namespace {

using simt::to_f;

constexpr int kWarps = 4;
constexpr uint32_t kMinusEight = 0x80088008u, kMinusEight16 = 0x80808080u;   // -8 x 2^-24, -8 x 2^-20, twice
constexpr float kSlack = 6.f;       // log2 units that the maximum may lag behind
constexpr float kShift = 7.f;       // p is scaled by 2^7: p s 2^-E < 2^15

struct FewParams {
    AttnParams a;
    CacheParams c;
    InType type;                    // of q and out
    int stages;
    int64_t tiles_r;                // tiles of 8 NQ rows
};

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 8 x 8 16-bit matrix, transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// BYTES (a multiple of two) from shared memory as words, the last one half.
template <int BYTES>
__device__ __forceinline__ void load_words(uint32_t (&w)[(BYTES + 3) / 4], const char* at) {
    if constexpr (BYTES == 16) {
        const uint4 x = *reinterpret_cast<const uint4*>(at);
        w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
    } else if constexpr (BYTES == 8) {
        const uint2 x = *reinterpret_cast<const uint2*>(at);
        w[0] = x.x, w[1] = x.y;
    } else if constexpr (BYTES == 6) {
        const uint16_t* x = reinterpret_cast<const uint16_t*>(at);
        w[0] = x[0] | static_cast<uint32_t>(x[1]) << 16;
        w[1] = x[2];
    } else if constexpr (BYTES == 2) {
        w[0] = *reinterpret_cast<const uint16_t*>(at);
    } else {
#pragma unroll
        for (int i = 0; i < BYTES / 4; ++i) w[i] = reinterpret_cast<const uint32_t*>(at)[i];
    }
}

__device__ __forceinline__ uint32_t add2(uint32_t a, uint32_t b) {
    uint32_t y;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
    return y;
}

__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Eight channels of a query row, zeros past the width.
__device__ __forceinline__ void load_query(float (&x)[8], const FewParams& f, int64_t at, int c0, bool on) {
    const AttnParams& p = f.a;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
    if (!on || c0 >= p.D) return;
    if (f.type == InType::F32) {
        const float* src = reinterpret_cast<const float*>(p.q.p) + at + c0;
        if (p.vec && c0 + 8 <= p.D) {
            const float4 u = reinterpret_cast<const float4*>(src)[0], v = reinterpret_cast<const float4*>(src)[1];
            x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c0 + i < p.D) x[i] = src[i];
        }
        return;
    }
    const uint16_t* src = reinterpret_cast<const uint16_t*>(p.q.p) + at + c0;
    uint16_t w[8];
    if (p.vec && c0 + 8 <= p.D) {
        *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(src);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = c0 + i < p.D ? src[i] : uint16_t(0);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        x[i] = f.type == InType::F16 ? __half2float(__ushort_as_half(w[i]))
                                     : __uint_as_float(static_cast<uint32_t>(w[i]) << 16);
}

template <int W, int NQ>
struct FewCfg {
    static constexpr int kGroups = (W + 1) / 2;
    static constexpr int kRows = 8 * NQ;
    static constexpr int kBlockBytes = 16 * 2 * (16 * W + 4 * kGroups);
    static constexpr int kStageBytes = 2 * kBlockBytes;
    // Eight rows take the codes' -8 as one more product, which the tensor pipe has time for (24
    // a block of 16 tokens, 48 of 104 clocks); more rows share additions on the codes.
    static constexpr bool kCentreByProduct = NQ == 1;
    static constexpr int kBlocksPerSm = NQ == 1 ? 4 : NQ == 2 ? 3 : 2;
    // Joining: rows of 32 W channels, and their lse, of every warp.
    static constexpr int kJoinBytes = (kRows * 32 * W + kRows) * 4;
};
constexpr int kMaxStages = 8;
// Exponent fields of bf16 numbers between which E moves: p 2^-E stays a normal
// float32 number, and values up to 2^102 are fine.
constexpr int kLeastExponent = 27, kMostExponent = 226;

template <int W, int NQ, bool SPLIT>
__global__ void __launch_bounds__(kWarps * 32, (FewCfg<W, NQ>::kBlocksPerSm))
cache_few_kernel(const __grid_constant__ FewParams f) {
    using K = FewCfg<W, NQ>;
    constexpr int G = K::kGroups, QS = SPLIT ? 2 : 1;
    const AttnParams& p = f.a;
    const CacheParams& c = f.c;
    extern __shared__ __align__(128) char smem[];
    __shared__ uint64_t full[kWarps][kMaxStages];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    char* ring = smem + warp * max(f.stages * K::kStageBytes, K::kJoinBytes);

    // Block -> (split, row tile, problem, key head).
    int64_t blk = blockIdx.x;
    const int split = static_cast<int>(blk % p.splits);
    blk /= p.splits;
    const int64_t tile = blk % f.tiles_r, bj = blk / f.tiles_r;
    const int b = static_cast<int>(bj / p.Hk), j0 = static_cast<int>(bj - static_cast<int64_t>(b) * p.Hk);
    if (lane == 0) {
        for (int s = 0; s < f.stages; ++s) mbar_init(&full[warp][s], 2);
        fence_mbar_init();
    }
    __syncwarp();
    pdl_wait();
    pdl_trigger();
    const int ql = attn_q_len(p, b), kl = attn_k_len(p, b);
    const int64_t rows_in = static_cast<int64_t>(ql) * p.G, r0 = tile * K::kRows;
    const int64_t last = min(r0 + K::kRows, rows_in) - 1;
    const int kend = last >= r0 ? attn_limit(static_cast<int>(last / p.G), ql, kl, p.causal) : 0;
    // Pairs of cache blocks (32 tokens): pairs s0 + warp + kWarps k.
    const int64_t all = (static_cast<int64_t>(kend) + 31) / 32;
    const int s0 = static_cast<int>(all * split / p.splits), s1 = static_cast<int>(all * (split + 1) / p.splits);
    const int steps = max(0, (s1 - s0 - warp + kWarps - 1) / kWarps);
    const int blocks = (kend + 15) >> 4;               // that hold a key some row sees

    // Copies: lanes 0 and 1 bring a block each.  Lane i has the page of block
    // i & 1 of pair i / 2 of the next 16 pairs, read ahead.
    const int per_page = c.tokens >> 4;
    const auto block_at = [&](int k) { return 2 * (s0 + warp + kWarps * k) + (lane & 1); };
    const auto page_of = [&](int k) {
        const int i = block_at(k);
        return k < steps && i < blocks ? cache_page(c, b, i << 4) : kNoPage;
    };
    int pages = page_of(lane >> 1), pages_next = page_of(16 + (lane >> 1));
    uint32_t bad = 0;                                  // two bits a stage: blocks that were not copied
    const char* base = c.data + j0 * c.sh;
    const auto issue = [&](int k, int stage) {
        if (k >= steps) return;
        if (k > 0 && (k & 15) == 0) {
            pages = pages_next;
            pages_next = page_of(k + 16 + (lane >> 1));
        }
        const int page = __shfl_sync(~0u, pages, 2 * (k & 15) + (lane & 1));
        const uint32_t none = __ballot_sync(~0u, page == kNoPage) & 3u;
        bad = (bad & ~(3u << (2 * stage))) | none << (2 * stage);
        if (lane < 2) {
            uint64_t* bar = &full[warp][stage];
            if (page == kNoPage) {
                mbar_arrive(bar);
            } else {
                const int i = block_at(k), in_page = c.shift >= 0 ? i & (per_page - 1) : i % per_page;
                mbar_arrive_expect_tx(bar, K::kBlockBytes);
                bulk_load(ring + stage * K::kStageBytes + lane * K::kBlockBytes,
                          base + page * c.sp + static_cast<int64_t>(in_page) * K::kBlockBytes, K::kBlockBytes, bar);
            }
        }
        __syncwarp();
    };
    for (int k = 0; k < f.stages; ++k) issue(k, k);

    // Queries: row 8 n + g as the second operand, scaled to at most 2^15.
    uint32_t qb[NQ][QS][W][4];
    float qsum[NQ][G][2], factor[NQ][2];               // of queries 2 t, 2 t + 1
    int lim[NQ][2];
    int lim_first = kl;                                // the least limit of a row of the tile
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int64_t r = r0 + 8 * n + g, m = r / p.G;
        const bool in = r < rows_in;
        const int64_t at = b * p.q.sb + m * p.q.sr + (j0 * p.G + static_cast<int>(r - m * p.G)) * p.q.sh;
        float x[W][8], top = 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            load_query(x[j], f, in ? at : 0, 32 * j + 8 * t, in);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[j][e]));
        }
        top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
        top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
        // 2^e top in [2^14, 2^15), e in -113 .. 100 (an empty row: 100).
        const int e = min(141 - static_cast<int>(__float_as_uint(top) >> 23), 100);
        const float up = __uint_as_float(static_cast<uint32_t>(min(max(e, -113), 100) + 127) << 23);
        float sums[G] = {};
#pragma unroll
        for (int j = 0; j < W; ++j) {
            float hi[8], lo[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = x[j][i] * up;
                hi[i] = __half2float(__float2half_rn(y));
                lo[i] = y - hi[i];
                sums[j / 2] += SPLIT ? y : hi[i];
            }
#pragma unroll
            for (int s = 0; s < QS; ++s) {
                const float* y = s == 0 ? hi : lo;
                qb[n][s][j][0] = pack_half2(y[0], y[4]);
                qb[n][s][j][1] = pack_half2(y[1] * 0.0625f, y[5] * 0.0625f);
                qb[n][s][j][2] = pack_half2(y[2], y[6]);
                qb[n][s][j][3] = pack_half2(y[3] * 0.0625f, y[7] * 0.0625f);
            }
        }
#pragma unroll
        for (int i = 0; i < G; ++i) {
            sums[i] += __shfl_xor_sync(~0u, sums[i], 1);
            sums[i] += __shfl_xor_sync(~0u, sums[i], 2);
            sums[i] *= 0x1p-24f;
            qsum[n][i][0] = __shfl_sync(~0u, sums[i], 8 * t);
            qsum[n][i][1] = __shfl_sync(~0u, sums[i], 8 * t + 4);
        }
        const float back = p.c * 0x1p24f / up;
        factor[n][0] = __shfl_sync(~0u, back, 8 * t);
        factor[n][1] = __shfl_sync(~0u, back, 8 * t + 4);
        const int mine = in ? attn_limit(static_cast<int>(m), ql, kl, p.causal) : 0;
        lim[n][0] = __shfl_sync(~0u, mine, 8 * t);
        lim[n][1] = __shfl_sync(~0u, mine, 8 * t + 4);
        lim_first = min(lim_first, in ? mine : kl);
    }
#pragma unroll
    for (int d = 4; d < 32; d *= 2) lim_first = min(lim_first, __shfl_xor_sync(~0u, lim_first, d));

    // p carries 2^(7 - E), E the exponent of the largest |m| or s so far.
    float o[NQ][W][2][4] = {}, least[NQ][G][2] = {}, sum[NQ][2] = {}, top[NQ][2], ref[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) top[n][0] = top[n][1] = -INFINITY, ref[n][0] = ref[n][1] = INFINITY;
    int exponent = kLeastExponent;                     // of bf16 numbers; E = exponent - 126
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int k = 0; k < steps; ++k) {
        if (!__all_sync(~0u, mbar_try_wait(&full[warp][stage], phase))) {
            ok = __all_sync(~0u, mbar_wait_bounded(&full[warp][stage], phase, nullptr, p.status));
            if (!ok) break;
        }
        const char* at = ring + stage * K::kStageBytes;
        const int n0 = (s0 + warp + kWarps * k) << 5;
        const uint32_t lost = (bad >> (2 * stage)) & 3u;
        const bool edge = n0 + 32 > lim_first;

        // S^T: rows are keys n0 + 16 z + g and + 8.
        float x[2][NQ][4];                             // key g + 8 (e / 2), query 2 t + e % 2
        uint32_t vgrp[2][2][G];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            const char* block = at + z * K::kBlockBytes;
            uint32_t kw[2][W], kgrp[2][G];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                load_words<4 * W>(kw[i], block + (g + 8 * i) * 16 * W + t * 4 * W);
                load_words<4 * G>(kgrp[i], block + 512 * W + (g + 8 * i) * 4 * G);
                load_words<4 * G>(vgrp[z][i], block + 512 * W + 64 * G + (g + 8 * i) * 4 * G);
            }
#pragma unroll
            for (int u = 0; u < G; ++u) {
                float acc[NQ][QS][4] = {};
#pragma unroll
                for (int j = 2 * u; j < W && j < 2 * u + 2; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t w0 = kw[0][j] >> (8 * h), w1 = kw[1][j] >> (8 * h);
#pragma unroll
                        for (int n = 0; n < NQ; ++n)
#pragma unroll
                            for (int s = 0; s < QS; ++s)
                                mma16816(acc[n][s], w0 & 0x000f000fu, w1 & 0x000f000fu, w0 & 0x00f000f0u,
                                         w1 & 0x00f000f0u, qb[n][s][j][2 * h], qb[n][s][j][2 * h + 1]);
                    }
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float sum_q = qsum[n][u][e & 1];
                        const float low = u == 0 ? high_bf16(kgrp[e / 2][u]) * sum_q
                                                 : fmaf(high_bf16(kgrp[e / 2][u]), sum_q, x[z][n][e]);
                        x[z][n][e] = fmaf(low_bf16(kgrp[e / 2][u]),
                                          SPLIT ? acc[n][0][e] + acc[n][QS - 1][e] : acc[n][0][e], low);
                    }
            }
        }
        float arg[2][NQ][4], most = -INFINITY;
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) arg[z][n][e] = fmaf(x[z][n][e], factor[n][e & 1], ref[n][e & 1]);
        if (edge || lost) {
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int key = n0 + 16 * z + g + 8 * i;
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 2 * i; e < 2 * i + 2; ++e) {
                            if ((lost >> z) & 1u) x[z][n][e] = arg[z][n][e] = NAN;
                            if (key >= lim[n][e & 1]) arg[z][n][e] = -INFINITY;
                        }
                    if (key >= kl || ((lost >> z) & 1u))
#pragma unroll
                        for (int u = 0; u < G; ++u) vgrp[z][i][u] = 0;
                }
        }
        // The values' sizes, a quarter of them per lane t (padding that lies in a block counts
        // here, but not past the slow path).
        uint32_t w[G];
        load_words<4 * G>(w, at + (t >> 1) * K::kBlockBytes + 512 * W + 64 * G + (g + 8 * (t & 1)) * 4 * G);
        uint32_t size = w[0] & 0x7fff7fffu;
#pragma unroll
        for (int u = 1; u < G; ++u) size = __vmaxu2(size, w[u] & 0x7fff7fffu);
        size = max(size & 0xffffu, size >> 16);
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) most = fmaxf(most, arg[z][n][e]);
        if (__any_sync(~0u, most > kSlack + kShift - (exponent - 126) ||
                                size >= static_cast<uint32_t>(exponent + 1) << 7)) {
            uint32_t largest = 0;                      // other than NaN and infinities
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int u = 0; u < G; ++u) {
                        const uint32_t lo = vgrp[z][i][u] & 0x7fffu, hi = (vgrp[z][i][u] >> 16) & 0x7fffu;
                        largest = max(largest, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
                    }
            const int to = min(max(exponent, static_cast<int>(__reduce_max_sync(~0u, largest) >> 7)), kMostExponent);
            const float f_e = __uint_as_float(static_cast<uint32_t>(max(127 + exponent - to, 0)) << 23);
            exponent = to;
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                float f_q[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float mt = -INFINITY;
#pragma unroll
                    for (int z = 0; z < 2; ++z)
#pragma unroll
                        for (int e = i; e < 4; e += 2)
                            if (arg[z][n][e] != -INFINITY) mt = fmaxf(mt, x[z][n][e] * factor[n][i]);
#pragma unroll
                    for (int d = 4; d < 32; d *= 2) mt = fmaxf(mt, __shfl_xor_sync(~0u, mt, d));
                    const bool up = mt > top[n][i] + kSlack;
                    f_q[i] = up ? ex2_approx(top[n][i] - mt) * f_e : f_e;        // 0 from -inf
                    if (up) top[n][i] = mt;
                    ref[n][i] = kShift - top[n][i] - (exponent - 126);
                    sum[n][i] *= f_q[i];
#pragma unroll
                    for (int u = 0; u < G; ++u) least[n][u][i] *= f_q[i];
                }
#pragma unroll
                for (int j = 0; j < W; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[n][j][h][e] *= f_q[e & 1];
#pragma unroll
                for (int z = 0; z < 2; ++z)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (arg[z][n][e] != -INFINITY)
                            arg[z][n][e] = fmaf(x[z][n][e], factor[n][e & 1], ref[n][e & 1]);
            }
        }

        // out^T += (codes of the values - 8)^T (p s)^T: lane (g, t) holds keys 2 t, 2 t + 1, + 8, + 9
        // and channels 4 g .. 4 g + 3 of every 32.
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            const char* block = at + z * K::kBlockBytes;
            float pr[NQ][4];
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    pr[n][e] = ex2_approx(arg[z][n][e]);
                    sum[n][e & 1] += pr[n][e];
                }
            uint32_t vw[4][(W + 1) / 2];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                load_words<2 * W>(vw[i], block + 256 * W + (2 * t + (i & 1) + 8 * (i / 2)) * 16 * W + g * 2 * W);
#pragma unroll
            for (int u = 0; u < G; ++u) {
                const float st0 = low_bf16(vgrp[z][0][u]), st1 = low_bf16(vgrp[z][1][u]);
                const float m0 = fmaf(st0, 8.f, high_bf16(vgrp[z][0][u]));
                const float m1 = fmaf(st1, 8.f, high_bf16(vgrp[z][1][u]));
                uint32_t pb[NQ][QS][2];
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    const float y0 = pr[n][0] * st0, y1 = pr[n][1] * st0, y2 = pr[n][2] * st1, y3 = pr[n][3] * st1;
                    least[n][u][0] = fmaf(pr[n][0], m0, fmaf(pr[n][2], m1, least[n][u][0]));
                    least[n][u][1] = fmaf(pr[n][1], m0, fmaf(pr[n][3], m1, least[n][u][1]));
                    const uint32_t w0 = pack_half2(y0, y1), w1 = pack_half2(y2, y3);
                    pb[n][0][0] = transpose8(w0);
                    pb[n][0][1] = transpose8(w1);
                    if constexpr (SPLIT) {
                        const float2 h0 = __half22float2(*reinterpret_cast<const __half2*>(&w0));
                        const float2 h1 = __half22float2(*reinterpret_cast<const __half2*>(&w1));
                        pb[n][QS - 1][0] = transpose8(pack_half2(y0 - h0.x, y1 - h0.y));
                        pb[n][QS - 1][1] = transpose8(pack_half2(y2 - h1.x, y3 - h1.y));
                    }
                }
#pragma unroll
                for (int j = 2 * u; j < W && j < 2 * u + 2; ++j) {
                    const uint32_t pick = j & 1 ? 0x7632u : 0x5410u;
                    const uint32_t xa = __byte_perm(vw[0][j / 2], vw[1][j / 2], pick);
                    const uint32_t xb = __byte_perm(vw[2][j / 2], vw[3][j / 2], pick);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t a0 = (xa >> (8 * h)) & 0x000f000fu, a1 = (xa >> (8 * h)) & 0x00f000f0u;
                        uint32_t a2 = (xb >> (8 * h)) & 0x000f000fu, a3 = (xb >> (8 * h)) & 0x00f000f0u;
                        if constexpr (K::kCentreByProduct && !SPLIT) {
                            mma16816(o[0][j][h], kMinusEight, kMinusEight16, kMinusEight, kMinusEight16,
                                     pb[0][0][0], pb[0][0][1]);
                        } else {
                            a0 = add2(a0, kMinusEight), a1 = add2(a1, kMinusEight16);
                            a2 = add2(a2, kMinusEight), a3 = add2(a3, kMinusEight16);
                        }
#pragma unroll
                        for (int n = 0; n < NQ; ++n) {
                            if constexpr (SPLIT) {
                                // Products into zeros, added in fp32: the products' own sums
                                // cut what lies 2^-24 below their largest term.
                                float y[QS][4] = {};
#pragma unroll
                                for (int s = 0; s < QS; ++s)
                                    mma16816(y[s], a0, a1, a2, a3, pb[n][s][0], pb[n][s][1]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[n][j][h][e] += y[0][e] + y[QS - 1][e];
                            } else {
                                mma16816(o[n][j][h], a0, a1, a2, a3, pb[n][0][0], pb[n][0][1]);
                            }
                        }
                    }
                }
            }
        }
        __syncwarp();                                  // every lane has read the stage
        issue(k + f.stages, stage);
        if (++stage == f.stages) {
            stage = 0;
            phase ^= 1u;
        }
    }

    // Each warp's normalised rows and their log2-sum-exp2, then their join.
    __syncthreads();
    float* rows = reinterpret_cast<float*>(ring);
    float* lse = rows + K::kRows * 32 * W;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int d = 4; d < 32; d *= 2) {
                sum[n][i] += __shfl_xor_sync(~0u, sum[n][i], d);
#pragma unroll
                for (int u = 0; u < G; ++u) least[n][u][i] += __shfl_xor_sync(~0u, least[n][u][i], d);
            }
            const bool has = ok && sum[n][i] != 0.f;   // (NaN: a row of NaN scores)
            const float inv = has ? 1.f / sum[n][i] : 0.f;
            const int row = 8 * n + 2 * t + i;
            if (g == 0)
                lse[row] = !has ? -INFINITY : sum[n][i] != sum[n][i] ? sum[n][i]
                                                                     : top[n][i] - kShift + (exponent - 126) + log2f(sum[n][i]);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const float low = least[n][j / 2][i];
                float4 y;
                y.x = has ? fmaf(o[n][j][0][i], 0x1p24f, low) * inv : 0.f;
                y.y = has ? fmaf(o[n][j][0][2 + i], 0x1p20f, low) * inv : 0.f;
                y.z = has ? fmaf(o[n][j][1][i], 0x1p24f, low) * inv : 0.f;
                y.w = has ? fmaf(o[n][j][1][2 + i], 0x1p20f, low) * inv : 0.f;
                *reinterpret_cast<float4*>(rows + row * 32 * W + 32 * j + 4 * g) = y;
            }
        }
    }
    __syncthreads();
    const int stride = max(f.stages * K::kStageBytes, K::kJoinBytes) / 4;
    const float* all_rows = reinterpret_cast<const float*>(smem);
    constexpr int kLse = K::kRows * 32 * W;
    const bool split_out = p.splits > 1;
    const int64_t rows_all = p.R;
    const int64_t part = (static_cast<int64_t>(split) * p.B * p.Hk + bj) * p.R + r0;
    for (int row = warp; row < K::kRows; row += kWarps) {
        const int64_t r = r0 + row;
        if (r >= rows_all) break;
        float l[kWarps], ref = -INFINITY, total = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            l[w] = all_rows[w * stride + kLse + row];
            ref = fmaxf(ref, l[w]);
        }
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            // (Padding queries come out empty, whatever their row did.)
            l[w] = l[w] == -INFINITY || r >= rows_in ? 0.f : exp2f(l[w] - ref);
            total += l[w];
        }
        const float inv = total == 0.f ? 0.f : 1.f / total;
        const float l2 = total == 0.f ? -INFINITY : ref + log2f(total);
        const int64_t m = r / p.G;
        const int hq = j0 * p.G + static_cast<int>(r - m * p.G);
        const int64_t to = b * p.out.sb + m * p.out.sr + hq * p.out.sh;
        for (int ch = lane; ch < p.C; ch += 32) {
            float y = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w)
                if (l[w] != 0.f) y = fmaf(l[w], all_rows[w * stride + row * 32 * W + ch], y);
            y *= inv;
            if (split_out)
                p.part_o[(part + row) * p.C + ch] = y;
            else if (f.type == InType::F32)
                reinterpret_cast<float*>(p.out.p)[to + ch] = y;
            else if (f.type == InType::F16)
                reinterpret_cast<__half*>(p.out.p)[to + ch] = __float2half_rn(y);
            else
                reinterpret_cast<__nv_bfloat16*>(p.out.p)[to + ch] = __float2bfloat16_rn(y);
        }
        if (lane == 0) {
            if (split_out)
                p.part_l[part + row] = l2;
            else if (p.lse)
                p.lse[(static_cast<int64_t>(b) * p.H + hq) * p.M + m] = l2 * kLn2;
        }
    }
}

template <int W, int NQ, bool SPLIT>
cudaError_t launch(FewParams& f, cudaStream_t s) {
    using K = FewCfg<W, NQ>;
    const AttnParams& p = f.a;
    f.tiles_r = (p.R + K::kRows - 1) / K::kRows;
    // As many stages as leave every SM its blocks.
    constexpr int kRing = 227 * 1024 / K::kBlocksPerSm - 2048;
    f.stages = std::max(2, std::min(kMaxStages, kRing / kWarps / K::kStageBytes));
    const size_t smem = kWarps * static_cast<size_t>(std::max(f.stages * K::kStageBytes, K::kJoinBytes));
    auto kern = cache_few_kernel<W, NQ, SPLIT>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               static_cast<int>(smem));
    if (e != cudaSuccess) return e;
    const int64_t blocks = f.tiles_r * p.B * p.Hk * p.splits;
    note_launches(1);
    return launch_kernel(kern, dim3(static_cast<unsigned>(blocks)), kWarps * 32, smem, s, f);
}

template <int W>
cudaError_t launch_w(FewParams& f, cudaStream_t s) {
    const int rows = cache_few_rows(f.a, f.type);
    if (f.type == InType::F32) return launch<W, 1, true>(f, s);
    if (rows == 8) return launch<W, 1, false>(f, s);
    if (rows == 16) return launch<W, 2, false>(f, s);
    return launch<W, 4, false>(f, s);
}

}  // namespace

int cache_few_rows(const AttnParams& p, InType t) {
    return t == InType::F32 || p.R <= 8 ? 8 : p.R <= 16 ? 16 : 32;
}

int cache_few_blocks_per_sm(int rows) { return rows == 8 ? 4 : rows == 16 ? 3 : 2; }

bool cache_few_takes(const CacheParams& c) { return c.kw == c.vw && c.kw <= 4; }

cudaError_t launch_cache_few(const AttnParams& p, const CacheParams& c, InType t, cudaStream_t s) {
    FewParams f{};
    f.a = p;
    f.c = c;
    f.type = t;
    if (c.kw == 1) return launch_w<1>(f, s);
    if (c.kw == 2) return launch_w<2>(f, s);
    if (c.kw == 3) return launch_w<3>(f, s);
    return launch_w<4>(f, s);
}

}  // namespace gs
