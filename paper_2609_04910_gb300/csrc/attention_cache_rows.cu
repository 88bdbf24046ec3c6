// Rows into and out of the 4-bit cache (include/gauss_sum/attention_cache.h).
//
// A lane takes eight channels of a row: one 32-bit word of its codes; eight
// lanes take a group, whose least and largest value three shuffles give.  Both
// kernels read and write every byte once; what bounds them is the instructions in between.  A block
// takes the tokens of one cache block (the same 16 places whatever the rows'
// offset), keys or values, and goes through a run of heads: a thread's row in the
// cache block, its page and its channels stay, and kRows heads are on their way
// before it works on the first (eight instead of four, as float32 numbers: 45 us read, not 41).
//
// 8 x 4096 tokens of 8 heads x 128, bf16, keys and values (134 MB as rows, 38 in the
// cache): written in 51 us (3.4 TB/s), bound by instructions (170 for eight values
// of a lane, 80 % of the issue slots; the conversion alone is 70); read in 34 us
// (5.1 TB/s; fp16 rows, which keep a second way for groups that fp16 does not hold, 41), issue
// slots at 64 % and the reads' latency.
#include <algorithm>
#include <type_traits>

#include "attention_cache.h"
#include "attention_simt.cuh"
#include "ptx.cuh"

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

// Eight channels from c0 on, of which `count` lie in the row; the others repeat the first.
template <bool VEC, typename E>
__device__ __forceinline__ Eight<E> load8(const E* src, int count) {
    if constexpr (VEC) {
        return *reinterpret_cast<const Eight<E>*>(src);
    } else {
        Eight<E> w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w.e[i] = src[i < count ? i : 0];
        return w;
    }
}

template <bool VEC, typename E>
__device__ __forceinline__ void store8(E* dst, const float (&x)[8], int count) {
    if constexpr (VEC) {
        Eight<E> w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w.e[i] = from_f<E>(x[i]);
        *reinterpret_cast<Eight<E>*>(dst) = w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) dst[i] = from_f<E>(x[i]);
    }
}

// m + s code of eight codes as pairs of E2 (s and m twice each), channels 2 i and 2 i + 1 in word i.
template <typename E2>
__device__ __forceinline__ uint4 values2(uint32_t word, uint32_t s, uint32_t m) {
    constexpr bool kHalf = std::is_same<E2, __half2>::value;
    constexpr uint32_t kOne = kHalf ? 0x64006400u : 0x43004300u;   // 1024, or 128: their codes in the low bits
    const uint32_t one = kOne;
    const auto as = [](const uint32_t& x) { return *reinterpret_cast<const E2*>(&x); };
    uint32_t y[4];                                                 // channels e and e + 4
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t v = ((word >> (4 * e)) & 0x000f000fu) | kOne;
        const E2 x = __hfma2(__hsub2(as(v), as(one)), as(s), as(m));
        y[e] = *reinterpret_cast<const uint32_t*>(&x);
    }
    return make_uint4(__byte_perm(y[0], y[1], 0x5410), __byte_perm(y[2], y[3], 0x5410),
                      __byte_perm(y[0], y[1], 0x7632), __byte_perm(y[2], y[3], 0x7632));
}

// low + s code for E: the nearest float32 number; for fp16, where it is rounded again, the one with an odd last
// bit of the two that it lies between, which no more lies on a border of fp16 numbers than the value does.
template <typename E>
__device__ __forceinline__ float value_of(float s, float code, float low) {
    if (!std::is_same<E, __half>::value) return fmaf(s, code, low);
    const float below = __fmaf_rd(s, code, low), above = __fmaf_ru(s, code, low);
    return __float_as_uint(below) & 1u ? below : above;
}
__device__ __forceinline__ bool is_half(float x) { return __half2float(__float2half_rn(x)) == x; }

template <bool VEC, typename E>
__device__ __forceinline__ void store_pairs(E* dst, const uint4& y, int count) {
    if constexpr (VEC) {
        *reinterpret_cast<uint4*>(dst) = y;
    } else {
        const E* x = reinterpret_cast<const E*>(&y);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) dst[i] = x[i];
    }
}

// Least and largest of two numbers, NaN if either is.
__device__ __forceinline__ float min_nan(float a, float b) {
    float y;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// The same over eight values.
__device__ __forceinline__ void range8(const Eight<float>& w, float& least, float& most) {
    least = most = w.e[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        least = min_nan(least, w.e[i]);
        most = max_nan(most, w.e[i]);
    }
}
template <typename E>
__device__ __forceinline__ void range8(const Eight<E>& w, float& least, float& most) {
    using E2 = typename std::conditional<std::is_same<E, __half>::value, __half2, __nv_bfloat162>::type;
    const E2* x = reinterpret_cast<const E2*>(&w);
    const E2 l = __hmin2_nan(__hmin2_nan(x[0], x[1]), __hmin2_nan(x[2], x[3]));
    const E2 g = __hmax2_nan(__hmax2_nan(x[0], x[1]), __hmax2_nan(x[2], x[3]));
    least = min_nan(to_f(l.x), to_f(l.y));
    most = max_nan(to_f(g.x), to_f(g.y));
}

// Where a thread is: its problem, side (keys or values), token (< 0: none) and row (< 0: none).
struct Place {
    int b;
    bool values;
    int m, token, kl;
    int head, step, last; // first head, the step to the next, the end
    int lane, c0, count;  // lane of a row; its channels
    int words, width;
};

// (`turn`: of a block that goes through several cache blocks.)
__device__ __forceinline__ Place place(const CacheRows& r, int turn = 0) {
    Place p;
    p.values = blockIdx.y != 0;
    p.width = p.values ? r.c.C : r.c.D;
    p.words = p.values ? r.c.vw : r.c.kw;
    const int shift = p.words <= 1 ? 2 : p.words <= 2 ? 3 : p.words <= 4 ? 4 : 5;    // log2 of a row's lanes
    const int tokens = min(4, 8 - shift);            // log2 of the tokens of a block (256 threads)
    p.b = static_cast<int>(blockIdx.x / r.grid_b);
    const int in_b = static_cast<int>(blockIdx.x - static_cast<unsigned>(p.b) * r.grid_b);
    p.kl = r.k_len ? min(max(r.k_len[p.b], 0), static_cast<int>(r.c.N)) : static_cast<int>(r.c.N);
    const int ql = r.all ? p.kl : r.q_len ? min(max(r.q_len[p.b], 0), r.M) : r.M;
    const int tile = r.head_blocks == 1 ? in_b : in_b / r.head_blocks, part = in_b - tile * r.head_blocks;
    const int row = threadIdx.x >> shift;
    // Row m is token m - ql + kl, also where it has no place (the shift rounds down).
    const int64_t off = static_cast<int64_t>(p.kl) - ql;
    const int64_t token = (((off >> tokens) + tile + static_cast<int64_t>(turn) * r.tiles) << tokens) +
                          (row & ((1 << tokens) - 1));
    const int64_t m = token - off;
    p.m = m >= 0 && m < r.M ? static_cast<int>(m) : -1;
    p.token = p.m >= 0 && p.m < ql && token >= 0 ? static_cast<int>(token) : -1;
    p.step = kThreads >> shift >> tokens;
    p.head = part * r.part_heads + (row >> tokens);
    p.last = min(r.heads, (part + 1) * r.part_heads);
    p.lane = threadIdx.x & ((1 << shift) - 1);
    p.c0 = p.lane * 8;
    p.count = p.width - p.c0;
    return p;
}

// Address of the cache block of a token in a page, for head 0.
__device__ __forceinline__ char* block_of(const CacheParams& c, int page, int token) {
    const int in_page = c.shift >= 0 ? token & (c.tokens - 1) : token % c.tokens;
    return c.data + page * c.sp + static_cast<int64_t>(in_page >> 4) * c.block_bytes;
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

// x / 15, correctly rounded where the result is a normal number (checked for every mantissa).
__device__ __forceinline__ float fifteenth(float x) {
    constexpr float kInv = 1.f / 15.f;
    const float q = __fmul_rn(x, kInv);
    return fmaf(fmaf(-15.f, q, x), kInv, q);
}

// Codes of eight values: (x - low) scale / step to the nearest, ties to even, four bits each.
//
// One Newton step on the product with the inverse gives the correctly rounded quotient, and that lies on a half only where the exact one does:
// y and (k + 1/2) s that differ at all differ by 2^-23 / mantissa(y) of their size, more than the
// half unit 2^-24 / mantissa(k + 1/2) of the quotient.  The addition of 1.5 x 2^23 then
// rounds as the definition does and leaves the code in the low bits.
// (The inverse is within a unit of its last place, for steps of 2^-60 .. 2^100.)
template <typename E>
__device__ __forceinline__ uint32_t codes8(const Eight<E>& w, float low, float step) {
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(step));
    uint32_t word = 0;
#pragma unroll
    for (int e = 7; e >= 0; --e) {
        const float y = __fsub_rn(to_f(w.e[e]), low), q = __fmul_rn(y, inv);
        word = word * 16u + __float_as_uint(fmaf(fmaf(-q, step, y), inv, q) + 12582912.f);
    }
    return word - 0x4b400000u * 0x11111111u;
}
// The same for other steps, of values and steps times a power of two: the remainders stay inside
// float32.
template <typename E>
__device__ __noinline__ uint32_t codes8_far(Eight<E> w, float low, float step) {
    const float scale = step < 1.f ? 0x1p60f : 0x1p-60f;
    Eight<float> x;
    for (int e = 0; e < 8; ++e) x.e[e] = __fsub_rn(to_f(w.e[e]), low) * scale;
    return codes8(x, 0.f, step * scale);
}

template <bool VEC, typename E>
__device__ __forceinline__ void write_rows(const CacheRows& r, const Place& p, const Arr& in) {
    const CacheParams& c = r.c;
    const int page = p.token >= 0 ? cache_page(c, p.b, p.token) : kNoPage;
    const bool there = page != kNoPage, on = p.count > 0, word_on = p.lane >> 2 < p.words;
    const int last = p.last;
    const int row = p.token & 15, j = p.lane >> 2, t = p.lane & 3;
    // (Places that nothing is written to stand for address 0.)
    char* block = there ? block_of(c, page, p.token) : nullptr;
    const int codes = codes_at(c, p.values, row) + (p.values ? 2 * (2 * t * p.words + j) : 4 * (t * p.words + j));
    const int group = groups_at(c, p.values, row) + 4 * (p.lane >> 3);
    const E* src = reinterpret_cast<const E*>(in.p) + p.b * in.sb + (p.m < 0 ? 0 : p.m) * in.sr + p.c0;
    const bool half_group = p.words == 1;
    if (!__any_sync(~0u, there)) return;
    src += p.head * in.sh;
    char* to = block + p.head * c.sh + codes;
    const int64_t src_step = p.step * in.sh, to_step = p.step * c.sh;
    const bool store = there && word_on, store_group = store && on && (p.lane & 7) == 0;
    // (A warp's rows are of the same head.)
    for (int h0 = p.head; h0 < last; h0 += kRows * p.step) {
        Eight<E> w[kRows] = {};
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (there && on && h0 + i * p.step < last) w[i] = load8<VEC>(src, p.count);
            src += src_step;
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (h0 + i * p.step >= last) break;
            float least, most;
            range8(w[i], least, most);
            if (!on) least = INFINITY, most = -INFINITY;
#pragma unroll
            for (int d = 1; d < 8; d *= 2) {      // (a row of four lanes has one half group)
                const float l = __shfl_xor_sync(~0u, least, d), g = __shfl_xor_sync(~0u, most, d);
                if (d < 4 || !half_group) {
                    least = min_nan(least, l);
                    most = max_nan(most, g);
                }
            }
            const float low = floor_bf16(least) + 0.f;         // (-0 becomes 0)
            float s = __bfloat162float(__float2bfloat16_rn(fifteenth(__fsub_rn(most, low))));
            if (s < 0x1p-126f) s = 0.f;
            // (A NaN or an infinity among the values makes s one; a group without values is not stored.)
            const bool fine = s <= 3.402823466e38f, some = fine && s > 0.f && on;
            uint32_t word = codes8(w[i], low, s);
            if (some && (s < 0x1p-60f || s > 0x1p100f)) word = codes8_far(w[i], low, s);
            if (!VEC && p.count < 8) word &= (1u << (4 * max(p.count, 0))) - 1u;
            word = some ? word : 0u;
            if (store) {
                if (p.values) {
                    *reinterpret_cast<uint16_t*>(to) = static_cast<uint16_t>(word);
                    *reinterpret_cast<uint16_t*>(to + 2 * p.words) = static_cast<uint16_t>(word >> 16);
                } else {
                    *reinterpret_cast<uint32_t*>(to) = word;
                }
            }
            if (store_group)
                *reinterpret_cast<uint32_t*>(to + (group - codes)) =
                    fine ? __byte_perm(__float_as_uint(s), __float_as_uint(low), 0x7632) : kNanGroup;
            to += to_step;
        }
    }
}

template <typename E>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(const __grid_constant__ CacheRows r) {
    pdl_wait();
    const Place p = place(r);
    const Arr& in = p.values ? r.v : r.k;
    if (p.values ? r.vec_v : r.vec_k)
        write_rows<true, E>(r, p, in);
    else
        write_rows<false, E>(r, p, in);
}

template <bool VEC, typename E>
__device__ __forceinline__ void read_rows(const CacheRows& r, const Place& p, const Arr& out) {
    const CacheParams& c = r.c;
    if (p.count <= 0 || p.m < 0 || (r.all && p.token < 0)) return;
    const int page = p.token >= 0 ? cache_page(c, p.b, p.token) : kNoPage;
    const int last = p.last;
    const int row = p.token & 15, j = p.lane >> 2, t = p.lane & 3;
    const char* block = page != kNoPage ? block_of(c, page, p.token) + r.head0 * c.sh : nullptr;
    const int codes = codes_at(c, p.values, row) + (p.values ? 2 * (2 * t * p.words + j) : 4 * (t * p.words + j));
    const int group = groups_at(c, p.values, row) + 4 * (p.lane >> 3);
    E* dst = reinterpret_cast<E*>(out.p) + p.b * out.sb + p.m * out.sr + p.head * out.sh + p.c0;
    const char* at = block + p.head * c.sh + codes;
    const int64_t dst_step = p.step * out.sh, at_step = p.step * c.sh;
    const uint2* sizes = r.sizes ? r.sizes + static_cast<int64_t>(p.b) * r.heads : nullptr;
    for (int h0 = p.head; h0 < last; h0 += kRows * p.step) {
        uint32_t word[kRows], pair[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            word[i] = 0;
            pair[i] = p.token >= 0 ? kNanGroup : 0u;
            if (block && h0 + i * p.step < last) {
                if (p.values)
                    word[i] = *reinterpret_cast<const uint16_t*>(at) |
                              static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(at + 2 * p.words)) << 16;
                else
                    word[i] = *reinterpret_cast<const uint32_t*>(at);
                pair[i] = *reinterpret_cast<const uint32_t*>(at + (group - codes));
            }
            at += at_step;
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (h0 + i * p.step >= last) break;
            if constexpr (std::is_same<E, __nv_bfloat16>::value) {
                // (Steps, least values and codes are bf16 numbers: one multiply-add rounds once.)
                store_pairs<VEC>(dst, values2<__nv_bfloat162>(word[i], __byte_perm(pair[i], 0, 0x1010),
                                                              __byte_perm(pair[i], 0, 0x3232)), p.count);
            } else {
                const float s = __uint_as_float(pair[i] << 16), low = __uint_as_float(pair[i] & 0xffff0000u);
                if (std::is_same<E, __half>::value && sizes) {
                    // (And fp16 numbers once scaled, those below 2^-27 of the head's largest value
                    // rounded to multiples of 2^-37 of it.)
                    const uint2 size = sizes[h0 + i * p.step];
                    const float down = __uint_as_float(
                        static_cast<uint32_t>(127 - scaled_exponent(p.values ? size.y : size.x)) << 23);
                    store_pairs<VEC>(dst, values2<__half2>(word[i], pack_half2(s * down, s * down),
                                                           pack_half2(low * down, low * down)), p.count);
                } else if (std::is_same<E, __half>::value && is_half(s) && is_half(low)) {
                    store_pairs<VEC>(dst, values2<__half2>(word[i], pack_half2(s, s), pack_half2(low, low)), p.count);
                } else {
                    // Pairs of codes as fp16 numbers 1024 + code, four channels apart.
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t v = ((word[i] >> (4 * e)) & 0x000f000fu) | 0x64006400u;
                        const float2 code =
                            __half22float2(__hsub2(*reinterpret_cast<const __half2*>(&v), __float2half2_rn(1024.f)));
                        x[e] = value_of<E>(s, code.x, low);
                        x[4 + e] = value_of<E>(s, code.y, low);
                    }
                    store8<VEC>(dst, x, p.count);
                }
            }
            dst += dst_step;
        }
    }
}

template <typename E>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const __grid_constant__ CacheRows r) {
    pdl_wait();
    for (int turn = 0; turn < r.turns; ++turn) {
        const Place p = place(r, turn);
        const Arr& out = p.values ? r.v : r.k;
        // (All tokens of a problem that has room for many more than it holds.)
        if (!out.p || (r.all && static_cast<int64_t>(turn) * r.tiles * 8 >= p.kl)) return;
        if (p.values ? r.vec_v : r.vec_k)
            read_rows<true, E>(r, p, out);
        else
            read_rows<false, E>(r, p, out);
    }
}

constexpr int kScanTokens = 1024;        // of a block of the scan
constexpr int kScaleHeads = 16, kScaleRows = 4;

template <typename E>
struct alignas(4 * sizeof(E)) Four {
    E e[4];
};

// Blocks below scan_blocks take the sizes of kScanTokens tokens of one problem and head, the others
// query rows.
template <typename E>
__global__ void __launch_bounds__(kThreads) cache_scale_kernel(const __grid_constant__ CacheScale r) {
    pdl_wait();
    const CacheParams& c = r.c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (blockIdx.x < r.scan_blocks) {
        const int bh = static_cast<int>(blockIdx.x / r.chunks), at = static_cast<int>(blockIdx.x) - bh * r.chunks;
        const int u0 = 2 * (at / r.token_chunks), chunk = at % r.token_chunks;    // first group, tokens
        const int b = bh / r.heads, h = bh - b * r.heads;
        const int kl = r.k_len ? min(max(r.k_len[b], 0), static_cast<int>(c.N)) : static_cast<int>(c.N);
        const int end = static_cast<int>(min(static_cast<int64_t>(chunk + 1) * kScanTokens, static_cast<int64_t>(kl)));
        // All pages of a thread's tokens, then two groups of each side, then the maxima.
        constexpr int kEach = kScanTokens / kThreads;
        uint32_t most[2] = {0, 0};
        int page[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int n = chunk * kScanTokens + i * kThreads + threadIdx.x;
            page[i] = n < end ? cache_page(c, b, n) : kNoPage;
        }
        uint32_t w[kEach][4] = {};
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int n = chunk * kScanTokens + i * kThreads + threadIdx.x;
            if (page[i] == kNoPage) continue;
            const char* block = block_of(c, page[i], n) + (r.head0 + h) * c.sh;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (u0 + (u & 1) < (u < 2 ? c.kg : c.vg))
                    w[i][u] = reinterpret_cast<const uint32_t*>(block + groups_at(c, u >= 2, n & 15))[u0 + (u & 1)];
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t s = w[i][u] & 0x7fffu, m = (w[i][u] >> 16) & 0x7fffu;   // (16 s: four exponents up)
                if (s < 0x7f80u && m < 0x7f80u) most[u >> 1] = max(most[u >> 1], max(s ? s + (4u << 7) : 0u, m));
            }
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            most[z] = __reduce_max_sync(~0u, most[z]);
            if (lane == 0 && most[z]) atomicMax(&(z ? r.sizes[bh].y : r.sizes[bh].x), most[z]);
        }
        return;
    }
    // A warp takes up to kScaleHeads heads of one token, four channels a lane (D <= 128), kScaleRows heads
    // read before the first is used: 2 x 1024 tokens of 32 heads x 128 with the scan of 8192 tokens of 8
    // heads 12 us; 19 with the place found row by row, 200 instructions of which half were its divisions
    // and products.
    const int H = r.heads * r.G, parts = (H + kScaleHeads - 1) / kScaleHeads;
    const int64_t item = static_cast<int64_t>(blockIdx.x - r.scan_blocks) * (kThreads / 32) + warp;
    const int64_t bm = divide(item, parts);
    const int b = static_cast<int>(divide(bm, r.M)), m = static_cast<int>(bm - static_cast<int64_t>(b) * r.M);
    if (b >= r.B) return;
    const int ql = r.q_len ? min(max(r.q_len[b], 0), r.M) : r.M;
    if (m >= ql) return;                               // (padding is not read)
    const int first = static_cast<int>(item - bm * parts) * kScaleHeads, last = min(first + kScaleHeads, H);
    const int c0 = 4 * lane;
    const E* src = reinterpret_cast<const E*>(r.q.p) + b * r.q.sb + m * r.q.sr + first * r.q.sh + c0;
    uint16_t* dst = r.q16 + (bm * H + first) * r.width + c0;
    float* scale = r.row_scale + (static_cast<int64_t>(b) * H + first) * r.M + m;
    for (int h0 = first; h0 < last; h0 += kScaleRows) {
        Four<E> w[kScaleRows];
#pragma unroll
        for (int i = 0; i < kScaleRows; ++i) {
            w[i] = Four<E>{};
            if (h0 + i < last) {
                if (r.vec) {
                    if (c0 < c.D) w[i] = *reinterpret_cast<const Four<E>*>(src);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (c0 + e < c.D) w[i].e[e] = src[e];
                }
            }
            src += r.q.sh;
        }
#pragma unroll
        for (int i = 0; i < kScaleRows; ++i) {
            if (h0 + i >= last) break;
            float x[4], top = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = to_f(w[i].e[e]);
                top = fmaxf(top, fabsf(x[e]));
            }
            top = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(top)));  // (top >= 0)
            // 2^e top in [2^14, 2^15), e in -113 .. 100.
            const int e = min(max(min(141 - static_cast<int>(__float_as_uint(top) >> 23), 100), -113), 100);
            const float up = __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
            if (c0 < r.width)                          // (whole multiples of eight)
                *reinterpret_cast<uint2*>(dst) = make_uint2(pack_half2(x[0] * up, x[1] * up), pack_half2(x[2] * up, x[3] * up));
            if (lane == 0) *scale = 1.f / up;
            dst += r.width;
            scale += r.M;
        }
    }
}

// Whether rows start on 16-byte boundaries and are whole vectors of eight.
bool eights(const Arr& a, int B, int M, int heads, int width, int es) {
    return width % 8 == 0 && reinterpret_cast<uintptr_t>(a.p) % 16 == 0 && (B == 1 || a.sb * es % 16 == 0) &&
           (M == 1 || a.sr * es % 16 == 0) && (heads == 1 || a.sh * es % 16 == 0);
}

// The heads in as many parts as give every SM four blocks, each thread kRows heads
// where there are enough.
cudaError_t plan(CacheRows& r, InType t, int sms, dim3* grid) {
    const int es = t == InType::F32 ? 4 : 2;
    r.vec_k = eights(r.k, r.B, r.M, r.heads, r.c.D, es);
    r.vec_v = eights(r.v, r.B, r.M, r.heads, r.c.C, es);
    const int words = std::max(r.c.kw, r.c.vw), least = std::min(r.c.kw, r.c.vw);
    const int tokens = words > 4 ? 8 : 16;                   // of a block, on the side that has fewer
    const int step = least <= 1 ? 4 : least <= 2 ? 2 : 1;    // heads at a time
    // Rows that do not start with a cache block take one block more.
    r.tiles = static_cast<int>((static_cast<int64_t>(r.M) + tokens - 1) / tokens + (r.all ? 0 : 1));
    r.turns = 1;
    if (r.all) {
        // At most 64 blocks an SM, however many tokens there is room for.
        const int64_t most = std::max<int64_t>(1, 64 * static_cast<int64_t>(sms) / r.B);
        r.turns = static_cast<int>((r.tiles + most - 1) / most);
        r.tiles = static_cast<int>((r.tiles + r.turns - 1) / r.turns);
    }
    r.part_heads = std::max(r.heads, 1);
    const auto blocks = [&]() {
        return static_cast<int64_t>(r.B) * r.tiles * ((r.heads + r.part_heads - 1) / r.part_heads);
    };
    while (r.part_heads > step && blocks() < 2 * sms) r.part_heads = (r.part_heads + 1) / 2;
    r.part_heads = (r.part_heads + step - 1) / step * step;
    r.head_blocks = (r.heads + r.part_heads - 1) / r.part_heads;
    r.grid_b = r.tiles * r.head_blocks;
    if (blocks() >= int64_t(1) << 31) return cudaErrorInvalidConfiguration;
    *grid = dim3(static_cast<unsigned>(blocks()), 2);
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

cudaError_t launch_cache_scale(CacheScale r, InType t, cudaStream_t s) {
    r.token_chunks = static_cast<int>(std::max<int64_t>(1, (r.c.N + kScanTokens - 1) / kScanTokens));
    r.chunks = r.token_chunks * ((std::max(r.c.kg, r.c.vg) + 1) / 2);
    const int64_t scan = static_cast<int64_t>(r.B) * r.heads * r.chunks;
    const int64_t items = static_cast<int64_t>(r.B) * r.M * ((r.heads * r.G + kScaleHeads - 1) / kScaleHeads);
    const int64_t blocks = scan + (items + kThreads / 32 - 1) / (kThreads / 32);
    r.vec = r.c.D % 4 == 0 && reinterpret_cast<uintptr_t>(r.q.p) % 8 == 0 && (r.B == 1 || r.q.sb % 4 == 0) &&
            (r.M == 1 || r.q.sr % 4 == 0) && (r.heads * r.G == 1 || r.q.sh % 4 == 0);
    if (blocks >= int64_t(1) << 31) return cudaErrorInvalidConfiguration;
    r.scan_blocks = static_cast<unsigned>(scan);
    const dim3 grid(static_cast<unsigned>(blocks));
    note_launches(1);
    if (t == InType::F16) return launch_kernel(cache_scale_kernel<__half>, grid, kThreads, 0, s, r);
    return launch_kernel(cache_scale_kernel<__nv_bfloat16>, grid, kThreads, 0, s, r);
}

}  // namespace gs
