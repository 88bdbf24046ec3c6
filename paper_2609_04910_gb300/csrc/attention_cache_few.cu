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
//   32 channels, fp32: 4.3e-5 without, 5.7e-6 before the parts of p s that are
//   summed exactly, 2e-6 before those of the queries; 5e-7 now).
//
// The products are mma.sync m16n8k16 with the codes as the 16-row operand in
// registers: S^T has keys as rows and queries as columns, out^T channels as rows;
// p s goes from the layout of a result to that of an operand by movmatrix.
// (tcgen05 would want the codes expanded to 16 bits in shared memory or TMEM: the
// kernel of many rows does that, in 75 us where this one takes 43 for 8 rows and
// 63 for 16, on 16 problems of 8192 tokens, 8 key heads x 128.  This card does 0.5
// m16n8k16 a clock and SM; 8 rows need 16 for 16 tokens, which HBM brings in 104
// clocks.)  Times here are of calls replayed from a graph where nothing else is said.
//
// Queries are scaled by a power of two per row to fp16 (exact down to 2^-28 of
// the row's largest); fp32 queries, and p s of such calls, are two fp16 numbers
// each (SPLIT), the first in fixed point.  p s 2^-E is rounded to fp16, E the
// exponent of the largest |m| or s that the warp has seen (p itself is scaled): it
// keeps fp16's 11 bits down to 2^-21 of the largest value and vanishes below 2^-32
// of it.  The running maximum lags by up to 2^6.
//
// A warp takes 32 tokens at a time through a ring of bulk copies of its own, no
// barrier between warps; their results are joined at the end of a set of rows
// (and those of several blocks by cache_join_kernel).
//
// What bounds it: the instructions of a block of 16 tokens, 300 a warp of which
// 140 on the ALU pipe (masks, shifts), at 2.2 issued a clock and SM; 64 problems
// of 8192 tokens run at 5.4 TB/s of the 6.75 that a copy does (copies alone, with
// the arithmetic taken out: 7).  Around that, 9 us of a call: lengths, page
// table, first tokens one after the other (4 us), the last block's join, the
// joining launch.  16 problems of 8191 .. 4352 tokens: 36 us with the join
// for 116 MB.  Tried: the -8 as a further product (24 of them, 6 % slower), four
// blocks an SM of 128 registers (8 % slower) and two (5 %), one block of 16 tokens
// at a time (6 %).
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
    int tiles_r;                    // tiles of 8 NQ rows
    int single;                     // a block takes whole sets of rows: no partial results
    int shared, sms;                // else: blocks that share the units, and SMs
    int stall;                      // test hook: block 0's first wait runs out
    int2* pieces;                   // of every set: its first block and its number of pieces
};

// Work is counted in units of 32 tokens: problem b has units_of(b) of them for
// each of its heads x tiles_r sets of rows.  Where sets are shared out, block i
// takes units [i len, (i + 1) len) of all, in the order (problem, tile and head,
// unit), whatever the lengths are.  A set of rows that lies in one block is
// written as it is; the others become partial results, in slot 2 i of block i
// when the piece starts inside the set, else in slot 2 i + 1.
//
// A block takes kMinUnits at least, and a set counts as that many, so that short
// ones do not queue up in one block while others are idle.
constexpr int kMinUnits = 8;

__device__ __forceinline__ int64_t units_of(int ql, int kl) {
    return ql > 0 ? max((static_cast<int64_t>(kl) + 31) / 32, static_cast<int64_t>(kMinUnits)) : kMinUnits;
}
__device__ __forceinline__ int64_t units_of(const AttnParams& p, int b) {
    return units_of(attn_q_len(p, b), attn_k_len(p, b));
}

// Units before this thread's first problem, and of all problems and the largest, for a block of
// kWarps warps of which thread i has problems [i m, (i + 1) m); `scan` has 2 kWarps words.
__device__ __forceinline__ int64_t scan_units(const AttnParams& p, int m, int64_t* scan, int64_t* all, int* most) {
    const int b0 = min(static_cast<int64_t>(threadIdx.x) * m, static_cast<int64_t>(p.B));
    const int b1 = min(b0 + static_cast<int64_t>(m), static_cast<int64_t>(p.B));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int64_t mine = 0;
    int top = 0;
    for (int b = b0; b < b1; ++b) {
        const int64_t n = units_of(p, b);
        mine += n;
        top = max(top, static_cast<int>(n));
    }
    int64_t sum = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int64_t y = __shfl_up_sync(~0u, sum, d);
        if (lane >= d) sum += y;
    }
    top = __reduce_max_sync(~0u, top);
    if (lane == 31) {
        scan[warp] = sum;
        scan[kWarps + warp] = top;
    }
    __syncthreads();
    int64_t before = 0;
    *all = 0;
    *most = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += scan[w];
        *all += scan[w];
        *most = max(*most, static_cast<int>(scan[kWarps + w]));
    }
    return before + sum - mine;
}

// Whether a block to a set is faster than equal shares: a warp takes 0.8, 0.85 or 0.95 us a unit (one, two,
// three blocks on an SM; a block has four warps), and shares cost about 8 us more for their pieces
// and the join.  Sets that do not all fit start as others end, so that the last one ends up to its own
// time after an equal share, half of it on average (`us` 16).  (One token, 8 key heads x 128, us of calls timed one by one: 64 problems
// of 900 tokens 35 and 43, of 1500 40 and 43, of 4096 77 and 67, of 8192 137 and 114; 8 of 1000
// tokens 16 and 24; 16 of 8191 .. 4352 tokens 42 shared, one block a set could not fill the card.)
__host__ __device__ __forceinline__ bool whole_sets(int64_t sets, int64_t units, int64_t most, int shared, int sms,
                                                    int us) {
    const int64_t rate = sets <= sms ? 80 : sets <= 2 * sms ? 85 : 95;
    return most * rate * shared - (sets <= shared ? units * 95 : 0) < int64_t(400) * us * shared;
}

// Units of a block of the grid.
__device__ __forceinline__ int64_t units_a_block(int64_t all, int64_t grid) {
    const int64_t len = divide(all + grid - 1, grid);
    return max((len + 3) / 4 * 4, static_cast<int64_t>(kMinUnits));
}

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The number whose addition and subtraction rounds numbers up to x >= 0 to multiples of 2^-10 of x's power of two
// (of 2^-24, the least fp16 number, at least).
__device__ __forceinline__ float rounder(float x) {
    const uint32_t e = min(max(__float_as_uint(x) >> 23, 113u), 230u);     // 2^-14 .. (NaN and infinity: any)
    return __uint_as_float((e + 13) << 23 | 0x400000u);                    // 1.5 x 2^(23 - 10) of its power of two
}
// The same for the x of all lanes with the same t.
__device__ __forceinline__ float column_rounder(float x) {
#pragma unroll
    for (int d = 4; d < 32; d *= 2) x = fmaxf(x, __shfl_xor_sync(~0u, x, d));
    return rounder(x);
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

// Channels 32 j + 8 t .. + 7 of a query row (null: zeros) for j < W, zeros past the width: read in one go,
// converted later.
template <int W, bool F32>
struct QueryRow {
    uint4 w[W][F32 ? 2 : 1];
    __device__ __forceinline__ void load(const char* row, const FewParams& f, int t) {
        const int D = f.a.D;
        constexpr int kPer = F32 ? 4 : 8;            // channels of a vector
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int z = 0; z < (F32 ? 2 : 1); ++z) {
                const int c0 = 32 * j + 8 * t + 4 * z;
                if (f.a.vec) {
                    w[j][z] = row && c0 < D ? *reinterpret_cast<const uint4*>(row + c0 * (16 / kPer)) : make_uint4(0, 0, 0, 0);
                    continue;
                }
                uint32_t e[kPer];
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const bool on = row && c0 + i < D;
                    if constexpr (F32)
                        e[i] = on ? reinterpret_cast<const uint32_t*>(row)[c0 + i] : 0u;
                    else
                        e[i] = on ? reinterpret_cast<const uint16_t*>(row)[c0 + i] : 0u;
                }
                if constexpr (F32)
                    w[j][z] = make_uint4(e[0], e[1], e[2], e[3]);
                else
                    w[j][z] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
            }
    }
    __device__ __forceinline__ void values(float (&x)[W][8], const FewParams& f) const {
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int z = 0; z < (F32 ? 2 : 1); ++z) {
                const uint32_t v[4] = {w[j][z].x, w[j][z].y, w[j][z].z, w[j][z].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (F32) {
                        x[j][4 * z + i] = __uint_as_float(v[i]);
                    } else if (f.type == InType::F16) {
                        const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&v[i]));
                        x[j][2 * i] = y.x, x[j][2 * i + 1] = y.y;
                    } else {
                        x[j][2 * i] = low_bf16(v[i]), x[j][2 * i + 1] = high_bf16(v[i]);
                    }
                }
            }
    }
};

// Channel ch, and the lse, of row r (all heads of a key head next to each other) of the outputs.
__device__ __forceinline__ void put_output(const FewParams& f, int b, int j, int r, int ch, float y) {
    const AttnParams& p = f.a;
    const int m = r / p.G;
    const int64_t at = b * p.out.sb + m * p.out.sr + static_cast<int64_t>(j * p.G + r - m * p.G) * p.out.sh + ch;
    if (f.type == InType::F32)
        reinterpret_cast<float*>(p.out.p)[at] = y;
    else if (f.type == InType::F16)
        reinterpret_cast<__half*>(p.out.p)[at] = __float2half_rn(y);
    else
        reinterpret_cast<__nv_bfloat16*>(p.out.p)[at] = __float2bfloat16_rn(y);
}
__device__ __forceinline__ void put_lse(const FewParams& f, int b, int j, int r, float l2) {
    const AttnParams& p = f.a;
    if (!p.lse) return;
    const int m = r / p.G;
    p.lse[(static_cast<int64_t>(b) * p.H + j * p.G + (r - m * p.G)) * p.M + m] = l2 * kLn2;
}

template <int W, int NQ>
struct FewCfg {
    static constexpr int kGroups = (W + 1) / 2;
    static constexpr int kRows = 8 * NQ;
    static constexpr int kBlockBytes = 16 * 2 * (16 * W + 4 * kGroups);
    static constexpr int kStageBytes = 2 * kBlockBytes;
    static constexpr int kBlocksPerSm = NQ == 1 ? 3 : 2;
    static constexpr int kRounds = NQ == 1 ? 1 : 2;    // of a unit: both its blocks at once, or one by one
    // Joining: rows of 32 W channels, and their lse, of every warp.
    static constexpr int kJoinBytes = (kRows * 32 * W + kRows) * 4;
};
constexpr int kMaxStages = 8;
// Exponent fields of bf16 numbers between which E moves: p 2^-E stays a normal
// float32 number, and values up to 2^102 are fine.  At the lower end (values of
// zero) p 2^(7 - E) is up to 2^106, and their sum fits for 2^22 keys a warp.
constexpr int kLeastExponent = 33, kMostExponent = 226;

template <int W, int NQ, bool SPLIT>
__global__ void __launch_bounds__(kWarps * 32, (FewCfg<W, NQ>::kBlocksPerSm))
cache_few_kernel(const __grid_constant__ FewParams f) {
    using K = FewCfg<W, NQ>;
    constexpr int G = K::kGroups, QS = SPLIT ? 2 : 1, Z = 2 / K::kRounds;
    const AttnParams& p = f.a;
    const CacheParams& c = f.c;
    extern __shared__ __align__(128) char smem[];
    __shared__ uint64_t full[kWarps][kMaxStages];
    __shared__ int64_t scan[2 * kWarps];
    __shared__ struct {
        int64_t at, left, units, len;                  // unit `at` of `units` of the set, units left, of a block
        int b, set, ql, kl;
    } work;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int key_row = g ^ ((g >> 1) & 1);
    char* ring = smem + warp * f.stages * K::kStageBytes;
    char* join = smem + kWarps * f.stages * K::kStageBytes;

    const int halves = (c.tokens >> 4) & 1;            // whether a unit may lie in two pages
    if (threadIdx.x == 0) {
        mbar_init(&full[0][0], 1 + halves + (blockIdx.x == 0 ? f.stall : 0));
#pragma unroll
        for (int i = 1; i < kWarps * kMaxStages; ++i) mbar_init(&full[0][0] + i, 1 + halves);
        fence_mbar_init();
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();

    // This block's units.
    const int64_t sets = static_cast<int64_t>(p.Hk) * f.tiles_r;
    if (f.single) {
        if (threadIdx.x == 0) {
            work.b = static_cast<int>(blockIdx.x / sets);
            work.set = static_cast<int>(blockIdx.x - work.b * sets);
            work.at = 0;
            work.ql = attn_q_len(p, work.b);
            work.kl = attn_k_len(p, work.b);
            work.left = work.units = units_of(work.ql, work.kl);
        }
    } else {
        const int m = (p.B + kWarps * 32 - 1) / (kWarps * 32);
        int64_t all;
        int most;
        int64_t before = scan_units(p, m, scan, &all, &most);
        all *= sets;
        const int64_t all_sets = p.B * sets;
        const bool whole = all_sets <= gridDim.x &&
                           whole_sets(all_sets, all, most, f.shared, f.sms, all_sets <= f.shared ? 8 : 16);
        if (whole && blockIdx.x >= all_sets) return;
        const int64_t len = units_a_block(all, f.shared), first = blockIdx.x * len;
        if (!whole && (blockIdx.x >= f.shared || first >= all)) return;
        if (whole && threadIdx.x == 0) {
            work.b = static_cast<int>(blockIdx.x / sets);
            work.set = static_cast<int>(blockIdx.x - work.b * sets);
            work.at = 0;
            work.ql = attn_q_len(p, work.b);
            work.kl = attn_k_len(p, work.b);
            work.left = work.units = units_of(work.ql, work.kl);
        }
        // The thread whose problems hold the first unit finds it.
        int b = min(static_cast<int64_t>(threadIdx.x) * m, static_cast<int64_t>(p.B));
        for (int i = 0; i < m && b < p.B; ++i, ++b) {
            const int ql = attn_q_len(p, b), kl = attn_k_len(p, b);
            const int64_t n = units_of(ql, kl), in_b = first - before * sets;
            if (!whole && in_b >= 0 && in_b < n * sets) {
                work.b = b;
                work.ql = ql;
                work.kl = kl;
                work.units = n;
                work.set = static_cast<int>(divide(in_b, n));
                work.at = in_b - work.set * n;
                work.left = min(len, all - first);
                work.len = len;
            }
            before += n;
        }
    }
    __syncthreads();
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    int b, j0, r0, rows_in, kend, s0, steps;           // of the piece at hand
    // Reads `work`; units that some row sees: s0 + warp + kWarps k, k < steps.
    const auto next_piece = [&]() {
        b = work.b;
        const int tile = work.set / p.Hk, ql = work.ql;
        j0 = work.set - tile * p.Hk;
        rows_in = ql * p.G;
        r0 = tile * K::kRows;
        const int last = min(r0 + K::kRows, rows_in) - 1;
        kend = last >= r0 ? attn_limit(last / p.G, ql, work.kl, p.causal) : 0;
        s0 = static_cast<int>(work.at);
        const int s1 = static_cast<int>(min(work.at + min(work.left, work.units - work.at),
                                            (static_cast<int64_t>(kend) + 31) / 32));
        steps = max(0, (s1 - s0 - warp + kWarps - 1) / kWarps);
    };

    // Copies.  In pages of whole units lane i brings the i-th of the next 32 units, else block i & 1
    // of the unit i / 2 of the next sixteen; the pages of those after them are read ahead.
    const int per_page = c.tokens >> 4;
    const auto block_at = [&](int k) {
        return 2 * (s0 + warp + kWarps * (k + (lane >> halves))) + (lane & halves);
    };
    const auto page_of = [&](int k) {
        const int i = block_at(k);
        return k + (lane >> halves) < steps && (i << 4) < kend ? cache_page(c, b, i << 4) : kNoPage;
    };
    int page_next = kNoPage;
    const char* src = nullptr;
    const auto issue = [&](int k, int stage) {
        if (k >= steps) return;
        const int turn = k & (31 >> halves);
        if (turn == 0) {
            const int i = block_at(k), in_page = c.shift >= 0 ? i & (per_page - 1) : i % per_page;
            src = page_next == kNoPage ? nullptr
                                       : c.data + j0 * c.sh + page_next * c.sp +
                                             static_cast<int64_t>(in_page) * K::kBlockBytes;
            page_next = page_of(k + (32 >> halves));
        }
        if ((lane >> halves) == turn) {
            uint64_t* bar = &full[warp][stage];
            char* to = ring + stage * K::kStageBytes + (lane & halves) * K::kBlockBytes;
            const uint32_t bytes = halves ? K::kBlockBytes : K::kStageBytes;
            if (src) {
                mbar_arrive_expect_tx(bar, bytes);
                bulk_load(to, src, bytes, bar);
            } else {
                // No page: keys of NaN (past the tokens none is looked at).
                for (uint32_t z = 0; z < bytes; z += K::kBlockBytes)
                    for (int w = 0; w < 32 * G; ++w)
                        reinterpret_cast<uint32_t*>(to + z + 512 * W)[w] = w < 16 * G ? kNanGroup : 0u;
                fence_proxy_async_smem();              // (before a copy to the same place)
                mbar_arrive(bar);
            }
        }
        __syncwarp();
    };
    const auto start = [&]() {
        for (int k = 0; k < f.stages; ++k) issue(k, stage + k < f.stages ? stage + k : stage + k - f.stages);
    };

    next_piece();
    page_next = page_of(0);
    bool started = false, lost;                        // lost: a wait ran out
    while (true) {
    const int ql = work.ql, kl = work.kl;
    // Queries: row 8 n + g as the second operand, scaled to at most 2^15.
    uint32_t qb[NQ][QS][W][4];
    float qsum[NQ][G][2], factor[NQ][2];               // of queries 2 t, 2 t + 1
    int lim[NQ][2];
    int lim_first = kl;                                // the least limit of a row of the tile
    QueryRow<W, SPLIT> query[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int r = r0 + 8 * n + g, m = r / p.G;
        const int64_t at = b * p.q.sb + m * p.q.sr + static_cast<int64_t>(j0 * p.G + r - m * p.G) * p.q.sh;
        query[n].load(r < rows_in ? p.q.p + at * (SPLIT ? 4 : 2) : nullptr, f, t);
    }
    if (!started) start();                             // (the first pages are read by now)
    started = true;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int r = r0 + 8 * n + g, m = r / p.G;
        const bool in = r < rows_in;
        float x[W][8], top = 0.f;
        query[n].values(x, f);
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[j][e]));
        top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
        top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
        // 2^e top in [2^14, 2^15), e in -113 .. 100 (an empty row: 100).
        const int e = min(141 - static_cast<int>(__float_as_uint(top) >> 23), 100);
        const float up = __uint_as_float(static_cast<uint32_t>(min(max(e, -113), 100) + 127) << 23);
        // (Of two parts the first is in multiples of 2^-10 of the row's largest: its products add up
        // without a rounding.)
        const float big = rounder(top * up);
        float sums[G] = {};
#pragma unroll
        for (int j = 0; j < W; ++j) {
            float hi[8], lo[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = x[j][i] * up;
                hi[i] = SPLIT ? __fsub_rn(__fadd_rn(y, big), big) : __half2float(__float2half_rn(y));
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
        const int mine = in ? attn_limit(m, ql, kl, p.causal) : 0;
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
    int k = 0;
    for (; k < steps; ++k) {
        if (!__all_sync(~0u, mbar_try_wait(&full[warp][stage], phase))) {
            ok = __all_sync(~0u, mbar_wait_bounded(&full[warp][stage], phase, nullptr, p.status));
            if (!ok) break;
        }
#pragma unroll 1
        for (int round = 0; round < K::kRounds; ++round) {
        const char* at = ring + stage * K::kStageBytes + (Z == 1 ? round * K::kBlockBytes : 0);
        const int n0 = (s0 + warp + kWarps * k) * 32 + 16 * round;
        const bool edge = n0 + 16 * Z > lim_first;

        // S^T: rows g and g + 8 are keys n0 + 16 z + row and + 8 (in an order that spreads the rows that the
        // value product reads together over the banks).
        float x[Z][NQ][4];                             // key g + 8 (e / 2), query 2 t + e % 2
        uint32_t vgrp[Z][2][G];
#pragma unroll
        for (int z = 0; z < Z; ++z) {
            const char* block = at + z * K::kBlockBytes;
            uint32_t kw[2][W], kgrp[2][G];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                load_words<4 * W>(kw[i], block + (key_row + 8 * i) * 16 * W + t * 4 * W);
                load_words<4 * G>(kgrp[i], block + 512 * W + (key_row + 8 * i) * 4 * G);
                load_words<4 * G>(vgrp[z][i], block + 512 * W + 64 * G + (key_row + 8 * i) * 4 * G);
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
        float arg[Z][NQ][4], most = -INFINITY;
#pragma unroll
        for (int z = 0; z < Z; ++z)
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) arg[z][n][e] = fmaf(x[z][n][e], factor[n][e & 1], ref[n][e & 1]);
        if (edge) {
#pragma unroll
            for (int z = 0; z < Z; ++z)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int key = n0 + 16 * z + key_row + 8 * i;
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 2 * i; e < 2 * i + 2; ++e)
                            if (key >= lim[n][e & 1]) arg[z][n][e] = -INFINITY;
                    if (key >= kl)
#pragma unroll
                        for (int u = 0; u < G; ++u) vgrp[z][i][u] = 0;
                }
        }
        // The values' sizes, a part of them per lane t (padding that lies in a block counts here,
        // but not past the slow path).
        uint32_t w[G];
        load_words<4 * G>(w, at + (Z == 2 ? (t >> 1) * K::kBlockBytes : 0) + 512 * W + 64 * G +
                                 (g + 8 * (t & 1)) * 4 * G);
        uint32_t size = w[0] & 0x7fff7fffu;
#pragma unroll
        for (int u = 1; u < G; ++u) size = __vmaxu2(size, w[u] & 0x7fff7fffu);
        size = max(size & 0xffffu, size >> 16);
#pragma unroll
        for (int z = 0; z < Z; ++z)
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) most = fmaxf(most, arg[z][n][e]);
        if (__any_sync(~0u, most > kSlack + kShift - (exponent - 126) ||
                                size >= static_cast<uint32_t>(exponent + 1) << 7)) {
            uint32_t largest = 0;                      // other than NaN and infinities
#pragma unroll
            for (int z = 0; z < Z; ++z)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int u = 0; u < G; ++u) {
                        const uint32_t lo = vgrp[z][i][u] & 0x7fffu, hi = (vgrp[z][i][u] >> 16) & 0x7fffu;
                        largest = max(largest, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
                    }
            // (One more than the block needs: larger blocks come.)
            const int need = static_cast<int>(__reduce_max_sync(~0u, largest) >> 7);
            const int to = min(need > exponent ? need + 1 : exponent, kMostExponent);
            if (to - exponent > 100) {
                // The sums of weights (2^100 a key and more where values were zero so far) take a step that is
                // longer than float32's range in two factors; 2^100 is enough for what it leaves of the
                // values' sums.
                const float f_far = __uint_as_float(static_cast<uint32_t>(127 + exponent - (to - 100)) << 23);
#pragma unroll
                for (int n = 0; n < NQ; ++n) sum[n][0] *= f_far, sum[n][1] *= f_far;
                exponent = to - 100;
            }
            const float f_e = __uint_as_float(static_cast<uint32_t>(127 + exponent - to) << 23);
            exponent = to;
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                float f_q[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float mt = -INFINITY;
#pragma unroll
                    for (int z = 0; z < Z; ++z)
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
                for (int z = 0; z < Z; ++z)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (arg[z][n][e] != -INFINITY)
                            arg[z][n][e] = fmaf(x[z][n][e], factor[n][e & 1], ref[n][e & 1]);
            }
        }

        // out^T += (codes of the values - 8)^T (p s)^T: lane (g, t) holds keys 2 t, 2 t + 1, + 8, + 9
        // and channels 4 g .. 4 g + 3 of every 32.
#pragma unroll
        for (int z = 0; z < Z; ++z) {
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
                load_words<2 * W>(vw[i], block + 256 * W + (((2 * t + (i & 1)) ^ (t & 1)) + 8 * (i / 2)) * 16 * W + g * 2 * W);
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
                    if constexpr (SPLIT) {
                        // The first part in multiples of 2^-10 of the column's largest (11 bits): its
                        // products add up without a rounding.  The second is the rest.
                        float h0, h1, h2, h3;
                        const float big0 = column_rounder(fmaxf(y0, y2)), big1 = column_rounder(fmaxf(y1, y3));
                        h0 = __fsub_rn(__fadd_rn(y0, big0), big0), h2 = __fsub_rn(__fadd_rn(y2, big0), big0);
                        h1 = __fsub_rn(__fadd_rn(y1, big1), big1), h3 = __fsub_rn(__fadd_rn(y3, big1), big1);
                        pb[n][0][0] = transpose8(pack_half2(h0, h1));
                        pb[n][0][1] = transpose8(pack_half2(h2, h3));
                        pb[n][QS - 1][0] = transpose8(pack_half2(y0 - h0, y1 - h1));
                        pb[n][QS - 1][1] = transpose8(pack_half2(y2 - h2, y3 - h3));
                    } else {
                        pb[n][0][0] = transpose8(pack_half2(y0, y1));
                        pb[n][0][1] = transpose8(pack_half2(y2, y3));
                    }
                }
#pragma unroll
                for (int j = 2 * u; j < W && j < 2 * u + 2; ++j) {
                    const uint32_t pick = j & 1 ? 0x7632u : 0x5410u;
                    const uint32_t xa = __byte_perm(vw[0][j / 2], vw[1][j / 2], pick);
                    const uint32_t xb = __byte_perm(vw[2][j / 2], vw[3][j / 2], pick);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t wa = xa >> (8 * h), wb = xb >> (8 * h);
                        const uint32_t a0 = add2(wa & 0x000f000fu, kMinusEight), a1 = add2(wa & 0x00f000f0u, kMinusEight16);
                        const uint32_t a2 = add2(wb & 0x000f000fu, kMinusEight), a3 = add2(wb & 0x00f000f0u, kMinusEight16);
#pragma unroll
                        for (int n = 0; n < NQ; ++n) {
                            if constexpr (SPLIT) {
                                // Into zeros, added in fp32: the products' own sums cut what lies
                                // 2^-24 below their largest term, always the same way.
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
        }
        __syncwarp();                                  // every lane has read the stage
        issue(k + f.stages, stage);
        if (++stage == f.stages) {
            stage = 0;
            phase ^= 1u;
        }
    }

    // (After a wait that ran out: the copies on their way still land before the block ends.)
    if (!ok)
        for (int i = 0; i < f.stages && k + i < steps; ++i) {
            mbar_wait_bounded(&full[warp][stage], phase, nullptr, p.status);
            if (++stage == f.stages) stage = 0, phase ^= 1u;
        }

    // The next piece's first copies run under the end of this one.
    const int b_of = b, j_of = j0, r_of = r0, rows_of = rows_in;
    const int64_t here = min(work.left, work.units - work.at);
    const bool whole = here == work.units;             // else a partial result
    const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (work.at == 0 ? 1 : 0);
    if (threadIdx.x == 0 && !f.single && work.at == 0)
        f.pieces[work.b * sets + work.set] =
            make_int2(blockIdx.x, whole ? 1 : 1 + static_cast<int>(divide(work.units - here + work.len - 1, work.len)));
    lost = __syncthreads_or(!ok);
    const bool more = !lost && work.left > here;
    if (more) {
        __syncthreads();
        if (threadIdx.x == 0) {
            work.left -= here;
            work.at = 0;
            if (++work.set == sets) {
                work.set = 0;
                ++work.b;
                work.ql = attn_q_len(p, work.b);
                work.kl = attn_k_len(p, work.b);
                work.units = units_of(work.ql, work.kl);
            }
        }
        __syncthreads();
        next_piece();
        page_next = page_of(0);
        start();
    }

    // Each warp's normalised rows and their log2-sum-exp2, then their join.
    float* rows = reinterpret_cast<float*>(join + warp * K::kJoinBytes);
    float* lse = rows + K::kRows * 32 * W;
    // A sum is in units of 2^(7 - E): taken off before the logarithm, which would else be some 100 for values
    // of zero and lose 2^-18 of itself.
    const float unit = __uint_as_float(static_cast<uint32_t>(127 + exponent - 126 - static_cast<int>(kShift)) << 23);
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
                lse[row] = !has ? -INFINITY : sum[n][i] != sum[n][i] ? sum[n][i] : top[n][i] + log2f(sum[n][i] * unit);
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
    constexpr int stride = K::kJoinBytes / 4;
    const float* all_rows = reinterpret_cast<const float*>(join);
    constexpr int kLse = K::kRows * 32 * W;
    for (int row = warp; row < K::kRows; row += kWarps) {
        const int r = r_of + row;
        if (r >= p.R) break;
        float l[kWarps], top_l = -INFINITY, total = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            l[w] = all_rows[w * stride + kLse + row];
            top_l = fmaxf(top_l, l[w]);
        }
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            // (Padding queries come out empty, whatever their row did.)
            l[w] = l[w] == -INFINITY || r >= rows_of ? 0.f : exp2f(l[w] - top_l);
            total += l[w];
        }
        const float inv = total == 0.f ? 0.f : 1.f / total;
        const float l2 = total == 0.f ? -INFINITY : top_l + log2f(total);
        for (int ch = lane; ch < p.C; ch += 32) {
            float y = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w)
                if (l[w] != 0.f) y = fmaf(l[w], all_rows[w * stride + row * 32 * W + ch], y);
            if (whole)
                put_output(f, b_of, j_of, r, ch, y * inv);
            else
                p.part_o[(slot * K::kRows + row) * p.C + ch] = y * inv;
        }
        if (lane == 0) {
            if (whole)
                put_lse(f, b_of, j_of, r, l2);
            else
                p.part_l[slot * K::kRows + row] = l2;
        }
    }
    if (!more) break;
    }
    if (lost && !f.single && threadIdx.x == 0) {
        // The sets that would have started here have no results, and nothing to join either.
        int64_t left = work.left - min(work.left, work.units - work.at);
        int of = work.b, set = work.set;
        while (left > 0) {
            if (++set == sets) set = 0, ++of;
            f.pieces[of * sets + set] = make_int2(blockIdx.x, 1);
            left -= units_of(p, of);
        }
    }
}

// Joins the pieces of a set of rows that lies in several blocks' units, a block per row: warp w sums
// the pieces w, w + kWarps, .. in order, and the warps' sums are added in order.
template <int ROWS>
__global__ void __launch_bounds__(kWarps * 32) cache_join_kernel(const __grid_constant__ FewParams f) {
    const AttnParams& p = f.a;
    __shared__ float sums[kWarps][129];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int sets = p.Hk * f.tiles_r;
    const int b = static_cast<int>(blockIdx.x / sets), set = static_cast<int>(blockIdx.x) - b * sets;
    const int tile = set / p.Hk, j0 = set - tile * p.Hk, row = blockIdx.y, r = tile * ROWS + row;
    if (r >= p.R) return;
    pdl_wait();
    const int2 piece = f.pieces[blockIdx.x];
    const int c0 = piece.x, n = piece.y;
    if (n == 1) return;
    // Slot of piece i: the second of its block's where the set starts in it.
    const auto at = [&](int i) { return (2 * static_cast<int64_t>(c0 + i) + (i == 0 ? 1 : 0)) * ROWS + row; };
    float top = -INFINITY;
    for (int i = lane; i < n; i += 32) top = fmaxf(top, p.part_l[at(i)]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
    const float ref = top == -INFINITY ? 0.f : top;
    float y[4] = {}, sum = 0.f;
    for (int i0 = warp; i0 < n; i0 += 4 * kWarps) {
        float w[4], x[4][4];
#pragma unroll
        for (int z = 0; z < 4; ++z) {
            const int i = i0 + z * kWarps;
            w[z] = i < n ? exp2f(p.part_l[at(i)] - ref) : 0.f;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int ch = lane + 32 * u;
                x[z][u] = i < n && ch < p.C ? p.part_o[at(i) * p.C + ch] : 0.f;
            }
        }
#pragma unroll
        for (int z = 0; z < 4; ++z) {
#pragma unroll
            for (int u = 0; u < 4; ++u) y[u] = w[z] != 0.f ? fmaf(w[z], x[z][u], y[u]) : y[u];
            sum += w[z];
        }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) sums[warp][lane + 32 * u] = y[u];
    if (lane == 0) sums[warp][128] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) sum += sums[w][128];
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int ch = threadIdx.x;
    float out = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) out += sums[w][ch];
    if (ch < p.C) put_output(f, b, j0, r, ch, out * inv);
    if (ch == 0) put_lse(f, b, j0, r, sum == 0.f ? -INFINITY : ref + log2f(sum));
}

template <int W, int NQ, bool SPLIT>
cudaError_t launch(FewParams& f, int grid, cudaStream_t s) {
    using K = FewCfg<W, NQ>;
    const AttnParams& p = f.a;
    // As many stages as leave every SM its blocks.
    constexpr int kRing = 227 * 1024 / K::kBlocksPerSm - 2048;
    f.stages = std::max(2, std::min(kMaxStages, (kRing / kWarps - K::kJoinBytes) / K::kStageBytes));
    const size_t smem = kWarps * static_cast<size_t>(f.stages * K::kStageBytes + K::kJoinBytes);
    auto kern = cache_few_kernel<W, NQ, SPLIT>;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
    note_launches(1);
    e = launch_kernel(kern, dim3(static_cast<unsigned>(grid)), kWarps * 32, smem, s, f);
    if (e != cudaSuccess || f.single) return e;
    note_launches(1);
    return launch_kernel(cache_join_kernel<K::kRows>, dim3(static_cast<unsigned>(f.tiles_r * p.B * p.Hk), std::min<int64_t>(p.R, K::kRows)),
                         kWarps * 32, 0, s, f);
}

template <int W>
cudaError_t launch_w(FewParams& f, const FewPlan& plan, cudaStream_t s) {
    if (f.type == InType::F32) return launch<W, 1, true>(f, plan.grid, s);
    if (plan.rows == 8) return launch<W, 1, false>(f, plan.grid, s);
    return launch<W, 2, false>(f, plan.grid, s);
}

}  // namespace

bool cache_few_takes(const CacheParams& c) { return c.kw == c.vw && c.kw <= 4; }

bool plan_cache_few(const AttnParams& p, InType t, int sms, FewPlan* plan) {
    plan->rows = t == InType::F32 || p.R <= 8 ? 8 : 16;
    const int64_t tiles = (p.R + plan->rows - 1) / plan->rows, sets = tiles * p.B * p.Hk;
    if (sets >= int64_t(1) << 31) return false;
    // One block to a set, and no join, where that costs 8 us at most whatever the lengths are (one
    // problem of all tokens among empty ones), or 16 where the sets fill the card; even lengths
    // are 5 us faster.
    plan->sms = sms;
    plan->shared = (plan->rows == 8 ? 3 : 2) * sms;
    plan->single = whole_sets(sets, 0, (static_cast<int64_t>(p.N) + 31) / 32, plan->shared, sms, sets <= 2 * sms ? 8 : 16);
    plan->grid = static_cast<int>(plan->single ? sets
                                  : sets <= 8 * plan->shared ? std::max<int64_t>(sets, plan->shared) : plan->shared);
    plan->slots = plan->single ? 0 : 2 * static_cast<size_t>(plan->shared) * plan->rows;
    plan->bytes = plan->single ? 0 : sets * sizeof(int2) + plan->slots * (p.C + 1) * sizeof(float);
    return true;
}

cudaError_t launch_cache_few(const AttnParams& p, const CacheParams& c, InType t, const FewPlan& plan, void* ws,
                             cudaStream_t s) {
    FewParams f{};
    f.a = p;
    f.c = c;
    f.type = t;
    f.tiles_r = static_cast<int>((p.R + plan.rows - 1) / plan.rows);
    f.single = plan.single;
    f.shared = plan.shared;
    f.sms = plan.sms;
    f.stall = testing_stall();
    if (!plan.single) {
        f.pieces = static_cast<int2*>(ws);
        f.a.part_o = reinterpret_cast<float*>(f.pieces + static_cast<size_t>(f.tiles_r) * p.B * p.Hk);
        f.a.part_l = f.a.part_o + plan.slots * p.C;
    }
    if (c.kw == 1) return launch_w<1>(f, plan, s);
    if (c.kw == 2) return launch_w<2>(f, plan, s);
    if (c.kw == 3) return launch_w<3>(f, plan, s);
    return launch_w<4>(f, plan, s);
}

}  // namespace gs
