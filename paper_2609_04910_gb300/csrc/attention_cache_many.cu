// Attention of many query rows over the 4-bit cache (drafts of several heads,
// parts of prompts) on the tensor cores: tcgen05, TMEM, bulk copies.
//
//   S  = q k^T          128 x 128 x D, A and B from shared memory, fp32 TMEM
//   P  = 2^(c S - m)    TMEM -> registers -> TMEM, fp16
//   O += P v            A = P from TMEM, B = the value tile, rows along the sum
//
// A block has 128 rows, all heads that share a key head next to each other, and
// two streams that take the even and the odd key tiles, each with its own
// softmax warpgroup, score tile and accumulator; the streams are joined at the
// end through shared memory.  Four warps for the keys and four for the values turn the cache's
// blocks, which another one brings by bulk copies, into swizzled fp16 tiles:
//
//   x & 0x000f000f is a pair of codes times 2^-24, x & 0x00f000f0 one times 2^-20,
//   and one fp16 multiply-add by s 2^(24 - E) (s 2^(20 - E)) and m 2^-E makes the
//   values times 2^-E; E puts the largest step of the tile into 2^-9 .. 2^-8, so
//   that the factors are fp16 numbers.  Values are rounded to fp16 (11 bits down
//   to 2^-5 of the largest step of the tile, multiples of 2^-15 of it below),
//   probabilities to fp16; both sums are fp32.
//
// Keys are exact: s (u - 8), which 11 bits hold (for steps down to 2^-9 of the tile's
// largest one), by the same multiply-add with -8 s; and the groups' centres m + 8 s times
// the sums of q over a group, as one more step of the product, 8 columns a group of bf16
// numbers, three for a centre and three for a sum (2^-25 of their product is left out).
// A row that sees few keys has no roundings to average: lse of 17 keys was 3e-5 off with
// keys rounded to 11 bits, and is 3e-7 now.
//
// At most 64 rows lie in a tile twice: the first copy takes the first half of every
// key tile, the second the other (its probabilities elsewhere are zero), so that a
// softmax thread has half the work and no warp is idle.  Copies have their own
// maximum, like streams, and are joined with them.
//
// K has an E of its own for every tile, which the scores' factor carries; V's E is
// the largest of the tiles so far, and a tile that raises it rescales O, as a
// moved maximum does.  Queries are scaled by a power of two a row to fp16, as in
// the kernel of few rows.  Channels lie in the order in which pairs of codes come
// out of a word: four apart in k (and q alike), 32 apart in v (undone at the end).
//
// What bounds it: the steps of a tile, which wait for one another, and the instruction
// caches.  16 problems of 8192 tokens, 8 key heads x 128, 64 rows (151 MB), replayed from a
// graph: 77 us, some 2000 clocks a tile of 128 keys, which HBM brings in 840; 128 rows 89
// us, 256 175.  Five roles' loops run at a time, and what does not fit the caches that they
// share makes all of them wait: with waits that report a time-out where they stand, and
// the softmax's code twice for the two halves of a tile, warps stood 3.6 times as long
// without an instruction as they issued (1.5 now), and 64 rows took 92 us.  (Taken apart
// when keys were still m + s u: E known after 600 clocks, 300 until the products have read
// the tile two before, 850 to convert and store, 400 to be heard; a stream's own chain 430
// for scores, 1400 .. 1800 softmax, 500 for values.)  The exact keys themselves cost nothing
// that shows.
// Shared memory moves 212 KB a tile, 1660 clocks at its 128 bytes.  Tried, before that: E
// from a warp of its own (115 us), V's E from the warps that fill it (4 us more), sleeping
// between polls (127 us), keys and values filled by the same warps (135 us), one copy of
// 64 rows (100 us).  And since: the centres by the value warps (64 rows 79 us, 128 rows 98) or by
// two warps of their own (105 us), the key warps' maxima a tile ahead (88 us).
#include <algorithm>

#include "attention_cache.h"
#include "attention_simt.cuh"
#include "attention_tc.cuh"

namespace gs {
namespace {

using namespace tc;

// Warps: two softmax warpgroups, one that fills key tiles and one that fills value tiles, and one with
// the copies' and the products' warps.
constexpr int kSoftmaxWarps = 8, kKeyWarp = 8, kValueWarp = 12, kFillWarps = 4, kLoadWarp = 16, kMmaWarp = 17;
constexpr int kThreads = 20 * 32;
constexpr int kRegsLaunch = 96, kRegsSoftmax = 144, kRegsFill = 72, kRegsCtrl = 48;
static_assert(kSoftmaxWarps * kRegsSoftmax + 2 * kFillWarps * kRegsFill + 4 * kRegsCtrl <= 20 * kRegsLaunch,
              "register split");
constexpr uint32_t kO = 256;              // TMEM: S of stream i at 128 i, O at kO + 128 i
constexpr float kMaxSlack = 8.f;          // log2 units the maximum may lag behind
constexpr float kShift = 7.f;
constexpr int kRawStages = 3;
// A wait of all lanes of a warp, with the time limit of every wait (ptx.cuh).  Who runs out of it leaves
// its warp, the barrier and the parity in the abort flag, which the block reports at its end: the
// caches that hold the roles' loops have no room for that at every wait (see below).
__device__ __forceinline__ bool wait_here(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    uint64_t t0 = 0;
    bool ok;
    for (uint32_t i = 0; !(ok = mbar_try_wait(bar, parity)); ++i)
        if ((i & 15u) == 0u) {
            const uint64_t now = global_timer_ns();
            if (i == 0) t0 = now;
            if (now - t0 > GS_WAIT_LIMIT_NS)
                *abort_flag = static_cast<int>((threadIdx.x >> 5) << 20 | smem_u32(bar) << 1 | parity);
            if (*abort_flag) break;
        }
    return __all_sync(~0u, ok);
}
__device__ __forceinline__ void report_timeout(unsigned flag, unsigned* status) {
    if (atomicCAS(status, kDevOk, kDevTimeout) != kDevOk) return;
    volatile unsigned* rec = status + 1;
    rec[0] = blockIdx.x;
    rec[1] = blockIdx.y;
    rec[2] = flag >> 20;
    rec[3] = flag >> 1 & 0x7ffffu;
    rec[4] = flag & 1u;
}
// bf16 exponent fields between which E moves (values up to 2^113 are fine).
constexpr int kLeastField = 16, kMostField = 240;

struct ManyParams {
    AttnParams a;
    CacheParams c;
    InType type;                          // of q and out
    int64_t tiles_r;
    int copies;                           // of each query row in a tile: 1, or 2 (see below)
    int dblocks, cblocks, ksteps;
    int raw_bytes;                        // 128 tokens as they lie in the cache
    int out_vec;                          // output rows start on four-element boundaries
    uint32_t idesc_s, idesc_x, idesc_o;
    int stall;                            // test hook: a wait of block 0's copies runs out
};

struct __align__(16) ManyBarriers {
    int fill_max[2][2][kFillWarps];
    uint64_t q_full, drain;
    uint64_t s_full[2], p_full[2], o_full[2];
    uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
    uint64_t raw_full[kRawStages], raw_empty[kRawStages];
    uint64_t exp_full[4];
    uint64_t never;                       // (nothing arrives on it)
    int exps[4][2];                       // E of k and v of a tile
    uint32_t lost[kRawStages];            // blocks of a stage without a page
    uint32_t tmem_base;
    int abort_flag;
};
constexpr uint32_t kBarBytes = 1024;      // (what follows starts on a boundary of 1024 bytes)
static_assert(sizeof(ManyBarriers) <= kBarBytes, "barriers");

__device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t y;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(y) : "r"(a), "r"(b), "r"(c));
    return y;
}

// 2^(-e) as a float for a bf16 exponent field e (value 2^(e - 126) above every number of the
// field), times 2^shift; 0 or infinity past float32's range.
__device__ __forceinline__ float scale_of(int field, int shift) {
    const int f = 127 - (field - 126) + shift;
    return __uint_as_float(static_cast<uint32_t>(min(max(f, 0), 254)) << 23);
}

// Eight values of a word of codes.
__device__ __forceinline__ uint4 eight(uint32_t w, uint32_t s24, uint32_t s20, uint32_t m) {
    uint4 y;
    y.x = fma2(w & 0x000f000fu, s24, m);
    y.y = fma2(w & 0x00f000f0u, s20, m);
    w >>= 8;
    y.z = fma2(w & 0x000f000fu, s24, m);
    y.w = fma2(w & 0x00f000f0u, s20, m);
    return y;
}

// Factors of a group word for values times 2^-E (of keys: s (u - 8) 2^-E, which is exact).
struct Pair {
    uint32_t s24, s20, m;
};
__device__ __forceinline__ Pair pair_of(uint32_t word, float up16, float up12, float down8) {
    const float s = __uint_as_float(word << 16), m = __uint_as_float(word & 0xffff0000u);
    Pair p;
    p.s24 = pack_half2(s * up16, s * up16);
    p.s20 = pack_half2(s * up12, s * up12);
    p.m = pack_half2(m * down8, m * down8);
    return p;
}

__device__ __forceinline__ Pair centred_pair(uint32_t word, float up16, float up12, float down5) {
    const float s = __uint_as_float(word << 16);
    Pair p;
    p.s24 = pack_half2(s * up16, s * up16);
    p.s20 = pack_half2(s * up12, s * up12);
    p.m = pack_half2(-s * down5, -s * down5);
    return p;
}

// Eight columns of a product x y of float32 numbers as bf16 operands: x = x1 + x2 + x3 and y alike,
// and all products of two parts but x3 y3.
__device__ __forceinline__ void three_parts(float x, float& a, float& b, float& c) {
    a = __bfloat162float(__float2bfloat16_rn(x));
    b = __bfloat162float(__float2bfloat16_rn(x - a));
    c = x - a - b;
}
__device__ __forceinline__ uint4 first_factor(float x) {
    float a, b, c;
    three_parts(x, a, b, c);
    return make_uint4(pack_bf162(a, a), pack_bf162(b, a), pack_bf162(b, c), pack_bf162(b, c));
}
__device__ __forceinline__ uint4 second_factor(float x) {
    float a, b, c;
    three_parts(x, a, b, c);
    return make_uint4(pack_bf162(a, b), pack_bf162(a, c), pack_bf162(b, a), pack_bf162(c, b));
}

__device__ __forceinline__ uint32_t mul_bf162(uint32_t a, uint32_t b) {
    uint32_t y;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
    return y;
}

// 128 rows of 16 bf16 columns: the 16-byte halves of the rows one after the other, half after half.
constexpr uint32_t kCentres = kTile * 32;
__device__ __forceinline__ uint64_t smem_desc_centres(uint32_t saddr) {
    uint64_t d = 0;
    d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
    d |= static_cast<uint64_t>((kTile * 16u) >> 4) << 16;      // from half to half
    d |= static_cast<uint64_t>(128u >> 4) << 32;               // from eight rows to the next eight
    d |= static_cast<uint64_t>(1u) << 46;
    return d;                                                  // (no swizzle)
}

// Shared memory by 32-bit addresses (half the registers of pointers).
__device__ __forceinline__ uint4 lds128(uint32_t at) {
    uint4 x;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at));
    return x;
}
__device__ __forceinline__ uint32_t lds32(uint32_t at) {
    uint32_t x;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(at));
    return x;
}
__device__ __forceinline__ uint32_t lds16(uint32_t at) {
    uint16_t x;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(at));
    return x;
}
__device__ __forceinline__ void sts128(uint32_t at, const uint4& x) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}

// The codes of a row of a key tile (four chunks of W words), and the row from them.  The row starts
// at a multiple of 128 bytes and its 16-byte chunk c lies at c ^ (row % 8); it takes its chunks in the
// order i ^ (row / 2 % 4), which spreads eight rows over the banks in reads and writes, and makes
// every address one exclusive or away from the first.
template <int W>
struct KeyRow {
    uint32_t w[4][W];
    __device__ __forceinline__ void load(uint32_t codes, int row) {
        const int rho = (row >> 1) & 3;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (W == 4) {
                const uint4 x = lds128((codes + 16 * rho) ^ (16 * i));       // (rows of 64 bytes)
                w[i][0] = x.x, w[i][1] = x.y, w[i][2] = x.z, w[i][3] = x.w;
            } else {
#pragma unroll
                for (int j = 0; j < W; ++j) w[i][j] = lds32(codes + 4 * (W * (rho ^ i) + j));
            }
        }
    }
    __device__ __forceinline__ void store(uint32_t tile, int row, const Pair (&g)[2]) const {
        const uint32_t at = tile + row * 128 + ((((row >> 1) & 3) ^ (row & 7)) << 4);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j)
                sts128((at ^ ((4 * (j & 1) + i) << 4)) + (j >> 1) * kBlock,
                       eight(w[i][j], g[j >> 1].s24, g[j >> 1].s20, g[j >> 1].m));
    }
};

// The same of a value tile (eight chunks of W 16-bit words, two at a time): column 8 g + 2 p + h of
// block b is channel 64 b + 32 h + 4 g + p.
template <int W>
struct ValueRow {
    static constexpr int kWords = (W + 1) / 2;
    uint32_t w[8][kWords];
    static __device__ __forceinline__ int first(int row) {
        const int rho = (row >> 1) & 3;
        return (0x1320 >> (4 * rho)) & 3;            // 0, 2, 3, 1
    }
    __device__ __forceinline__ void load(uint32_t codes, int row) {
        const int f = first(row);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (W == 4) {
                const uint4 x = lds128((codes + 16 * f) ^ (16 * i));
                w[2 * i][0] = x.x, w[2 * i][1] = x.y, w[2 * i + 1][0] = x.z, w[2 * i + 1][1] = x.w;
            } else {
                const uint32_t at = codes + 4 * W * (f ^ i);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    w[2 * i + h][0] = lds16(at + 2 * W * h);
                    if constexpr (W > 1) w[2 * i + h][0] |= lds16(at + 2 * W * h + 2) << 16;
                    if constexpr (W > 2) w[2 * i + h][1] = lds16(at + 2 * W * h + 4);
                }
            }
        }
    }
    __device__ __forceinline__ void store(uint32_t tile, int row, const Pair (&g)[2]) const {
        const uint32_t at = tile + row * 128 + (((2 * first(row)) ^ (row & 7)) << 4);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int b = 0; b < kWords; ++b)
                sts128((at ^ (i << 4)) + b * kBlock, eight(w[i][b], g[b].s24, g[b].s20, g[b].m));
    }
};

// A thread of the filling warps: its row in a tile, and where it lies in the raw tile.
struct FillAt {
    int row, lane, warp, raw_row, block_row, groups;
};
__device__ __forceinline__ FillAt fill_at(const CacheParams& c, int tid) {
    FillAt a;
    a.row = tid & (kTile - 1);
    a.lane = tid & 31;
    a.warp = a.row >> 5;
    a.block_row = a.row & 15;
    a.raw_row = (a.row >> 4) * c.block_bytes;
    a.groups = a.raw_row + 256 * (c.kw + c.vw);
    return a;
}

// Bits of the larger of s and |m| 2^-20 of a group word, not of NaN or infinities.
__device__ __forceinline__ uint32_t sized(uint32_t word) {
    const uint32_t s = word & 0x7fffu, m = (word >> 16) & 0x7fffu;
    return max(s < 0x7f80u ? s : 0u, m < 0x7f80u && m > (20u << 7) ? m - (20u << 7) : 0u);
}

// Key tiles t < n, and the E of both tiles.  (After a wait that ran out the warps still meet at
// every barrier.)
template <int W>
__device__ __forceinline__ void fill_keys(const ManyParams& f, ManyBarriers* bars, uint32_t raw, uint32_t k_smem,
                                          uint32_t k_mid, int tid, int n, int tile0, int kl) {
    const CacheParams& c = f.c;
    const FillAt a = fill_at(c, tid);
    volatile int* abort_flag = &bars->abort_flag;
    bool ok = true;
    int v_field = kLeastField;
    int s = 0;
    if (W <= 2)                                      // (one group: the other's columns stay 0)
        for (int i = 0; i < 2; ++i) sts128(k_mid + i * kCentres + kTile * 16 + a.row * 16, make_uint4(0, 0, 0, 0));
    uint32_t phase = 0;
    for (int t = 0; t < n; ++t) {
        const int i = t & 1;
        ok = ok && wait_here(&bars->raw_full[s], phase, abort_flag);
        const uint32_t at = raw + s * f.raw_bytes;
        const bool none = (bars->lost[s] >> (a.row >> 4)) & 1u, out = (tile0 + t) * kTile + a.row >= kl;
        KeyRow<W> codes;
        uint32_t word[2] = {0, 0}, size[2] = {0, 0};
        if (ok) codes.load(at + a.raw_row + a.block_row * 16 * W, a.row);
        if (ok && !out && !none) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (u < (W + 1) / 2) {
                    word[u] = lds32(at + a.groups + (a.block_row * ((W + 1) / 2) + u) * 4);
                    size[0] = max(size[0], sized(word[u]));
                }
                if (u < c.vg)
                    size[1] = max(size[1], sized(lds32(at + a.groups + 64 * ((W + 1) / 2) + (a.block_row * c.vg + u) * 4)));
            }
        }
        if (none && !out) word[0] = word[1] = kNanGroup;
        size[0] = __reduce_max_sync(~0u, size[0]);
        size[1] = __reduce_max_sync(~0u, size[1]);
        // The groups' centres m + 8 s, in parts before E is known.
        uint4 mid[(W + 1) / 2];
#pragma unroll
        for (int u = 0; u < (W + 1) / 2; ++u)
            mid[u] = first_factor(fmaf(__uint_as_float(word[u] << 16), 8.f, __uint_as_float(word[u] & 0xffff0000u)));
        __syncwarp();
        if (a.lane == 0) {
            bars->fill_max[i][0][a.warp] = static_cast<int>(size[0]);
            bars->fill_max[i][1][a.warp] = static_cast<int>(size[1]);
            if (ok) mbar_arrive(&bars->raw_empty[s]);    // (its codes and groups are in registers)
        }
        barrier_sync<2, kFillWarps * 32>();
        int most[2];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            const int4 x = *reinterpret_cast<const int4*>(bars->fill_max[i][z]);
            most[z] = max(max(x.x, x.y), max(x.z, x.w));
        }
        const int k_field = min(max(most[0] >> 7, kLeastField), kMostField);
        v_field = min(max(v_field, most[1] >> 7), kMostField);
        ok = ok && wait_here(&bars->k_empty[i], ((t >> 1) & 1) ^ 1, abort_flag);
        if (ok) {
            if (a.row == 0) {
                bars->exps[t & 3][0] = k_field;
                bars->exps[t & 3][1] = v_field;
                mbar_arrive(&bars->exp_full[t & 3]);
            }
            const float up16 = scale_of(k_field, 16), up12 = scale_of(k_field, 12), down5 = scale_of(k_field, -5);
            Pair g[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) g[u] = centred_pair(word[u], up16, up12, down5);    // (zeros past the tokens)
            codes.store(k_smem + i * f.dblocks * kBlock, a.row, g);
            const uint32_t down8 = __byte_perm(__float_as_uint(down5 * 0.125f), 0, 0x3232);
#pragma unroll
            for (int u = 0; u < (W + 1) / 2; ++u)
                sts128(k_mid + i * kCentres + u * kTile * 16 + a.row * 16,
                       make_uint4(mul_bf162(mid[u].x, down8), mul_bf162(mid[u].y, down8), mul_bf162(mid[u].z, down8),
                                  mul_bf162(mid[u].w, down8)));
            fence_proxy_async_smem();
            __syncwarp();
            mbar_arrive_if_zero(&bars->k_full[i], a.lane);
        }
        if (++s == kRawStages) s = 0, phase ^= 1u;
    }
}

template <int W>
__device__ __forceinline__ void fill_values(const ManyParams& f, ManyBarriers* bars, uint32_t raw, uint32_t v_smem,
                                            int tid, int n, int tile0, int kl) {
    const CacheParams& c = f.c;
    const FillAt a = fill_at(c, tid);
    volatile int* abort_flag = &bars->abort_flag;
    int s = 0;
    uint32_t phase = 0;
    for (int t = 0; t < n; ++t) {
        const int i = t & 1;
        if (!wait_here(&bars->raw_full[s], phase, abort_flag)) return;
        const uint32_t at = raw + s * f.raw_bytes;
        const bool zero = (tile0 + t) * kTile + a.row >= kl || ((bars->lost[s] >> (a.row >> 4)) & 1u);
        ValueRow<W> codes;
        uint32_t word[2] = {0, 0};
        codes.load(at + a.raw_row + 256 * c.kw + a.block_row * 16 * W, a.row);
        if (!zero)
#pragma unroll
            for (int u = 0; u < (W + 1) / 2; ++u)
                word[u] = lds32(at + a.groups + 64 * c.kg + (a.block_row * ((W + 1) / 2) + u) * 4);
        __syncwarp();
        mbar_arrive_if_zero(&bars->raw_empty[s], a.lane);
        if (!wait_here(&bars->exp_full[t & 3], (t >> 2) & 1, abort_flag) ||
            !wait_here(&bars->v_empty[i], ((t >> 1) & 1) ^ 1, abort_flag))
            return;
        const int field = bars->exps[t & 3][1];
        const float up16 = scale_of(field, 16), up12 = scale_of(field, 12), down8 = scale_of(field, -8);
        Pair g[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) g[u] = pair_of(word[u], up16, up12, down8);
        codes.store(v_smem + i * f.cblocks * kBlock, a.row, g);
        fence_proxy_async_smem();
        __syncwarp();
        mbar_arrive_if_zero(&bars->v_full[i], a.lane);
        if (++s == kRawStages) s = 0, phase ^= 1u;
    }
}

__global__ void __launch_bounds__(kThreads, 1) cache_many_kernel(const __grid_constant__ ManyParams f) {
    const AttnParams& p = f.a;
    const CacheParams& cp = f.c;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* smem = smem_raw + kBarBytes;
    const uint32_t k_bytes = f.dblocks * kBlock, v_bytes = f.cblocks * kBlock;
    uint8_t* q_smem = smem;
    uint8_t* k_smem = q_smem + k_bytes;
    uint8_t* v_smem = k_smem + 2 * k_bytes;
    uint8_t* q_mid = v_smem + 2 * v_bytes;             // sums of q, and the keys' centres (two tiles)
    uint8_t* k_mid = q_mid + kCentres;
    uint8_t* raw = k_mid + 2 * kCentres;
    ManyBarriers* bars = reinterpret_cast<ManyBarriers*>(smem_raw);
    volatile int* abort_flag = &bars->abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // Block -> (split, row tile, problem and key head); later row tiles see more keys and go first.
    int64_t blk = blockIdx.x;
    const int split = static_cast<int>(blk % p.splits);
    blk /= p.splits;
    const int64_t heads_all = static_cast<int64_t>(p.B) * p.Hk;
    const int64_t tile = f.tiles_r - 1 - blk / heads_all, bh = blk % heads_all;
    const int b = static_cast<int>(bh / p.Hk), h = static_cast<int>(bh - static_cast<int64_t>(b) * p.Hk);
    const int ql = attn_q_len(p, b), kl = attn_k_len(p, b);
    const int tile_rows = kTile / f.copies;
    const int rows_in = ql * p.G, r0 = static_cast<int>(tile) * tile_rows;
    const int last = min(r0 + tile_rows, rows_in) - 1;
    const int kend = last >= r0 ? attn_limit(last / p.G, ql, kl, p.causal) : 0;
    const int64_t all = (static_cast<int64_t>(kend) + kTile - 1) / kTile;
    const int tile0 = static_cast<int>(all * split / p.splits), tile1 = static_cast<int>(all * (split + 1) / p.splits);
    const int n = tile1 - tile0;                       // key tiles: tile t belongs to stream t & 1
    const int nt[2] = {(n + 1) / 2, n / 2};

    if (tid == 0) {
        mbar_init(&bars->q_full, kSoftmaxWarps);
        mbar_init(&bars->drain, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars->s_full[i], 1);
            mbar_init(&bars->p_full[i], 4);
            mbar_init(&bars->o_full[i], 1);
            mbar_init(&bars->k_full[i], kFillWarps);
            mbar_init(&bars->k_empty[i], 1);
            mbar_init(&bars->v_full[i], kFillWarps);
            mbar_init(&bars->v_empty[i], 1);
        }
        for (int s = 0; s < kRawStages; ++s) {
            mbar_init(&bars->raw_full[s], 8);
            mbar_init(&bars->raw_empty[s], 2 * kFillWarps);
            bars->lost[s] = 0;
        }
        for (int s = 0; s < 4; ++s) mbar_init(&bars->exp_full[s], 1);
        mbar_init(&bars->never, 1);
        bars->abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(&bars->tmem_base, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();
    pdl_trigger();
    const uint32_t tmem = bars->tmem_base;

    if (warp == kLoadWarp) {
        reg_dealloc<kRegsCtrl>();
        // Lane i < 8 brings block i of a tile; pages are read one tile ahead.
        const int per_page = cp.tokens >> 4;
        const auto page_of = [&](int t) {
            const int i = 8 * (tile0 + t) + (lane & 7);
            return t < n && (i << 4) < kend ? cache_page(cp, b, i << 4) : kNoPage;
        };
        int page = page_of(0);
        const int stall_at = f.stall && blockIdx.x == 0 ? min(n - 1, 6) : -1;
        int issued = 0;
        RingPos at;
        for (int t = 0; t < n; ++t) {
            const int next = page_of(t + 1);
            if (!wait_here(&bars->raw_empty[at.idx], at.phase ^ 1u, abort_flag)) break;
            if (t == stall_at && !wait_here(&bars->never, 0, abort_flag)) break;
            const uint32_t none = __ballot_sync(~0u, page == kNoPage) & 0xffu;
            if (lane == 0) bars->lost[at.idx] = none;
            __syncwarp();
            if (lane < 8) {
                if (page == kNoPage) {
                    mbar_arrive(&bars->raw_full[at.idx]);
                } else {
                    const int i = 8 * (tile0 + t) + lane;
                    const int in_page = cp.shift >= 0 ? i & (per_page - 1) : i % per_page;
                    mbar_arrive_expect_tx(&bars->raw_full[at.idx], cp.block_bytes);
                    bulk_load(raw + at.idx * f.raw_bytes + lane * cp.block_bytes,
                              cp.data + page * cp.sp + h * cp.sh + static_cast<int64_t>(in_page) * cp.block_bytes,
                              cp.block_bytes, &bars->raw_full[at.idx]);
                }
            }
            __syncwarp();
            page = next;
            at.advance(kRawStages);
            ++issued;
        }
        // Every copy started here lands before the block can end, whoever gave up.
        for (int t = max(0, issued - kRawStages); t < issued; ++t)
            mbar_wait_bounded(&bars->raw_full[t % kRawStages], static_cast<uint32_t>(t / kRawStages) & 1u, nullptr, p.status);
    } else if (warp >= kKeyWarp && warp < kValueWarp) {
        reg_dealloc<kRegsFill>();
        if (cp.kw == 4) fill_keys<4>(f, bars, smem_u32(raw), smem_u32(k_smem), smem_u32(k_mid), tid, n, tile0, kl);
        else if (cp.kw == 3) fill_keys<3>(f, bars, smem_u32(raw), smem_u32(k_smem), smem_u32(k_mid), tid, n, tile0, kl);
        else if (cp.kw == 2) fill_keys<2>(f, bars, smem_u32(raw), smem_u32(k_smem), smem_u32(k_mid), tid, n, tile0, kl);
        else fill_keys<1>(f, bars, smem_u32(raw), smem_u32(k_smem), smem_u32(k_mid), tid, n, tile0, kl);
    } else if (warp >= kValueWarp && warp < kLoadWarp) {
        reg_dealloc<kRegsFill>();
        if (cp.vw == 4) fill_values<4>(f, bars, smem_u32(raw), smem_u32(v_smem), tid, n, tile0, kl);
        else if (cp.vw == 3) fill_values<3>(f, bars, smem_u32(raw), smem_u32(v_smem), tid, n, tile0, kl);
        else if (cp.vw == 2) fill_values<2>(f, bars, smem_u32(raw), smem_u32(v_smem), tid, n, tile0, kl);
        else fill_values<1>(f, bars, smem_u32(raw), smem_u32(v_smem), tid, n, tile0, kl);
    } else if (warp == kMmaWarp) {
        reg_dealloc<kRegsCtrl>();
        if (n > 0) {
            const uint32_t leader = elect_one() ? 1u : 0u;
            bool ok = wait_here(&bars->q_full, 0, abort_flag);
            const uint32_t q_at = smem_u32(q_smem), k_at = smem_u32(k_smem), v_at = smem_u32(v_smem);
            const uint32_t k_mid_at = smem_u32(k_mid);
            const uint64_t q_mid_desc = smem_desc_centres(smem_u32(q_mid));
            const auto scores = [&](int t) {
                const int i = t & 1;
                if (ok) ok = wait_here(&bars->k_full[i], (t >> 1) & 1, abort_flag);
                if (!ok) return;
                tc_fence_after();
                mma_scores(leader, tmem + 128 * i, q_at, k_at + i * k_bytes, f.ksteps, f.idesc_s);
                mma_ss_on(leader, tmem + 128 * i, q_mid_desc, smem_desc_centres(k_mid_at + i * kCentres), f.idesc_x, 1u);
                mma_commit_on(leader, &bars->s_full[i]);
                mma_commit_on(leader, &bars->k_empty[i]);
            };
            const auto values = [&](int t) {
                const int i = t & 1;
                if (ok) ok = wait_here(&bars->v_full[i], (t >> 1) & 1, abort_flag);
                if (ok) ok = wait_here(&bars->p_full[i], (t >> 1) & 1, abort_flag);
                if (!ok) return;
                tc_fence_after();
                mma_rows<16>(leader, tmem + kO + 128 * i, tmem + 128 * i, v_at + i * v_bytes, f.idesc_o, t < 2);
                mma_commit_on(leader, &bars->v_empty[i]);
                if (t + 2 >= n) mma_commit_on(leader, &bars->o_full[i]);
            };
            for (int t = 0; t < 2 && t < n; ++t) scores(t);
            for (int t = 0; ok && t < n; ++t) {
                values(t);
                if (t + 2 < n) scores(t + 2);
            }
            // No MMA may still be running when TMEM is released.
            if (leader) mma_commit(&bars->drain);
            __syncwarp();
            mbar_wait_bounded(&bars->drain, 0, nullptr, p.status);
            __syncwarp();
        }
    } else if (warp > kMmaWarp) {
        reg_dealloc<kRegsCtrl>();
    } else {
        reg_alloc<kRegsSoftmax>();
        const int i = warp >> 2, row = tid & (kTile - 1);
        const int r = r0 + (row & (tile_rows - 1)), m = r / p.G, hq = h * p.G + r - m * p.G;
        const bool in = r < rows_in;
        const int lim = in ? attn_limit(m, ql, kl, p.causal) : 0;
        const int lim_first = attn_limit(r0 / p.G, ql, kl, p.causal);
        const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;   // (32 x quarter) << 16
        const uint32_t t_s = tmem + lanes + 128 * i, t_o = tmem + lanes + kO + 128 * i;
        float c_row = 0.f;                             // of scores times 2^-E

        if (n > 0) {
            // This row's queries; every other chunk of eight goes to shared memory from here.
            const int64_t at = b * p.q.sb + m * p.q.sr + static_cast<int64_t>(hq) * p.q.sh;
            const uint16_t* src = reinterpret_cast<const uint16_t*>(p.q.p) + at;
            uint4 x[8];
            float top = 0.f, sums[2] = {0.f, 0.f};         // (of all channels of a group)
            const auto two = [&](uint32_t w) {
                return f.type == InType::F16 ? __half22float2(*reinterpret_cast<const __half2*>(&w))
                                             : make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
            };
#pragma unroll
            for (int z = 0; z < 2; ++z) {              // the other stream's chunks, then this one's
                const int par = z == 0 ? 1 - i : i;
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int c0 = 8 * (2 * u + par);
                    x[u] = make_uint4(0, 0, 0, 0);
                    if (in && c0 < p.D) {
                        if (p.vec) {
                            x[u] = *reinterpret_cast<const uint4*>(src + c0);
                        } else {
                            uint32_t e[8];
#pragma unroll
                            for (int d = 0; d < 8; ++d) e[d] = c0 + d < p.D ? src[c0 + d] : 0u;
                            x[u] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        const float2 y = two(w[d]);
                        top = fmaxf(top, fmaxf(fabsf(y.x), fabsf(y.y)));
                        sums[u >> 2] += y.x + y.y;
                    }
                }
            }
            // 2^e top in [2^14, 2^15), e in -113 .. 100.
            const int e = min(max(min(141 - static_cast<int>(__float_as_uint(top) >> 23), 100), -113), 100);
            const float up = __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
            c_row = p.c / up;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int c8 = 2 * u + i;
                if (c8 >= f.dblocks * 8) continue;
                const float2 a = two(x[u].x), bb = two(x[u].y), cc = two(x[u].z), d = two(x[u].w);
                uint4 y;                               // channels 0 4, 1 5, 2 6, 3 7
                y.x = pack_half2(a.x * up, cc.x * up);
                y.y = pack_half2(a.y * up, cc.y * up);
                y.z = pack_half2(bb.x * up, d.x * up);
                y.w = pack_half2(bb.y * up, d.y * up);
                *reinterpret_cast<uint4*>(q_smem + (c8 >> 3) * kBlock + row * 128 + (((c8 & 7) ^ (row & 7)) << 4)) = y;
            }
            *reinterpret_cast<uint4*>(q_mid + i * kTile * 16 + row * 16) = second_factor((i == 0 ? sums[0] : sums[1]) * up);
            fence_proxy_async_smem();
            __syncwarp();
            mbar_arrive_if_zero(&bars->q_full, lane);
        }

        // A tile may leave whole warps without rows: they only keep the barriers going.
        const bool active = r0 + (((warp & 3) * 32) & (tile_rows - 1)) < rows_in;
        const int own = row >> 6;                      // with two copies: this one's half of a tile
        float top = -INFINITY, sum = 0.f;              // m in log2 units, row sum of 2^(c s - m + shift)
        int v_field = kLeastField;
        bool ok = true;
        for (int j = 0; ok && j < nt[i]; ++j) {
            const int t = 2 * j + i;
            ok = wait_here(&bars->s_full[i], j & 1, abort_flag);
            if (!ok) break;
            tc_fence_after();
            ok = wait_here(&bars->exp_full[t & 3], (t >> 2) & 1, abort_flag);
            if (!ok) break;
            const int n0 = (tile0 + t) * kTile;
            const int field = bars->exps[t & 3][1];
            if (active) {
                // (E of k: values are k 2^(126 - 8 - field).)
                // Never 0, which makes NaN of a masked score: where the product is so small that 2^-126 more
                // changes it, the scores (below 2^40) are nothing either way.
                const float c = fmaf(c_row, __uint_as_float(
                    static_cast<uint32_t>(min(bars->exps[t & 3][0] - 126 + 8 + 127, 254)) << 23), 0x1p-126f);
                const bool edge = n0 + kTile > lim_first;
                // 64 scores at a time: their maxima, the later half first kept for its exponentials,
                // and the other read again (P lies over the first half of each 32 columns).
                uint32_t s[2][32];
                const auto load = [&](int half) {
                    tmem_ld_32x32b_x32(t_s + 64 * half, s[0]);
                    tmem_ld_32x32b_x32(t_s + 64 * half + 32, s[1]);
                    tmem_wait_ld_regs(s[0], s[1]);
                    if (edge) {
                        const int seen = lim - n0 - 64 * half;
#pragma unroll
                        for (int q = 0; q < 2; ++q)
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (q * 32 + e >= seen) s[q][e] = 0xff800000u;   // -inf
                    }
                };
                const auto highest = [&]() {
                    float mx[2] = {__uint_as_float(s[0][0]), __uint_as_float(s[1][0])};
#pragma unroll
                    for (int e = 1; e < 32; ++e) {
                        mx[0] = fmaxf(mx[0], __uint_as_float(s[0][e]));
                        mx[1] = fmaxf(mx[1], __uint_as_float(s[1][e]));
                    }
                    return fmaxf(mx[0], mx[1]);
                };
                // (One copy of the code for both halves: the roles' loops share the instruction caches.)
                const int first = f.copies == 1 ? 0 : own, last = f.copies == 1 ? 1 : own;
                float mt = -INFINITY;
#pragma unroll 1
                for (int half = first; half <= last; ++half) {
                    load(half);
                    mt = fmaxf(mt, highest());
                }
                mt *= c;
                const bool move = mt - top > kMaxSlack;   // (also from -inf)
                if (__any_sync(~0u, move) || field != v_field) {
                    const float to = move ? mt : top;
                    const float fq = move ? ex2_approx(top - to) : 1.f;      // 0 from -inf
                    const float fo = fq * __uint_as_float(static_cast<uint32_t>(max(127 + v_field - field, 0)) << 23);
                    top = to;
                    sum *= fq;
                    if (j > 0) {
                        for (int cc = 0; cc < f.cblocks * 64; cc += 32) {
                            uint32_t o[2][16];
                            tmem_ld_32x32b_x16(t_o + cc, o[0]);
                            tmem_ld_32x32b_x16(t_o + cc + 16, o[1]);
                            tmem_wait_ld_regs(o[0], o[1]);
#pragma unroll
                            for (int z = 0; z < 2; ++z) {
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[z][e] = __float_as_uint(__uint_as_float(o[z][e]) * fo);
                                tmem_st_32x32b_x16(t_o + cc + 16 * z, o[z]);
                            }
                        }
                    }
                }
                v_field = field;
                const float ref = (top == -INFINITY ? 0.f : -top) + kShift;
                const uint64_t c2 = f32x2_pack(c, c), r2 = f32x2_pack(ref, ref);
                uint64_t acc[2] = {0, 0};
                const auto exponentials = [&](int half) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        uint32_t w[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            const uint64_t y = f32x2_fma(
                                f32x2_pack(__uint_as_float(s[q][e]), __uint_as_float(s[q][e + 1])), c2, r2);
                            float x0, x1;
                            f32x2_unpack(y, x0, x1);
                            x0 = ex2_approx(x0);
                            x1 = ex2_approx(x1);
                            acc[(e >> 1) & 1] = f32x2_add(acc[(e >> 1) & 1], f32x2_pack(x0, x1));
                            w[e >> 1] = pack2<false>(x0, x1);
                        }
                        tmem_st_32x32b_x16(t_s + 64 * half + 32 * q, w);
                    }
                };
#pragma unroll 1
                for (int half = last; half >= first; --half) {
                    if (half != last) load(half);
                    exponentials(half);
                }
                if (f.copies != 1) {
                    const uint32_t zero[16] = {};
                    tmem_st_32x32b_x16(t_s + 64 * (1 - own), zero);
                    tmem_st_32x32b_x16(t_s + 64 * (1 - own) + 32, zero);
                }
                float a0, a1;
                f32x2_unpack(f32x2_add(acc[0], acc[1]), a0, a1);
                sum += a0 + a1;
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            mbar_arrive_if_zero(&bars->p_full[i], lane);
        }

        // Epilogue: out = O / sum, lse = m + log2 sum, through shared memory (the tiles are no longer read).
        if (ok && nt[i] > 0) ok = wait_here(&bars->o_full[i], 0, abort_flag);
        tc_fence_after();
        // (A row of NaN scores has no maximum, but its sum is NaN.)
        const bool has = ok && nt[i] > 0 && lim > 0 && (top != -INFINITY || sum != sum);
        const float inv = has ? 1.f / sum : 0.f;
        const float l2 = has ? top - kShift + log2f(sum) : -INFINITY;
        // V's scale, as two factors that float32 holds.
        const int ve = v_field - 126 + 8;
        const float up_a = __uint_as_float(static_cast<uint32_t>(127 + ve / 2) << 23);
        const float up_b = __uint_as_float(static_cast<uint32_t>(127 + ve - ve / 2) << 23);
        // Every stream's and copy's rows, column by column, and their lse; then each thread joins a
        // run of columns of one row.
        const int cols = f.cblocks * 64;
        float* part_l = reinterpret_cast<float*>(k_smem);
        float* part_o = part_l + 2 * kTile;
        barrier_sync<1, kSoftmaxWarps * 32>();
        part_l[i * kTile + row] = l2;
        for (int c = 0; active && nt[i] > 0 && c < cols; c += 32) {
            uint32_t o[32];
            tmem_ld_32x32b_x32(t_o + c, o);
            tmem_wait_ld_regs(o);
#pragma unroll
            for (int e = 0; e < 32; ++e)
                if (has) part_o[(i * cols + c + e) * kTile + row] = __uint_as_float(o[e]) * inv * up_a * up_b;
            __syncwarp();
        }
        barrier_sync<1, kSoftmaxWarps * 32>();
        const int parts = 2 * f.copies, of_row = tid & (tile_rows - 1), part = tid / tile_rows;
        const int ro = r0 + of_row, mo = ro / p.G, ho = h * p.G + ro - mo * p.G;
        float l[4], top_l = -INFINITY, total = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            l[e] = e < parts ? part_l[(e & 1) * kTile + (e >> 1) * tile_rows + of_row] : -INFINITY;
            top_l = fmaxf(top_l, l[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            l[e] = l[e] == -INFINITY ? 0.f : exp2f(l[e] - top_l);      // (NaN: a row of NaN scores)
            total += l[e];
        }
        const float norm = total != 0.f ? 1.f / total : 0.f;
        const float l_row = total != 0.f ? top_l + log2f(total) : -INFINITY;
        const bool mine = ro < p.R, split_out = p.splits > 1;
        const int64_t at_part = (static_cast<int64_t>(split) * p.B * p.Hk + bh) * p.R + ro;
        if (mine && part == 0) {
            if (split_out)
                p.part_l[at_part] = l_row;
            else if (p.lse)
                p.lse[(static_cast<int64_t>(b) * p.H + ho) * p.M + mo] = l_row * kLn2;
        }
        const int64_t to = b * p.out.sb + mo * p.out.sr + static_cast<int64_t>(ho) * p.out.sh;
        const int run = cols / parts;
        for (int c = part * run; mine && c < (part + 1) * run; c += 8) {
            float x[8] = {};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (l[e] != 0.f) {
                    const float* from = part_o + ((e & 1) * cols + c) * kTile + (e >> 1) * tile_rows + of_row;
#pragma unroll
                    for (int z = 0; z < 8; ++z) x[z] = fmaf(l[e] * norm, from[z * kTile], x[z]);
                }
            // Columns c + 2 q + z are channels 64 (c / 64) + 32 z + 4 (c % 64 / 8) + q.
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const int ch = (c & 64) + 32 * z + (c & 63) / 2;
                const float y[4] = {x[z], x[2 + z], x[4 + z], x[6 + z]};
                if (split_out) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (total != 0.f && ch + q < p.C) p.part_o[at_part * p.C + ch + q] = y[q];
                    continue;
                }
                uint16_t* dst = reinterpret_cast<uint16_t*>(p.out.p) + to + ch;
                uint2 w;
                w.x = f.type == InType::BF16 ? round2<true>(y[0], y[1]) : round2<false>(y[0], y[1]);
                w.y = f.type == InType::BF16 ? round2<true>(y[2], y[3]) : round2<false>(y[2], y[3]);
                if (f.out_vec && ch + 4 <= p.C) {
                    *reinterpret_cast<uint2*>(dst) = w;
                } else {
                    if (ch < p.C) dst[0] = static_cast<uint16_t>(w.x);
                    if (ch + 1 < p.C) dst[1] = static_cast<uint16_t>(w.x >> 16);
                    if (ch + 2 < p.C) dst[2] = static_cast<uint16_t>(w.y);
                    if (ch + 3 < p.C) dst[3] = static_cast<uint16_t>(w.y >> 16);
                }
            }
        }
        tc_fence_before();
    }
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (tid == 0 && *abort_flag) report_timeout(static_cast<unsigned>(*abort_flag), p.status);
}

}  // namespace

bool cache_many_takes(const CacheParams& c, InType t) { return t != InType::F32 && c.kw <= 4 && c.vw <= 4; }

cudaError_t launch_cache_many(const AttnParams& p, const CacheParams& c, InType t, bool out_vec, cudaStream_t s) {
    ManyParams f{};
    f.a = p;
    f.c = c;
    f.type = t;
    f.copies = p.R <= kTile / 2 ? 2 : 1;
    f.tiles_r = (p.R * f.copies + kTile - 1) / kTile;
    f.dblocks = (c.kw + 1) / 2;
    f.cblocks = (c.vw + 1) / 2;
    f.ksteps = 2 * c.kw;
    f.raw_bytes = 8 * c.block_bytes;
    f.out_vec = out_vec;
    f.stall = testing_stall();
    f.idesc_s = idesc_f16(kTile, kTile, 0, 0);
    f.idesc_o = idesc_f16(kTile, f.cblocks * 64, 0, 0) | kIdescTransposeB;
    f.idesc_x = idesc_f16(kTile, kTile, 1, 1);
    // (Joining takes the columns of both streams where the tiles were.)
    const size_t tiles = (3 * f.dblocks + 2 * f.cblocks) * static_cast<size_t>(kBlock) + 3 * kCentres;
    const size_t join = f.dblocks * static_cast<size_t>(kBlock) + 2 * (f.cblocks * 64 + 1) * kTile * sizeof(float);
    const size_t smem = kBarBytes + std::max(tiles + kRawStages * static_cast<size_t>(f.raw_bytes), join);
    const cudaError_t e = cudaFuncSetAttribute(cache_many_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
    if (e != cudaSuccess) return e;
    note_launches(1);
    return launch_kernel(cache_many_kernel, dim3(static_cast<unsigned>(f.tiles_r * p.B * p.Hk * p.splits)), kThreads,
                         smem, s, f);
}

}  // namespace gs
