// Gradients of softmax attention on the tensor cores (tcgen05, TMA, TMEM),
// fp16 / bf16, D, C <= 128.
//
// The probabilities are recomputed, p = 2^(c s - lse log2 e), in two passes,
// so that every gradient is one accumulation in TMEM in a fixed order:
//   query pass  (128 query rows of a head, streaming key tiles)
//       S = q k^T,  dP = g v^T,  dS = p (dP - delta),  dq += dS k
//   key pass    (128 keys of a key head, streaming the query tiles of all
//                heads that share it), with keys as rows
//       S' = k q^T,  dP' = v g^T,  dv += P' g,  dk += dS' q
// Seven products instead of the five of a single pass, but no atomic
// additions, no fp32 gradient buffer in memory and no transposes: P, dS, P'
// and dS' are written where they are read, as A operands in TMEM, and the
// streamed tiles serve as B operands both ways (channels along the sum for
// the scores, rows along the sum for the gradients).
//
// One thread issues the products in an order that keeps the tensor pipe busy
// while the softmax warps work (query pass: S(j+1), dP(j+1), dq(j); key
// pass: dv(j), S(j+1), dk(j), dP(j+1)).  Softmax warps: thread = row,
// warpgroup w takes the columns 32 w .. 32 w + 31 of a tile.
//
// What bounds it: the tensor pipe with 128 channels (2 x 4096 tokens, 32 / 8
// heads, causal, bf16: 639 us with the row terms, 1.08 PFLOP/s of the five
// products a single pass would need, 1.51 of the seven; shared-memory reads of
// the operands at 85 % of 128 B a clock).  With 64 channels nothing is busy
// (4 x 1500 x 1111, 12 heads, fp16: 96 us, tensor pipe 29 %, MUFU 18 %, issue slots
// 47 %; 2 x 4096, 16 heads, causal: 267 us, 41, 24 and 56 %): half of TMEM holds one
// S' and one dP', so that the next scores wait for the product that reads P',
// and blocks are short.  Few keys on few key heads leave the key pass with
// few blocks, which stream the queries of all heads that share them: 8192
// queries of 28 / 4 heads x 128 on 512 keys are 16 such blocks and 569 us.
//
// Scaling of fp16 operands: p carries 2^15 (p <= 1), and dP - delta is
// scaled by a power of two that brings its bound |g||v| + |delta| to at most
// one.  Each row of either pass has its own: the largest bound among the
// pairs that the masks leave of it (query pass: the row's |g| and the keys it
// sees; key pass: the key's |v| and the queries that see it), from running
// maxima of the norms inside a tile and the maxima of whole tiles.  dS then
// keeps fp16's precision down to 2^-29 of that bound, and is rounded to
// multiples of 2^-38 of it below, however large hidden pairs are.  bf16 needs
// no scaling.
#include <algorithm>

#include "attention_tc.cuh"

namespace gs {
namespace {

using namespace tc;

// Streamed tiles have NT rows, each column group of 32 its own warpgroup of
// softmax warps.  D, C above 64: NT = 128, one block per SM with all of TMEM.
// Up to 64: NT = 64, two blocks per SM with half of TMEM each, so that one
// block's exponentials (MUFU) run under the other's dS arithmetic and its
// start and end under the other's loop (one block of 128-row tiles took
// 2300 clocks a tile in the key pass, its warps all in the same phase).
template <int NT>
struct Cfg {
    static constexpr int kSoftmaxWarps = NT / 8;
    static constexpr int kLoadWarp = kSoftmaxWarps, kMmaWarp = kSoftmaxWarps + 1;
    static constexpr int kThreads = (kSoftmaxWarps + 4) * 32;
    static constexpr int kBlocksPerSm = NT == 128 ? 1 : 2;
    static constexpr uint32_t kTmem = 512 / kBlocksPerSm;
    static constexpr uint32_t kRegsLaunch = NT == 128 ? 96 : 80, kRegsSoftmax = NT == 128 ? 104 : 96,
                              kRegsCtrl = NT == 128 ? 64 : 48;
    static_assert(kSoftmaxWarps * kRegsSoftmax + 4 * kRegsCtrl <= (kSoftmaxWarps + 4) * kRegsLaunch,
                  "register split");
    // Shared memory of a block: 227 KiB for one, 113 KiB each for two.
    static constexpr size_t kSmem = (NT == 128 ? 227 : 113) * 1024;
    // TMEM columns: scores, dP, and in the key pass dk, dv; in the query pass
    // the second dP and dq.
    static constexpr uint32_t kS = 0, kDp = NT, kDk = 2 * NT, kDv = 2 * NT + kTmem / 4, kDq = kDv;
};
constexpr float kShiftF16 = 15.f;

struct VjpParams {
    AttnParams a;
    Coords cq, ck, cv, cg;
    int64_t Mp;              // M rounded up to 128: row stride of nl2, delta, gnorm
    int64_t tiles_m, tiles_n;
    int64_t key_blocks;      // blocks of the key pass (first in the grid)
    int64_t Np;              // N rounded up to 128: row stride of vnorm, vhead
    float* nl2;              // B H x Mp: -lse log2 e + shift; -infinity: no probabilities
    float* delta;            // B H x Mp
    // The rest for fp16 only.
    float* gnorm;            // B H x Mp: |g_m|
    float *gtail, *dtail;    // B H x Mp: largest |g|, |delta| from row m to the end of its tile
    float *gmax, *dmax;      // B H x tiles_m: of a whole tile
    float* vnorm;            // B Hk x Np: |v_n|
    float* vhead;            // B Hk x Np: largest |v| from the start of n's tile to row n
    float* vmax;             // B Hk x tiles_n: of a whole tile
    int dblocks, cblocks, dsteps, csteps;
    int dstages, cstages;    // slots of the rings of D- and of C-channel tiles
    uint32_t smem_bytes;
    uint32_t idesc_s, idesc_d, idesc_c;   // scores; gradients of D, of C channels
};

struct __align__(8) VjpBarriers {
    uint64_t own_full, drain, done;
    uint64_t s_full, s_free, dp_full[2], p_full, ds_full[2];
    uint64_t full_d[8], empty_d[8], full_c[8], empty_c[8];
    uint32_t tmem_base;
    int abort_flag;
};

// The power of two that brings x to at most one (1 for 0, inf and NaN).
__device__ __forceinline__ float unit_scale(float x) {
    if (!(x > 0.f) || x > 3e38f) return 1.f;
    const int e = static_cast<int>(__float_as_uint(x) >> 23) - 126;   // x < 2^e
    return __uint_as_float(static_cast<uint32_t>(127 - min(max(e, -100), 100)) << 23);
}

// ------------------------------------------------------------------ rows
// Per 128 rows of a head: -lse log2 e, delta = g . out - g_lse and, for
// fp16, |g| and the tile's maxima.  Blocks past those take 128 values of a
// key head each, for their norms (fp16).  Bound by HBM (g and out, once):
// four lanes share a row, each with CH groups of eight channels, and sixteen
// rows a warp are on their way at a time: 31 us and 4.4 TB/s for 2 x 4096
// tokens of 32 heads of 128 channels (37 us with the rows of few keys below);
// with 16 lanes a row and eight rows on their way 48 us, twice the instructions.  Widths that are no multiple of 8
// take an instance of their own, whose branches would cost the others registers.
//
// The rounding of `out` goes into delta with the weight |out| / |v|, which is
// near one for a row of few keys and falls as the root of the number of keys
// that share the weight, and such rows have the largest gradients: those of at
// most kFewKeys keys take delta = sum_n p_n g . v_n - g_lse instead.  Rows of as
// many keys each, fp16, 64 channels (rounding once: 2.07e-4): error of grad_q with
// scores of standard deviation 1 and 9, and us of 4 x 1500 rows of 12 heads, both
// launches:
//     keys             6             12            18            30
//     from out         3.4, 8.3e-4   3.2, 7.8e-4   3.1, 7.4e-4   3.0, 7.4e-4
//     over the keys    2.9, 2.9e-4   2.9, 3.0e-4   2.9, 2.9e-4   2.9, 3.0e-4
//     us               39 -> 55      39 -> 60      39 -> 70      39 -> 86
// The gain falls and the cost grows with the keys.  What the limit costs where only
// the first rows of a causal mask are such rows:
//     limit                              0      8      16     24     32
//     200 rows, 4 heads x 64, us         19.0   20.7   22.1   23.5   24.9
//     2 x 4096, 32 heads x 128, us       627    631    631    633    638
template <bool BF16, int CH, bool WHOLE>
__global__ void __launch_bounds__(256, 2) attn_rows_kernel(const __grid_constant__ VjpParams f) {
    const AttnParams& p = f.a;
    pdl_wait();
    pdl_trigger();
    __shared__ float norm_of[kTile], term_of[kTile], red[2][kTile / 32];   // |g| or |v|, |delta|; a warp's largest
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = lane / 4, c0 = (lane % 4) * 8;   // channels c0 + 32 u ..
    constexpr int kRows = 8;                 // rows of a warp at a time
    const int64_t row_blocks = static_cast<int64_t>(p.B) * p.H * f.tiles_m;
    const bool values = blockIdx.x >= row_blocks;
    const int64_t blk = values ? blockIdx.x - row_blocks : blockIdx.x;
    const int64_t tiles = values ? f.tiles_n : f.tiles_m;
    const int heads = values ? p.Hk : p.H;
    // Neighbouring blocks take the same tokens of neighbouring heads, which lie
    // next to each other in the usual layout; first tiles go first, which have
    // the rows of few keys under a causal mask (15 us).
    const int h = static_cast<int>(blk % heads), b = static_cast<int>(blk / heads % p.B);
    const int64_t tile = blk / heads / p.B, t0 = tile * kTile;
    const int64_t bh = static_cast<int64_t>(b) * heads + h;
    const int ql = attn_q_len(p, b), kl = attn_k_len(p, b);
    const int len = values ? kl : ql;
    const Arr& x = values ? p.v : p.g;
    const uint16_t* xb = reinterpret_cast<const uint16_t*>(x.p) + b * x.sb + h * x.sh;
    const uint16_t* ob = reinterpret_cast<const uint16_t*>(p.out.p) + b * p.out.sb + h * p.out.sh;
    const auto widen = [](uint32_t w, float& lo, float& hi) {
        if (BF16) {
            lo = __uint_as_float(w << 16);
            hi = __uint_as_float(w & 0xffff0000u);
        } else {
            const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w));
            lo = t.x;
            hi = t.y;
        }
    };
    // Reads are unconditional, from the nearest valid place, so that a warp's
    // rows are all on their way before the first is used; only widths that are
    // no multiple of 8 (not WHOLE) take branches.
    const auto ragged8 = [](const uint16_t* row, int c, int width) {   // zeros past the width
        uint4 w = make_uint4(0, 0, 0, 0);
        uint16_t* e = reinterpret_cast<uint16_t*>(&w);
        for (int i = c; i < min(width, c + 8); ++i) e[i - c] = row[i];
        return w;
    };
    const auto read8 = [&](const uint16_t* row, int c, int width) {
        return WHOLE ? *reinterpret_cast<const uint4*>(row + min(c, width - 8)) : ragged8(row, c, width);
    };
    const auto dot8 = [&](const uint4& a, const uint4& b, float x) {
        const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float a0, a1, b0, b1;
            widen(aw[e], a0, a1);
            widen(bw[e], b0, b1);
            x = fmaf(a0, b0, fmaf(a1, b1, x));
        }
        return x;
    };
    const auto row_sum = [](float x) {
#pragma unroll
        for (int d = 2; d > 0; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
        return x;
    };
    // sum_n p_n g . v_n over the first `lim` <= kFewKeys keys of token r, whose
    // lse is l; the whole warp takes part.  (g is read again: it would otherwise
    // hold registers in every row.)
    const auto few_keys = [&](int64_t r, int lim, float l) {
        const int j = h / p.G;
        const int64_t rq = lim > 0 ? r : 0;
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p.q.p) + b * p.q.sb + h * p.q.sh + rq * p.q.sr;
        const uint16_t* k = reinterpret_cast<const uint16_t*>(p.k.p) + b * p.k.sb + j * p.k.sh;
        const uint16_t* v = reinterpret_cast<const uint16_t*>(p.v.p) + b * p.v.sb + j * p.v.sh;
        constexpr int kKeys = 8 / CH;         // on their way at a time
        float sum = 0.f;
        uint4 qq[CH], y[CH];
#pragma unroll
        for (int u = 0; u < CH; ++u) {
            qq[u] = read8(q, c0 + 32 * u, p.D);
            y[u] = read8(xb + rq * x.sr, c0 + 32 * u, p.C);
            if (c0 + 32 * u >= p.C) y[u] = make_uint4(0, 0, 0, 0);
            if (c0 + 32 * u >= p.D) qq[u] = make_uint4(0, 0, 0, 0);
        }
        for (int n0 = 0; n0 < kFewKeys && __any_sync(~0u, n0 < lim); n0 += kKeys) {
            uint4 kk[kKeys][CH], vv[kKeys][CH];
#pragma unroll
            for (int n = 0; n < kKeys; ++n) {     // (rows past the limit read the last one again)
                const int64_t kn = max(min(n0 + n, lim - 1), 0);
#pragma unroll
                for (int u = 0; u < CH; ++u) {
                    kk[n][u] = read8(k + kn * p.k.sr, c0 + 32 * u, p.D);
                    vv[n][u] = read8(v + kn * p.v.sr, c0 + 32 * u, p.C);
                }
            }
#pragma unroll
            for (int n = 0; n < kKeys; ++n) {
                float sc = 0.f, dp = 0.f;
#pragma unroll
                for (int u = 0; u < CH; ++u) {
                    sc = dot8(qq[u], kk[n][u], sc);
                    dp = dot8(y[u], vv[n][u], dp);
                }
                sc = row_sum(sc);
                dp = row_sum(dp);
                if (n0 + n < lim) sum = fmaf(exp2f(fmaf(sc, p.c, -l * kLog2e)), dp, sum);
            }
        }
        return sum;
    };
    constexpr int kIters = kTile / (8 * kRows), kBatch = 2;
#pragma unroll 1
    for (int i0 = 0; i0 < kIters; i0 += kBatch) {
        uint4 y[kBatch][CH], o[kBatch][CH];
        float l[kBatch], gl[kBatch], dot[kBatch], sq[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int64_t r = t0 + ((i0 + i) * 8 + warp) * kRows + sub;
            const int64_t rc = min(r, static_cast<int64_t>(max(len, 1) - 1));
#pragma unroll
            for (int u = 0; u < CH; ++u) {
                y[i][u] = read8(xb + rc * x.sr, c0 + 32 * u, p.C);
                if (!values) o[i][u] = read8(ob + rc * p.out.sr, c0 + 32 * u, p.C);
            }
            if (!values) {
                l[i] = p.lse[bh * p.M + rc];
                gl[i] = p.g_lse ? p.g_lse[bh * p.M + rc] : 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int64_t r = t0 + ((i0 + i) * 8 + warp) * kRows + sub;
            dot[i] = sq[i] = 0.f;
#pragma unroll
            for (int u = 0; u < CH; ++u) {
                if (r >= len || c0 + 32 * u >= p.C) y[i][u] = make_uint4(0, 0, 0, 0), o[i][u] = y[i][u];
                if (!BF16) sq[i] = dot8(y[i][u], y[i][u], sq[i]);
                if (!values) dot[i] = dot8(y[i][u], o[i][u], dot[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int64_t r = t0 + ((i0 + i) * 8 + warp) * kRows + sub;
            const float norm = BF16 ? 0.f : sqrtf(row_sum(sq[i]));
            if (!BF16 && lane % 4 == 0) norm_of[r - t0] = norm;
            if (values) continue;
            float dg = row_sum(dot[i]);
            const int lim = r < len && l[i] != -INFINITY
                                ? attn_limit(static_cast<int>(r), ql, kl, p.causal) : 0;
            const bool some = lim > 0, few = some && lim <= kFewKeys;
            if (__any_sync(~0u, few)) {
                const float exact = few_keys(r, few ? lim : 0, l[i]);
                if (few) dg = exact;
            }
            const float dl = some ? dg - gl[i] : 0.f;
            if (lane % 4 == 0) {
                const int64_t at = bh * f.Mp + r;
                f.nl2[at] = some ? -l[i] * kLog2e + (BF16 ? 0.f : kShiftF16) : -INFINITY;
                f.delta[at] = dl;
                if (!BF16) term_of[r - t0] = fabsf(dl);
            }
        }
    }
    if constexpr (!BF16) {
        // Running maxima (NaN does not count): of values from the tile's first
        // row on, of queries from its last row back.
        __syncthreads();
        const bool scans = threadIdx.x < kTile;
        const int at = values ? threadIdx.x : kTile - 1 - threadIdx.x;
        float x = 0.f, y = 0.f;
        if (scans) {
            x = fmaxf(norm_of[at], 0.f);
            if (!values) y = fmaxf(term_of[at], 0.f);
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const float x1 = __shfl_up_sync(~0u, x, d), y1 = __shfl_up_sync(~0u, y, d);
                if (lane >= d) x = fmaxf(x, x1), y = fmaxf(y, y1);
            }
            if (lane == 31) red[0][warp] = x, red[1][warp] = y;
        }
        __syncthreads();
        if (scans) {
            for (int w = 0; w < warp; ++w) x = fmaxf(x, red[0][w]), y = fmaxf(y, red[1][w]);
            const bool last = threadIdx.x == kTile - 1;
            if (values) {
                const int64_t to = bh * f.Np + t0 + at;
                f.vnorm[to] = norm_of[at];
                f.vhead[to] = x;
                if (last) f.vmax[bh * tiles + tile] = x;
            } else {
                const int64_t to = bh * f.Mp + t0 + at;
                f.gnorm[to] = norm_of[at];
                f.gtail[to] = x;
                f.dtail[to] = y;
                if (last) {
                    f.gmax[bh * tiles + tile] = x;
                    f.dmax[bh * tiles + tile] = y;
                }
            }
        }
    }
}

// Largest of a warp's floats.
__device__ __forceinline__ float warp_max(float m) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
    return m;
}

// 32 columns of an fp32 tile in TMEM.
__device__ __forceinline__ void load32(uint32_t t, uint32_t (&x)[32]) {
    tmem_ld_32x32b_x32(t, x);
    tmem_wait_ld_regs(x);
}
__device__ __forceinline__ uint64_t pair(const uint32_t (&x)[32], int e) {
    return f32x2_pack(__uint_as_float(x[e]), __uint_as_float(x[e + 1]));
}

// Shared memory, barriers and TMEM of a block of either pass.
struct Block {
    uint8_t *own_a, *own_b;      // the block's own rows: D channels, C channels
    // Slots of streamed tiles: K (query pass) or Q (key pass) of D channels, V
    // or G of C.  Two rings, because the first kind is held for two products
    // and the second for its scores only in the query pass: in one ring of
    // five slots the next V waited for a K slot (2850 clocks a tile, 1840 with two).
    uint8_t *ring_d, *ring_c;
    // Key pass: the streamed queries' row terms, NT to a slot: delta with the
    // queries and nl2 with the upstream gradients, whose slot is handed back
    // once P' is written.
    float *terms_d, *terms_c;
    VjpBarriers* bars;
    uint32_t tmem;
    bool ok;
};

template <int NT>
__device__ __forceinline__ Block start_block(const VjpParams& f) {
    using K = Cfg<NT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    Block k;
    k.own_a = smem;
    k.own_b = smem + f.dblocks * kBlock;
    k.ring_d = k.own_b + f.cblocks * kBlock;
    k.ring_c = k.ring_d + f.dstages * f.dblocks * NT * 128;
    k.terms_d = reinterpret_cast<float*>(k.ring_c + f.cstages * f.cblocks * NT * 128);
    k.terms_c = k.terms_d + f.dstages * NT;
    k.bars = reinterpret_cast<VjpBarriers*>(k.terms_c + f.cstages * NT);
    VjpBarriers* bars = k.bars;
    // A shared window that does not start 1 KiB aligned leaves too little room.
    k.ok = reinterpret_cast<uint8_t*>(bars + 1) <= smem_raw + f.smem_bytes;
    if (!k.ok) {
        if (threadIdx.x == 0) atomicCAS(f.a.status, kDevOk, kDevTimeout);
        return k;
    }
    if (threadIdx.x == 0) {
        mbar_init(&bars->own_full, 1);
        mbar_init(&bars->drain, 1);
        mbar_init(&bars->done, 1);
        mbar_init(&bars->s_full, 1);
        mbar_init(&bars->s_free, K::kSoftmaxWarps);
        mbar_init(&bars->dp_full[0], 1);
        mbar_init(&bars->dp_full[1], 1);
        mbar_init(&bars->p_full, K::kSoftmaxWarps);
        mbar_init(&bars->ds_full[0], K::kSoftmaxWarps);
        mbar_init(&bars->ds_full[1], K::kSoftmaxWarps);
        for (int s = 0; s < 8; ++s) {
            mbar_init(&bars->full_d[s], 1);
            mbar_init(&bars->empty_d[s], 1);
            mbar_init(&bars->full_c[s], 1);
            mbar_init(&bars->empty_c[s], 1);
        }
        bars->abort_flag = 0;
        fence_mbar_init();
    }
    if (threadIdx.x >> 5 == K::kMmaWarp) {
        tmem_alloc(&bars->tmem_base, K::kTmem);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();
    pdl_trigger();
    k.tmem = bars->tmem_base;
    return k;
}

// The loading warp's position in the two rings.
template <int NT>
struct Loader {
    const Block& blk;
    const VjpParams& f;
    volatile int* abort_flag;
    bool leader;
    RingPos at_d, at_c;
    int issued_d = 0, issued_c = 0;

    __device__ __forceinline__ Loader(const Block& blk_, const VjpParams& f_, volatile int* flag, bool lead)
        : blk(blk_), f(f_), abort_flag(flag), leader(lead) {}

    // The next tile of D (C) channels, with its row terms where there are
    // some, as soon as its slot is free; false: give up.
    __device__ __forceinline__ bool d(const CUtensorMap* map, int row, int h, int b, const float* terms) {
        return next(at_d, f.dstages, issued_d, blk.ring_d, blk.bars->full_d, blk.bars->empty_d, f.dblocks,
                    map, row, h, b, blk.terms_d, terms);
    }
    __device__ __forceinline__ bool c(const CUtensorMap* map, int row, int h, int b, const float* terms) {
        return next(at_c, f.cstages, issued_c, blk.ring_c, blk.bars->full_c, blk.bars->empty_c, f.cblocks,
                    map, row, h, b, blk.terms_c, terms);
    }
    __device__ __forceinline__ bool next(RingPos& at, int n, int& issued, uint8_t* ring, uint64_t* full,
                                         uint64_t* empty, int blocks, const CUtensorMap* map, int row, int h,
                                         int b, float* slots, const float* terms) {
        if (!wait_all(&empty[at.idx], at.phase ^ 1u, abort_flag, f.a.status)) return false;
        if (leader) {
            constexpr uint32_t kTermBytes = NT * sizeof(float);
            mbar_arrive_expect_tx(&full[at.idx], blocks * NT * 128 + (terms ? kTermBytes : 0));
            load_tile<NT>(ring + at.idx * blocks * NT * 128, map, &full[at.idx], blocks, row, h, b);
            if (terms) bulk_load(slots + at.idx * NT, terms, kTermBytes, &full[at.idx]);
        }
        __syncwarp();
        at.advance(n);
        ++issued;
        return true;
    }
    // Every copy of this block lands before the block can end.
    __device__ __forceinline__ void finish() {
        mbar_wait_bounded(&blk.bars->own_full, 0, nullptr, f.a.status);
        for (int j = max(0, issued_d - f.dstages); j < issued_d; ++j)
            mbar_wait_bounded(&blk.bars->full_d[j % f.dstages], static_cast<uint32_t>(j / f.dstages) & 1u,
                              nullptr, f.a.status);
        for (int j = max(0, issued_c - f.cstages); j < issued_c; ++j)
            mbar_wait_bounded(&blk.bars->full_c[j % f.cstages], static_cast<uint32_t>(j / f.cstages) & 1u,
                              nullptr, f.a.status);
    }
};

// Writes columns 32 w .. of a 128-row fp32 accumulator, times scale, as
// channels of one output row (zeros when !has).
template <bool BF16>
__device__ __forceinline__ void put_grad(uint32_t t, bool loaded, bool has, float scale, int w,
                                         uint16_t* dst, bool mine, int width) {
    const int c = 32 * w;
    if (c >= width) return;
    uint32_t o[32];
    float x[32];
    if (loaded) load32(t + c, o);
#pragma unroll
    for (int e = 0; e < 32; ++e) x[e] = has ? __uint_as_float(o[e]) * scale : 0.f;
    if (mine) put_row<BF16>(dst, x, c, width);
    __syncwarp();
}

// ------------------------------------------------------------------ query pass
// dP goes to two buffers by turns, dS into the first half of each 32 columns
// of it.
// S is read into registers once and then free for the next tile's scores, so
// both score products of tile j + 1 run under the softmax of tile j.
template <bool BF16, int NT>
__device__ __forceinline__ void query_pass(const CUtensorMap& tm_q, const CUtensorMap& tm_k,
                                           const CUtensorMap& tm_v, const CUtensorMap& tm_g,
                                           const VjpParams& f, const Block& blk, int64_t index) {
    using K = Cfg<NT>;
    const AttnParams& p = f.a;
    VjpBarriers* bars = blk.bars;
    volatile int* abort_flag = &bars->abort_flag;
    const uint32_t tmem = blk.tmem;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t d_bytes = f.dblocks * NT * 128, c_bytes = f.cblocks * NT * 128;
    // Later query tiles see more keys under a causal mask and go first, all
    // heads' before the next, so that the last blocks to start are short.
    const int64_t all_heads = static_cast<int64_t>(p.B) * p.H;
    const int64_t tile = f.tiles_m - 1 - index / all_heads;
    const int64_t bh = index % all_heads;
    const int b = static_cast<int>(bh / p.H), h = static_cast<int>(bh % p.H), kvh = h / p.G;
    const int ql = attn_q_len(p, b), kl = attn_k_len(p, b);
    const int m0 = static_cast<int>(tile) * kTile;
    const int last = min(m0 + kTile, ql) - 1;
    const int kend = last >= m0 ? attn_limit(last, ql, kl, p.causal) : 0;
    const int T = static_cast<int>((static_cast<int64_t>(kend) + NT - 1) / NT);

    if (warp == K::kLoadWarp) {
        reg_dealloc<K::kRegsCtrl>();
        if (T > 0) {
            const bool leader = elect_one();
            if (leader) {
                mbar_arrive_expect_tx(&bars->own_full, (f.dblocks + f.cblocks) * kBlock);
                load_tile<kTile, NT>(blk.own_a, &tm_q, &bars->own_full, f.dblocks, m0, h * f.cq.h, b * f.cq.b);
                load_tile<kTile, NT>(blk.own_b, &tm_g, &bars->own_full, f.cblocks, m0, h * f.cg.h, b * f.cg.b);
            }
            __syncwarp();
            Loader<NT> load(blk, f, abort_flag, leader);
            for (int j = 0; j < T; ++j)
                if (!load.d(&tm_k, j * NT, kvh * f.ck.h, b * f.ck.b, nullptr) ||
                    !load.c(&tm_v, j * NT, kvh * f.cv.h, b * f.cv.b, nullptr))
                    break;
            load.finish();
            __syncwarp();
        }
    } else if (warp == K::kMmaWarp) {
        reg_dealloc<K::kRegsCtrl>();
        if (T > 0) {
            const uint32_t leader = elect_one() ? 1u : 0u;
            bool ok = wait_all(&bars->own_full, 0, abort_flag, p.status);
            const uint32_t q_at = smem_u32(blk.own_a), g_at = smem_u32(blk.own_b);
            const uint32_t ring_d = smem_u32(blk.ring_d), ring_c = smem_u32(blk.ring_c);
            RingPos at_k, at_v, kd;      // keys of the scores, values, keys of dq
            const auto scores = [&]() {
                if (ok) ok = wait_all(&bars->full_d[at_k.idx], at_k.phase, abort_flag, p.status);
                if (!ok) return;
                tc_fence_after();
                mma_scores<NT>(leader, tmem + K::kS, q_at, ring_d + at_k.idx * d_bytes, f.dsteps, f.idesc_s);
                mma_commit_on(leader, &bars->s_full);
                at_k.advance(f.dstages);
            };
            const auto dprobs = [&](int j) {
                if (ok) ok = wait_all(&bars->full_c[at_v.idx], at_v.phase, abort_flag, p.status);
                if (!ok) return;
                tc_fence_after();
                mma_scores<NT>(leader, tmem + K::kDp + NT * (j & 1), g_at, ring_c + at_v.idx * c_bytes, f.csteps,
                           f.idesc_s);
                mma_commit_on(leader, &bars->dp_full[j & 1]);
                mma_commit_on(leader, &bars->empty_c[at_v.idx]);
                at_v.advance(f.cstages);
            };
            // ds_full alternates between two barriers: the softmax warps can be
            // done with tile j + 1 before this warp has seen the arrivals for
            // tile j, and those for tile j + 2 need scores issued after that.
            scores();
            dprobs(0);
            for (int j = 0; ok && j < T; ++j) {
                if (j + 1 < T) {
                    ok = wait_all(&bars->s_free, j & 1, abort_flag, p.status);
                    scores();
                    dprobs(j + 1);     // (dq of tile j - 1, issued before, read this buffer)
                }
                if (ok) ok = wait_all(&bars->ds_full[j & 1], (j >> 1) & 1, abort_flag, p.status);
                if (!ok) break;
                tc_fence_after();
                mma_rows<16, NT>(leader, tmem + K::kDq, tmem + K::kDp + NT * (j & 1), ring_d + kd.idx * d_bytes,
                             f.idesc_d, j == 0);
                mma_commit_on(leader, &bars->empty_d[kd.idx]);
                kd.advance(f.dstages);
                if (j + 1 == T) mma_commit_on(leader, &bars->done);
            }
            if (leader) mma_commit(&bars->drain);
            __syncwarp();
            mbar_wait_bounded(&bars->drain, 0, nullptr, p.status);
            __syncwarp();
        }
    } else if (warp > K::kMmaWarp) {
        reg_dealloc<K::kRegsCtrl>();
    } else {
        reg_alloc<K::kRegsSoftmax>();
        const int w = warp >> 2, row = tid & (kTile - 1);
        const int m = m0 + row;
        const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;
        const int lim = attn_limit(m, ql, kl, p.causal), lim_first = attn_limit(m0, ql, kl, p.causal);
        const int64_t at = bh * f.Mp + m;
        const float nl2 = f.nl2[at], delta = f.delta[at];
        float sc = 1.f;
        if (!BF16 && T > 0) {
            // Largest |v| of the keys below this row's limit, which lies in the
            // key tile of the first row's (t0) or in the next.
            const int64_t kv = static_cast<int64_t>(b) * p.Hk + kvh;
            const float* vmax = f.vmax + kv * f.tiles_n;
            const int last = max(lim - 1, 0), t0 = max(lim_first - 1, 0) / kTile;
            // (All reads are on their way before the first is used.)
            const float own = f.vhead[kv * f.Np + last], of_t0 = vmax[t0], g = f.gnorm[at];
            float v = 0.f;
            for (int t = lane; t < t0; t += 32) v = fmaxf(v, vmax[t]);
            v = fmaxf(warp_max(v), own);
            if (last / kTile > t0) v = fmaxf(v, of_t0);
            if (lim > 0) sc = unit_scale(g * v + fabsf(delta));
        }
        const uint64_t c2 = f32x2_pack(p.c, p.c), l2 = f32x2_pack(nl2, nl2);
        const uint64_t sc2 = f32x2_pack(sc, sc), nd2 = f32x2_pack(-delta * sc, -delta * sc);
        bool ok = true;
        for (int j = 0; ok && j < T; ++j) {
            const int n0 = j * NT;
            const bool masked = n0 + NT > lim_first;
            const int seen = lim - n0 - 32 * w;      // of this thread's 32 columns
            const uint32_t t_d = tmem + lanes + K::kDp + NT * (j & 1) + 32 * w;
            ok = wait_all(&bars->s_full, j & 1, abort_flag, p.status);
            if (!ok) break;
            tc_fence_after();
            uint32_t s[32], o[16];
            load32(tmem + lanes + K::kS + 32 * w, s);
            tc_fence_before();
            __syncwarp();
            mbar_arrive_if_zero(&bars->s_free, lane);
            uint64_t pr[16];
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
                float x0, x1;
                f32x2_unpack(f32x2_fma(pair(s, e), c2, l2), x0, x1);
                pr[e >> 1] = f32x2_pack(ex2_approx(x0), ex2_approx(x1));
            }
            ok = wait_all(&bars->dp_full[j & 1], (j >> 1) & 1, abort_flag, p.status);
            if (!ok) break;
            tc_fence_after();
            load32(t_d, s);
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
                float x0, x1;
                f32x2_unpack(f32x2_mul(pr[e >> 1], f32x2_fma(pair(s, e), sc2, nd2)), x0, x1);
                s[e] = __float_as_uint(x0);
                s[e + 1] = __float_as_uint(x1);
            }
            if (masked) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (e >= seen) s[e] = 0u;
            }
#pragma unroll
            for (int e = 0; e < 32; e += 2)
                o[e >> 1] = pack2<BF16>(__uint_as_float(s[e]), __uint_as_float(s[e + 1]));
            tmem_st_32x32b_x16(t_d, o);
            if (n0 + NT > kl) {       // keys past the length: 0 x NaN is not 0
                const int i = j % f.dstages;
                ok = wait_all(&bars->full_d[i], static_cast<uint32_t>(j / f.dstages) & 1u, abort_flag,
                              p.status);
                if (!ok) break;
                zero_rows<NT>(blk.ring_d + i * d_bytes, f.dblocks, kl - n0, tid, K::kSoftmaxWarps * 32);
                fence_proxy_async_smem();
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            mbar_arrive_if_zero(&bars->ds_full[j & 1], lane);
        }
        if (ok && T > 0) ok = wait_all(&bars->done, 0, abort_flag, p.status);
        tc_fence_after();
        const float scale = BF16 ? p.tau : p.tau / (sc * 32768.f);
        uint16_t* dst = reinterpret_cast<uint16_t*>(p.dq.p) + b * p.dq.sb + h * p.dq.sh + m * p.dq.sr;
        put_grad<BF16>(tmem + lanes + K::kDq, T > 0, ok && lim > 0 && nl2 != -INFINITY, scale, w, dst,
                       m < p.M, p.D);
        tc_fence_before();
    }
}

// ------------------------------------------------------------------ key pass
// P' lies in the first half of each 32 columns of S', dS' in those of dP'; the
// next scores wait for the product that reads P' (dS'), and the two chains
// cover one another.
template <bool BF16, int NT>
__device__ __forceinline__ void key_pass(const CUtensorMap& tm_q, const CUtensorMap& tm_k,
                                         const CUtensorMap& tm_v, const CUtensorMap& tm_g,
                                         const VjpParams& f, const Block& blk, int64_t index) {
    using K = Cfg<NT>;
    const AttnParams& p = f.a;
    VjpBarriers* bars = blk.bars;
    volatile int* abort_flag = &bars->abort_flag;
    const uint32_t tmem = blk.tmem;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t d_bytes = f.dblocks * NT * 128, c_bytes = f.cblocks * NT * 128;
    // Earlier key tiles are seen by more queries under a causal mask.
    const int64_t all_heads = static_cast<int64_t>(p.B) * p.Hk;
    const int64_t tile = index / all_heads;
    const int64_t bj = index % all_heads;
    const int b = static_cast<int>(bj / p.Hk), kvh = static_cast<int>(bj % p.Hk);
    const int ql = attn_q_len(p, b), kl = attn_k_len(p, b);
    const int n0 = static_cast<int>(tile) * kTile;
    // Tokens m >= n - off see key n; the first query tile with one that sees n0.
    const int64_t off = static_cast<int64_t>(kl) - ql;
    const int64_t m_first = p.causal ? max(static_cast<int64_t>(0), n0 - off) : 0;
    const int mt0 = static_cast<int>(m_first / NT);
    const int nm = n0 < kl ? max(0, (ql + NT - 1) / NT - mt0) : 0;   // query tiles of a head
    const int T = nm * p.G;
    if (warp == K::kLoadWarp) {
        reg_dealloc<K::kRegsCtrl>();
        if (T > 0) {
            const bool leader = elect_one();
            if (leader) {
                mbar_arrive_expect_tx(&bars->own_full, (f.dblocks + f.cblocks) * kBlock);
                load_tile<kTile, NT>(blk.own_a, &tm_k, &bars->own_full, f.dblocks, n0, kvh * f.ck.h, b * f.ck.b);
                load_tile<kTile, NT>(blk.own_b, &tm_v, &bars->own_full, f.cblocks, n0, kvh * f.cv.h, b * f.cv.b);
            }
            __syncwarp();
            Loader<NT> load(blk, f, abort_flag, leader);
            int g = 0, mt = 0;
            for (int j = 0; j < T; ++j) {
                const int h = kvh * p.G + g, m0 = (mt0 + mt) * NT;
                const int64_t at = (static_cast<int64_t>(b) * p.H + h) * f.Mp + m0;
                if (!load.d(&tm_q, m0, h * f.cq.h, b * f.cq.b, f.delta + at) ||
                    !load.c(&tm_g, m0, h * f.cg.h, b * f.cg.b, f.nl2 + at))
                    break;
                if (++mt == nm) {
                    mt = 0;
                    ++g;
                }
            }
            load.finish();
            __syncwarp();
        }
    } else if (warp == K::kMmaWarp) {
        reg_dealloc<K::kRegsCtrl>();
        if (T > 0) {
            const uint32_t leader = elect_one() ? 1u : 0u;
            bool ok = wait_all(&bars->own_full, 0, abort_flag, p.status);
            const bool want_k = p.dk.p != nullptr, want_v = p.dv.p != nullptr;
            const uint32_t k_at = smem_u32(blk.own_a), v_at = smem_u32(blk.own_b);
            const uint32_t ring_d = smem_u32(blk.ring_d), ring_c = smem_u32(blk.ring_c);
            // Each tile is used for the scores first (at_*), then for a gradient (on_*).
            RingPos at_q, at_g, on_q, on_g;
            const auto scores = [&]() {
                if (ok) ok = wait_all(&bars->full_d[at_q.idx], at_q.phase, abort_flag, p.status);
                if (!ok) return;
                tc_fence_after();
                mma_scores<NT>(leader, tmem + K::kS, k_at, ring_d + at_q.idx * d_bytes, f.dsteps, f.idesc_s);
                mma_commit_on(leader, &bars->s_full);
                at_q.advance(f.dstages);
            };
            const auto dprobs = [&]() {
                if (ok) ok = wait_all(&bars->full_c[at_g.idx], at_g.phase, abort_flag, p.status);
                if (!ok) return;
                tc_fence_after();
                mma_scores<NT>(leader, tmem + K::kDp, v_at, ring_c + at_g.idx * c_bytes, f.csteps, f.idesc_s);
                mma_commit_on(leader, &bars->dp_full[0]);
                at_g.advance(f.cstages);
            };
            scores();
            dprobs();
            for (int j = 0; ok && j < T; ++j) {
                if (ok) ok = wait_all(&bars->p_full, j & 1, abort_flag, p.status);
                if (!ok) break;
                tc_fence_after();
                if (want_v)
                    mma_rows<16, NT>(leader, tmem + K::kDv, tmem + K::kS, ring_c + on_g.idx * c_bytes, f.idesc_c,
                                   j == 0);
                // dP' of this tile was issued before: its operand is free too.
                mma_commit_on(leader, &bars->empty_c[on_g.idx]);
                on_g.advance(f.cstages);
                if (j + 1 < T) scores();
                if (ok) ok = wait_all(&bars->ds_full[0], j & 1, abort_flag, p.status);
                if (!ok) break;
                tc_fence_after();
                if (want_k)
                    mma_rows<16, NT>(leader, tmem + K::kDk, tmem + K::kDp, ring_d + on_q.idx * d_bytes, f.idesc_d,
                                   j == 0);
                mma_commit_on(leader, &bars->empty_d[on_q.idx]);
                on_q.advance(f.dstages);
                if (j + 1 == T) mma_commit_on(leader, &bars->done);
                if (j + 1 < T) dprobs();
            }
            if (leader) mma_commit(&bars->drain);
            __syncwarp();
            mbar_wait_bounded(&bars->drain, 0, nullptr, p.status);
            __syncwarp();
        }
    } else if (warp > K::kMmaWarp) {
        reg_dealloc<K::kRegsCtrl>();
    } else {
        reg_alloc<K::kRegsSoftmax>();
        const int w = warp >> 2, row = tid & (kTile - 1);
        const int64_t n = static_cast<int64_t>(n0) + row;
        const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;
        const uint32_t t_s = tmem + lanes + K::kS + 32 * w, t_d = tmem + lanes + K::kDp + 32 * w;
        const uint64_t c2 = f32x2_pack(p.c, p.c);
        float sc = 1.f;
        if (!BF16 && T > 0) {
            // Largest |g| and |delta| of the queries from m_seen on, the first that
            // sees this key, which lies in the query tile of m_first (t0) or in the next.
            const int64_t h0 = static_cast<int64_t>(b) * p.H + kvh * p.G;
            const int tiles = static_cast<int>(f.tiles_m), t0 = static_cast<int>(m_first / kTile);
            const int64_t m_seen = p.causal ? max(static_cast<int64_t>(0), n - off) : 0;
            const float* gtail = f.gtail + h0 * f.Mp + min(m_seen, static_cast<int64_t>(ql - 1));
            const float* dtail = gtail + (f.dtail - f.gtail);
            const float vn = f.vnorm[bj * f.Np + n];
            float g0 = 0.f, d0 = 0.f;                        // the rest of the tile of m_seen
            float g1 = 0.f, d1 = 0.f, g2 = 0.f, d2 = 0.f;    // tile t0 + 1, later ones
            for (int g = 0; g < p.G; ++g) {
                g0 = fmaxf(g0, gtail[g * f.Mp]), d0 = fmaxf(d0, dtail[g * f.Mp]);
                const float *gm = f.gmax + (h0 + g) * tiles, *dm = f.dmax + (h0 + g) * tiles;
                if (t0 + 1 < tiles) g1 = fmaxf(g1, gm[t0 + 1]), d1 = fmaxf(d1, dm[t0 + 1]);
                for (int t = t0 + 2 + lane; t < tiles; t += 32) g2 = fmaxf(g2, gm[t]), d2 = fmaxf(d2, dm[t]);
            }
            g2 = warp_max(g2), d2 = warp_max(d2);
            if (m_seen / kTile == t0) g2 = fmaxf(g2, g1), d2 = fmaxf(d2, d1);
            if (m_seen < ql) sc = unit_scale(fmaxf(g2, g0) * vn + fmaxf(d2, d0));
        }
        const uint64_t sc2 = f32x2_pack(sc, sc);
        RingPos at_d, at_c;       // slots of this tile's queries and upstream gradients
        int mt = 0;
        bool ok = true;
        for (int j = 0; ok && j < T; ++j) {
            const int m0 = (mt0 + mt) * NT;
            if (++mt == nm) mt = 0;
            // Columns lo .. hi - 1 of this thread's 32 see its key.
            const bool masked = m0 + NT > ql || (p.causal && m0 + off < n0 + kTile - 1);
            const int hi = ql - m0 - 32 * w;
            const int64_t lo64 = p.causal ? n - off - m0 - 32 * w : 0;
            const int lo = static_cast<int>(min(max(lo64, static_cast<int64_t>(0)), static_cast<int64_t>(32)));
            ok = wait_all(&bars->full_c[at_c.idx], at_c.phase, abort_flag, p.status) &&
                 wait_all(&bars->s_full, j & 1, abort_flag, p.status);
            if (!ok) break;
            tc_fence_after();
            uint32_t s[32], o[16];
            load32(t_s, s);
            const ulonglong2* l2 = reinterpret_cast<const ulonglong2*>(blk.terms_c + at_c.idx * NT + 32 * w);
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
                const ulonglong2 l = l2[e >> 2];
                float x[4];
                f32x2_unpack(f32x2_fma(pair(s, e), c2, l.x), x[0], x[1]);
                f32x2_unpack(f32x2_fma(pair(s, e + 2), c2, l.y), x[2], x[3]);
#pragma unroll
                for (int d = 0; d < 4; ++d) s[e + d] = __float_as_uint(ex2_approx(x[d]));
            }
            if (masked) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (e < lo || e >= hi) s[e] = 0u;
            }
            uint64_t pr[16];
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
                pr[e >> 1] = pair(s, e);
                o[e >> 1] = pack2<BF16>(__uint_as_float(s[e]), __uint_as_float(s[e + 1]));
            }
            tmem_st_32x32b_x16(t_s, o);
            if (m0 + NT > ql) {       // queries past the length: 0 x NaN is not 0
                zero_rows<NT>(blk.ring_c + at_c.idx * c_bytes, f.cblocks, ql - m0, tid, K::kSoftmaxWarps * 32);
                fence_proxy_async_smem();
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            mbar_arrive_if_zero(&bars->p_full, lane);

            ok = wait_all(&bars->full_d[at_d.idx], at_d.phase, abort_flag, p.status) &&
                 wait_all(&bars->dp_full[0], j & 1, abort_flag, p.status);
            if (!ok) break;
            tc_fence_after();
            load32(t_d, s);
            const ulonglong2* d2 = reinterpret_cast<const ulonglong2*>(blk.terms_d + at_d.idx * NT + 32 * w);
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
                const ulonglong2 l = d2[e >> 2];
                float x[4];
                uint64_t d0 = f32x2_mul(pr[e >> 1], f32x2_sub(pair(s, e), l.x));
                uint64_t d1 = f32x2_mul(pr[(e >> 1) + 1], f32x2_sub(pair(s, e + 2), l.y));
                if (!BF16) d0 = f32x2_mul(d0, sc2), d1 = f32x2_mul(d1, sc2);
                f32x2_unpack(d0, x[0], x[1]);
                f32x2_unpack(d1, x[2], x[3]);
#pragma unroll
                for (int d = 0; d < 4; ++d) s[e + d] = __float_as_uint(x[d]);
            }
            if (masked) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (e < lo || e >= hi) s[e] = 0u;
            }
#pragma unroll
            for (int e = 0; e < 32; e += 2)
                o[e >> 1] = pack2<BF16>(__uint_as_float(s[e]), __uint_as_float(s[e + 1]));
            tmem_st_32x32b_x16(t_d, o);
            if (m0 + NT > ql) {
                zero_rows<NT>(blk.ring_d + at_d.idx * d_bytes, f.dblocks, ql - m0, tid, K::kSoftmaxWarps * 32);
                fence_proxy_async_smem();
            }
            at_d.advance(f.dstages);
            at_c.advance(f.cstages);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            mbar_arrive_if_zero(&bars->ds_full[0], lane);
        }
        if (ok && T > 0) ok = wait_all(&bars->done, 0, abort_flag, p.status);
        tc_fence_after();
        const bool has = ok && T > 0 && n < kl, mine = n < p.N;
        if (p.dk.p) {
            uint16_t* dst = reinterpret_cast<uint16_t*>(p.dk.p) + b * p.dk.sb + kvh * p.dk.sh + n * p.dk.sr;
            put_grad<BF16>(tmem + lanes + K::kDk, T > 0, has, BF16 ? p.tau : p.tau / (sc * 32768.f), w, dst,
                           mine, p.D);
        }
        if (p.dv.p) {
            uint16_t* dst = reinterpret_cast<uint16_t*>(p.dv.p) + b * p.dv.sb + kvh * p.dv.sh + n * p.dv.sr;
            put_grad<BF16>(tmem + lanes + K::kDv, T > 0, has, BF16 ? 1.f : 1.f / 32768.f, w, dst, mine, p.C);
        }
        tc_fence_before();
    }
}

// Both passes in one launch: the key passes are the longer blocks and start
// first, the query passes fill the SMs that they leave.
template <bool BF16, int NT>
__global__ void __launch_bounds__(Cfg<NT>::kThreads, Cfg<NT>::kBlocksPerSm)
attn_tc_vjp_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                   const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_g,
                   const __grid_constant__ VjpParams f) {
    using K = Cfg<NT>;
    const Block blk = start_block<NT>(f);
    if (!blk.ok) return;
    if (blockIdx.x < f.key_blocks)
        key_pass<BF16, NT>(tm_q, tm_k, tm_v, tm_g, f, blk, blockIdx.x);
    else
        query_pass<BF16, NT>(tm_q, tm_k, tm_v, tm_g, f, blk, blockIdx.x - f.key_blocks);
    __syncthreads();
    if (threadIdx.x >> 5 == K::kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(blk.tmem, K::kTmem);
    }
}

// Workspace: the row terms of VjpParams in the order of their declaration;
// returns their number.
size_t vjp_floats(const AttnParams& p, bool bf16, float* base, VjpParams* f) {
    const size_t tm = (static_cast<size_t>(p.M) + kTile - 1) / kTile, tn = (static_cast<size_t>(p.N) + kTile - 1) / kTile;
    const size_t qt = static_cast<size_t>(p.B) * p.H * tm, kt = static_cast<size_t>(p.B) * p.Hk * tn;
    size_t at = 0;
    const auto take = [&](float*& to, size_t n) {
        to = base + at;
        at += n;
    };
    take(f->nl2, qt * kTile);
    take(f->delta, qt * kTile);
    if (bf16) return at;
    take(f->gnorm, qt * kTile);
    take(f->gtail, qt * kTile);
    take(f->dtail, qt * kTile);
    take(f->gmax, qt);
    take(f->dmax, qt);
    take(f->vnorm, kt * kTile);
    take(f->vhead, kt * kTile);
    take(f->vmax, kt);
    return at;
}

template <bool BF16, int NT>
cudaError_t launch_vjp(const AttnParams& p, float* ws, cudaStream_t s) {
    using K = Cfg<NT>;
    VjpParams f{};
    f.a = p;
    CUtensorMap mq, mk, mv, mg;
    if (!attn_map(&mq, &f.cq, BF16, p.q, p.B, p.M, p.H, p.D, NT) ||
        !attn_map(&mk, &f.ck, BF16, p.k, p.B, p.N, p.Hk, p.D, NT) ||
        !attn_map(&mv, &f.cv, BF16, p.v, p.B, p.N, p.Hk, p.C, NT) ||
        !attn_map(&mg, &f.cg, BF16, p.g, p.B, p.M, p.H, p.C, NT))
        return cudaErrorInvalidValue;
    f.tiles_m = (static_cast<int64_t>(p.M) + kTile - 1) / kTile;
    f.tiles_n = (static_cast<int64_t>(p.N) + kTile - 1) / kTile;
    f.Mp = f.tiles_m * kTile;
    f.Np = f.tiles_n * kTile;
    vjp_floats(p, BF16, ws, &f);
    f.dblocks = (p.D + 63) / 64;
    f.cblocks = (p.C + 63) / 64;
    f.dsteps = (p.D + 15) / 16;
    f.csteps = (p.C + 15) / 16;
    const uint32_t bf = BF16 ? 1 : 0;
    f.idesc_s = idesc_f16(kTile, NT, bf, bf);
    f.idesc_d = idesc_f16(kTile, f.dsteps * 16, bf, bf) | kIdescTransposeB;
    f.idesc_c = idesc_f16(kTile, f.csteps * 16, bf, bf) | kIdescTransposeB;
    // Row terms and barriers after the rings; the shared window starts 1 KiB
    // aligned (checked in the kernel), so no room is kept for aligning it.
    constexpr size_t kSmem = K::kSmem, kTerms = NT * sizeof(float);
    const size_t own = static_cast<size_t>(f.dblocks + f.cblocks) * kBlock;
    const size_t room = kSmem - sizeof(VjpBarriers) - own;
    const size_t d_bytes = f.dblocks * NT * 128 + kTerms, c_bytes = f.cblocks * NT * 128 + kTerms;
    f.dstages = 3;
    f.cstages = 2;
    while (f.dstages < 8 && (f.dstages + 1) * d_bytes + (f.cstages + 1) * c_bytes <= room) {
        ++f.dstages;
        ++f.cstages;
    }
    const size_t used = own + f.dstages * d_bytes + f.cstages * c_bytes + sizeof(VjpBarriers);
    f.smem_bytes = static_cast<uint32_t>(std::min(kSmem, used + 1024));

    const int64_t row_blocks = static_cast<int64_t>(p.B) * p.H * f.tiles_m;
    const int64_t value_blocks = BF16 ? 0 : static_cast<int64_t>(p.B) * p.Hk * f.tiles_n;
    constexpr int kGroups = NT == 64 ? 2 : 4;   // of 32 channels
    auto rows = p.C % 8 == 0 && p.D % 8 == 0 ? attn_rows_kernel<BF16, kGroups, true>
                                             : attn_rows_kernel<BF16, kGroups, false>;
    note_launches(1);
    cudaError_t e = launch_kernel(rows, dim3(static_cast<unsigned>(row_blocks + value_blocks)), 256, 0, s, f);
    if (e != cudaSuccess) return e;
    f.key_blocks = p.dk.p || p.dv.p ? static_cast<int64_t>(p.B) * p.Hk * f.tiles_n : 0;
    const int64_t blocks = f.key_blocks + (p.dq.p ? row_blocks : 0);
    auto kern = attn_tc_vjp_kernel<BF16, NT>;
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmem));
    if (e != cudaSuccess) return e;
    note_launches(1);
    return launch_kernel(kern, dim3(static_cast<unsigned>(blocks)), K::kThreads, f.smem_bytes, s, mq, mk, mv,
                         mg, f);
}

}  // namespace

size_t attn_tc_vjp_workspace(const AttnParams& p, InType t) {
    VjpParams f{};
    return vjp_floats(p, t == InType::BF16, nullptr, &f) * sizeof(float);
}

cudaError_t launch_attn_tc_vjp(const AttnParams& p, InType t, void* ws, cudaStream_t s) {
    float* w = static_cast<float*>(ws);
    if (p.D > 64 || p.C > 64)
        return t == InType::BF16 ? launch_vjp<true, 128>(p, w, s) : launch_vjp<false, 128>(p, w, s);
    return t == InType::BF16 ? launch_vjp<true, 64>(p, w, s) : launch_vjp<false, 64>(p, w, s);
}

}  // namespace gs
