// Softmax attention on the tensor cores (tcgen05, TMA, TMEM), fp16 / bf16,
// D, C <= 128.
//
//   S  = q k^T          128 x 128 x D, A and B from shared memory, fp32 TMEM
//   P  = 2^(c S - m)    TMEM -> registers -> TMEM, rounded to 16 bits
//   O += P v            A = P from TMEM, B = the value tile as it lies in
//                       memory (rows along the summation index)
//
// A block keeps two streams of tiles going, each with its own softmax
// warpgroup, so that one stream's exponentials run under the other's
// products; both products of a stream are issued by one thread in the order
// P v (tile j), q k^T (tile j + 1), so a completed S tile also says that O is
// up to date and that P has been read (P lies in the first half of S).
//  - Long queries: the streams are two neighbouring tiles of 128 query rows
//    of one head over the same keys.
//  - Long queries with D, C <= 64, where the exponentials are the larger part:
//    two blocks of one stream each per SM (half of TMEM and shared memory),
//    key tiles of 64 and two S buffers, so that q k^T of tile j + 1 runs under
//    the softmax of tile j and the softmax warps never wait for a product.
//  - Few queries (packed): the rows are all heads that share a key head times
//    the tokens, and the streams take the even and the odd key tiles; the
//    second stream hands its rows to the first through shared memory.
//
// The running maximum m moves only when a tile's maximum exceeds it by more
// than 8 (a factor 256): P is then at most 2^8 and no accuracy is lost, since
// P and the fp32 row sum use the same m; the warp that needs it rescales its
// rows of O itself, which is safe between the last P v's completion and the
// hand-over of P.  fp16 P carries a factor 2^7 (P <= 2^15), so that
// probabilities down to 2^-21 of the row's largest stay normal numbers.
//
// What bounds it: the tensor pipe and its shared-memory reads for long queries
// of 128 channels (2 x 8192 tokens, 16 heads, causal: 355 us, 1.55 PFLOP/s of
// the 1.91 measured for a plain product; 1.44 back to back at the power
// limit); for 64 channels the chain of a tile in each softmax thread, TMEM
// load - mask - maximum - exponentials - TMEM store, of which two warps a
// scheduler hide too little (the same tokens: 296 us, tensor pipe 39 %, MUFU
// 40 %, issue slots 55 %; the exponentials alone would take 108 us); HBM for few
// tokens (16 tokens against caches of 8191 .. 4352 keys, 32 / 8 heads x 128:
// 72 us, 5.7 TB/s).
//
// A warpgroup of softmax warps per stream, one thread per row; then one warp
// for the TMA copies, one for TMEM and the products, and two idle ones (they
// make up the warpgroup that hands registers to the softmax warps).
#include <algorithm>

#include "attention_tc.cuh"

namespace gs {
namespace {

using namespace tc;

template <int STREAMS>
struct Cfg {
    static constexpr int kSoftmaxWarps = 4 * STREAMS;
    static constexpr int kLoadWarp = kSoftmaxWarps, kMmaWarp = kSoftmaxWarps + 1;
    static constexpr int kThreads = (kSoftmaxWarps + 4) * 32;
    static constexpr int kBlocksPerSm = STREAMS == 2 ? 1 : 2;
    static constexpr uint32_t kRegsLaunch = STREAMS == 2 ? 168 : 128, kRegsSoftmax = STREAMS == 2 ? 224 : 200,
                              kRegsCtrl = 56;
    static_assert(kSoftmaxWarps * kRegsSoftmax + 4 * kRegsCtrl <= (kSoftmaxWarps + 4) * kRegsLaunch,
                  "register split");
    static constexpr uint32_t kTmem = 512 / kBlocksPerSm;
    static constexpr int NT = STREAMS == 2 ? 128 : 64;      // keys of a tile
    // TMEM: S of stream i at 128 i (of buffer i at 64 i), O at kO + 128 i.
    static constexpr uint32_t kO = 128 * STREAMS;
    static constexpr size_t kSmem = (STREAMS == 2 ? 227 : 113) * 1024;
};
constexpr float kMaxSlack = 8.f;      // log2 units the maximum may lag behind
constexpr float kShiftF16 = 7.f;

struct FwdParams {
    AttnParams a;
    Coords cq, ck, cv;
    int64_t group;        // heads that run together
    int64_t tiles_r;      // row tiles of a block per (problem, head; packed: key head)
    int dblocks, cblocks; // 64-channel blocks of D and C
    int ksteps;           // 16-channel steps of D
    int stages;
    uint32_t stage_bytes;
    uint32_t idesc_s, idesc_o;
};

struct __align__(8) FwdBarriers {
    uint64_t q_full, drain;
    uint64_t s_full[2], p_full[2];   // per stream, or per S buffer of one stream
    uint64_t o_full[2];              // per stream: O complete
    uint64_t pv_done;                // one stream: O up to date with a tile
    uint64_t kv_full[8], kv_empty[8];
    uint32_t tmem_base;
    int abort_flag;
};

template <bool BF16, bool PACKED, int STREAMS, bool SCALED>
__global__ void __launch_bounds__(Cfg<STREAMS>::kThreads, Cfg<STREAMS>::kBlocksPerSm)
attn_tc_fwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                   const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ FwdParams fp) {
    using K = Cfg<STREAMS>;
    constexpr int NT = K::NT;
    static_assert(!PACKED || STREAMS == 2, "packed rows: the streams share the keys out");
    const AttnParams& p = fp.a;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t q_tile_bytes = fp.dblocks * kBlock;
    uint8_t* q_smem = smem;
    uint8_t* ring = smem + (PACKED ? 1 : STREAMS) * q_tile_bytes;
    FwdBarriers* bars = reinterpret_cast<FwdBarriers*>(ring + fp.stages * fp.stage_bytes);
    volatile int* abort_flag = &bars->abort_flag;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // Block -> (split, row tile, problem and head).  Heads go in groups whose
    // keys and values fit in L2 together; within a group the later row tiles,
    // which see more keys under a causal mask, go first.
    const int heads = PACKED ? p.Hk : p.H;
    int64_t blk = blockIdx.x;
    const int split = static_cast<int>(blk % p.splits);
    blk /= p.splits;
    const int64_t all_heads = static_cast<int64_t>(p.B) * heads;
    const int64_t group0 = blk / (fp.group * fp.tiles_r) * fp.group;
    const int64_t in_group = blk - group0 * fp.tiles_r, group = min(fp.group, all_heads - group0);
    const int64_t tile = fp.tiles_r - 1 - in_group / group;
    const int64_t bh = group0 + in_group % group;
    const int b = static_cast<int>(bh / heads), h = static_cast<int>(bh % heads);
    const int kvh = PACKED ? h : h / p.G;
    const int ql = attn_q_len(p, b), kl = attn_k_len(p, b);
    const int64_t rows_all = PACKED ? p.R : p.M;                       // rows with outputs
    const int64_t rows_in = PACKED ? static_cast<int64_t>(ql) * p.G : ql;
    const int64_t r0 = tile * (PACKED ? kTile : STREAMS * kTile);

    // Keys that some row of row tile i sees, and the key tiles of this split.
    // Packed: both streams share the row tile and take alternate key tiles.
    int nt[2];
    int64_t tiles[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t first = r0 + (PACKED ? 0 : i * kTile);
        const int64_t last = i < STREAMS ? min(first + kTile, rows_in) - 1 : -1;
        const int kend =
            last >= first
                ? attn_limit(static_cast<int>(PACKED ? last / p.G : last), ql, kl, p.causal) : 0;
        tiles[i] = (static_cast<int64_t>(kend) + NT - 1) / NT;
    }
    const int64_t all = max(tiles[0], tiles[1]);
    const int key_tile0 = static_cast<int>(all * split / p.splits);
    const int key_tile1 = static_cast<int>(all * (split + 1) / p.splits);
#pragma unroll
    for (int i = 0; i < 2; ++i)
        nt[i] = PACKED ? (key_tile1 - key_tile0 + 1 - i) / 2
                       : max(0, static_cast<int>(min(static_cast<int64_t>(key_tile1), tiles[i])) - key_tile0);
    const int steps = max(nt[0], nt[1]);
    const int tile_step = PACKED ? 2 : 1;

    if (tid == 0) {
        mbar_init(&bars->q_full, PACKED ? K::kSoftmaxWarps : 1);
        mbar_init(&bars->drain, 1);
        mbar_init(&bars->pv_done, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars->s_full[i], 1);
            mbar_init(&bars->p_full[i], 4);
            mbar_init(&bars->o_full[i], 1);
        }
        for (int s = 0; s < fp.stages; ++s) {
            mbar_init(&bars->kv_full[s], 1);
            mbar_init(&bars->kv_empty[s], 1);
        }
        bars->abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == K::kMmaWarp) {
        tmem_alloc(&bars->tmem_base, K::kTmem);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();
    pdl_trigger();
    const uint32_t tmem = bars->tmem_base;
    auto slot = [&](int i) { return ring + i * fp.stage_bytes; };

    if (warp == K::kLoadWarp) {
        reg_dealloc<K::kRegsCtrl>();
        const bool leader = elect_one();
        int issued = 0;
        bool ok = true;
        RingPos at;
        const auto load = [&](bool value, int key_tile) {
            if (!ok) return;
            ok = wait_all(&bars->kv_empty[at.idx], at.phase ^ 1u, abort_flag, p.status);
            if (!ok) return;
            if (leader) {
                const int blocks = value ? fp.cblocks : fp.dblocks;
                const Coords& c = value ? fp.cv : fp.ck;
                mbar_arrive_expect_tx(&bars->kv_full[at.idx], blocks * NT * 128);
                load_tile<NT>(slot(at.idx), value ? &tm_v : &tm_k, &bars->kv_full[at.idx], blocks,
                          key_tile * NT, kvh * c.h, b * c.b);
            }
            __syncwarp();
            at.advance(fp.stages);
            ++issued;
        };
        if (steps > 0) {
            if (leader && !PACKED) {
                const int n = (nt[0] > 0) + (nt[1] > 0);
                mbar_arrive_expect_tx(&bars->q_full, n * q_tile_bytes);
                for (int i = 0; i < 2; ++i)
                    if (nt[i] > 0)
                        load_tile<kTile, NT>(q_smem + i * q_tile_bytes, &tm_q, &bars->q_full, fp.dblocks,
                                  static_cast<int>(r0) + i * kTile, h * fp.cq.h, b * fp.cq.b);
            }
            __syncwarp();
            if (PACKED) {
                for (int i = 0; i < 2; ++i)
                    if (nt[i] > 0) load(false, key_tile0 + i);
                for (int j = 0; j < nt[0]; ++j)
                    for (int i = 0; i < 2; ++i) {
                        if (j < nt[i]) load(true, key_tile0 + 2 * j + i);
                        if (j + 1 < nt[i]) load(false, key_tile0 + 2 * j + 2 + i);
                    }
            } else if (STREAMS == 1) {
                load(false, key_tile0);
                for (int j = 0; j < steps; ++j) {
                    if (j + 1 < steps) load(false, key_tile0 + j + 1);
                    load(true, key_tile0 + j);
                }
            } else {
                for (int j = 0; j < steps; ++j) {
                    load(false, key_tile0 + j);
                    load(true, key_tile0 + j);
                }
            }
            // Every copy started here lands before the block can end.
            if (!PACKED) mbar_wait_bounded(&bars->q_full, 0, nullptr, p.status);
            for (int j = max(0, issued - fp.stages); j < issued; ++j)
                mbar_wait_bounded(&bars->kv_full[j % fp.stages],
                                  static_cast<uint32_t>(j / fp.stages) & 1u, nullptr, p.status);
            __syncwarp();
        }
    } else if (warp == K::kMmaWarp) {
        reg_dealloc<K::kRegsCtrl>();
        if (steps > 0) {
            const uint32_t leader = elect_one() ? 1u : 0u;
            bool ok = wait_all(&bars->q_full, 0, abort_flag, p.status);
            RingPos at;
            const auto acquire = [&]() {   // the next loaded tile's slot
                const int s = at.idx;
                if (ok) ok = wait_all(&bars->kv_full[s], at.phase, abort_flag, p.status);
                at.advance(fp.stages);
                return s;
            };
            const uint32_t q_at = smem_u32(q_smem), ring_at = smem_u32(ring);
            const auto scores = [&](int i, int s) {
                if (!ok) return;
                tc_fence_after();
                mma_scores<NT>(leader, tmem + NT * i, q_at + (PACKED || STREAMS == 1 ? 0 : i * q_tile_bytes),
                           ring_at + s * fp.stage_bytes, fp.ksteps, fp.idesc_s);
                mma_commit_on(leader, &bars->s_full[i]);
            };
            // (i: the stream; the S buffer of one stream)
            const auto values = [&](int i, int s, int j) {
                const int phase = STREAMS == 1 ? j >> 1 : j;
                if (ok) ok = wait_all(&bars->p_full[i], phase & 1, abort_flag, p.status);
                if (!ok) return;
                tc_fence_after();
                if (STREAMS == 1) {
                    mma_rows<64, NT>(leader, tmem + K::kO, tmem + NT * i, ring_at + s * fp.stage_bytes,
                                     fp.idesc_o, j == 0);
                    mma_commit_on(leader, &bars->pv_done);
                    if (j + 1 == nt[0]) mma_commit_on(leader, &bars->o_full[0]);
                    return;
                }
                mma_rows<64>(leader, tmem + K::kO + 128 * i, tmem + 128 * i, ring_at + s * fp.stage_bytes,
                             fp.idesc_o, j == 0);
                if (j + 1 == nt[i]) mma_commit_on(leader, &bars->o_full[i]);
            };
            const auto release = [&](int s) {
                if (ok) mma_commit_on(leader, &bars->kv_empty[s]);
            };
            if (PACKED) {
                for (int i = 0; i < 2; ++i)
                    if (nt[i] > 0) {
                        const int s = acquire();
                        scores(i, s);
                        release(s);
                    }
                for (int j = 0; ok && j < nt[0]; ++j)
                    for (int i = 0; i < 2; ++i) {
                        if (j < nt[i]) {
                            const int s = acquire();
                            values(i, s, j);
                            release(s);
                        }
                        if (j + 1 < nt[i]) {
                            const int s = acquire();
                            scores(i, s);
                            release(s);
                        }
                    }
            } else if (STREAMS == 1) {
                // p_full alternates between the buffers: the softmax warps can
                // be done with tile j + 1 before this warp has seen P of tile j.
                int s = acquire();
                scores(0, s);
                release(s);
                for (int j = 0; ok && j < steps; ++j) {
                    if (j + 1 < steps) {
                        s = acquire();
                        scores((j + 1) & 1, s);      // (P v of tile j - 1 has read this buffer)
                        release(s);
                    }
                    s = acquire();
                    values(j & 1, s, j);
                    release(s);
                }
            } else {
                int ks = acquire();
                if (nt[0] > 0) scores(0, ks);
                if (nt[1] > 0) scores(1, ks);
                release(ks);
                for (int j = 0; ok && j < steps; ++j) {
                    const int vs = acquire();
                    if (j < nt[0]) values(0, vs, j);
                    const bool more = j + 1 < steps;
                    if (more) ks = acquire();
                    if (j + 1 < nt[0]) scores(0, ks);
                    if (j < nt[1]) values(1, vs, j);
                    release(vs);
                    if (j + 1 < nt[1]) scores(1, ks);
                    if (more) release(ks);
                }
            }
            // No MMA may still be running when TMEM is released.
            if (leader) mma_commit(&bars->drain);
            __syncwarp();
            mbar_wait_bounded(&bars->drain, 0, nullptr, p.status);
            __syncwarp();
        }
    } else if (warp > K::kMmaWarp) {
        reg_dealloc<K::kRegsCtrl>();
    } else {
        reg_alloc<K::kRegsSoftmax>();
        const int i = warp >> 2;                        // stream
        const int row = tid & (kTile - 1);
        const int64_t r = r0 + (PACKED ? 0 : i * kTile) + row;
        const int64_t m = PACKED ? r / p.G : r;
        const int hq = PACKED ? h * p.G + static_cast<int>(r - m * p.G) : h;
        const int lim = r < rows_in ? attn_limit(static_cast<int>(m), ql, kl, p.causal) : 0;
        const int64_t first = r0 + (PACKED ? 0 : i * kTile);
        const int lim_first =
            attn_limit(static_cast<int>(PACKED ? first / p.G : first), ql, kl, p.causal);
        const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;   // (32 x quarter) << 16
        const uint32_t t_o = tmem + lanes + K::kO + 128 * i;

        if (PACKED && steps > 0) {
            // Query rows into the swizzled layout TMA would have written.
            const uint16_t* src = reinterpret_cast<const uint16_t*>(p.q.p) + b * p.q.sb + hq * p.q.sh +
                                  m * p.q.sr;
            uint4 x[8];              // all reads before the first write
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int c = 2 * u + i;
                x[u] = make_uint4(0, 0, 0, 0);
                if (r < rows_in && c * 8 + 8 <= p.D) x[u] = *reinterpret_cast<const uint4*>(src + c * 8);
            }
            if (r < rows_in && p.D % 8 && ((p.D / 8) & 1) == i) {      // the last, ragged 16 bytes
                uint4 y = make_uint4(0, 0, 0, 0);
                uint16_t* e = reinterpret_cast<uint16_t*>(&y);
                for (int d = p.D / 8 * 8; d < p.D; ++d) e[d & 7] = src[d];
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (2 * u + i == p.D / 8) x[u] = y;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int c = 2 * u + i;
                if (c < fp.dblocks * 8)
                    *reinterpret_cast<uint4*>(q_smem + (c >> 3) * kBlock + row * 128 +
                                              (((c & 7) ^ (row & 7)) << 4)) = x[u];
            }
            fence_proxy_async_smem();
            __syncwarp();
            mbar_arrive_if_zero(&bars->q_full, lane);
        }

        const float shift = BF16 ? 0.f : kShiftF16;
        float c_row = p.c, v_up = 1.f;                  // SCALED: of this row's scores, and of O
        if constexpr (SCALED) {
            const uint2 size = p.head_sizes[static_cast<int64_t>(b) * p.Hk + kvh];
            if (r < rows_in)
                // (Never 0, which makes NaN of a masked score: where the product is below 2^-126, the scores,
                // below 2^40, are nothing either way.)
                c_row = fmaxf(c_row * p.row_scale[(static_cast<int64_t>(b) * p.H + hq) * p.M + m] *
                                  exp2f(static_cast<float>(scaled_exponent(size.x))), 0x1p-126f);
            v_up = exp2f(static_cast<float>(scaled_exponent(size.y)));
        }
        const float c_log = SCALED ? c_row : p.c;
        // Packed tiles may leave whole warps without rows: they only keep the
        // barriers going.
        const bool active = !PACKED || first + (warp & 3) * 32 < rows_in;
        float top = -INFINITY, sum = 0.f;    // m in log2 units, row sum of 2^(c s - m + shift)
        bool ok = true;
        for (int j = 0; ok && j < nt[i]; ++j) {
            const int buf = STREAMS == 1 ? j & 1 : i;
            const uint32_t t_s = tmem + lanes + NT * buf;
            ok = wait_all(&bars->s_full[buf], (STREAMS == 1 ? j >> 1 : j) & 1, abort_flag, p.status);
            if (!ok) break;
            tc_fence_after();
            const int n0 = (key_tile0 + tile_step * j + (PACKED ? i : 0)) * NT;
            if (active) {
                constexpr int kQ = NT / 32;
                uint32_t s[kQ][32];
#pragma unroll
                for (int q = 0; q < kQ; ++q) tmem_ld_32x32b_x32(t_s + 32 * q, s[q]);
#pragma unroll
                for (int q = 0; q < kQ; q += 2) tmem_wait_ld_regs(s[q], s[q + 1]);
                if (n0 + NT > lim_first) {
                    const int seen = lim - n0;
#pragma unroll
                    for (int q = 0; q < kQ; ++q)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (q * 32 + e >= seen) s[q][e] = 0xff800000u;   // -inf
                }
                float mx[kQ];
#pragma unroll
                for (int q = 0; q < kQ; ++q) {
                    mx[q] = __uint_as_float(s[q][0]);
#pragma unroll
                    for (int e = 1; e < 32; ++e) mx[q] = fmaxf(mx[q], __uint_as_float(s[q][e]));
                }
                float mt = fmaxf(mx[0], mx[1]);
                if (kQ == 4) mt = fmaxf(mt, fmaxf(mx[kQ - 2], mx[kQ - 1]));
                mt *= c_log;
                const bool move = mt - top > kMaxSlack;   // (also from -inf)
                if (__any_sync(~0u, move)) {
                    const float to = move ? mt : top;
                    const float f = move ? ex2_approx(top - to) : 1.f;   // 0 from -inf
                    top = to;
                    sum *= f;
                    // The phase is j - 1's: the scores of tile j completed after P v
                    // of tile j - 2, and P v of tile j waits for this warp.
                    if (STREAMS == 1 && j > 0) {
                        ok = wait_all(&bars->pv_done, (j - 1) & 1, abort_flag, p.status);
                        tc_fence_after();
                    }
                    if (j > 0) {
                        for (int c = 0; c < fp.cblocks * 64; c += 32) {
                            uint32_t o[32];
                            tmem_ld_32x32b_x32(t_o + c, o);
                            tmem_wait_ld_regs(o);
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                            tmem_st_32x32b_x32(t_o + c, o);
                        }
                    }
                }
                const float ref = (top == -INFINITY ? 0.f : -top) + shift;
                const uint64_t c2 = f32x2_pack(c_log, c_log), r2 = f32x2_pack(ref, ref);
                uint64_t acc[2] = {0, 0};
#pragma unroll
                for (int q = 0; q < kQ; ++q) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        const uint64_t x = f32x2_fma(
                            f32x2_pack(__uint_as_float(s[q][e]), __uint_as_float(s[q][e + 1])), c2, r2);
                        float x0, x1;
                        f32x2_unpack(x, x0, x1);
                        x0 = ex2_approx(x0);
                        x1 = ex2_approx(x1);
                        acc[(e >> 1) & 1] = f32x2_add(acc[(e >> 1) & 1], f32x2_pack(x0, x1));
                        w[e >> 1] = pack2<BF16>(x0, x1);
                    }
                    tmem_st_32x32b_x16(t_s + 16 * q, w);
                }
                float a0, a1;
                f32x2_unpack(f32x2_add(acc[0], acc[1]), a0, a1);
                sum += a0 + a1;
            }
            if (n0 + NT > kl) {
                // The value tile runs past the keys: its other rows become 0.
                int idx = STREAMS == 1 && j + 1 < nt[i] ? 2 * j + 2 : 2 * j + 1;   // in the load order
                if (PACKED)
                    idx = i == 0 ? 1 + (nt[1] > 0) + 4 * j - (j > 0 && j >= nt[1] ? 1 : 0)
                                 : 3 + 4 * j + (j + 1 < nt[0] ? 1 : 0);
                ok = wait_all(&bars->kv_full[idx % fp.stages],
                              static_cast<uint32_t>(idx / fp.stages) & 1u, abort_flag, p.status);
                if (!ok) break;
                zero_rows<NT>(slot(idx % fp.stages), fp.cblocks, kl - n0, row, kTile);
                fence_proxy_async_smem();
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            mbar_arrive_if_zero(&bars->p_full[buf], lane);
        }

        // Epilogue: out = O / sum, lse = m + log2 sum.
        if (ok && nt[i] > 0) ok = wait_all(&bars->o_full[i], 0, abort_flag, p.status);
        tc_fence_after();
        // (A row of NaN scores has no maximum, but its sum is NaN.)
        const bool has = ok && nt[i] > 0 && lim > 0 && (top != -INFINITY || sum != sum);
        const float inv = has ? (SCALED ? v_up / sum : 1.f / sum) : 0.f;
        float l2 = has ? top - shift + log2f(sum) : -INFINITY;
        const bool split_out = p.splits > 1;
        const int64_t rr = PACKED ? r : m * p.G + (h - kvh * p.G);
        const int64_t at = (static_cast<int64_t>(split) * p.B * p.Hk + static_cast<int64_t>(b) * p.Hk + kvh) *
                               p.R + rr;
        const bool mine = r < rows_all && (!PACKED || i == 0);
        // Packed: the second stream's lse and rows (channel by channel) go
        // through the ring, once both streams have read all their tiles, and
        // the first adds them: out = sum_i 2^(l_i - l) out_i, as for splits.
        float* other_l = reinterpret_cast<float*>(ring);
        float* other_o = other_l + kTile;
        float w_own = inv, w_other = 0.f;
        bool any = has;
        if constexpr (PACKED) {
            barrier_sync<1, K::kSoftmaxWarps * 32>();
            if (i == 1) {
                other_l[row] = l2;
                for (int c = 0; active && nt[1] > 0 && c < p.C; c += 32) {
                    uint32_t o[32];
                    tmem_ld_32x32b_x32(t_o + c, o);
                    tmem_wait_ld_regs(o);
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (has && c + e < p.C) other_o[(c + e) * kTile + row] = __uint_as_float(o[e]) * inv;
                    __syncwarp();
                }
            }
            barrier_sync<1, K::kSoftmaxWarps * 32>();
            if (i == 0) {
                const float l1 = other_l[row], ref0 = fmaxf(l2, l1), ref = ref0 == -INFINITY ? 0.f : ref0;
                const float f0 = exp2f(l2 - ref), f1 = exp2f(l1 - ref);
                any = f0 + f1 != 0.f;           // (NaN: a row of NaN scores)
                const float norm = any ? 1.f / (f0 + f1) : 0.f;
                w_own = inv * f0 * norm;
                w_other = f1 * norm;
                l2 = any ? ref + log2f(f0 + f1) : -INFINITY;
            }
        }
        if (mine) {
            if (split_out) {
                p.part_l[at] = l2;
            } else if (p.lse) {
                p.lse[(static_cast<int64_t>(b) * p.H + hq) * p.M + m] = l2 * kLn2;
            }
        }
        uint16_t* dst = reinterpret_cast<uint16_t*>(p.out.p) + b * p.out.sb + hq * p.out.sh + m * p.out.sr;
        if ((active || !split_out) && (!PACKED || i == 0)) {
            for (int c = 0; c < p.C; c += 32) {
                uint32_t o[32];
                float x[32];
                if (nt[i] > 0) {
                    tmem_ld_32x32b_x32(t_o + c, o);
                    tmem_wait_ld_regs(o);
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = has ? __uint_as_float(o[e]) * w_own : 0.f;
                if (PACKED && w_other != 0.f) {
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (c + e < p.C) x[e] = fmaf(other_o[(c + e) * kTile + row], w_other, x[e]);
                }
                if (mine && !split_out) {
                    if (SCALED && p.out_bf16)
                        put_row<true>(dst, x, c, p.C);
                    else
                        put_row<BF16>(dst, x, c, p.C);
                }
                if (mine && split_out && any) {
                    float* to = p.part_o + at * p.C + c;
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        if (p.C % 4 == 0) {
                            if (c + e < p.C)
                                *reinterpret_cast<float4*>(to + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                        } else {
#pragma unroll
                            for (int d = 0; d < 4; ++d)
                                if (c + e + d < p.C) to[e + d] = x[e + d];
                        }
                    }
                }
                __syncwarp();
            }
        }
        tc_fence_before();
    }
    __syncthreads();
    if (warp == K::kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, K::kTmem);
    }
}

template <bool BF16, bool PACKED, int STREAMS, bool SCALED = false>
cudaError_t launch_fwd(FwdParams& f, cudaStream_t s) {
    using K = Cfg<STREAMS>;
    const AttnParams& p = f.a;
    CUtensorMap mq, mk, mv;
    if (!attn_map(&mq, &f.cq, BF16, p.q, p.B, p.M, p.H, p.D, K::NT) ||
        !attn_map(&mk, &f.ck, BF16, p.k, p.B, p.N, p.Hk, p.D, K::NT) ||
        !attn_map(&mv, &f.cv, BF16, p.v, p.B, p.N, p.Hk, p.C, K::NT))
        return cudaErrorInvalidValue;
    f.dblocks = (p.D + 63) / 64;
    f.cblocks = (p.C + 63) / 64;
    f.ksteps = (p.D + 15) / 16;
    constexpr int NT = K::NT;
    f.stage_bytes = std::max(f.dblocks, f.cblocks) * NT * 128;
    const size_t q_bytes = (PACKED ? 1 : STREAMS) * f.dblocks * kBlock;
    constexpr size_t kSmem = K::kSmem, kExtra = 1024 + sizeof(FwdBarriers);
    f.stages = static_cast<int>(std::min<size_t>(8, (kSmem - kExtra - q_bytes) / f.stage_bytes));
    const uint32_t bf = BF16 ? 1 : 0;
    f.idesc_s = idesc_f16(kTile, NT, bf, bf);
    f.idesc_o = idesc_f16(kTile, (p.C + 15) / 16 * 16, bf, bf) | kIdescTransposeB;
    const int64_t rows = PACKED ? p.R : p.M, heads = PACKED ? p.Hk : p.H;
    constexpr int64_t kRows = PACKED ? kTile : STREAMS * kTile;
    f.tiles_r = (rows + kRows - 1) / kRows;
    const int64_t blocks = f.tiles_r * p.B * heads * p.splits;
    constexpr int64_t kKeysInL2 = int64_t(48) << 20;
    const int64_t head_bytes = 2 * static_cast<int64_t>(p.N) * (p.D + p.C) / (PACKED ? 1 : p.G) + 1;
    f.group = std::max<int64_t>(1, std::min<int64_t>(static_cast<int64_t>(p.B) * heads, kKeysInL2 / head_bytes));
    const size_t smem = kExtra + q_bytes + static_cast<size_t>(f.stages) * f.stage_bytes;
    auto kern = attn_tc_fwd_kernel<BF16, PACKED, STREAMS, SCALED>;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         static_cast<int>(kSmem));
    if (e != cudaSuccess) return e;
    note_launches(1);
    return launch_kernel(kern, dim3(static_cast<unsigned>(blocks)), K::kThreads, smem, s, mq, mk, mv, f);
}

}  // namespace

bool attn_tc_takes(const Arr& a, int64_t B, int64_t rows, int64_t heads, int width) {
    if (width > 128 || reinterpret_cast<uintptr_t>(a.p) % 16) return false;
    constexpr int64_t kMaxStride = int64_t(1) << 39;    // elements; maps take < 2^40 bytes
    const int64_t n[3] = {B, rows, heads}, st[3] = {a.sb, a.sr, a.sh};
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && (st[i] % 8 || st[i] >= kMaxStride || (i == 1 && st[i] == 0))) return false;
    return true;
}

bool attn_tc_narrow(const AttnParams& p) { return p.D <= 64 && p.C <= 64; }

cudaError_t launch_attn_tc_fwd(const AttnParams& p, InType t, bool packed, bool scaled, cudaStream_t s) {
    FwdParams f{};
    f.a = p;
    if (scaled)
        return packed ? launch_fwd<false, true, 2, true>(f, s)
               : attn_tc_narrow(p) ? launch_fwd<false, false, 1, true>(f, s)
                                   : launch_fwd<false, false, 2, true>(f, s);
    const bool bf16 = t == InType::BF16;
    if (packed) return bf16 ? launch_fwd<true, true, 2>(f, s) : launch_fwd<false, true, 2>(f, s);
    if (attn_tc_narrow(p))
        return bf16 ? launch_fwd<true, false, 1>(f, s) : launch_fwd<false, false, 1>(f, s);
    return bf16 ? launch_fwd<true, false, 2>(f, s) : launch_fwd<false, false, 2>(f, s);
}

}  // namespace gs
