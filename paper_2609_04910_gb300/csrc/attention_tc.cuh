// Shared parts of the tensor-core attention kernels.
#pragma once

#include <cuda.h>

#include "attention.h"
#include "ptx.cuh"
#include "tensor_map.h"

namespace gs {
namespace tc {

constexpr int kTile = 128;               // rows of a tile: queries or keys
constexpr uint32_t kBlock = kTile * 128; // bytes of 128 rows x 64 16-bit channels

// Factors that turn (problem, head) into the coordinates of a TMA map: 1, or 0
// where the dimension has one element or a stride of zero (broadcast).
struct Coords {
    int b, h;
};

__device__ __forceinline__ bool wait_all(uint64_t* bar, uint32_t parity, volatile int* abort_flag,
                                         unsigned* status) {
    const bool ok = mbar_wait_bounded(bar, parity, abort_flag, status);
    return __all_sync(0xffffffffu, ok);
}

// Barrier ID (1 .. 15) of the THREADS threads that call it.
template <int ID, int THREADS>
__device__ __forceinline__ void barrier_sync() {
    asm volatile("barrier.cta.sync %0, %1;" ::"n"(ID), "n"(THREADS) : "memory");
}

// ROWS rows x `blocks` 64-channel blocks of one (problem, head), block after
// block, from row `row` on, in boxes of BOX rows (the map's).
template <int ROWS = kTile, int BOX = ROWS>
__device__ __forceinline__ void load_tile(uint8_t* dst, const CUtensorMap* map, uint64_t* bar,
                                          int blocks, int row, int h, int b) {
    for (int i = 0; i < blocks; ++i)
#pragma unroll
        for (int r = 0; r < ROWS; r += BOX)
            tma_load_4d(dst + (i * ROWS + r) * 128, map, bar, i * 64, row + r, h, b);
}

// Zeroes rows r0 .. ROWS - 1 of a tile in shared memory (`threads` threads,
// thread t of them): padding may hold NaN, which 0 x NaN would spread.
template <int ROWS = kTile>
__device__ __forceinline__ void zero_rows(uint8_t* tile, int blocks, int r0, int t, int threads) {
    const int chunks = (ROWS - r0) * 8;
    for (int i = 0; i < blocks; ++i)
        for (int c = t; c < chunks; c += threads)
            *reinterpret_cast<uint4*>(tile + (i * ROWS + r0) * 128 + c * 16) = make_uint4(0, 0, 0, 0);
}

// Matrix products are issued by the whole warp with warp-uniform operands,
// each instruction predicated on `on` (1 in the elected lane, else 0): the
// operands then stay in uniform registers.  (A loop in a branch that only the
// elected lane takes, building both descriptors for every instruction, took
// 130 clocks an instruction, twice the 64 of the product itself.)
__device__ __forceinline__ void mma_ss_on(uint32_t on, uint32_t d, uint64_t a, uint64_t b,
                                          uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(on)
        : "memory");
}
__device__ __forceinline__ void mma_ts_on(uint32_t on, uint32_t d, uint32_t a, uint64_t b,
                                          uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(on)
        : "memory");
}
__device__ __forceinline__ void mma_commit_on(uint32_t on, uint64_t* bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(
            smem_u32(bar)),
        "r"(on)
        : "memory");
}

// Scores of 128 x NT pairs: D[tmem] = rows(a) . rows(b) over `steps` (at
// most 8) x 16 channels of two tiles at shared addresses a and b.
template <int NT = kTile>
__device__ __forceinline__ void mma_scores(uint32_t on, uint32_t d, uint32_t a, uint32_t b, int steps,
                                           uint32_t idesc) {
    const uint64_t ad = smem_desc_kmajor_sw128(a), bd = smem_desc_kmajor_sw128(b);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
        if (kk < steps) {
            // (addresses in descriptor units of 16 bytes)
            const uint32_t a_off = ((kk >> 2) * kBlock + (kk & 3) * 32) >> 4;
            const uint32_t b_off = ((kk >> 2) * NT * 128 + (kk & 3) * 32) >> 4;
            mma_ss_on(on, d, ad + a_off, bd + b_off, idesc, kk > 0 ? 1u : 0u);
        }
}

// D[tmem] (+)= (16-bit tile in TMEM) x (NT rows at shared address b); the
// NT columns of the tile lie in runs of RUN 32-bit columns, 32 apart.
template <int RUN, int NT = kTile>
__device__ __forceinline__ void mma_rows(uint32_t on, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                         bool first) {
    const uint64_t bd = smem_desc_mnmajor_sw128(b, NT * 128);
#pragma unroll
    for (int kk = 0; kk < NT / 16; ++kk)
        mma_ts_on(on, d, a + (kk * 8 % RUN) + kk * 8 / RUN * 32, bd + ((kk * 2048) >> 4), idesc,
                  (!first || kk > 0) ? 1u : 0u);
}

template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    return BF16 ? pack_bf162(lo, hi) : pack_half2_satfinite(lo, hi);
}

// Two outputs (which may overflow to infinity), against operands of a product,
// which pack2 keeps finite.
template <bool BF16>
__device__ __forceinline__ uint32_t round2(float lo, float hi) {
    return BF16 ? pack_bf162(lo, hi) : pack_half2(lo, hi);
}

// Writes channels c0 .. c0 + 31 of one row of 16-bit outputs, those below
// `width`; dst 16-byte aligned at channel 0.
template <bool BF16>
__device__ __forceinline__ void put_row(uint16_t* dst, const float (&x)[32], int c0, int width) {
#pragma unroll
    for (int c = 0; c < 32; c += 8) {
        if (c0 + c >= width) break;
        uint4 w;
        w.x = round2<BF16>(x[c], x[c + 1]);
        w.y = round2<BF16>(x[c + 2], x[c + 3]);
        w.z = round2<BF16>(x[c + 4], x[c + 5]);
        w.w = round2<BF16>(x[c + 6], x[c + 7]);
        if (c0 + c + 8 <= width) {
            *reinterpret_cast<uint4*>(dst + c0 + c) = w;
        } else {
            const uint16_t* e = reinterpret_cast<const uint16_t*>(&w);
            for (int i = 0; c0 + c + i < width; ++i) dst[c0 + c + i] = e[i];
        }
    }
}

}  // namespace tc

// Map of a (B, rows, heads, width) array of 16-bit elements, in boxes of
// box_rows rows x 64 channels.
inline bool attn_map(CUtensorMap* map, tc::Coords* at, bool bf16, const Arr& a, int64_t B,
                     int64_t rows, int64_t heads, int width, int box_rows) {
    at->b = B > 1 && a.sb > 0 ? 1 : 0;
    at->h = heads > 1 && a.sh > 0 ? 1 : 0;
    const uint64_t dim[4] = {static_cast<uint64_t>(width), static_cast<uint64_t>(rows > 0 ? rows : 1),
                             at->h ? static_cast<uint64_t>(heads) : 1u,
                             at->b ? static_cast<uint64_t>(B) : 1u};
    // Strides of dimensions of one element are not used.
    const uint64_t stride[3] = {rows > 1 ? 2u * static_cast<uint64_t>(a.sr) : 16u,
                                at->h ? 2u * static_cast<uint64_t>(a.sh) : 16u,
                                at->b ? 2u * static_cast<uint64_t>(a.sb) : 16u};
    return encode_tile_map_4d(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                              a.p, dim, stride, static_cast<uint32_t>(box_rows));
}

}  // namespace gs
