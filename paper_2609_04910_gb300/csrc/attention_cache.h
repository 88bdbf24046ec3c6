// Internal interface of the 4-bit cache: its entry points
// (attention_cache_api.cu) and kernels.
#pragma once

#include "attention.h"
#include "gauss_sum/attention_cache.h"

namespace gs {

// A cache as the kernels see it (stored form: gauss_sum/attention_cache.h).
struct CacheParams {
    char* data;
    int64_t sp, sh;             // bytes from page to page and from head to head
    int pages, tokens;          // of the pool; of a page
    int shift;                  // log2 of tokens, or -1
    int heads, D, C;
    int kw, vw;                 // 32-channel words of a key row, of a value row
    int kg, vg;                 // groups of a key row, of a value row
    int block_bytes;
    const int* table;           // or null
    int64_t stride_table;
    int64_t N;                  // tokens of a problem
};

constexpr int kNoPage = -1;
constexpr uint32_t kNanGroup = 0x7fc07fc0u;

// a / b of numbers >= 0 that mostly fit 32 bits.
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}

// Page of token n of problem b, or kNoPage.
__device__ __forceinline__ int cache_page(const CacheParams& c, int b, int n) {
    if (!c.table) return b < c.pages ? b : kNoPage;
    const int at = c.shift >= 0 ? n >> c.shift : n / c.tokens;
    const int page = c.table[b * c.stride_table + at];
    return static_cast<unsigned>(page) < static_cast<unsigned>(c.pages) ? page : kNoPage;
}

// Rows of tokens to write from or read to.
struct CacheRows {
    CacheParams c;
    int B, M;
    const int* q_len;
    const int* k_len;
    Arr k, v;
    int vec_k, vec_v;           // rows in 16-byte vectors
    const uint2* sizes;         // read: rows times 2^-scaled_exponent of their problem's and head's; or null
    int all;                    // read: row m is token m, those past k_length are left as they are
    int head0, heads;           // heads of the rows
    int tiles, head_blocks;     // blocks of a problem: runs of tokens x parts of the heads
    int turns;                  // runs of tokens of a block, r.tiles apart
    unsigned grid_b;            // their number
    int part_heads;             // heads of a part
};

// attention_cache_rows.cu
cudaError_t launch_cache_write(CacheRows r, InType t, int sms, cudaStream_t s);
cudaError_t launch_cache_read(CacheRows r, InType t, int sms, cudaStream_t s);

// What scaled fp16 operands need: the sizes of every problem's and head's keys and values (bits of the
// largest |m| and 16 s; zero before the launch), and (M > 0, D <= 128) the queries as fp16 rows of `width`
// elements (B, M, heads x G, width), each times a power of two whose inverse is row_scale (B, heads x G, M).
struct CacheScale {
    CacheParams c;
    int B, M, G, head0, heads;
    const int* q_len;
    const int* k_len;
    Arr q;                      // of the first head's queries
    int vec;                    // its rows start on four-element boundaries
    uint16_t* q16;
    int width;
    float* row_scale;
    uint2* sizes;               // B x heads
    int chunks, token_chunks;   // blocks of a problem's head: two groups of a side of a run of tokens each
    unsigned scan_blocks;
};
cudaError_t launch_cache_scale(CacheScale r, InType t, cudaStream_t s);

// attention_cache_few.cu: attention of few rows (M x G) of a key head.
// Whether it takes the cache's widths; rows of a set, blocks, rows of partial results and bytes of
// workspace of a call (false: too many sets); and its launches.
struct FewPlan {
    int rows, grid, shared, sms;
    bool single;
    size_t slots, bytes;
};
bool cache_few_takes(const CacheParams& c);
bool plan_cache_few(const AttnParams& p, InType t, int sms, FewPlan* plan);
cudaError_t launch_cache_few(const AttnParams& p, const CacheParams& c, InType t, const FewPlan& plan, void* ws,
                             cudaStream_t s);

// attention_cache_many.cu: 16-bit queries, D, C <= 128, tiles of kCacheManyRows rows (M x G); each of
// the p.splits key splits yields one partial output.  out_vec: rows of `out` start on the
// boundary of four elements.
constexpr int kCacheManyRows = 128, kCacheManyKeys = 128;
bool cache_many_takes(const CacheParams& c, InType t);
cudaError_t launch_cache_many(const AttnParams& p, const CacheParams& c, InType t, bool out_vec, cudaStream_t s);

}  // namespace gs
