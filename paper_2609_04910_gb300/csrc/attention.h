// Internal interface between the attention entry points (attention_api.cu)
// and their kernels.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "gauss_sum/attention.h"
#include "internal.h"

namespace gs {

// A (B, rows, heads, width) array on the device; strides in elements.
struct Arr {
    char* p;
    int64_t sb, sr, sh;
};

// One attention call.  Query rows are numbered r = m G + g inside a key head
// j (query head j G + g), so that the G heads sharing a key head are
// neighbouring rows; R = M G of them.
struct AttnParams {
    int B, M, N, H, Hk, G, D, C;
    int64_t R;
    float c;                 // tau log2 e: probabilities are 2^(c s - lse2)
    float tau;
    int causal;
    const int* q_len;
    const int* k_len;
    Arr q, k, v, out, g, dq, dk, dv;
    float* lse;              // B x H x M, natural logarithm
    const float* g_lse;
    float* delta;            // B x H x M: g . out - g_lse
    int splits;              // key splits of a row tile
    float* part_o;           // splits x (B Hk) x R x C normalised partial outputs
    float* part_l;           // splits x (B Hk) x R: their log2-sum-exp2
    int row_splits;          // fp32-pipe gradient: row splits of a key tile
    float *part_dq, *part_dk, *part_dv;   // its partial sums: splits x (B Hk) x rows x width
    int vec;                 // fp32-pipe kernels: rows start on four-element boundaries
    unsigned* status;
    // fp16 operands scaled by powers of two (launch_attn_tc_fwd with `scaled`; else unused): the
    // scores of row (b, h, m) and key head j are row_scale[b, h, m] 2^x times the products, out
    // is 2^y times O, x and y the scaled_exponent of head_sizes[b, j].  out_bf16: type of out.
    // On the fp32 pipe head_sizes (or null) means the same of keys and values, queries are as they are.
    const float* row_scale;
    const uint2* head_sizes;
    int out_bf16;
};

// Values below twice the bf16 number of these bits, times 2^-scaled_exponent, are below 2^14.
__host__ __device__ constexpr int scaled_exponent(unsigned bits) {
    const int field = static_cast<int>(bits >> 7);
    return (field < 16 ? 16 : field > 240 ? 240 : field) - 139;
}

// Lengths of problem b, clamped to the arrays.
__device__ __forceinline__ int attn_q_len(const AttnParams& p, int b) {
    return p.q_len ? min(max(p.q_len[b], 0), p.M) : p.M;
}
__device__ __forceinline__ int attn_k_len(const AttnParams& p, int b) {
    return p.k_len ? min(max(p.k_len[b], 0), p.N) : p.N;
}

// Every mask is a limit per query: token m sees the keys n < limit.
// (64-bit sum: m + k_len - q_len + 1 stays below 2^32.)
__device__ __forceinline__ int attn_limit(int m, int ql, int kl, int causal) {
    if (m >= ql) return 0;
    if (!causal) return kl;
    const int64_t lim = static_cast<int64_t>(m) + kl - ql + 1;
    return static_cast<int>(lim < 0 ? 0 : lim > kl ? kl : lim);
}

// Gradients of 16-bit arrays take delta of rows of at most this many keys as
// sum_n p_n g . v_n - g_lse, without the rounding of `out` (attention_tc_vjp.cu
// has the errors and times of the choice).
constexpr int kFewKeys = 24;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// attention_simt_fwd.cu / attention_simt_vjp.cu: any type, alignment and
// D, C <= 256, on the fp32 pipe.
constexpr int kSimtAttnRows = 64;
constexpr int kSimtAttnKeys = 64;
cudaError_t launch_attn_simt_fwd(const AttnParams& p, InType t, cudaStream_t s);
cudaError_t launch_attn_simt_vjp(const AttnParams& p, InType t, cudaStream_t s);
// Joins the partial outputs of p.splits key splits.
cudaError_t launch_attn_join(const AttnParams& p, InType t, cudaStream_t s);
// delta of every query row, for launch_attn_simt_vjp (attention_simt_vjp.cu).
cudaError_t launch_attn_delta(const AttnParams& p, InType t, cudaStream_t s);

// attention_tc_fwd.cu: fp16 / bf16, D, C <= 128, arrays a TMA map can describe.
// `packed`: the heads sharing a key head are neighbouring rows of one tile
// (few tokens).  Each of the p.splits key splits yields one partial output.
bool attn_tc_takes(const Arr& a, int64_t B, int64_t rows, int64_t heads, int width);
// Whether (not packed) blocks take 128 query rows and key tiles of 64, two to
// an SM; else 256 rows and tiles of 128, one to an SM.
bool attn_tc_narrow(const AttnParams& p);
cudaError_t launch_attn_tc_fwd(const AttnParams& p, InType t, bool packed, bool scaled, cudaStream_t s);

// attention_tc_vjp.cu: the same range; workspace bytes, and the launches.
size_t attn_tc_vjp_workspace(const AttnParams& p, InType t);
cudaError_t launch_attn_tc_vjp(const AttnParams& p, InType t, void* ws, cudaStream_t s);

// attention_api.cu
// Attention of checked arguments: the choice of kernels, workspace and launches.  `scaled` (fp16
// arrays that attn_tc_takes, p.row_scale and p.head_sizes set): the output type is p.out_bf16's.
struct DeviceContext;
gs_status attn_forward(AttnParams p, InType t, bool scaled, const DeviceContext& dc, cudaStream_t s);
// Checks a (B, rows, heads, width) array of es-byte elements that the call
// touches unless it is empty; returns what is wrong with it, or null.
// Outputs may not overlap themselves: along dimensions longer than one,
// ordered by stride, each stride must span the extent of the ones below.
const char* check_array(const gs_array& a, int64_t es, int64_t B, int64_t rows, int64_t heads,
                        int64_t width, bool output);
inline Arr make_arr(const gs_array& a) {
    return {static_cast<char*>(a.data), a.stride_b, a.stride_row, a.stride_head};
}

// api.cu
// The current device's number, status word, SM count and whether it is an
// sm_103; and stream-ordered memory from the library's pool.
struct DeviceContext {
    int dev;
    unsigned* status;
    int sms;
    bool sm103;
};
gs_status device_context(DeviceContext* d);
// (GS_ERR_OUT_OF_MEMORY when there is none, or the test hook says so.)
gs_status workspace_alloc(void** ptr, size_t bytes, cudaStream_t s);
gs_status cuda_status(cudaError_t e, const char* where);

}  // namespace gs
