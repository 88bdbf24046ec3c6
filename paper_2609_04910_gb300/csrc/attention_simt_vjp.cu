// Gradients of softmax attention on the fp32 pipe: any element type,
// alignment and D, C <= 256, and the row term delta that both gradient paths
// use.
//
// Two passes over the pairs, so that every gradient is a sum in a fixed
// order and nothing is added atomically: the query pass owns 64 query rows
// and streams keys (grad_q), the key pass owns 64 keys and streams the rows
// of all query heads that share them (grad_k, grad_v).  Both recompute
//     p = 2^(c s - lse log2 e),  ds = p (g . v - delta).
#include "attention_simt.cuh"

namespace gs {
namespace {

using namespace simt;

// delta_m = g_m . out_m - g_lse_m; one warp per (problem, head, token).
template <typename E>
__global__ void __launch_bounds__(256) attn_delta_kernel(const AttnParams p) {
    pdl_wait();
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (row >= static_cast<int64_t>(p.B) * p.H * p.M) return;
    const int m = static_cast<int>(row % p.M);
    const int h = static_cast<int>(row / p.M % p.H), b = static_cast<int>(row / p.M / p.H);
    float x = 0.f;
    if (m < attn_q_len(p, b)) {
        const E* g = base<E>(p.g, b, h) + m * p.g.sr;
        const E* o = base<E>(p.out, b, h) + m * p.out.sr;
        for (int c = lane; c < p.C; c += 32) x = fmaf(to_f(g[c]), to_f(o[c]), x);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    if (lane == 0) p.delta[row] = p.g_lse ? x - p.g_lse[row] : x;
}

template <typename E, int NB>
__global__ void __launch_bounds__(kThreads) attn_simt_dq_kernel(const AttnParams p) {
    __shared__ __align__(16) float stage[2 * KC * LD];
    __shared__ __align__(16) float w[T * LD];
    pdl_wait();
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    const int64_t tiles_r = (p.R + T - 1) / T;
    const int64_t r0 = (blockIdx.x % tiles_r) * T;
    const int bj = static_cast<int>(blockIdx.x / tiles_r);
    const int b = bj / p.Hk, j = bj % p.Hk;
    const int ql = attn_q_len(p, b), kl = attn_k_len(p, b);
    const int64_t rows = static_cast<int64_t>(ql) * p.G;
    int lim[4];
    float l2[4], delta[4];
    E* dst[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = r0 + ty * 4 + i, m = r / p.G;
        const int h = j * p.G + static_cast<int>(r - m * p.G);
        lim[i] = r < rows ? attn_limit(static_cast<int>(m), ql, kl, p.causal) : 0;
        const int64_t at = (static_cast<int64_t>(b) * p.H + h) * p.M + m;
        l2[i] = lim[i] > 0 ? p.lse[at] * kLog2e : 0.f;
        if (l2[i] == -INFINITY) lim[i] = 0;   // every score was -inf: no probabilities
        delta[i] = lim[i] > 0 ? p.delta[at] : 0.f;
        dst[i] = r < p.R ? const_cast<E*>(base<E>(p.dq, b, h)) + m * p.dq.sr : nullptr;
    }
    const int64_t last = min(r0 + T, rows) - 1;
    const int kend = last >= r0 ? attn_limit(static_cast<int>(last / p.G), ql, kl, p.causal) : 0;
    const E* qrow = query_row<E>(p.q, p, b, j, r0 + (tid & (T - 1)), rows);
    const E* grow = query_row<E>(p.g, p, b, j, r0 + (tid & (T - 1)), rows);
    float dq[NB][4][4] = {};
    for (int64_t n0 = 0; n0 < kend; n0 += T) {
        float s[4][4], dp[4][4];
        scores(s, stage, stage + KC * LD, qrow, key_row<E>(p.k, b, j, n0 + (tid & (T - 1)), kl),
               p.D);
        scores(dp, stage, stage + KC * LD, grow, key_row<E>(p.v, b, j, n0 + (tid & (T - 1)), kl),
               p.C);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                s[i][e] = n0 + tx * 4 + e < lim[i]
                              ? exp2f(fmaf(s[i][e], p.c, -l2[i])) * (dp[i][e] - delta[i]) : 0.f;
        put_t(w, s);
        accumulate(dq, w, stage, key_row<E>(p.k, b, j, n0 + (tid >> 2), kl), p.D);
    }
    const float scale[4] = {p.tau, p.tau, p.tau, p.tau};
    put_rows(dq, dst, scale, p.D);
}

template <typename E, int NB>
__global__ void __launch_bounds__(kThreads) attn_simt_dkv_kernel(const AttnParams p) {
    __shared__ __align__(16) float stage[2 * KC * LD];
    __shared__ __align__(16) float w[T * LD];
    pdl_wait();
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    const int64_t tiles_n = (p.N + T - 1) / T;
    const int64_t n0 = (blockIdx.x % tiles_n) * T;
    const int bj = static_cast<int>(blockIdx.x / tiles_n);
    const int b = bj / p.Hk, j = bj % p.Hk;
    const int ql = attn_q_len(p, b), kl = attn_k_len(p, b);
    // First token that sees key n0: its limit m + kl - ql + 1 exceeds n0.
    int64_t m0 = p.causal ? max(static_cast<int64_t>(0), n0 - (static_cast<int64_t>(kl) - ql)) : 0;
    const int64_t rows = n0 < kl ? static_cast<int64_t>(ql) * p.G : 0;
    const E* krow = key_row<E>(p.k, b, j, n0 + (tid & (T - 1)), kl);
    const E* vrow = key_row<E>(p.v, b, j, n0 + (tid & (T - 1)), kl);
    float dk[NB][4][4] = {}, dv[NB][4][4] = {};
    for (int64_t r0 = m0 * p.G; r0 < rows; r0 += T) {
        const int64_t rt = r0 + (tid & (T - 1)), rn = r0 + (tid >> 2);
        float s[4][4], dp[4][4];
        scores(s, stage, stage + KC * LD, krow, query_row<E>(p.q, p, b, j, rt, rows), p.D);
        scores(dp, stage, stage + KC * LD, vrow, query_row<E>(p.g, p, b, j, rt, rows), p.C);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t r = r0 + tx * 4 + e, m = r / p.G;
            int lim = r < rows ? attn_limit(static_cast<int>(m), ql, kl, p.causal) : 0;
            const int64_t at = (static_cast<int64_t>(b) * p.H + j * p.G + (r - m * p.G)) * p.M + m;
            const float l2 = lim > 0 ? p.lse[at] * kLog2e : 0.f;
            if (l2 == -INFINITY) lim = 0;
            const float delta = lim > 0 ? p.delta[at] : 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[i][e] = n0 + ty * 4 + i < lim ? exp2f(fmaf(s[i][e], p.c, -l2)) : 0.f;
                dp[i][e] = n0 + ty * 4 + i < lim ? s[i][e] * (dp[i][e] - delta) : 0.f;
            }
        }
        put_t(w, s);
        accumulate(dv, w, stage, query_row<E>(p.g, p, b, j, rn, rows), p.C);
        __syncthreads();
        put_t(w, dp);
        accumulate(dk, w, stage, query_row<E>(p.q, p, b, j, rn, rows), p.D);
    }
    E *dk_rows[4], *dv_rows[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t n = n0 + ty * 4 + i;
        dk_rows[i] = n < p.N && p.dk.p ? const_cast<E*>(base<E>(p.dk, b, j)) + n * p.dk.sr : nullptr;
        dv_rows[i] = n < p.N && p.dv.p ? const_cast<E*>(base<E>(p.dv, b, j)) + n * p.dv.sr : nullptr;
    }
    const float sk[4] = {p.tau, p.tau, p.tau, p.tau}, sv[4] = {1.f, 1.f, 1.f, 1.f};
    put_rows(dk, dk_rows, sk, p.D);
    put_rows(dv, dv_rows, sv, p.C);
}

template <typename E, int NB>
cudaError_t launch_vjp(const AttnParams& p, cudaStream_t s) {
    cudaError_t e = cudaSuccess;
    if (p.dq.p) {
        note_launches(1);
        e = launch_kernel(attn_simt_dq_kernel<E, NB>,
                          dim3(static_cast<unsigned>((p.R + T - 1) / T * p.B * p.Hk)), kThreads, 0,
                          s, p);
    }
    if (e == cudaSuccess && (p.dk.p || p.dv.p) && p.N > 0) {
        note_launches(1);
        e = launch_kernel(attn_simt_dkv_kernel<E, NB>,
                          dim3(static_cast<unsigned>((p.N + T - 1) / T * static_cast<int64_t>(p.B) * p.Hk)),
                          kThreads, 0, s, p);
    }
    return e;
}

template <typename E>
cudaError_t launch_vjp(const AttnParams& p, cudaStream_t s) {
    const int width = p.D > p.C ? p.D : p.C;
    if (width <= 64) return launch_vjp<E, 1>(p, s);
    if (width <= 128) return launch_vjp<E, 2>(p, s);
    return launch_vjp<E, 4>(p, s);
}

}  // namespace

cudaError_t launch_attn_simt_vjp(const AttnParams& p, InType t, cudaStream_t s) {
    if (t == InType::F32) return launch_vjp<float>(p, s);
    if (t == InType::F16) return launch_vjp<__half>(p, s);
    return launch_vjp<__nv_bfloat16>(p, s);
}

cudaError_t launch_attn_delta(const AttnParams& p, InType t, cudaStream_t s) {
    const int64_t rows = static_cast<int64_t>(p.B) * p.H * p.M;
    const dim3 grid(static_cast<unsigned>((rows + 7) / 8));
    note_launches(1);
    if (t == InType::F32) return launch_kernel(attn_delta_kernel<float>, grid, 256, 0, s, p);
    if (t == InType::F16) return launch_kernel(attn_delta_kernel<__half>, grid, 256, 0, s, p);
    return launch_kernel(attn_delta_kernel<__nv_bfloat16>, grid, 256, 0, s, p);
}

}  // namespace gs
