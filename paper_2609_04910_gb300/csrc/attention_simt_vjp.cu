// Gradients of softmax attention on the fp32 pipe: any element type,
// alignment and D, C <= 256, with its row term delta.
//
// Two passes over the pairs, so that every gradient is a sum in a fixed
// order and nothing is added atomically: the query pass owns 64 query rows
// and streams keys (grad_q), the key pass owns 64 keys and streams the rows
// of all query heads that share them (grad_k, grad_v).  Both recompute
//     p = 2^(c s - lse log2 e),  ds = p (g . v - delta).
// Few tiles are shared out further (key splits of the query pass, row splits
// of the key pass), their partial sums added in order by a last kernel.
//
// Bound like the forward pass by the latency of its steps (four warps a
// scheduler, 45 % of the issue slots): 500 x 900 points, 4 heads x 32 channels,
// 51 us for the three launches, 11 TFLOP/s of the five products.
#include "attention_simt.cuh"

namespace gs {
namespace {

using namespace simt;

// delta_m = g_m . out_m - g_lse_m; one warp per (problem, head, token).  16-bit
// rows of few keys sum p_n g . v_n over them instead, as on the tensor cores:
// `out` is rounded, and such rows do not average that out.
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
        const int lim = attn_limit(m, attn_q_len(p, b), attn_k_len(p, b), p.causal);
        const float l2 = lim > 0 ? p.lse[row] * kLog2e : -INFINITY;
        if (sizeof(E) == 2 && lim <= kFewKeys && l2 != -INFINITY) {
            const int j = h / p.G;
            const E* q = base<E>(p.q, b, h) + m * p.q.sr;
            constexpr int kKeys = 4;     // on their way at a time
            for (int n0 = 0; n0 < lim; n0 += kKeys) {
                const E *k[kKeys], *v[kKeys];
                float s[kKeys] = {}, dp[kKeys] = {};
#pragma unroll
                for (int i = 0; i < kKeys; ++i) {
                    const int n = min(n0 + i, lim - 1);
                    k[i] = base<E>(p.k, b, j) + n * p.k.sr;
                    v[i] = base<E>(p.v, b, j) + n * p.v.sr;
                }
#pragma unroll 8
                for (int d = lane; d < p.D; d += 32) {
                    const float y = to_f(q[d]);
#pragma unroll
                    for (int i = 0; i < kKeys; ++i) s[i] = fmaf(y, to_f(k[i][d]), s[i]);
                }
#pragma unroll 8
                for (int c = lane; c < p.C; c += 32) {
                    const float y = to_f(g[c]);
#pragma unroll
                    for (int i = 0; i < kKeys; ++i) dp[i] = fmaf(y, to_f(v[i][c]), dp[i]);
                }
#pragma unroll
                for (int i = 0; i < kKeys; ++i) {
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) s[i] += __shfl_xor_sync(~0u, s[i], d);
                    if (n0 + i < lim) x = fmaf(exp2f(fmaf(s[i], p.c, -l2)), dp[i], x);
                }
            }
        } else {
            for (int c = lane; c < p.C; c += 32) x = fmaf(to_f(g[c]), to_f(o[c]), x);
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    if (lane == 0) p.delta[row] = p.g_lse ? x - p.g_lse[row] : x;
}

// Where the rows 4 ty + i of a block's gradient go: the output, or with key
// (row) splits a partial sum in float32.
template <typename E>
struct Target {
    E* out[4];
    float* part[4];
};

template <int NB, int CW, typename E>
__device__ __forceinline__ void put(const float (&acc)[NB][4][CW], const Target<E>& to, bool split,
                                    float scale, int width) {
    const float one[4] = {1.f, 1.f, 1.f, 1.f}, sc[4] = {scale, scale, scale, scale};
    if (split)
        put_rows(acc, to.part, one, width);
    else
        put_rows(acc, to.out, sc, width);
}

template <typename E, int NB, int CW>
__device__ __forceinline__ void query_pass(const AttnParams& p, float* stage, float* w, int64_t blk) {
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    const int64_t tiles_r = (p.R + T - 1) / T;
    const int split = static_cast<int>(blk % p.splits);
    blk /= p.splits;
    const int64_t r0 = (tiles_r - 1 - blk % tiles_r) * T;   // (most keys first)
    const int bj = static_cast<int>(blk / tiles_r);
    const int b = bj / p.Hk, j = bj % p.Hk;
    const int ql = attn_q_len(p, b), kl = attn_k_len(p, b);
    const int64_t rows = static_cast<int64_t>(ql) * p.G;
    int lim[4];
    float l2[4], delta[4];
    Target<E> to;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = r0 + ty * 4 + i, m = row_token(p, r);
        const int h = j * p.G + static_cast<int>(r - m * p.G);
        lim[i] = r < rows ? attn_limit(static_cast<int>(m), ql, kl, p.causal) : 0;
        const int64_t at = (static_cast<int64_t>(b) * p.H + h) * p.M + m;
        l2[i] = lim[i] > 0 ? p.lse[at] * kLog2e : 0.f;
        if (l2[i] == -INFINITY) lim[i] = 0;   // every score was -inf: no probabilities
        delta[i] = lim[i] > 0 ? p.delta[at] : 0.f;
        to.out[i] = r < p.R ? const_cast<E*>(base<E>(p.dq, b, h)) + m * p.dq.sr : nullptr;
        to.part[i] = r < p.R ? p.part_dq + ((static_cast<int64_t>(split) * p.B * p.Hk + bj) * p.R + r) * p.D
                             : nullptr;
    }
    // Keys below `open` are seen by all four rows of the thread.
    const int open = min(min(lim[0], lim[1]), min(lim[2], lim[3]));
    const int64_t last = min(r0 + T, rows) - 1;
    const int kend = last >= r0 ? attn_limit(static_cast<int>(last / p.G), ql, kl, p.causal) : 0;
    const int64_t tiles = (static_cast<int64_t>(kend) + T - 1) / T;
    const int64_t t0 = tiles * split / p.splits, t1 = tiles * (split + 1) / p.splits;
    const E *qrow[2], *grow[2], *krow[2], *vrow[2], *kn[4];
    query_rows(qrow, p.q, p, b, j, r0, rows);
    query_rows(grow, p.g, p, b, j, r0, rows);
    float dq[NB][4][CW] = {};
    for (int64_t t = t0; t < t1; ++t) {
        const int64_t n0 = t * T;
        key_rows(krow, p.k, b, j, n0, kl);
        key_rows(vrow, p.v, b, j, n0, kl);
        key_rows(kn, p.k, b, j, n0, kl);
        float s[4][4], dp[4][4];
        scores(s, stage, stage + KC * T, qrow, krow, p.D, p.vec);
        scores(dp, stage, stage + KC * T, grow, vrow, p.C, p.vec);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                s[i][e] = ex2_approx(fmaf(s[i][e], p.c, -l2[i])) * (dp[i][e] - delta[i]);
        if (n0 + T > open) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n0 + tx * 4 + e >= lim[i]) s[i][e] = 0.f;
        }
        put_t(w, s);
        accumulate(dq, w, stage, kn, p.D, p.vec);
    }
    put(dq, to, p.splits > 1, p.tau, p.D);
}

// lse log2 e, delta and the limit of a streamed row.
struct RowTerms {
    float l2, delta;
    int lim;
};

template <typename E, int NB, int CW>
__device__ __forceinline__ void key_pass(const AttnParams& p, float* stage, float* w, RowTerms* terms, int64_t blk) {
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    const int64_t tiles_n = (static_cast<int64_t>(p.N) + T - 1) / T;
    const int split = static_cast<int>(blk % p.row_splits);
    blk /= p.row_splits;
    const int64_t n0 = (blk % tiles_n) * T;
    const int bj = static_cast<int>(blk / tiles_n);
    const int b = bj / p.Hk, j = bj % p.Hk;
    const int ql = attn_q_len(p, b), kl = attn_k_len(p, b);
    // First token that sees key n0: its limit m + kl - ql + 1 exceeds n0.
    const int64_t m0 = p.causal ? max(static_cast<int64_t>(0), n0 - (static_cast<int64_t>(kl) - ql)) : 0;
    const int64_t rows = n0 < kl ? static_cast<int64_t>(ql) * p.G : 0;
    const int64_t tiles = max(static_cast<int64_t>(0), rows - m0 * p.G + T - 1) / T;
    const int64_t t0 = tiles * split / p.row_splits, t1 = tiles * (split + 1) / p.row_splits;
    const E *krow[2], *vrow[2], *qrow[2], *grow[2], *qn[4], *gn[4];
    key_rows(krow, p.k, b, j, n0, kl);
    key_rows(vrow, p.v, b, j, n0, kl);
    float dk[NB][4][CW] = {}, dv[NB][4][CW] = {};
    for (int64_t t = t0; t < t1; ++t) {
        const int64_t r0 = m0 * p.G + t * T;
        query_rows(qrow, p.q, p, b, j, r0, rows);
        query_rows(grow, p.g, p, b, j, r0, rows);
        // (The last tile's terms were read before the barriers of its products.)
        if (threadIdx.x < T) {
            const int64_t r = r0 + threadIdx.x, m = row_token(p, r);
            int lim = r < rows ? attn_limit(static_cast<int>(m), ql, kl, p.causal) : 0;
            const int64_t at = (static_cast<int64_t>(b) * p.H + j * p.G + (r - m * p.G)) * p.M + m;
            const float l2 = lim > 0 ? p.lse[at] * kLog2e : 0.f;
            if (l2 == -INFINITY) lim = 0;
            terms[threadIdx.x] = {l2, lim > 0 ? p.delta[at] : 0.f, lim};
        }
        float s[4][4], dp[4][4];
        scores(s, stage, stage + KC * T, krow, qrow, p.D, p.vec);
        scores(dp, stage, stage + KC * T, vrow, grow, p.C, p.vec);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const RowTerms x = terms[tx * 4 + e];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool on = n0 + ty * 4 + i < x.lim;
                s[i][e] = on ? ex2_approx(fmaf(s[i][e], p.c, -x.l2)) : 0.f;
                dp[i][e] = on ? s[i][e] * (dp[i][e] - x.delta) : 0.f;
            }
        }
        query_rows(gn, p.g, p, b, j, r0, rows);
        put_t(w, s);
        accumulate(dv, w, stage, gn, p.C, p.vec);
        query_rows(qn, p.q, p, b, j, r0, rows);
        __syncthreads();
        put_t(w, dp);
        accumulate(dk, w, stage, qn, p.D, p.vec);
    }
    Target<E> tk, tv;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t n = n0 + ty * 4 + i;
        const int64_t at = (static_cast<int64_t>(split) * p.B * p.Hk + bj) * p.N + n;
        tk.out[i] = n < p.N && p.dk.p ? const_cast<E*>(base<E>(p.dk, b, j)) + n * p.dk.sr : nullptr;
        tv.out[i] = n < p.N && p.dv.p ? const_cast<E*>(base<E>(p.dv, b, j)) + n * p.dv.sr : nullptr;
        tk.part[i] = n < p.N && p.dk.p ? p.part_dk + at * p.D : nullptr;
        tv.part[i] = n < p.N && p.dv.p ? p.part_dv + at * p.C : nullptr;
    }
    put(dk, tk, p.row_splits > 1, p.tau, p.D);
    put(dv, tv, p.row_splits > 1, 1.f, p.C);
}

// Both passes in one launch, the longer key passes first.
template <typename E, int NB, int CW>
__global__ void __launch_bounds__(kThreads, NB == 1 ? 2 : 1) attn_simt_vjp_kernel(const AttnParams p, int64_t key_blocks) {
    __shared__ __align__(16) float stage[2 * KC * T];
    __shared__ __align__(16) float w[T * T];
    __shared__ RowTerms terms[T];
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x < key_blocks)
        key_pass<E, NB, CW>(p, stage, w, terms, blockIdx.x);
    else
        query_pass<E, NB, CW>(p, stage, w, blockIdx.x - key_blocks);
}

// Sums partial gradients over their splits, in order: one thread per channel
// of a row of dq, then dk, then dv.
template <typename E>
__global__ void __launch_bounds__(256) attn_simt_sum_kernel(const AttnParams p, int64_t nq, int64_t nk, int64_t nv) {
    pdl_wait();
    int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= nq + nk + nv) return;
    const bool is_q = i < nq, is_k = !is_q && i < nq + nk;
    i -= is_q ? 0 : is_k ? nq : nq + nk;
    const int width = is_q || is_k ? p.D : p.C;
    const int64_t all = is_q ? nq : is_k ? nk : nv, per = is_q ? p.R : p.N;
    const float* part = is_q ? p.part_dq : is_k ? p.part_dk : p.part_dv;
    const int splits = is_q ? p.splits : p.row_splits;
    float x = 0.f;
    for (int s = 0; s < splits; ++s) x += part[s * all + i];
    const int c = static_cast<int>(i % width);
    const int64_t row = i / width % per;
    const int bj = static_cast<int>(i / width / per), b = bj / p.Hk, j = bj % p.Hk;
    if (is_q) {
        const int64_t m = row / p.G;
        const_cast<E*>(base<E>(p.dq, b, j * p.G + static_cast<int>(row - m * p.G)))[m * p.dq.sr + c] =
            from_f<E>(x * p.tau);
    } else {
        const Arr& a = is_k ? p.dk : p.dv;
        const_cast<E*>(base<E>(a, b, j))[row * a.sr + c] = from_f<E>(is_k ? x * p.tau : x);
    }
}

template <typename E, int NB, int CW>
cudaError_t launch_vjp(const AttnParams& p, cudaStream_t s) {
    const int64_t heads = static_cast<int64_t>(p.B) * p.Hk;
    const int64_t key_blocks =
        p.dk.p || p.dv.p ? (static_cast<int64_t>(p.N) + T - 1) / T * heads * p.row_splits : 0;
    const int64_t blocks = key_blocks + (p.dq.p ? (p.R + T - 1) / T * heads * p.splits : 0);
    if (blocks == 0) return cudaSuccess;
    note_launches(1);
    cudaError_t e = launch_kernel(attn_simt_vjp_kernel<E, NB, CW>, dim3(static_cast<unsigned>(blocks)), kThreads, 0,
                                  s, p, key_blocks);
    const int64_t nq = p.dq.p && p.splits > 1 ? heads * p.R * p.D : 0;
    const int64_t nk = p.dk.p && p.row_splits > 1 ? heads * p.N * p.D : 0;
    const int64_t nv = p.dv.p && p.row_splits > 1 ? heads * p.N * p.C : 0;
    if (e != cudaSuccess || nq + nk + nv == 0) return e;
    note_launches(1);
    return launch_kernel(attn_simt_sum_kernel<E>, dim3(static_cast<unsigned>((nq + nk + nv + 255) / 256)), 256,
                         0, s, p, nq, nk, nv);
}

template <typename E>
cudaError_t launch_vjp(const AttnParams& p, cudaStream_t s) {
    const int width = p.D > p.C ? p.D : p.C;
    if (width <= 32) return launch_vjp<E, 1, 2>(p, s);
    if (width <= 64) return launch_vjp<E, 1, 4>(p, s);
    if (width <= 128) return launch_vjp<E, 2, 4>(p, s);
    return launch_vjp<E, 4, 4>(p, s);
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
