// Softmax attention on the fp32 pipe: any element type, alignment and
// D, C <= 256 (fp32 arrays, and fp16 / bf16 arrays the tensor-core kernel
// does not take), and the join of key splits that both forward kernels use.
//
// One block takes 64 query rows of one key head (the heads that share it are
// neighbouring rows, so a single token of 8 heads fills 8 rows) and streams
// the keys in tiles of 64 once, with the running maximum m and sum l of each
// row in log2 units:
//     m' = max(m, max_n c s_n),  l' = l 2^(m - m') + sum_n 2^(c s_n - m'),
//     o' = o 2^(m - m') + sum_n 2^(c s_n - m') v_n,   out = o / l.
// Bound by the latency of its steps: 128 registers leave four warps a
// scheduler, which issue 59 % of the time and keep the FMA pipe a third busy
// (2 x 700 x 1501 points, 4 heads x 32 channels: 54 us with the join, 20
// TFLOP/s).  Packed two-term FMAs (12 % fewer instructions) gained nothing;
// 64-row tiles, because point clouds are short and a tile of 128 pads more.
#include "attention_simt.cuh"

namespace gs {
namespace {

using namespace simt;

template <typename E, int NB, int CW>
__global__ void __launch_bounds__(kThreads, NB == 1 ? 2 : 1) attn_simt_fwd_kernel(const AttnParams p) {
    __shared__ __align__(16) float stage[2 * KC * T];   // score operands, then values
    __shared__ __align__(16) float w[T * T];
    static_assert(2 * KC == T, "values reuse the score operands' space");
    pdl_wait();
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    const int64_t tiles_r = (p.R + T - 1) / T;
    int64_t blk = blockIdx.x;
    const int split = static_cast<int>(blk % p.splits);
    blk /= p.splits;
    const int64_t r0 = (blk % tiles_r) * T;
    const int bj = static_cast<int>(blk / tiles_r);
    const int b = bj / p.Hk, j = bj % p.Hk;
    const int ql = attn_q_len(p, b), kl = attn_k_len(p, b);
    const int64_t rows = static_cast<int64_t>(ql) * p.G;

    int lim[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = r0 + ty * 4 + i;
        lim[i] = r < rows ? attn_limit(static_cast<int>(row_token(p, r)), ql, kl, p.causal) : 0;
    }
    // Limits grow with the row: the tile's last row has the largest.
    const int64_t last = min(r0 + T, rows) - 1;
    const int kend = last >= r0 ? attn_limit(static_cast<int>(last / p.G), ql, kl, p.causal) : 0;
    const int64_t tiles = (kend + T - 1) / T;
    const int64_t t0 = tiles * split / p.splits, t1 = tiles * (split + 1) / p.splits;

    // Keys below `open` are seen by all four rows of the thread.
    const int open = min(min(lim[0], lim[1]), min(lim[2], lim[3]));

    // Keys and values times powers of two of their head: the scores' and the results' factors.
    // (The first never 0, which would make NaN of a masked score.)
    float c = p.c, v_up = 1.f;
    if (p.head_sizes) {
        const uint2 size = p.head_sizes[static_cast<int64_t>(b) * p.Hk + j];
        c = fmaxf(c * exp2f(static_cast<float>(scaled_exponent(size.x))), 0x1p-126f);
        v_up = exp2f(static_cast<float>(scaled_exponent(size.y)));
    }

    float o[NB][4][CW] = {};
    float top[4], sum[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) top[i] = -INFINITY, sum[i] = 0.f;
    const E *qrow[2], *krow[2], *vrow[4];
    query_rows(qrow, p.q, p, b, j, r0, rows);

    for (int64_t t = t0; t < t1; ++t) {
        const int64_t n0 = t * T;
        float s[4][4];
        key_rows(krow, p.k, b, j, n0, kl);
        key_rows(vrow, p.v, b, j, n0, kl);
        scores(s, stage, stage + KC * T, qrow, krow, p.D, p.vec);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (n0 + T > open) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n0 + tx * 4 + e >= lim[i]) s[i][e] = -INFINITY;
            }
            float mx = fmaxf(fmaxf(s[i][0], s[i][1]), fmaxf(s[i][2], s[i][3]));
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, d));
            const float m1 = fmaxf(top[i], mx * c);
            const float ref = m1 == -INFINITY ? 0.f : m1;   // nothing seen yet: 2^(-inf) = 0
            const float f = ex2_approx(top[i] - ref);
            float add = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[i][e] = ex2_approx(fmaf(s[i][e], c, -ref));   // (rounded once)
                add += s[i][e];
            }
            sum[i] = sum[i] * f + add;
            top[i] = m1;
#pragma unroll
            for (int u = 0; u < NB; ++u)
#pragma unroll
                for (int e = 0; e < CW; ++e) o[u][i][e] *= f;
        }
        put_t(w, s);
        accumulate(o, w, stage, vrow, p.C, p.vec);
    }

    E* out_rows[4];
    float* part_rows[4];
    float inv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) sum[i] += __shfl_xor_sync(~0u, sum[i], d);
        const int64_t r = r0 + ty * 4 + i;
        inv[i] = lim[i] > 0 && t1 > t0 && top[i] != -INFINITY ? 1.f / sum[i] : 0.f;
        const float l2 = inv[i] != 0.f || sum[i] != sum[i] ? top[i] + log2f(sum[i]) : -INFINITY;
        inv[i] *= v_up;
        out_rows[i] = nullptr;
        part_rows[i] = nullptr;
        if (r >= p.R) continue;
        const int64_t at = (static_cast<int64_t>(split) * p.B * p.Hk + bj) * p.R + r;
        if (p.splits > 1) {
            part_rows[i] = p.part_o + at * p.C;
            if (tx == 0) p.part_l[at] = l2;
        } else {
            const int64_t m = row_token(p, r);
            const int h = j * p.G + static_cast<int>(r - m * p.G);
            out_rows[i] = const_cast<E*>(base<E>(p.out, b, h)) + m * p.out.sr;
            if (p.lse && tx == 0)
                p.lse[(static_cast<int64_t>(b) * p.H + h) * p.M + m] = l2 * kLn2;
        }
    }
    if (p.splits > 1)
        put_rows(o, part_rows, inv, p.C);
    else
        put_rows(o, out_rows, inv, p.C);
}

// out = sum_s 2^(l_s - l) out_s, l = log2 sum_s 2^(l_s).  WARPS warps share a
// query row: warp w sums the splits w, w + WARPS, .. in order (four of them on
// their way at a time), and the warps' sums are added in order.  A split
// without keys has l_s = -infinity and no partial output: what lies in its
// place is read, but not used.
template <typename E, int WARPS>
__global__ void __launch_bounds__(128) attn_join_kernel(const AttnParams p) {
    __shared__ float sums[4][257];
    pdl_wait();
    constexpr int kRows = 4 / WARPS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % WARPS;
    const int64_t all = static_cast<int64_t>(p.B) * p.Hk * p.R;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + warp / WARPS;
    if (WARPS == 1 && row >= all) return;
    const int bj = static_cast<int>(row / p.R);
    const int64_t r = row % p.R, m = r / p.G;
    const int b = bj / p.Hk, h = (bj % p.Hk) * p.G + static_cast<int>(r - m * p.G);
    float top = -INFINITY;
    for (int s = lane; s < p.splits; s += 32) top = fmaxf(top, p.part_l[s * all + row]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
    const float ref = top == -INFINITY ? 0.f : top;
    float o[8] = {}, sum = 0.f;
    for (int s0 = part; s0 < p.splits; s0 += 4 * WARPS) {
        float wgt[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = s0 + i * WARPS;
            wgt[i] = s < p.splits ? exp2f(p.part_l[s * all + row] - ref) : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int c = lane + 32 * u;
            if (c >= p.C) break;
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[i] = p.part_o[(min(s0 + i * WARPS, p.splits - 1) * all + row) * p.C + c];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[u] = wgt[i] != 0.f ? fmaf(wgt[i], x[i], o[u]) : o[u];
        }
        sum += wgt[0] + wgt[1] + wgt[2] + wgt[3];
    }
    if (WARPS > 1) {
#pragma unroll
        for (int u = 0; u < 8; ++u) sums[warp][lane + 32 * u] = o[u];
        if (lane == 0) sums[warp][256] = sum;
        __syncthreads();
        if (part != 0) return;
#pragma unroll
        for (int w = 1; w < WARPS; ++w) {
#pragma unroll
            for (int u = 0; u < 8; ++u) o[u] += sums[warp + w][lane + 32 * u];
            sum += sums[warp + w][256];
        }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    E* dst = const_cast<E*>(base<E>(p.out, b, h)) + m * p.out.sr;
#pragma unroll
    for (int u = 0; u < 8; ++u)
        if (lane + 32 * u < p.C) dst[lane + 32 * u] = from_f<E>(o[u] * inv);
    if (p.lse && lane == 0)
        p.lse[(static_cast<int64_t>(b) * p.H + h) * p.M + m] =
            sum == 0.f ? -INFINITY : (ref + log2f(sum)) * kLn2;
}

template <typename E>
cudaError_t launch_fwd(const AttnParams& p, cudaStream_t s) {
    const int64_t blocks = (p.R + T - 1) / T * p.B * p.Hk * p.splits;
    const dim3 grid(static_cast<unsigned>(blocks));
    note_launches(1);
    if (p.C <= 32) return launch_kernel(attn_simt_fwd_kernel<E, 1, 2>, grid, kThreads, 0, s, p);
    if (p.C <= 64) return launch_kernel(attn_simt_fwd_kernel<E, 1, 4>, grid, kThreads, 0, s, p);
    if (p.C <= 128) return launch_kernel(attn_simt_fwd_kernel<E, 2, 4>, grid, kThreads, 0, s, p);
    return launch_kernel(attn_simt_fwd_kernel<E, 4, 4>, grid, kThreads, 0, s, p);
}

}  // namespace

cudaError_t launch_attn_simt_fwd(const AttnParams& p, InType t, cudaStream_t s) {
    if (t == InType::F32) return launch_fwd<float>(p, s);
    if (t == InType::F16) return launch_fwd<__half>(p, s);
    return launch_fwd<__nv_bfloat16>(p, s);
}

template <typename E>
static cudaError_t launch_join(const AttnParams& p, cudaStream_t s) {
    const int64_t rows = static_cast<int64_t>(p.B) * p.Hk * p.R;
    note_launches(1);
    if (p.splits > 8)
        return launch_kernel(attn_join_kernel<E, 4>, dim3(static_cast<unsigned>(rows)), 128, 0, s, p);
    return launch_kernel(attn_join_kernel<E, 1>, dim3(static_cast<unsigned>((rows + 3) / 4)), 128, 0, s, p);
}

cudaError_t launch_attn_join(const AttnParams& p, InType t, cudaStream_t s) {
    if (t == InType::F32) return launch_join<float>(p, s);
    if (t == InType::F16) return launch_join<__half>(p, s);
    return launch_join<__nv_bfloat16>(p, s);
}

}  // namespace gs
