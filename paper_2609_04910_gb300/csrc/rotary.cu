// Rotary positions of queries and keys (include/gauss_sum/attention.h).
//
// A pair turns by angle = position x frequency.  Frequencies are 64-bit
// fractions of a turn, so the product modulo 2^64 is the exact angle modulo
// one turn for any position: its top 32 bits, as a signed fraction of half a
// turn, go to sincospif.
//
// The kernel reads and writes every element once and is bound by that.  A
// block takes up to four tokens and a share of the heads: its threads write
// the tokens' cosines and sines to shared memory (once for all heads, while
// the first vectors are on their way) and then stream the heads, two 16-byte
// vectors of eight (fp32: four) pairs an item, two items read before the
// first is written (outputs may be the inputs, so the compiler cannot move
// a read past a write).
#include <algorithm>
#include <cmath>

#include "attention_simt.cuh"

namespace gs {
namespace {

using simt::from_f;
using simt::to_f;

// Two items in flight a thread at 64 registers (four blocks an SM) and four
// tokens a block: 59 us on q and k of 16384 tokens x 40 heads x 128 channels
// in bf16 (5.7 TB/s; 57 us replayed; a plain copy of the same bytes takes 58 us).  At the time
// of the choice, 64 us: four items at 104 registers took 71, eight tokens 66.
constexpr int kBatch = 2;       // items a thread reads before it writes the first
constexpr int kMaxTokens = 4;   // tokens of a block
constexpr int kMaxRotated = 4096;

struct RotaryParams {
    int64_t M, tokens;       // tokens: B x M
    int H, Hk, D, R;
    float scale;
    int interleaved, transpose, pos64;
    const void* pos;
    int64_t pos_b, pos_m;
    const int64_t* freq;
    Arr q, k, qo, ko;
    int copy_q, copy_k;      // channels R .. D - 1 are copied (out of place)
    int units;               // per token: R / (2 V) turned ones, then copied ones
    int block_tokens;        // tokens of a block
    int head_blocks;         // blocks that share a token's heads
    int rounds;              // heads of a thread
};

template <typename E, int V>
struct alignas(sizeof(E) * V < 16 ? sizeof(E) * V : 16) Vec {
    E e[V];
};

// Unit u of a head: pairs V u .. V u + V - 1, i.e. channels [a, a + V) and
// [b, b + V); half layout a = V u, b = a + R / 2, interleaved a = 2 V u,
// b = a + V.  Units past the turned ones copy 2 V channels from R on.  V = 1
// takes any stride and alignment.  threadIdx.x: unit, threadIdx.y: head.
template <typename E, int V>
__global__ void __launch_bounds__(256, 4) rotary_kernel(const __grid_constant__ RotaryParams p) {
    extern __shared__ float table[];      // block_tokens x R / 2 cosines, then as many sines
    using X = Vec<E, V>;
    pdl_wait();
    const int64_t token0 = static_cast<int64_t>(blockIdx.x / p.head_blocks) * p.block_tokens;
    const int64_t b0 = token0 / p.M, m0 = token0 - b0 * p.M;
    const int here = static_cast<int>(min(static_cast<int64_t>(p.block_tokens), p.tokens - token0));
    const int heads = p.H + p.Hk;
    const int h0 = static_cast<int>(blockIdx.x % p.head_blocks) * blockDim.y * p.rounds + threadIdx.y;
    const int turned = p.R / (2 * V);
    const int items = here * p.rounds;
    const int half = p.R / 2;
    const int tid = threadIdx.y * blockDim.x + threadIdx.x, threads = blockDim.x * blockDim.y;
    // Problem and row of token tk of this block.
    const auto place = [&](int tk, int64_t& b, int64_t& m) {
        b = b0;
        m = m0 + tk;
        while (m >= p.M) {
            m -= p.M;
            ++b;
        }
    };

    for (int u0 = 0; u0 < p.units; u0 += blockDim.x) {
        const int u = min(u0 + static_cast<int>(threadIdx.x), p.units - 1);
        const bool mine = u0 + static_cast<int>(threadIdx.x) < p.units;
        const bool copy = u >= turned;
        const int at = copy ? p.R + (u - turned) * 2 * V : p.interleaved ? 2 * V * u : V * u;
        const int second = copy || p.interleaved ? at + V : at + half;
        const int bt = second < p.D ? second : at;    // a copied unit may end in a single half
        int tk = 0, round = 0;                        // of the next item
        for (int k0 = 0; k0 < items; k0 += kBatch) {
            X x[kBatch], y[kBatch];
            E* to[kBatch];
            int tok[kBatch];
            bool put[kBatch];
#pragma unroll
            for (int n = 0; n < kBatch; ++n) {
                // Items past the end read the last one again and write nothing.
                const int h_of = h0 + round * static_cast<int>(blockDim.y);
                const int h = min(h_of, heads - 1);
                int64_t b, m;
                place(tk, b, m);
                const bool is_q = h < p.H;
                const Arr& in = is_q ? p.q : p.k;
                const Arr& out = is_q ? p.qo : p.ko;
                const int hh = is_q ? h : h - p.H;
                const E* src = reinterpret_cast<const E*>(in.p) + b * in.sb + m * in.sr + hh * in.sh;
                to[n] = reinterpret_cast<E*>(out.p) + b * out.sb + m * out.sr + hh * out.sh;
                put[n] = mine && k0 + n < items && h_of < heads && (!copy || (is_q ? p.copy_q : p.copy_k));
                tok[n] = tk;
                x[n] = *reinterpret_cast<const X*>(src + at);
                y[n] = *reinterpret_cast<const X*>(src + bt);
                if (k0 + n + 1 < items && ++round == p.rounds) {
                    round = 0;
                    ++tk;
                }
            }
            if (u0 == 0 && k0 == 0) {
                for (int i = tid; i < here * half; i += threads) {
                    const int tk = i / half, f = i - tk * half;
                    int64_t b, m;
                    place(tk, b, m);
                    const int64_t at_pos = b * p.pos_b + m * p.pos_m;
                    const int64_t pos = p.pos64 ? static_cast<const int64_t*>(p.pos)[at_pos]
                                                : static_cast<const int*>(p.pos)[at_pos];
                    const uint64_t turn = static_cast<uint64_t>(pos) * static_cast<uint64_t>(p.freq[f]);
                    // Top half as a signed fraction of 2^32; sincospif takes half turns.
                    float si, co;
                    sincospif(static_cast<float>(static_cast<int>(turn >> 32)) * 0x1p-31f, &si, &co);
                    table[i] = co * p.scale;
                    table[p.block_tokens * half + i] = p.transpose ? -si * p.scale : si * p.scale;
                }
                __syncthreads();
            }
#pragma unroll
            for (int n = 0; n < kBatch; ++n) {
                if (!copy) {
                    const float* co = table + tok[n] * half + V * u;
                    const Vec<float, V> c = *reinterpret_cast<const Vec<float, V>*>(co);
                    const Vec<float, V> t =
                        *reinterpret_cast<const Vec<float, V>*>(co + p.block_tokens * half);
                    float v[2 * V], w[2 * V];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        v[e] = to_f(x[n].e[e]);
                        v[V + e] = to_f(y[n].e[e]);
                    }
                    const auto turn = [&](int ia, int ib, int e) {
                        w[ia] = v[ia] * c.e[e] - v[ib] * t.e[e];
                        w[ib] = v[ia] * t.e[e] + v[ib] * c.e[e];
                    };
                    if (p.interleaved) {
#pragma unroll
                        for (int e = 0; e < V; ++e) turn(2 * e, 2 * e + 1, e);
                    } else {
#pragma unroll
                        for (int e = 0; e < V; ++e) turn(e, V + e, e);
                    }
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        x[n].e[e] = from_f<E>(w[e]);
                        y[n].e[e] = from_f<E>(w[V + e]);
                    }
                }
                if (put[n]) {
                    *reinterpret_cast<X*>(to[n] + at) = x[n];
                    if (second < p.D) *reinterpret_cast<X*>(to[n] + bt) = y[n];
                }
            }
        }
    }
}

template <typename E, int V>
cudaError_t launch(RotaryParams p, int sms, cudaStream_t s) {
    const int heads = p.H + p.Hk;
    p.units = p.R / (2 * V) + (p.copy_q || p.copy_k ? (p.D - p.R + 2 * V - 1) / (2 * V) : 0);
    if (p.units == 0) return cudaSuccess;
    // All units of as many heads as make 256 threads; the heads in equal
    // rounds, shared between blocks and with fewer tokens to a block while
    // that is what it takes to give every SM four blocks.
    const int bx = std::min(p.units, 256), slots = std::max(1, 256 / bx);
    p.rounds = (heads + slots - 1) / slots;
    const int by = (heads + p.rounds - 1) / p.rounds;
    p.block_tokens = kMaxTokens;
    while (p.block_tokens > 1 && p.block_tokens * p.R * sizeof(float) > 48 * 1024) p.block_tokens /= 2;
    p.head_blocks = 1;
    while (p.block_tokens > 1 && (p.tokens + p.block_tokens - 1) / p.block_tokens < 4 * sms)
        p.block_tokens /= 2;
    while (p.rounds > 1 && p.tokens * p.head_blocks < 4 * sms) {
        p.rounds = (p.rounds + 1) / 2;
        p.head_blocks = (heads + by * p.rounds - 1) / (by * p.rounds);
    }
    const int64_t blocks = (p.tokens + p.block_tokens - 1) / p.block_tokens * p.head_blocks;
    if (blocks >= int64_t(1) << 31) return cudaErrorInvalidConfiguration;
    note_launches(1);
    return launch_kernel(rotary_kernel<E, V>, dim3(static_cast<unsigned>(blocks)), dim3(bx, by),
                         static_cast<size_t>(p.block_tokens) * (p.R / 2) * 2 * sizeof(float), s, p);
}

// 16-byte vectors need every address of a unit on a 16-byte boundary
// (the strides of dimensions of one element do not count).
bool vectors(const RotaryParams& p, int64_t B, int es) {
    const int v = 16 / es;
    if (p.R % (2 * v) || p.D % v) return false;
    const Arr* all[4] = {&p.q, &p.qo, &p.k, &p.ko};
    for (int i = 0; i < 4; ++i) {
        const Arr& a = *all[i];
        const int heads = i < 2 ? p.H : p.Hk;
        if (heads == 0) continue;
        if (reinterpret_cast<uintptr_t>(a.p) % 16 || (B > 1 && a.sb % v) || (p.M > 1 && a.sr % v) ||
            (heads > 1 && a.sh % v))
            return false;
    }
    return true;
}

}  // namespace
}  // namespace gs

extern "C" gs_status gauss_sum_rotary(const gs_rotary* a, void* stream) {
    using namespace gs;
    pdl_reset();
    const auto invalid = [](const char* msg) { return set_last_error(GS_ERR_INVALID_ARGUMENT, msg); };
    if (!a) return invalid("null arguments");
    if (a->dtype != GS_FP32 && a->dtype != GS_FP16 && a->dtype != GS_BF16) return invalid("unknown dtype");
    const bool with_k = a->k.data != nullptr || a->k_out.data != nullptr;
    if (a->B < 0 || a->M < 0 || a->H < 0 || a->D < 0 || (with_k && a->Hk < 0)) return invalid("negative size");
    if (a->R < 0 || a->R > a->D || a->R % 2) return invalid("R must be even and in 0 .. D");
    if (!std::isfinite(a->scale) || !std::isfinite(static_cast<float>(a->scale)))
        return invalid("scale must be finite");
    if ((a->interleaved & ~int64_t(1)) || (a->transpose & ~int64_t(1)) || (a->positions_64 & ~int64_t(1)))
        return invalid("interleaved, transpose and positions_64 must be 0 or 1");
    if (a->R > kMaxRotated) return set_last_error(GS_ERR_UNSUPPORTED, "R must be at most 4096");
    constexpr int64_t kMax = (int64_t(1) << 30) - 1;
    const int64_t Hk = with_k ? a->Hk : 0;
    if (a->B > kMax || a->M > kMax || a->H > kMax || Hk > kMax || a->D > kMax)
        return set_last_error(GS_ERR_UNSUPPORTED, "sizes must be below 2^30");
    const int es = a->dtype == GS_FP32 ? 4 : 2;
    const char* why = nullptr;
    if (a->H > 0) why = check_array(a->q, es, a->B, a->M, a->H, a->D, false);
    if (!why && a->H > 0) why = check_array(a->q_out, es, a->B, a->M, a->H, a->D, true);
    if (!why && with_k) why = check_array(a->k, es, a->B, a->M, Hk, a->D, false);
    if (!why && with_k) why = check_array(a->k_out, es, a->B, a->M, Hk, a->D, true);
    const auto shifted = [](const gs_array& x, const gs_array& y) {
        return x.data && x.data == y.data &&
               (x.stride_b != y.stride_b || x.stride_row != y.stride_row || x.stride_head != y.stride_head);
    };
    if (!why && (shifted(a->q, a->q_out) || (with_k && shifted(a->k, a->k_out))))
        why = "an in-place output must have its input's strides";
    if (why) return invalid(why);
    if (a->B == 0 || a->M == 0 || a->D == 0 || a->H + Hk == 0) return GS_OK;
    if (a->R > 0) {
        if (!a->positions || !a->frequencies) return invalid("null positions or frequencies");
        if (reinterpret_cast<uintptr_t>(a->positions) % (a->positions_64 ? 8 : 4) ||
            reinterpret_cast<uintptr_t>(a->frequencies) % 8)
            return invalid("positions and frequencies must be aligned to their element");
        if (a->stride_pos_b < 0 || a->stride_pos_m < 0) return invalid("strides must be >= 0");
    }
    DeviceContext dc;
    const gs_status st = device_context(&dc);
    if (st != GS_OK) return st;
    RotaryParams p{};
    p.M = a->M;
    p.tokens = a->B * a->M;
    p.H = static_cast<int>(a->H);
    p.Hk = static_cast<int>(Hk);
    p.D = static_cast<int>(a->D);
    p.R = static_cast<int>(a->R);
    p.scale = static_cast<float>(a->scale);
    p.interleaved = a->interleaved != 0;
    p.transpose = a->transpose != 0;
    p.pos64 = a->positions_64 != 0;
    p.pos = a->positions;
    p.pos_b = a->stride_pos_b;
    p.pos_m = a->stride_pos_m;
    p.freq = a->frequencies;
    p.q = make_arr(a->q);
    p.k = make_arr(a->k);
    p.qo = make_arr(a->q_out);
    p.ko = make_arr(a->k_out);
    p.copy_q = p.R < p.D && p.H > 0 && p.q.p != p.qo.p;
    p.copy_k = p.R < p.D && p.Hk > 0 && p.k.p != p.ko.p;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool vec = vectors(p, a->B, es);
    cudaError_t e;
    if (a->dtype == GS_FP32)
        e = vec ? launch<float, 4>(p, dc.sms, s) : launch<float, 1>(p, dc.sms, s);
    else if (a->dtype == GS_FP16)
        e = vec ? launch<__half, 8>(p, dc.sms, s) : launch<__half, 1>(p, dc.sms, s);
    else
        e = vec ? launch<__nv_bfloat16, 8>(p, dc.sms, s)
                : launch<__nv_bfloat16, 1>(p, dc.sms, s);
    return cuda_status(e, "rotary kernel");
}
