// Rotary positions of queries and keys (include/gauss_sum/attention.h).
//
// A pair turns by angle = position x frequency.  Frequencies are 64-bit
// fractions of a turn, so the product modulo 2^64 is the exact angle modulo
// one turn for any position: its top 32 bits, as a signed fraction of half a
// turn, go to sincospif.  One thread computes the cosines and sines of eight
// (fp32: four) neighbouring pairs of a token and applies them to that
// token's heads in turn, two 16-byte loads and two 16-byte stores a head, so
// the kernel is bound by the reading and writing of the arrays.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "attention.h"
#include "ptx.cuh"

namespace gs {
namespace {

struct RotaryParams {
    int64_t M;
    int H, Hk, D, R;
    float scale;
    int interleaved, transpose, pos64;
    const void* pos;
    int64_t pos_b, pos_m;
    const int64_t* freq;
    Arr q, k, qo, ko;
    int copy_q, copy_k;      // channels R .. D - 1 are copied (out of place)
    int units;               // per token: R / (2 V) turned units, then copied ones
    int groups, per_group;   // heads (queries, then keys) are shared out over `groups` threads
    int64_t total;           // threads
};

template <typename E>
__device__ __forceinline__ float to_float(E x);
template <>
__device__ __forceinline__ float to_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_float<__half>(__half x) { return __half2float(x); }
template <>
__device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename E>
__device__ __forceinline__ E from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

template <typename E, int V>
struct alignas(sizeof(E) * V) Vec {
    E e[V];
};

// V pairs a thread: channels [a, a + V) and [b, b + V) of every head of its
// group; half layout a = V u, b = a + R / 2, interleaved a = 2 V u, b = a + V.
// Units past the turned ones copy the 2 V channels from R on.  V = 1 takes
// any stride and alignment.
template <typename E, int V>
__global__ void __launch_bounds__(256) rotary_kernel(const RotaryParams p) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= p.total) return;
    const int u = static_cast<int>(i % p.units);
    int64_t rest = i / p.units;
    const int grp = static_cast<int>(rest % p.groups);
    rest /= p.groups;
    const int64_t m = rest % p.M, b = rest / p.M;
    const int turned = p.R / (2 * V);
    const bool copy = u >= turned;

    int at, bt;
    float co[V], si[V];
    if (copy) {
        at = p.R + (u - turned) * 2 * V;
        bt = at + V;
    } else {
        at = p.interleaved ? 2 * V * u : V * u;
        bt = p.interleaved ? at + V : at + p.R / 2;
        const int64_t at_pos = b * p.pos_b + m * p.pos_m;
        const int64_t pos = p.pos64 ? static_cast<const int64_t*>(p.pos)[at_pos]
                                    : static_cast<const int*>(p.pos)[at_pos];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const uint64_t turn = static_cast<uint64_t>(pos) * static_cast<uint64_t>(p.freq[V * u + e]);
            // Top half as a signed fraction of 2^32; sincospif takes half turns.
            const float half = static_cast<float>(static_cast<int>(turn >> 32)) * 0x1p-31f;
            sincospif(half, &si[e], &co[e]);
            co[e] *= p.scale;
            si[e] *= p.transpose ? -p.scale : p.scale;
        }
    }

    const int h0 = grp * p.per_group, h1 = min(h0 + p.per_group, p.H + p.Hk);
#pragma unroll 4
    for (int h = h0; h < h1; ++h) {
        const bool is_q = h < p.H;
        if (copy && !(is_q ? p.copy_q : p.copy_k)) continue;
        const Arr& in = is_q ? p.q : p.k;
        const Arr& out = is_q ? p.qo : p.ko;
        const int hh = is_q ? h : h - p.H;
        const E* src = reinterpret_cast<const E*>(in.p) + b * in.sb + m * in.sr + hh * in.sh;
        E* dst = reinterpret_cast<E*>(out.p) + b * out.sb + m * out.sr + hh * out.sh;
        using X = Vec<E, V>;
        const bool two = bt < p.D;   // a copied unit may end in a single half
        X x = *reinterpret_cast<const X*>(src + at), y = x;
        if (two) y = *reinterpret_cast<const X*>(src + bt);
        if (!copy) {
            float v[2 * V], w[2 * V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                v[e] = to_float(x.e[e]);
                v[V + e] = to_float(y.e[e]);
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int ia = p.interleaved ? 2 * e : e, ib = p.interleaved ? 2 * e + 1 : V + e;
                w[ia] = v[ia] * co[e] - v[ib] * si[e];
                w[ib] = v[ia] * si[e] + v[ib] * co[e];
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x.e[e] = from_float<E>(w[e]);
                y.e[e] = from_float<E>(w[V + e]);
            }
        }
        *reinterpret_cast<X*>(dst + at) = x;
        if (two) *reinterpret_cast<X*>(dst + bt) = y;
    }
}

template <typename E, int V>
cudaError_t launch(RotaryParams p, int64_t B, int sms, cudaStream_t s) {
    const int heads = p.H + p.Hk;
    p.units = p.R / (2 * V) + (p.copy_q || p.copy_k ? (p.D - p.R + 2 * V - 1) / (2 * V) : 0);
    if (p.units == 0) return cudaSuccess;
    // Threads take as many heads as keeps 2048 threads on every SM, up to
    // eight, so that the sines are shared.
    const int64_t one = B * p.M * p.units;
    const int64_t want = int64_t(2048) * sms;
    p.per_group = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(8, one * heads / want)));
    p.groups = (heads + p.per_group - 1) / p.per_group;
    p.total = one * p.groups;
    const int64_t blocks = (p.total + 255) / 256;
    if (blocks >= int64_t(1) << 31) return cudaErrorInvalidConfiguration;
    note_launches(1);
    return launch_kernel(rotary_kernel<E, V>, dim3(static_cast<unsigned>(blocks)), 256, 0, s, p);
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
        e = vec ? launch<float, 4>(p, a->B, dc.sms, s) : launch<float, 1>(p, a->B, dc.sms, s);
    else if (a->dtype == GS_FP16)
        e = vec ? launch<__half, 8>(p, a->B, dc.sms, s) : launch<__half, 1>(p, a->B, dc.sms, s);
    else
        e = vec ? launch<__nv_bfloat16, 8>(p, a->B, dc.sms, s)
                : launch<__nv_bfloat16, 1>(p, a->B, dc.sms, s);
    return cuda_status(e, "rotary kernel");
}
