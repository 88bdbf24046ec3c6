// Entry points of include/gauss_sum/attention.h: argument checks, workspace
// and the choice of kernels.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "attention.h"

namespace gs {

const char* check_array(const gs_array& a, int64_t es, int64_t B, int64_t rows, int64_t heads,
                        int64_t width, bool output) {
    if (B == 0 || rows == 0 || heads == 0 || width == 0) return nullptr;
    if (!a.data) return "null array pointer";
    if (reinterpret_cast<uintptr_t>(a.data) % static_cast<uintptr_t>(es))
        return "array pointers must be aligned to their element";
    if (a.stride_b < 0 || a.stride_row < 0 || a.stride_head < 0) return "strides must be >= 0";
    // Offsets stay far inside 64 bits.
    constexpr int64_t kMaxExtent = int64_t(1) << 60;
    const int64_t n[3] = {B, rows, heads}, st[3] = {a.stride_b, a.stride_row, a.stride_head};
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && st[i] > kMaxExtent / n[i]) return "array extent overflows 2^60 elements";
    if (!output) return nullptr;
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int x, int y) { return st[x] < st[y]; });
    int64_t extent = width;
    for (int i = 0; i < 3; ++i) {
        const int d = order[i];
        if (n[d] <= 1) continue;
        if (st[d] < extent) return "output arrays must not overlap themselves";
        extent += st[d] * (n[d] - 1);
    }
    return nullptr;
}

}  // namespace gs

namespace {

using namespace gs;

gs_status invalid(const char* msg) { return set_last_error(GS_ERR_INVALID_ARGUMENT, msg); }
gs_status unsupported(const char* msg) { return set_last_error(GS_ERR_UNSUPPORTED, msg); }

bool known_dtype(int64_t t) { return t == GS_FP32 || t == GS_FP16 || t == GS_BF16; }
InType in_type(int64_t t) {
    return t == GS_FP16 ? InType::F16 : t == GS_BF16 ? InType::BF16 : InType::F32;
}
int64_t elem_size(int64_t t) { return t == GS_FP32 ? 4 : 2; }

// Checks shared by both attention entry points; fills *p.
gs_status check(const gs_attention* a, AttnParams* p) {
    if (!a) return invalid("null arguments");
    if (!known_dtype(a->dtype)) return invalid("unknown dtype");
    if (a->B < 0 || a->M < 0 || a->N < 0 || a->H < 0) return invalid("negative size");
    if (a->Hk < 1 || a->H % a->Hk) return invalid("H must be a multiple of Hk >= 1");
    if (a->D < 1 || a->C < 1) return invalid("D and C must be >= 1");
    if (!(std::isfinite(a->tau) && a->tau > 0.0)) return invalid("tau must be finite and > 0");
    if (a->causal != 0 && a->causal != 1) return invalid("causal must be 0 or 1");
    if (a->D > 256 || a->C > 256) return unsupported("attention takes D, C <= 256");
    constexpr int64_t kMax = (int64_t(1) << 31) - 1;
    if (a->B > kMax || a->H > kMax || a->N > kMax - 256 || a->M > kMax - 256)
        return unsupported("B, H, M and N must be below 2^31");
    const int64_t G = a->H / a->Hk;
    if (a->M > 0 && G > (kMax - 256) / a->M) return unsupported("M x H / Hk must be below 2^31");
    if (a->H > kMax / std::max<int64_t>(1, a->B)) return unsupported("B x H must be below 2^31");
    const float tau = static_cast<float>(a->tau);
    const float c = static_cast<float>(a->tau * 1.4426950408889634);
    if (!(std::isfinite(c) && tau > 0.f)) return invalid("tau is outside the float32 range");
    if (reinterpret_cast<uintptr_t>(a->q_lengths) & 3u || reinterpret_cast<uintptr_t>(a->k_lengths) & 3u)
        return invalid("lengths must be aligned to their element");
    if (reinterpret_cast<uintptr_t>(a->lse) & 3u) return invalid("lse must be aligned to its element");
    const int64_t es = elem_size(a->dtype);
    const char* why = check_array(a->q, es, a->B, a->M, a->H, a->D, false);
    if (!why) why = check_array(a->k, es, a->B, a->N, a->Hk, a->D, false);
    if (!why) why = check_array(a->v, es, a->B, a->N, a->Hk, a->C, false);
    if (why) return invalid(why);
    *p = AttnParams{};
    p->B = static_cast<int>(a->B);
    p->M = static_cast<int>(a->M);
    p->N = static_cast<int>(a->N);
    p->H = static_cast<int>(a->H);
    p->Hk = static_cast<int>(a->Hk);
    p->G = static_cast<int>(G);
    p->D = static_cast<int>(a->D);
    p->C = static_cast<int>(a->C);
    p->R = a->M * G;
    p->c = c;
    p->tau = tau;
    p->causal = a->causal != 0;
    p->q_len = a->q_lengths;
    p->k_len = a->k_lengths;
    p->q = make_arr(a->q);
    p->k = make_arr(a->k);
    p->v = make_arr(a->v);
    p->out = make_arr(a->out);
    p->lse = a->lse;
    p->splits = 1;
    return GS_OK;
}

// A grid of `tiles` blocks per (problem, key head) must stay below 2^31.
bool grid_fits(int64_t tiles, const AttnParams& p, int64_t splits) {
    return tiles <= ((int64_t(1) << 31) - 1) / splits / (static_cast<int64_t>(p.B) * p.Hk);
}

// Whether every row of the arrays starts on the boundary of four elements.
bool four_aligned(std::initializer_list<const Arr*> arrays, const AttnParams& p, int64_t es) {
    for (const Arr* a : arrays)
        if (reinterpret_cast<uintptr_t>(a->p) % (4 * es) || (p.B > 1 && a->sb % 4) || a->sr % 4 ||
            (p.H > 1 && a->sh % 4))
            return false;
    return true;
}

// Key splits of the fp32-pipe kernel: at least four tiles a split, until
// every SM has two blocks.
int simt_splits(int64_t blocks, int64_t key_tiles, int sms) {
    if (blocks >= 2 * sms) return 1;
    return static_cast<int>(
        std::max<int64_t>(1, std::min<int64_t>(key_tiles / 4, 2 * sms / blocks)));
}

// Key splits of the tensor-core kernel (`slots` blocks at a time): the number
// with the fewest tile times over all waves, a block's start and end counted as
// four tiles, and as four more the joining launch that splits of packed rows
// bring with them (one token, 8 heads x 64, GPU us without / with that launch's
// share: 333 keys 10.9 / 9.8, 1000 keys 10.9 / 11.1 and one launch less for the
// host; 8 x 600 keys of 8 heads x 128 15.8 / 13.5; with eight tiles instead of
// four 1000 keys take 12.7).
int tensor_splits(int64_t blocks, int64_t key_tiles, int slots, bool packed) {
    if (blocks >= 8 * slots) return 1;   // the last wave is a small part of the whole
    int best = 1;
    int64_t least = INT64_MAX, most = std::min<int64_t>(64, (key_tiles + 1) / 2);
    if (!packed) most = std::min<int64_t>(most, std::max<int64_t>(1, slots / blocks));
    for (int64_t s = 1; s <= most; ++s) {
        const int64_t cost = (blocks * s + slots - 1) / slots * ((key_tiles + s - 1) / s + 4) +
                             (packed && s > 1 ? 4 : 0);
        if (cost < least) {
            least = cost;
            best = static_cast<int>(s);
        }
    }
    return best;
}

// Stream-ordered workspace of one call.
struct Workspace {
    void* ptr = nullptr;
    cudaStream_t s;
    explicit Workspace(cudaStream_t stream) : s(stream) {}
    gs_status alloc(size_t bytes) { return workspace_alloc(&ptr, bytes, s); }
    // Frees on the stream; the status of the call is `st` unless that fails.
    gs_status done(gs_status st) {
        if (!ptr) return st;
        const cudaError_t e = cudaFreeAsync(ptr, s);
        ptr = nullptr;
        return st != GS_OK ? st : cuda_status(e, "workspace free");
    }
};

}  // namespace

extern "C" {

gs_status gauss_sum_attention(const gs_attention* a, void* stream) {
    pdl_reset();
    AttnParams p;
    gs_status st = check(a, &p);
    if (st != GS_OK) return st;
    const char* why = check_array(a->out, elem_size(a->dtype), a->B, a->M, a->H, a->C, true);
    if (why) return invalid(why);
    if (p.B == 0 || p.R == 0) return GS_OK;
    DeviceContext dc;
    st = device_context(&dc);
    if (st != GS_OK) return st;
    p.status = dc.status;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const InType t = in_type(a->dtype);

    const bool tc = t != InType::F32 && dc.sm103 && p.N > 0 &&
                    attn_tc_takes(p.q, p.B, p.M, p.H, p.D) && attn_tc_takes(p.k, p.B, p.N, p.Hk, p.D) &&
                    attn_tc_takes(p.v, p.B, p.N, p.Hk, p.C) && attn_tc_takes(p.out, p.B, p.M, p.H, p.C);
    // Fewer tokens than a tile: the heads that share keys fill it together.
    const bool packed = tc && p.M < 128;
    const int64_t rows = !tc || packed ? p.R : p.M, heads = !tc || packed ? p.Hk : p.H;
    const int64_t tile_r = !tc ? kSimtAttnRows : packed || attn_tc_narrow(p) ? 128 : 256;
    const bool narrow = tc && !packed && attn_tc_narrow(p);
    const int64_t tile_n = !tc ? kSimtAttnKeys : narrow ? 64 : 128;
    const int64_t row_tiles = (rows + tile_r - 1) / tile_r;
    const int64_t key_tiles = (static_cast<int64_t>(p.N) + tile_n - 1) / tile_n;
    if (row_tiles > ((int64_t(1) << 31) - 1) / (p.B * heads))
        return unsupported("too many row tiles for one launch");
    const int64_t blocks = row_tiles * p.B * heads;
    const int slots = narrow ? 2 * dc.sms : dc.sms;
    p.splits = tc ? tensor_splits(blocks, key_tiles, slots, packed) : simt_splits(blocks, key_tiles, dc.sms);
    p.vec = four_aligned({&p.q, &p.k, &p.v}, p, elem_size(a->dtype));
    Workspace ws(s);
    if (p.splits > 1) {
        const size_t all = static_cast<size_t>(p.splits) * p.B * p.Hk * p.R;
        st = ws.alloc(all * (p.C + 1) * sizeof(float));
        if (st != GS_OK) return st;
        p.part_o = static_cast<float*>(ws.ptr);
        p.part_l = p.part_o + all * p.C;
    }
    st = cuda_status(tc ? launch_attn_tc_fwd(p, t, packed, s) : launch_attn_simt_fwd(p, t, s),
                     "attention kernel");
    if (st == GS_OK && p.splits > 1) st = cuda_status(launch_attn_join(p, t, s), "attention join kernel");
    return ws.done(st);
}

gs_status gauss_sum_attention_vjp(const gs_attention* a, const gs_attention_grad* d, void* stream) {
    pdl_reset();
    AttnParams p;
    gs_status st = check(a, &p);
    if (st != GS_OK) return st;
    if (!d) return invalid("null arguments");
    const int64_t es = elem_size(a->dtype);
    const char* why = check_array(a->out, es, a->B, a->M, a->H, a->C, false);
    if (!why) why = check_array(d->g, es, a->B, a->M, a->H, a->C, false);
    if (!why && d->grad_q.data) why = check_array(d->grad_q, es, a->B, a->M, a->H, a->D, true);
    if (!why && d->grad_k.data) why = check_array(d->grad_k, es, a->B, a->N, a->Hk, a->D, true);
    if (!why && d->grad_v.data) why = check_array(d->grad_v, es, a->B, a->N, a->Hk, a->C, true);
    if (!why && reinterpret_cast<uintptr_t>(d->g_lse) & 3u)
        why = "g_lse must be aligned to its element";
    if (!why && !a->lse && a->B > 0 && p.R > 0) why = "null lse pointer";
    if (why) return invalid(why);
    if (p.B == 0 || !(d->grad_q.data || d->grad_k.data || d->grad_v.data)) return GS_OK;
    if (p.R == 0 && p.N == 0) return GS_OK;
    p.g = make_arr(d->g);
    p.g_lse = d->g_lse;
    p.dq = make_arr(d->grad_q);
    p.dk = make_arr(d->grad_k);
    p.dv = make_arr(d->grad_v);
    if (p.R == 0) p.dq.p = nullptr;
    DeviceContext dc;
    st = device_context(&dc);
    if (st != GS_OK) return st;
    p.status = dc.status;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const InType t = in_type(a->dtype);
    if (!grid_fits((p.R + kSimtAttnRows - 1) / kSimtAttnRows, p, 1) ||
        !grid_fits((static_cast<int64_t>(p.N) + kSimtAttnKeys - 1) / kSimtAttnKeys, p, 1) ||
        !grid_fits((static_cast<int64_t>(p.G) * p.M + 7) / 8, p, 1))
        return unsupported("too many tiles for one launch");

    Workspace ws(s);
    const auto takes = [&](const Arr& x, int64_t rows, int heads, int width) {
        return !x.p || attn_tc_takes(x, p.B, rows, heads, width);
    };
    if (t != InType::F32 && dc.sm103 && p.R > 0 && p.N > 0 && takes(p.q, p.M, p.H, p.D) &&
        takes(p.k, p.N, p.Hk, p.D) && takes(p.v, p.N, p.Hk, p.C) && takes(p.out, p.M, p.H, p.C) &&
        takes(p.g, p.M, p.H, p.C) && takes(p.dq, p.M, p.H, p.D) && takes(p.dk, p.N, p.Hk, p.D) &&
        takes(p.dv, p.N, p.Hk, p.C)) {
        st = ws.alloc(attn_tc_vjp_workspace(p, t));
        if (st != GS_OK) return st;
        return ws.done(cuda_status(launch_attn_tc_vjp(p, t, ws.ptr, s), "attention gradient kernels"));
    }
    // Few tiles: share each out until every SM has two blocks, at least two
    // tiles to a block.
    const int64_t heads = static_cast<int64_t>(p.B) * p.Hk;
    const int64_t tiles_r = (p.R + kSimtAttnRows - 1) / kSimtAttnRows;
    const int64_t tiles_n = (static_cast<int64_t>(p.N) + kSimtAttnKeys - 1) / kSimtAttnKeys;
    const int64_t blocks = std::max<int64_t>(1, heads * (tiles_r + tiles_n));
    const int64_t share = std::min<int64_t>(8, 2 * dc.sms / blocks);
    p.splits = static_cast<int>(std::max<int64_t>(1, std::min(share, tiles_n / 2)));
    p.row_splits = static_cast<int>(std::max<int64_t>(1, std::min(share, tiles_r / 2)));
    const size_t rows = static_cast<size_t>(p.B) * p.H * p.M;
    const size_t nq = p.splits > 1 && p.dq.p ? rows * p.D * p.splits : 0;
    const size_t keys = p.row_splits > 1 ? static_cast<size_t>(heads) * p.N * p.row_splits : 0;
    const size_t nk = p.dk.p ? keys * p.D : 0, nv = p.dv.p ? keys * p.C : 0;
    if (p.R > 0) {
        st = ws.alloc((rows + nq + nk + nv) * sizeof(float));
        if (st != GS_OK) return st;
        p.delta = static_cast<float*>(ws.ptr);
        p.part_dq = p.delta + rows;
        p.part_dk = p.part_dq + nq;
        p.part_dv = p.part_dk + nk;
        st = cuda_status(launch_attn_delta(p, t, s), "attention row-term kernel");
    }
    p.vec = four_aligned({&p.q, &p.k, &p.v, &p.g}, p, es);
    if (st == GS_OK) st = cuda_status(launch_attn_simt_vjp(p, t, s), "attention gradient kernel");
    return ws.done(st);
}

}  // extern "C"
