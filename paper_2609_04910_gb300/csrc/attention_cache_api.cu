// Entry points of include/gauss_sum/attention_cache.h: argument checks,
// workspace and the choice of kernels.
#include <algorithm>
#include <cmath>

#include "attention_cache.h"

namespace {

using namespace gs;

gs_status invalid(const char* msg) { return set_last_error(GS_ERR_INVALID_ARGUMENT, msg); }
gs_status unsupported(const char* msg) { return set_last_error(GS_ERR_UNSUPPORTED, msg); }

bool known_dtype(int64_t t) { return t == GS_FP32 || t == GS_FP16 || t == GS_BF16; }
InType in_type(int64_t t) {
    return t == GS_FP16 ? InType::F16 : t == GS_BF16 ? InType::BF16 : InType::F32;
}
int64_t elem_size(int64_t t) { return t == GS_FP32 ? 4 : 2; }

constexpr int64_t kMax = (int64_t(1) << 31) - 1 - 256;

// Checks the cache for a call of B problems; fills *p.
gs_status check_cache(const gs_cache* c, int64_t B, bool written, CacheParams* p) {
    if (!c) return invalid("null arguments");
    if (c->pages < 0 || c->heads < 0) return invalid("negative size");
    if (c->D < 1 || c->C < 1) return invalid("D and C must be >= 1");
    if (c->tokens < 1 || c->tokens % GS_CACHE_BLOCK_TOKENS)
        return invalid("the tokens of a page must be a multiple of 16, at least 16");
    if (c->page_table && (c->table_pages < 0 || c->stride_table < 0)) return invalid("negative size");
    if (c->D > 256 || c->C > 256) return unsupported("the cache takes D, C <= 256");
    if (c->heads > 65535) return unsupported("the cache takes at most 65535 heads");
    if (c->pages > kMax || c->tokens > kMax) return unsupported("pages and tokens must be below 2^31");
    const int64_t per = c->page_table ? c->table_pages : 1;
    if (per > kMax / c->tokens) return unsupported("the tokens of a problem must be below 2^31");
    if (!c->page_table && c->pages < B) return invalid("without a page table every problem needs a page");
    if (reinterpret_cast<uintptr_t>(c->page_table) & 3u)
        return invalid("the page table must be aligned to its element");
    constexpr int64_t kMaxExtent = int64_t(1) << 60;
    if (c->page_table && B > 1 && c->stride_table > kMaxExtent / B)
        return invalid("page table extent overflows 2^60 elements");
    p->block_bytes = static_cast<int>(GS_CACHE_BLOCK_BYTES(c->D, c->C));
    // (Strides of dimensions of one element are not used.)
    p->sp = c->pages > 1 ? c->stride_page : 0;
    p->sh = c->heads > 1 ? c->stride_head : 0;
    if (c->pages > 0 && c->heads > 0 && B > 0) {
        if (!c->data) return invalid("null cache pointer");
        if (reinterpret_cast<uintptr_t>(c->data) % 16 || p->sp % 16 || p->sh % 16)
            return invalid("the cache and its strides must be multiples of 16 bytes");
        if (p->sp < 0 || p->sh < 0) return invalid("strides must be >= 0");
        if (p->sp > kMaxExtent / c->pages || p->sh > kMaxExtent / c->heads)
            return invalid("cache extent overflows 2^60 bytes");
        const int64_t inner = c->tokens / GS_CACHE_BLOCK_TOKENS * p->block_bytes;
        if (written) {
            // Along dimensions longer than one, ordered by stride, each stride
            // must span the extent of the ones below.
            const int64_t n[2] = {c->pages, c->heads}, st[2] = {p->sp, p->sh};
            const int low = st[0] < st[1] ? 0 : 1;
            int64_t extent = inner;
            for (int i = 0; i < 2; ++i) {
                const int d = i == 0 ? low : 1 - low;
                if (n[d] <= 1) continue;
                if (st[d] < extent) return invalid("a cache that is written must not overlap itself");
                extent += st[d] * (n[d] - 1);
            }
        }
    }
    p->data = static_cast<char*>(c->data);
    p->pages = static_cast<int>(c->pages);
    p->tokens = static_cast<int>(c->tokens);
    p->shift = -1;
    for (int i = 0; i < 31; ++i)
        if (c->tokens == int64_t(1) << i) p->shift = i;
    p->heads = static_cast<int>(c->heads);
    p->D = static_cast<int>(c->D);
    p->C = static_cast<int>(c->C);
    p->kw = (p->D + 31) / 32;
    p->vw = (p->C + 31) / 32;
    p->kg = (p->D + 63) / 64;
    p->vg = (p->C + 63) / 64;
    p->table = c->page_table;
    p->stride_table = c->stride_table;
    p->N = c->tokens * per;
    return GS_OK;
}

gs_status check_lengths(const int32_t* q, const int32_t* k) {
    if (reinterpret_cast<uintptr_t>(q) & 3u || reinterpret_cast<uintptr_t>(k) & 3u)
        return invalid("lengths must be aligned to their element");
    return GS_OK;
}

// Checks shared by both calls on rows; fills *p.
gs_status check_rows(const gs_cache* c, const gs_cache_rows* r, bool write, CacheRows* p) {
    if (!c || !r) return invalid("null arguments");
    if (!known_dtype(r->dtype)) return invalid("unknown dtype");
    if (r->B < 0 || r->M < 0) return invalid("negative size");
    if (r->B > kMax || r->M > kMax) return unsupported("B and M must be below 2^31");
    *p = CacheRows{};
    gs_status st = check_cache(c, r->B, write, &p->c);
    if (st == GS_OK) st = check_lengths(r->q_lengths, r->k_lengths);
    if (st != GS_OK) return st;
    const int64_t es = elem_size(r->dtype);
    const char* why = nullptr;
    if (write || r->k.data) why = check_array(r->k, es, r->B, r->M, c->heads, c->D, !write);
    if (!why && (write || r->v.data)) why = check_array(r->v, es, r->B, r->M, c->heads, c->C, !write);
    if (why) return invalid(why);
    p->B = static_cast<int>(r->B);
    p->M = static_cast<int>(r->M);
    p->q_len = r->q_lengths;
    p->k_len = r->k_lengths;
    p->k = make_arr(r->k);
    p->v = make_arr(r->v);
    p->heads = p->c.heads;
    return GS_OK;
}

// Whether every row of q or out starts on the boundary of n elements.
bool aligned_rows(const Arr& a, const AttnParams& p, int64_t n, int64_t es) {
    return reinterpret_cast<uintptr_t>(a.p) % (n * es) == 0 && (p.B == 1 || a.sb % n == 0) &&
           (p.M == 1 || a.sr % n == 0) && (p.H == 1 || a.sh % n == 0);
}

// Stream-ordered workspace of one call.
struct Workspace {
    void* ptr = nullptr;
    cudaStream_t s;
    explicit Workspace(cudaStream_t stream) : s(stream) {}
    gs_status alloc(size_t bytes) { return workspace_alloc(&ptr, bytes, s); }
    gs_status done(gs_status st) {
        if (!ptr) return st;
        const cudaError_t e = cudaFreeAsync(ptr, s);
        ptr = nullptr;
        return st != GS_OK ? st : cuda_status(e, "workspace free");
    }
};

// Largest rows (M x G) of 16-bit calls for the kernel of few rows, and for the kernel that fills tiles
// from the cache; more rows have the cache's rows read back first.  us (here and below of calls replayed
// from a graph), 8192 tokens, 8 key heads x 128:
//   16 problems, 16 rows: few 63, tiles 75; 24 rows: few 104, tiles 75
//   16 problems, 256 rows: tiles 175, read back 310; 1 problem, 512 rows: 47 and 60
//   2 problems, 4096 rows: 433 and 222
// float32 queries always take the kernel of few rows, tile by tile (4 problems, 512 rows of 64
// channels: 395; read back, on the fp32 pipe, some 1300).
constexpr int64_t kFewRows = 16, kManyRows = 512;

// Rows read back are keys rounded to 11 bits, which moves a score by some 2e-4 and the log-sum-exp of n keys
// by 5e-4 / sqrt(n); the other kernels have exact keys.  Caches with room for so many tokens, all of whose
// rows see few keys, are never read back.  (The first rows of longer prompts see few keys too.  Taking their
// tiles once more with exact keys cost 20 to 70 us of 80 for 8 x 512 tokens, their lse alone by fp32
// products 8 to 30.)
constexpr int64_t kExactTokens = 256;

// Nor are they for calls whose tiles fit the card at once, up to kSmallTokens (one sequence of 32/8 heads x 128,
// us: 512 queries on 512 keys, tiles 19, read back 37; 512 on 2048 33 and 48, on 8192 88 and 90; 2 x 300 on 300
// of 8/4 heads x 64 13 and 23; not at once: 8 x 512 on 512 113 and 78).
constexpr int64_t kSmallTokens = 8192;
bool tiles_fit(const AttnParams& p, int sms) {
    return p.N <= kSmallTokens && (p.R + kCacheManyRows - 1) / kCacheManyRows * p.B * p.Hk <= sms;
}

// On caches with so little room the kernel of few rows is the faster one as long as its sets of 16 rows fit
// the card at once, two blocks to an SM (32/8 heads x 128, 256 tokens, us: 1 x 64 queries, 128 sets, few 13.0,
// tiles 15.8; 1 x 256, 512 sets, 25.6 and 15.9; 8 x 64, 1024 sets, 52.7 and 16.4).
bool few_short(const AttnParams& p, int sms) {
    return p.N <= kExactTokens && (p.R + 15) / 16 * p.B * p.Hk <= 2 * sms;
}

AttnParams attention_params(const gs_cached_attention* a, const CacheParams& c, const DeviceContext& dc) {
    AttnParams p{};
    p.B = static_cast<int>(a->B);
    p.M = static_cast<int>(a->M);
    p.N = static_cast<int>(c.N);
    p.H = static_cast<int>(a->H);
    p.Hk = c.heads;
    p.G = p.H / p.Hk;
    p.D = c.D;
    p.C = c.C;
    p.R = a->M * p.G;
    p.tau = static_cast<float>(a->tau);
    p.c = static_cast<float>(a->tau * 1.4426950408889634);
    p.causal = a->causal != 0;
    p.q_len = a->q_lengths;
    p.k_len = a->k_lengths;
    p.q = make_arr(a->q);
    p.out = make_arr(a->out);
    p.lse = a->lse;
    p.status = dc.status;
    p.splits = 1;
    const int64_t es = elem_size(a->dtype);
    p.vec = p.D % 8 == 0 && aligned_rows(p.q, p, 16 / es, es);
    return p;
}

// Attention over rows read back into a workspace, for as many problems (of one
// problem: key heads) at a time as kRowsBytes hold.  16-bit calls that the tensor cores take, and other
// fp16 calls, get fp16 rows scaled by a power of two per problem and head (values keep 11 bits and
// any size), the first also queries scaled by one per row; others rows in their own type.
constexpr int64_t kRowsBytes = int64_t(1) << 31;

gs_status attend_rows(const AttnParams& a, const CacheParams& c, InType t, const DeviceContext& dc, cudaStream_t s) {
    const bool scaled = t != InType::F32 && dc.sm103 && c.D <= 128 && attn_tc_takes(a.out, a.B, a.M, a.H, a.C);
    const bool sized = scaled || t == InType::F16;
    const int64_t es = t == InType::F32 ? 4 : 2, G = a.G, N = c.N;
    // Rows on 16-byte boundaries, so that every kernel can take them.
    const int64_t dw = (c.D + 7) / 8 * 8, cw = (c.C + 7) / 8 * 8;
    const int64_t head_bytes = N * (dw + cw) * es + (scaled ? G * a.M * (2 * dw + 4) : 0) + (sized ? 8 : 0);
    const int64_t nb = std::max<int64_t>(1, std::min<int64_t>(a.B, kRowsBytes / (head_bytes * c.heads + 1)));
    const int64_t nh = nb > 1 ? c.heads : std::max<int64_t>(1, std::min<int64_t>(c.heads, kRowsBytes / (head_bytes + 1)));
    Workspace ws(s);
    gs_status st = ws.alloc(static_cast<size_t>(nb * nh * head_bytes + 64));
    if (st != GS_OK) return st;
    char* k = static_cast<char*>(ws.ptr);
    char* v = k + nb * nh * N * dw * es;
    char* q16 = v + nb * nh * N * cw * es;
    uint2* sizes = reinterpret_cast<uint2*>(q16 + (scaled ? nb * nh * G * a.M * dw * 2 : 0));
    float* row_scale = reinterpret_cast<float*>(sizes + nb * nh);
    for (int64_t b = 0; st == GS_OK && b < a.B; b += nb)
        for (int64_t h = 0; st == GS_OK && h < c.heads; h += nh) {
            const int64_t bs = std::min<int64_t>(nb, a.B - b), hs = std::min<int64_t>(nh, c.heads - h);
            const auto at = [&](const Arr& x) {
                return Arr{x.p + (b * x.sb + h * G * x.sh) * es, x.sb, x.sr, x.sh};
            };
            CacheRows r{};
            r.c = c;
            if (c.table)
                r.c.table += b * c.stride_table;
            else {
                r.c.data += b * c.sp;
                r.c.pages -= static_cast<int>(b);
            }
            r.B = static_cast<int>(bs);
            r.M = static_cast<int>(N);
            r.k_len = a.k_len ? a.k_len + b : nullptr;
            r.k = {k, hs * N * dw, dw, N * dw};
            r.v = {v, hs * N * cw, cw, N * cw};
            r.all = 1;
            r.head0 = static_cast<int>(h);
            r.heads = static_cast<int>(hs);
            AttnParams p = a;
            p.B = static_cast<int>(bs);
            p.Hk = static_cast<int>(hs);
            p.H = static_cast<int>(hs * G);
            p.q_len = a.q_len ? a.q_len + b : nullptr;
            p.k_len = r.k_len;
            p.q = at(a.q);
            p.out = at(a.out);
            p.lse = a.lse ? a.lse + (b * a.H + h * G) * a.M : nullptr;
            p.k = r.k;
            p.v = r.v;
            pdl_reset();
            if (sized) {
                CacheScale x{};
                x.c = r.c;
                x.B = r.B;
                x.G = a.G;
                x.head0 = r.head0;
                x.heads = r.heads;
                x.k_len = p.k_len;
                x.sizes = sizes;
                if (scaled) {
                    x.M = a.M;
                    x.q_len = p.q_len;
                    x.q = p.q;
                    x.q16 = reinterpret_cast<uint16_t*>(q16);
                    x.width = static_cast<int>(dw);
                    x.row_scale = row_scale;
                    p.q = {q16, a.M * hs * G * dw, hs * G * dw, dw};
                    p.row_scale = row_scale;
                    p.out_bf16 = t == InType::BF16;
                }
                st = cuda_status(cudaMemsetAsync(sizes, 0, bs * hs * sizeof(uint2), s), "memset");
                if (st == GS_OK) st = cuda_status(launch_cache_scale(x, t, s), "cache scale kernel");
                r.sizes = sizes;
                p.head_sizes = sizes;
            }
            if (st == GS_OK && N > 0)
                st = cuda_status(launch_cache_read(r, scaled ? InType::F16 : t, dc.sms, s), "cache read kernel");
            if (st == GS_OK) st = attn_forward(p, scaled ? InType::F16 : t, scaled, dc, s);
        }
    return ws.done(st);
}

gs_status attend_few(const AttnParams& p, const CacheParams& c, InType t, const FewPlan& plan, cudaStream_t s) {
    Workspace ws(s);
    gs_status st = plan.bytes > 0 ? ws.alloc(plan.bytes) : GS_OK;
    if (st != GS_OK) return st;
    st = cuda_status(launch_cache_few(p, c, t, plan, ws.ptr, s), "cached attention kernels");
    return ws.done(st);
}

// Key splits of the tensor-core kernel: the number with the fewest tile times
// over all waves, a block's start and end counted as four tiles, and the joining launch
// as four more.
int many_splits(int64_t blocks, int64_t key_tiles, int sms) {
    if (blocks >= 8 * sms) return 1;   // the last wave is a small part of the whole
    int best = 1;
    int64_t least = INT64_MAX;
    const int64_t most = std::min<int64_t>(64, (key_tiles + 1) / 2);
    for (int64_t s = 1; s <= most; ++s) {
        const int64_t cost = (blocks * s + sms - 1) / sms * ((key_tiles + s - 1) / s + 4) + (s > 1 ? 4 : 0);
        if (cost < least) {
            least = cost;
            best = static_cast<int>(s);
        }
    }
    return best;
}

gs_status attend_many(AttnParams p, const CacheParams& c, InType t, const DeviceContext& dc, cudaStream_t s) {
    const int64_t tiles = (p.R + kCacheManyRows - 1) / kCacheManyRows;
    if (tiles > kMax / (static_cast<int64_t>(p.B) * p.Hk)) return unsupported("too many row tiles for one launch");
    const int64_t blocks = tiles * p.B * p.Hk;
    p.splits = many_splits(blocks, (c.N + kCacheManyKeys - 1) / kCacheManyKeys, dc.sms);
    Workspace ws(s);
    gs_status st = GS_OK;
    if (p.splits > 1) {
        const size_t all = static_cast<size_t>(p.splits) * p.B * p.Hk * p.R;
        st = ws.alloc(all * (p.C + 1) * sizeof(float));
        if (st != GS_OK) return st;
        p.part_o = static_cast<float*>(ws.ptr);
        p.part_l = p.part_o + all * p.C;
    }
    st = cuda_status(launch_cache_many(p, c, t, aligned_rows(p.out, p, 4, 2), s), "cached attention kernel");
    if (st == GS_OK && p.splits > 1) st = cuda_status(launch_attn_join(p, t, s), "attention join kernel");
    return ws.done(st);
}

}  // namespace

extern "C" {

gs_status gauss_sum_cache_write(const gs_cache* c, const gs_cache_rows* r, void* stream) {
    pdl_reset();
    CacheRows p;
    gs_status st = check_rows(c, r, true, &p);
    if (st != GS_OK) return st;
    if (p.B == 0 || p.M == 0 || p.heads == 0 || p.c.pages == 0 || p.c.N == 0) return GS_OK;
    DeviceContext dc;
    st = device_context(&dc);
    if (st != GS_OK) return st;
    return cuda_status(launch_cache_write(p, in_type(r->dtype), dc.sms, static_cast<cudaStream_t>(stream)),
                       "cache write kernel");
}

gs_status gauss_sum_cache_read(const gs_cache* c, const gs_cache_rows* r, void* stream) {
    pdl_reset();
    CacheRows p;
    gs_status st = check_rows(c, r, false, &p);
    if (st != GS_OK) return st;
    if (p.B == 0 || p.M == 0 || p.heads == 0 || !(p.k.p || p.v.p)) return GS_OK;
    DeviceContext dc;
    st = device_context(&dc);
    if (st != GS_OK) return st;
    return cuda_status(launch_cache_read(p, in_type(r->dtype), dc.sms, static_cast<cudaStream_t>(stream)),
                       "cache read kernel");
}

gs_status gauss_sum_attention_cached(const gs_cached_attention* a, const gs_cache* c, void* stream) {
    pdl_reset();
    if (!a || !c) return invalid("null arguments");
    if (!known_dtype(a->dtype)) return invalid("unknown dtype");
    if (a->B < 0 || a->M < 0 || a->H < 0) return invalid("negative size");
    if (a->B > kMax || a->M > kMax || a->H > kMax) return unsupported("B, M and H must be below 2^31");
    if (c->heads < 1 || a->H % c->heads) return invalid("H must be a multiple of the cache's heads >= 1");
    const int64_t G = a->H / c->heads;
    if (a->M > 0 && G > kMax / a->M) return unsupported("M x H / heads must be below 2^31");
    if (a->H > kMax / std::max<int64_t>(1, a->B)) return unsupported("B x H must be below 2^31");
    if (!(std::isfinite(a->tau) && a->tau > 0.0)) return invalid("tau must be finite and > 0");
    if (a->causal != 0 && a->causal != 1) return invalid("causal must be 0 or 1");
    const float factor = static_cast<float>(a->tau * 1.4426950408889634);
    if (!(std::isfinite(factor) && static_cast<float>(a->tau) > 0.f))
        return invalid("tau is outside the float32 range");
    CacheParams p{};
    gs_status st = check_cache(c, a->B, false, &p);
    if (st == GS_OK) st = check_lengths(a->q_lengths, a->k_lengths);
    if (st != GS_OK) return st;
    if (reinterpret_cast<uintptr_t>(a->lse) & 3u) return invalid("lse must be aligned to its element");
    const int64_t es = elem_size(a->dtype);
    const char* why = check_array(a->q, es, a->B, a->M, a->H, c->D, false);
    if (!why) why = check_array(a->out, es, a->B, a->M, a->H, c->C, true);
    if (why) return invalid(why);
    if (a->B == 0 || a->M == 0 || a->H == 0) return GS_OK;
    DeviceContext dc;
    st = device_context(&dc);
    if (st != GS_OK) return st;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const InType t = in_type(a->dtype);
    const AttnParams call = attention_params(a, p, dc);
    FewPlan plan;
    if ((call.R <= kFewRows || t == InType::F32 || few_short(call, dc.sms)) && cache_few_takes(p) &&
        plan_cache_few(call, t, dc.sms, &plan))
        return attend_few(call, p, t, plan, s);
    if (dc.sm103 && cache_many_takes(p, t) &&
        (call.R <= kManyRows || p.N <= kExactTokens || tiles_fit(call, dc.sms) || !attn_tc_takes(call.out, call.B, call.M, call.H, call.C)))
        return attend_many(call, p, t, dc, s);
    return attend_rows(call, p, t, dc, s);
}

}  // extern "C"
