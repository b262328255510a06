// C ABI of the 8-bit cache (append, attention, eviction): argument checks and the carve-up of the caller's scratch.
// Nothing is allocated here.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <utility>

#include "bct_internal.h"
#include "bct_qcache.h"

namespace {

using bct::QcView;

bct_status_t fail(bct_status_t st, const char* fmt, ...) {
    char msg[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof(msg), fmt, ap);
    va_end(ap);
    bct::set_last_error(msg);
    return st;
}
bct_status_t fail_cuda(const char* what, cudaError_t e) { return fail(BCT_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e)); }

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t round256(size_t x) { return (x + 255) / 256 * 256; }

struct Span {
    const char* name;
    const void* p;
    size_t bytes;
};
bool overlap(const Span& x, const Span& y) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(x.p), b = reinterpret_cast<uintptr_t>(y.p);
    return x.p != nullptr && y.p != nullptr && a < b + y.bytes && b < a + x.bytes;
}
// No written operand (the first n_written) overlaps any other.
bct_status_t check_overlap(const Span* s, int n, int n_written) {
    for (int i = 0; i < n_written; ++i)
        for (int j = i + 1; j < n; ++j)
            if (overlap(s[i], s[j])) return fail(BCT_ERR_INVALID_ARG, "%s overlaps %s", s[i].name, s[j].name);
    return BCT_OK;
}

// The cache's sizes alone.
bct_status_t check_sizes(const bct_qcache_t* c, QcView* v) {
    if (c == nullptr) return fail(BCT_ERR_INVALID_ARG, "cache is NULL");
    if (c->batch < 1 || c->n_kv_heads < 1 || c->capacity < 1)
        return fail(BCT_ERR_INVALID_ARG, "batch, n_kv_heads and capacity must be >= 1");
    if ((long long)c->batch * c->n_kv_heads > (1LL << 20)) return fail(BCT_ERR_INVALID_ARG, "batch * n_kv_heads too large");
    if (c->capacity > (1 << 24)) return fail(BCT_ERR_INVALID_ARG, "capacity too large");
    if (c->head_dim < 1) return fail(BCT_ERR_INVALID_ARG, "head_dim must be >= 1");
    if (c->head_dim != 64 && c->head_dim != 128)
        return fail(BCT_ERR_UNSUPPORTED, "head_dim %d: this library has kernels for 64 and 128", c->head_dim);
    v->B = c->batch, v->Hkv = c->n_kv_heads, v->D = c->head_dim, v->C = c->capacity;
    v->NB = (v->C + bct::kQcBlock - 1) / bct::kQcBlock;
    return BCT_OK;
}
enum { kWeightSpan = 4, kCacheSpans = 7 };
bct_status_t check_cache(const bct_qcache_t* c, QcView* v, Span* spans) {
    if (const bct_status_t st = check_sizes(c, v)) return st;
    const size_t units = (size_t)v->B * v->Hkv, slots = units * v->C, nb = units * v->NB;
    const Span s[kCacheSpans] = {{"k", c->k, slots * v->D},        {"v", c->v, slots * v->D},
                                 {"k_scale", c->k_scale, nb * 4},  {"v_scale", c->v_scale, nb * 4},
                                 {"weight", c->weight, slots * 4}, {"position", c->position, slots * 4},
                                 {"state", c->state, (size_t)v->B * 12}};
    for (int i = 0; i < kCacheSpans; ++i) {
        if (s[i].p == nullptr) return fail(BCT_ERR_INVALID_ARG, "%s must not be NULL", s[i].name);
        if (!aligned(s[i].p, 16)) return fail(BCT_ERR_INVALID_ARG, "%s must be 16-byte aligned", s[i].name);
        spans[i] = s[i];
    }
    v->codes[0] = c->k, v->codes[1] = c->v;
    v->scale[0] = c->k_scale, v->scale[1] = c->v_scale;
    v->weight = c->weight, v->position = c->position, v->state = c->state;
    return BCT_OK;
}
bct_status_t check_tokens(int64_t T, int32_t dtype, const int32_t* lens) {
    if (T < 1 || T > 0x7fffffff) return fail(BCT_ERR_INVALID_ARG, "T must be in 1..2^31 - 1");
    if (dtype != BCT_F32 && dtype != BCT_BF16) return fail(BCT_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (!aligned(lens, 4)) return fail(BCT_ERR_INVALID_ARG, "lens must be 4-byte aligned");
    return BCT_OK;
}
bct_status_t check_operand(const char* name, const void* p) {
    if (p == nullptr) return fail(BCT_ERR_INVALID_ARG, "%s must not be NULL", name);
    if (!aligned(p, 16)) return fail(BCT_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
    return BCT_OK;
}
bct_status_t check_scratch(const void* scratch, size_t bytes, size_t need) {
    if (need == 0) return BCT_OK;
    if (scratch == nullptr) return fail(BCT_ERR_INVALID_ARG, "scratch must not be NULL: this call needs %zu bytes", need);
    if (!aligned(scratch, 256)) return fail(BCT_ERR_INVALID_ARG, "scratch must be 256-byte aligned");
    if (bytes < need) return fail(BCT_ERR_INVALID_ARG, "scratch has %zu bytes, this call needs %zu", bytes, need);
    return BCT_OK;
}
inline bool grid_fits(int64_t units, int64_t ctas) { return ctas <= 0x7fffffff / units; }

// Many bfloat16 rows go to the tensor path, whose time hardly depends on how many there are up to 128.  The other serves rows in
// groups alike of 8, 16 or 24 (16 in float, whose queries and probabilities are two terms each), a reading of the codes for
// each.  28 rows take 108 us there and 118 on the tensor path with 16 x 4096 slots x 8 heads, 202 / 233 with 64 x 2048, 79 / 112
// with 64 x 512, 58 / 52 with one sequence of 8192; 48 rows 177 / 120, 325 / 243, 126 / 120, 87 / 54.  (So one sequence alone loses
// 6 us at 28 rows; the rule goes by the rows, since batches lose more on the other side: 10 to 33 us.)
bct_status_t plan_attend(const QcView& v, int64_t T, int32_t n_q_heads, int32_t dtype, int32_t accumulate, bct::QcPlan* p) {
    if (n_q_heads < 1 || n_q_heads > (1 << 16) || n_q_heads % v.Hkv != 0)
        return fail(BCT_ERR_INVALID_ARG, "n_q_heads (%d) must be a multiple of n_kv_heads (%d) in 1..65536", n_q_heads, v.Hkv);
    const int64_t R = T * (n_q_heads / v.Hkv), units = (int64_t)v.B * v.Hkv;
    if (!grid_fits(units, std::max<int64_t>(v.NB, R))) return fail(BCT_ERR_INVALID_ARG, "batch, heads and T too large for one call");
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += round256(bytes); return here; };
    *p = bct::QcPlan{};
    p->prompt = dtype == BCT_BF16 && R > bct::kQcScoredRows;
    if (p->prompt) {
        const int64_t tiles = (R + 255) / 256;
        // a CTA per SM, but four tiles of 128 slots to each at least
        p->pr.tiles = (int)tiles;
        p->pr.splits = (int)std::max<int64_t>(1, std::min<int64_t>(148 / (units * tiles), v.C / 512));
        p->pr.by_slots = R <= 128;
        p->pr.parts = p->pr.splits * (p->pr.by_slots ? 2 : 1);
        if (p->pr.parts > 1) {
            p->part_o = take((size_t)units * R * p->pr.parts * v.D * 4);
            p->part_ml = take((size_t)units * R * p->pr.parts * 8);
        }
        if (accumulate) {
            p->q_tiles = take((size_t)units * tiles * 256 * v.D * 2);
            p->records = take((size_t)units * tiles * 2 * 1536);
        }
        p->total = at;
        return BCT_OK;
    }
    const int most = dtype == BCT_BF16 ? 3 : 2;
    const int64_t groups = (R + 8 * most - 1) / (8 * most);
    p->tiles = (int)((R + 8 * groups - 1) / (8 * groups));        // (groups alike)
    p->rows = 8 * p->tiles;
    p->n_groups = (R + p->rows - 1) / p->rows;
    p->by_scores = accumulate != 0 && R <= bct::kQcScoredRows;
    p->n_warps = (int)std::min<int64_t>(bct::qc_attend_max_warps(), units * p->n_groups * v.NB);
    p->part_o = take((size_t)2 * p->n_warps * p->rows * v.D * 4);
    p->part_ml = take((size_t)2 * p->n_warps * p->rows * 8);
    p->spans = take((size_t)units * p->n_groups * 8);
    p->ml = take((size_t)units * R * 8);
    p->scores = take(p->by_scores ? (size_t)units * R * v.NB * bct::kQcBlock * 4 : 0);
    p->total = at;
    return BCT_OK;
}

struct EvictPlan {
    int max_moves, max_blocks;
    size_t n_out, n_blocks, cut_scale, blocks, movers, total;
};
bct_status_t plan_evict(const QcView& v, int32_t keep, EvictPlan* p) {
    if (keep < 0 || keep > v.C) return fail(BCT_ERR_INVALID_ARG, "keep (%d) must be in 0..capacity (%d)", keep, v.C);
    const size_t units = (size_t)v.B * v.Hkv;
    p->max_moves = std::min(v.C - keep, keep);
    p->max_blocks = std::min(p->max_moves, (keep + bct::kQcBlock - 1) / bct::kQcBlock);
    if (!grid_fits((int64_t)units, std::max(1, p->max_blocks))) return fail(BCT_ERR_INVALID_ARG, "batch, heads and capacity too large for one call");
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += round256(bytes); return here; };
    p->n_out = take(units * 4);
    p->n_blocks = take(units * 4);
    p->cut_scale = take(units * 8);
    p->blocks = take(units * p->max_blocks * sizeof(int4));
    p->movers = take(units * p->max_moves * 4);
    p->total = keep == v.C ? 0 : at;
    return BCT_OK;
}

}  // namespace

extern "C" bct_status_t bct_qcache_append(const bct_qcache_t* cache, int64_t T, int32_t dtype, const void* k, const void* v,
                                          const int32_t* lens, void* cuda_stream) {
    bct::QcAppend a;
    Span s[kCacheSpans + 3];
    if (bct_status_t st = check_cache(cache, &a.c, s)) return st;
    if (bct_status_t st = check_tokens(T, dtype, lens)) return st;
    if (bct_status_t st = check_operand("new k", k)) return st;
    if (bct_status_t st = check_operand("new v", v)) return st;
    const size_t bytes = (size_t)a.c.B * T * a.c.Hkv * a.c.D * (dtype == BCT_F32 ? 4 : 2);
    s[kCacheSpans] = {"new k", k, bytes};
    s[kCacheSpans + 1] = {"new v", v, bytes};
    s[kCacheSpans + 2] = {"lens", lens, (size_t)a.c.B * 4};
    if (bct_status_t st = check_overlap(s, kCacheSpans + 3, kCacheSpans)) return st;
    a.x[0] = k, a.x[1] = v, a.lens = lens, a.T = T, a.ctas = 0;
    a.W = (int)std::min<int64_t>((T + bct::kQcBlock - 2) / bct::kQcBlock + 1, a.c.NB);   // (one token touches one)
    if (!grid_fits((int64_t)a.c.B * a.c.Hkv, a.W)) return fail(BCT_ERR_INVALID_ARG, "batch, heads and T too large for one call");
    const cudaError_t e = bct::qc_append(a, dtype, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? BCT_OK : fail_cuda("bct_qcache_append", e);
}

extern "C" bct_status_t bct_qcache_attend_scratch_bytes(const bct_qcache_t* cache, int64_t T, int32_t n_q_heads, int32_t dtype,
                                                        int32_t accumulate, size_t* bytes) {
    QcView v;
    bct::QcPlan p;
    if (bytes == nullptr) return fail(BCT_ERR_INVALID_ARG, "bytes is NULL");
    if (bct_status_t st = check_sizes(cache, &v)) return st;
    if (bct_status_t st = check_tokens(T, dtype, nullptr)) return st;
    if (bct_status_t st = plan_attend(v, T, n_q_heads, dtype, accumulate, &p)) return st;
    *bytes = p.total;
    return BCT_OK;
}

extern "C" bct_status_t bct_qcache_attend(const bct_qcache_t* cache, int64_t T, int32_t n_q_heads, int32_t dtype, const void* q,
                                          const int32_t* lens, float scale, float score_cap, int32_t accumulate, void* out,
                                          void* scratch, size_t scratch_bytes, void* cuda_stream) {
    bct::QcAttend a;
    bct::QcPlan p;
    Span s[kCacheSpans + 4];
    if (bct_status_t st = check_cache(cache, &a.c, s + 2)) return st;
    if (bct_status_t st = check_tokens(T, dtype, lens)) return st;
    if (bct_status_t st = plan_attend(a.c, T, n_q_heads, dtype, accumulate, &p)) return st;
    if (bct_status_t st = check_operand("q", q)) return st;
    if (bct_status_t st = check_operand("out", out)) return st;
    if (std::isnan(scale) || std::isinf(scale)) return fail(BCT_ERR_INVALID_ARG, "scale must be finite");
    if (!(score_cap >= 0.f) || std::isinf(score_cap)) return fail(BCT_ERR_INVALID_ARG, "score_cap must be finite and not below 0");
    if (!(scale > 0.f)) scale = 1.0f / std::sqrt((float)a.c.D);
    if (score_cap > 0.f && (!std::isfinite(scale / score_cap) || scale / score_cap < 1.17549435e-38f))
        return fail(BCT_ERR_INVALID_ARG, "scale / score_cap is out of fp32's range");
    if (!std::isfinite(scale * 1.4426950408889634f) || !std::isfinite(score_cap * 1.4426950408889634f))   // (scores are powers of two)
        return fail(BCT_ERR_INVALID_ARG, "scale or score_cap, times log2(e), is out of fp32's range");
    if (bct_status_t st = check_scratch(scratch, scratch_bytes, p.total)) return st;
    const size_t bytes = (size_t)a.c.B * T * n_q_heads * a.c.D * (dtype == BCT_F32 ? 4 : 2);
    s[0] = {"out", out, bytes};
    s[1] = {"scratch", scratch, p.total};
    s[kCacheSpans + 2] = {"q", q, bytes};
    s[kCacheSpans + 3] = {"lens", lens, (size_t)a.c.B * 4};
    std::swap(s[2], s[2 + kWeightSpan]);   // written only if `accumulate`
    if (bct_status_t st = check_overlap(s, kCacheSpans + 4, accumulate != 0 ? 3 : 2)) return st;
    a.q = q, a.out = out, a.lens = lens, a.T = T;
    a.G = n_q_heads / a.c.Hkv;
    a.R = T * a.G;
    a.n_groups = p.n_groups;
    a.scale = scale, a.cap = score_cap, a.accumulate = accumulate != 0;
    a.n_warps = p.n_warps;
    unsigned char* base = static_cast<unsigned char*>(scratch);
    a.part_o = reinterpret_cast<float*>(base + p.part_o);
    a.part_ml = reinterpret_cast<float2*>(base + p.part_ml);
    a.spans = reinterpret_cast<int2*>(base + p.spans);
    a.ml = reinterpret_cast<float2*>(base + p.ml);
    a.scores = p.by_scores ? reinterpret_cast<float*>(base + p.scores) : nullptr;
    a.Cs = a.c.NB * bct::kQcBlock;
    cudaError_t e;
    if (p.prompt) {
        if (accumulate != 0) {
            p.pr.q_tiles = base + p.q_tiles;
            p.pr.records = base + p.records;
        }
        e = bct::qc_prompt(a, p.pr, static_cast<cudaStream_t>(cuda_stream));
    } else {
        e = bct::qc_attend(a, p, dtype, static_cast<cudaStream_t>(cuda_stream));
    }
    return e == cudaSuccess ? BCT_OK : fail_cuda("bct_qcache_attend", e);
}

extern "C" bct_status_t bct_qcache_evict_scratch_bytes(const bct_qcache_t* cache, int32_t keep, size_t* bytes) {
    QcView v;
    EvictPlan p;
    if (bytes == nullptr) return fail(BCT_ERR_INVALID_ARG, "bytes is NULL");
    if (bct_status_t st = check_sizes(cache, &v)) return st;
    if (bct_status_t st = plan_evict(v, keep, &p)) return st;
    *bytes = p.total;
    return BCT_OK;
}

extern "C" bct_status_t bct_qcache_evict(const bct_qcache_t* cache, int32_t keep, int32_t recent, void* scratch,
                                         size_t scratch_bytes, void* cuda_stream) {
    bct::QcEvict a;
    EvictPlan p;
    Span s[kCacheSpans + 1];
    if (bct_status_t st = check_cache(cache, &a.c, s + 1)) return st;
    if (bct_status_t st = plan_evict(a.c, keep, &p)) return st;
    if (recent < 0 || recent > keep) return fail(BCT_ERR_INVALID_ARG, "recent (%d) must be in 0..keep (%d)", recent, keep);
    if (bct_status_t st = check_scratch(scratch, scratch_bytes, p.total)) return st;
    s[0] = {"scratch", scratch, p.total};
    if (bct_status_t st = check_overlap(s, kCacheSpans + 1, kCacheSpans + 1)) return st;
    if (keep == a.c.C) return BCT_OK;   // no cache holds more
    a.keep = keep, a.recent = recent, a.max_moves = p.max_moves, a.max_blocks = p.max_blocks;
    unsigned char* base = static_cast<unsigned char*>(scratch);
    a.n_out = reinterpret_cast<int32_t*>(base + p.n_out);
    a.n_blocks = reinterpret_cast<int32_t*>(base + p.n_blocks);
    a.cut_scale = reinterpret_cast<float*>(base + p.cut_scale);
    a.blocks = reinterpret_cast<int4*>(base + p.blocks);
    a.movers = reinterpret_cast<int32_t*>(base + p.movers);
    const cudaError_t e = bct::qc_evict(a, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? BCT_OK : fail_cuda("bct_qcache_evict", e);
}
