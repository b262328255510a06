// C ABI of the linear-attention calls and of the norm and rotation of queries and keys: argument checks, the
// roles of a call's scans and the carve-up of the caller's scratch.  Nothing is allocated here.
#include <cuda_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "bct_internal.h"
#include "bct_linear.h"

namespace {

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

// a named operand: where it is and how long
struct Span {
    const char* name;
    const void* p;
    size_t bytes;
    bool may_be_null;
};
bool overlap(const Span& x, const Span& y) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(x.p), b = reinterpret_cast<uintptr_t>(y.p);
    return x.p != nullptr && y.p != nullptr && x.bytes > 0 && y.bytes > 0 && a < b + y.bytes && b < a + x.bytes;
}
bct_status_t check_spans(const Span* s, int n) {   // the operands that kernels read and write 16 bytes at a time
    for (int i = 0; i < n; ++i) {
        if (s[i].p == nullptr && !s[i].may_be_null) return fail(BCT_ERR_INVALID_ARG, "%s must not be NULL", s[i].name);
        if (!aligned(s[i].p, 16)) return fail(BCT_ERR_INVALID_ARG, "%s must be 16-byte aligned", s[i].name);
    }
    return BCT_OK;
}
// No output overlaps an input or another output, except an output on exactly the place of an input where the
// call allows that (in_place[i] = index of that input, or -1).
bct_status_t check_overlap(const Span* in, int n_in, const Span* out, int n_out, const int* in_place) {
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < n_in; ++j)
            if (overlap(out[i], in[j]) && !(in_place[i] == j && out[i].p == in[j].p))
                return fail(BCT_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, in[j].name);
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return fail(BCT_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, out[j].name);
    }
    return BCT_OK;
}

bct_status_t resolve(const bct_linear_params_t* in, bct_linear_params_t* p) {
    if (in == nullptr) return fail(BCT_ERR_INVALID_ARG, "params is NULL");
    *p = *in;
    if (p->batch < 1 || p->n_q_heads < 1 || p->n_kv_heads < 1)
        return fail(BCT_ERR_INVALID_ARG, "batch, n_q_heads and n_kv_heads must be >= 1");
    if (p->n_q_heads % p->n_kv_heads != 0)
        return fail(BCT_ERR_INVALID_ARG, "n_q_heads (%d) is not a multiple of n_kv_heads (%d)", p->n_q_heads, p->n_kv_heads);
    if (p->dtype != BCT_F32 && p->dtype != BCT_BF16) return fail(BCT_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
    if (p->head_dim < 1) return fail(BCT_ERR_INVALID_ARG, "head_dim must be >= 1");
    if (p->head_dim != 64 && p->head_dim != 128)
        return fail(BCT_ERR_UNSUPPORTED, "head_dim %d: this library has kernels for 64 and 128", p->head_dim);
    if ((long long)p->batch * p->n_kv_heads > (1LL << 20) || p->n_q_heads > (1 << 16))
        return fail(BCT_ERR_INVALID_ARG, "batch * n_kv_heads or n_q_heads too large");
    if (std::isnan(p->scale)) return fail(BCT_ERR_INVALID_ARG, "scale is not a number");
    if (!(p->scale > 0.f)) p->scale = 1.0f / std::sqrt((float)p->head_dim);
    if (!std::isfinite(p->scale) || !std::isfinite(1.f / p->scale))
        return fail(BCT_ERR_INVALID_ARG, "scale must be finite, and its reciprocal too");
    return BCT_OK;
}

// Sizes of one call's tensors.
struct Sizes {
    size_t q, kv, state, decay, lens;
};
Sizes sizes_of(const bct_linear_params_t& p, int64_t T) {
    const size_t eb = p.dtype == BCT_F32 ? 4 : 2;
    Sizes s;
    s.q = (size_t)p.batch * (size_t)T * p.n_q_heads * p.head_dim * eb;
    s.kv = (size_t)p.batch * (size_t)T * p.n_kv_heads * p.head_dim * eb;
    s.state = (size_t)p.batch * p.n_kv_heads * p.head_dim * p.head_dim * sizeof(float);
    s.decay = (size_t)p.n_kv_heads * sizeof(float);
    s.lens = (size_t)p.batch * sizeof(int32_t);
    return s;
}
bct_status_t check_tokens(const bct_linear_params_t& p, int64_t T) {
    if (T < 1 || T > bct::kMaxCallTokens) return fail(BCT_ERR_INVALID_ARG, "T must be in [1, 2^30] (got %lld)", (long long)T);
    if ((double)p.batch * (double)T * p.n_q_heads * p.head_dim > 4.0e15) return fail(BCT_ERR_INVALID_ARG, "tensors too large");
    return BCT_OK;
}
bct_status_t check_scratch(const void* scratch, size_t bytes, size_t need) {
    if (need == 0) return BCT_OK;
    if (scratch == nullptr || bytes < need || !aligned(scratch, 256))
        return fail(BCT_ERR_INVALID_ARG, "scratch must be 256-byte aligned and hold %zu bytes (got %zu)", need, bytes);
    return BCT_OK;
}
// One launch serves roles that all have several heads on A's side, or none: the backward of shared heads takes two.
bool two_launches(const bct_linear_params_t& p) { return p.dtype == BCT_BF16 && p.n_q_heads > p.n_kv_heads; }
// What every segment adds to the state in reverse, by head.
size_t by_head_bytes(const bct_linear_params_t& p, const bct::LinPlan& plan) {
    return round256((size_t)p.batch * p.n_q_heads * plan.nseg * p.head_dim * p.head_dim * sizeof(float));
}
// kind: 0 the forward, 1 the backward, 2 the backward without d_state_in
size_t scratch_need(const bct_linear_params_t& p, int64_t T, int kind) {
    if (kind == 0) return round256(bct::lin_plan(p, T, 0).seg_bytes);
    if (!two_launches(p)) return 2 * round256(bct::lin_plan(p, T, 1).seg_bytes);
    const bct::LinPlan last = bct::lin_plan(p, T, 3);
    const size_t a = round256(bct::lin_plan(p, T, 2).seg_bytes);
    const size_t b = round256(last.seg_bytes) + (kind == 2 ? 0 : by_head_bytes(p, last));
    return a > b ? a : b;   // one after the other, in the same place
}
bct_status_t check_lens(const int32_t* lens) {
    if (!aligned(lens, 4)) return fail(BCT_ERR_INVALID_ARG, "lens must be 4-byte aligned");
    return BCT_OK;
}
bct_status_t check_decay(const float* log_decay) {
    if (log_decay == nullptr || !aligned(log_decay, 4))
        return fail(BCT_ERR_INVALID_ARG, "log_decay must not be NULL and 4-byte aligned");
    return BCT_OK;
}

}  // namespace

extern "C" {

bct_status_t bct_linear_scratch_bytes(const bct_linear_params_t* params, int64_t T, int32_t backward, size_t* bytes) {
    bct_linear_params_t p;
    bct_status_t st = resolve(params, &p);
    if (st == BCT_OK) st = check_tokens(p, T);
    if (st != BCT_OK) return st;
    if (bytes == nullptr) return fail(BCT_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = scratch_need(p, T, backward == 0 ? 0 : (backward == 2 ? 2 : 1));
    return BCT_OK;
}

bct_status_t bct_linear_step(const bct_linear_params_t* params, const void* q, const void* k, const void* v,
                             const float* log_decay, const float* state, float* state_out, void* out, void* cuda_stream) {
    bct_linear_params_t p;
    bct_status_t st = resolve(params, &p);
    if (st == BCT_OK) st = check_decay(log_decay);
    if (st != BCT_OK) return st;
    const Sizes s = sizes_of(p, 1);
    const Span in[] = {{"q", q, s.q, false}, {"k", k, s.kv, false}, {"v", v, s.kv, false}, {"state", state, s.state, false},
                       {"log_decay", log_decay, s.decay, false}};
    const Span outs[] = {{"out", out, s.q, false}, {"state_out", state_out, s.state, false}};
    const int in_place[] = {-1, 3};
    if ((st = check_spans(in, 4)) != BCT_OK || (st = check_spans(outs, 2)) != BCT_OK) return st;
    if ((st = check_overlap(in, 5, outs, 2, in_place)) != BCT_OK) return st;
    const cudaError_t e = bct::launch_linear_step(p, q, k, v, log_decay, state, state_out, out, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? BCT_OK : fail_cuda("linear step launch", e);
}

bct_status_t bct_linear_forward(const bct_linear_params_t* params, int64_t T, const void* q, const void* k, const void* v,
                                const float* log_decay, const int32_t* lens, const float* state, float* state_out,
                                void* out, void* scratch, size_t scratch_bytes, void* cuda_stream) {
    bct_linear_params_t p;
    bct_status_t st = resolve(params, &p);
    if (st == BCT_OK) st = check_tokens(p, T);
    if (st == BCT_OK) st = check_decay(log_decay);
    if (st == BCT_OK) st = check_lens(lens);
    if (st != BCT_OK) return st;
    const Sizes s = sizes_of(p, T);
    const bct::LinPlan plan = bct::lin_plan(p, T, 0);
    const size_t need = scratch_need(p, T, 0);
    if ((st = check_scratch(scratch, scratch_bytes, need)) != BCT_OK) return st;
    const Span in[] = {{"q", q, s.q, false}, {"k", k, s.kv, false}, {"v", v, s.kv, false}, {"state", state, s.state, true},
                       {"log_decay", log_decay, s.decay, false}, {"lens", lens, s.lens, true}};
    const Span outs[] = {{"out", out, s.q, false}, {"state_out", state_out, s.state, true}, {"scratch", need ? scratch : nullptr, need, true}};
    const int in_place[] = {-1, 3, -1};
    if ((st = check_spans(in, 4)) != BCT_OK || (st = check_spans(outs, 3)) != BCT_OK) return st;
    if ((st = check_overlap(in, 6, outs, 3, in_place)) != BCT_OK) return st;

    const int G = p.n_q_heads / p.n_kv_heads;
    bct::LinArgs a = {};
    a.log_decay = log_decay;
    a.lens = lens;
    a.n_roles = 1;
    a.B = p.batch, a.Hkv = p.n_kv_heads, a.T = (int)T;
    a.nseg = plan.nseg, a.seg_len = plan.seg_len;
    float* seg = plan.nseg > 1 ? static_cast<float*>(scratch) : nullptr;
    a.role[0] = {q, k, v, out, state, state_out, seg, G, 1, 0, 0, p.scale, 1.f, 1.f};
    bct::LinStates states = {};
    states.b[0] = k, states.c[0] = v, states.seg[0] = seg, states.first[0] = state, states.in_mul[0] = 1.f, states.G[0] = 1;
    const cudaError_t e = bct::launch_linear_scan(p, plan, a, states, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? BCT_OK : fail_cuda("linear forward launch", e);
}

bct_status_t bct_linear_backward(const bct_linear_params_t* params, int64_t T, const void* d_out, const void* q,
                                 const void* k, const void* v, const float* log_decay, const int32_t* lens,
                                 const float* state, const float* d_state, void* d_q, void* d_k, void* d_v,
                                 float* d_state_in, void* scratch, size_t scratch_bytes, void* cuda_stream) {
    bct_linear_params_t p;
    bct_status_t st = resolve(params, &p);
    if (st == BCT_OK) st = check_tokens(p, T);
    if (st == BCT_OK) st = check_decay(log_decay);
    if (st == BCT_OK) st = check_lens(lens);
    if (st != BCT_OK) return st;
    const Sizes s = sizes_of(p, T);
    const size_t need = scratch_need(p, T, d_state_in != nullptr ? 1 : 2);
    if ((st = check_scratch(scratch, scratch_bytes, need)) != BCT_OK) return st;
    const Span in[] = {{"d_out", d_out, s.q, false}, {"q", q, s.q, false},          {"k", k, s.kv, false},
                       {"v", v, s.kv, false},        {"state", state, s.state, true}, {"d_state", d_state, s.state, true},
                       {"log_decay", log_decay, s.decay, false}, {"lens", lens, s.lens, true}};
    const Span outs[] = {{"d_q", d_q, s.q, false},
                         {"d_k", d_k, s.kv, false},
                         {"d_v", d_v, s.kv, false},
                         {"d_state_in", d_state_in, s.state, true},
                         {"scratch", need ? scratch : nullptr, need, true}};
    const int in_place[] = {-1, -1, -1, -1, -1};
    if ((st = check_spans(in, 6)) != BCT_OK || (st = check_spans(outs, 5)) != BCT_OK) return st;
    if ((st = check_overlap(in, 8, outs, 5, in_place)) != BCT_OK) return st;

    const int G = p.n_q_heads / p.n_kv_heads;
    // In reverse the state is carried without the scale that q has in it: R = sum lambda^.. q^T do, times `scale`
    // where it is used, so what comes in is divided by it and what goes out multiplied.
    const float inv = 1.f / p.scale;
    const bool two = two_launches(p);
    for (int launch = 0; launch < (two ? 2 : 1); ++launch) {
        const int kind = two ? 2 + launch : 1;
        const bct::LinPlan plan = bct::lin_plan(p, T, kind);
        float* seg = static_cast<float*>(scratch);      // forward in time, then in reverse
        float* seg0 = plan.nseg > 1 && kind != 3 ? seg : nullptr;
        if (seg0 != nullptr) seg += round256(plan.seg_bytes) / sizeof(float);
        float* seg1 = plan.nseg > 1 && kind != 2 ? seg : nullptr;
        if (seg1 != nullptr) seg += round256(plan.seg_bytes) / sizeof(float);
        float* by_head = kind == 3 && d_state_in != nullptr ? seg : nullptr;
        const bct::LinRole roles[3] = {{d_out, v, k, d_q, state, nullptr, seg0, G, 1, 0, 1, p.scale, 1.f, 1.f},
                                       {v, d_out, q, d_k, d_state, nullptr, seg1, 1, G, 1, 1, p.scale, inv, 1.f},
                                       {k, q, d_out, d_v, d_state, by_head ? nullptr : d_state_in, seg1, 1, G, 1, 0, p.scale, inv, p.scale}};
        bct::LinArgs a = {};
        a.log_decay = log_decay;
        a.lens = lens;
        a.B = p.batch, a.Hkv = p.n_kv_heads, a.T = (int)T;
        a.nseg = plan.nseg, a.seg_len = plan.seg_len;
        for (int i = kind == 3 ? 1 : 0; i < (kind == 2 ? 1 : 3); ++i) a.role[a.n_roles++] = roles[i];
        bct::LinStates states = {};
        states.b[0] = k, states.c[0] = v, states.seg[0] = seg0, states.first[0] = state, states.in_mul[0] = 1.f, states.G[0] = 1;
        states.b[1] = q, states.c[1] = d_out, states.seg[1] = seg1, states.first[1] = d_state, states.in_mul[1] = inv, states.G[1] = G;
        states.by_head = by_head, states.heads = G, states.last = d_state_in, states.last_mul = p.scale;
        const cudaError_t e = bct::launch_linear_scan(p, plan, a, states, static_cast<cudaStream_t>(cuda_stream));
        if (e != cudaSuccess) return fail_cuda("linear backward launch", e);
    }
    return BCT_OK;
}

}  // extern "C"

namespace {

// The sizes and switches that both norm_rotate calls share.
bct_status_t check_norm_rotate(int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                               float eps, const int64_t* positions, const double* freq, int32_t rot_dim, uint32_t flags,
                               size_t* q_bytes, size_t* k_bytes, size_t* w_bytes) {
    if (n_tokens < 1 || n_tokens > bct::kMaxCallTokens)
        return fail(BCT_ERR_INVALID_ARG, "n_tokens must be in [1, 2^30] (got %lld)", (long long)n_tokens);
    if (n_q_heads < 1 || n_kv_heads < 1 || n_q_heads > (1 << 16) || n_kv_heads > (1 << 16))
        return fail(BCT_ERR_INVALID_ARG, "n_q_heads and n_kv_heads must be in [1, 65536]");
    if (dtype != BCT_F32 && dtype != BCT_BF16) return fail(BCT_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (head_dim != 64 && head_dim != 128)
        return fail(BCT_ERR_UNSUPPORTED, "head_dim %d: this library has kernels for 64 and 128", head_dim);
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(BCT_ERR_INVALID_ARG, "eps must be finite and not negative");
    if (rot_dim < 0 || rot_dim > head_dim) return fail(BCT_ERR_INVALID_ARG, "rot_dim %d outside 0..head_dim", rot_dim);
    if (rot_dim % 16 != 0) return fail(BCT_ERR_UNSUPPORTED, "rot_dim %d is not a multiple of 16", rot_dim);
    if (flags & ~BCT_ROTATE_INTERLEAVED) return fail(BCT_ERR_INVALID_ARG, "unknown flag bits 0x%x", flags);
    if (rot_dim > 0 && (positions == nullptr || freq == nullptr || !aligned(positions, 8) || !aligned(freq, 8)))
        return fail(BCT_ERR_INVALID_ARG, "positions and freq must not be NULL and 8-byte aligned");
    const size_t eb = dtype == BCT_F32 ? 4 : 2;
    *q_bytes = (size_t)n_tokens * n_q_heads * head_dim * eb;
    *k_bytes = (size_t)n_tokens * n_kv_heads * head_dim * eb;
    *w_bytes = (size_t)head_dim * eb;
    return BCT_OK;
}

}  // namespace

extern "C" {

bct_status_t bct_norm_rotate(int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                             const void* q, const void* k, const void* w_q, const void* w_k, float eps,
                             const int64_t* positions, const double* freq, int32_t rot_dim, uint32_t flags, void* q_out,
                             void* k_out, void* cuda_stream) {
    size_t qb = 0, kb = 0, wb = 0;
    bct_status_t st = check_norm_rotate(n_tokens, n_q_heads, n_kv_heads, head_dim, dtype, eps, positions, freq, rot_dim,
                                        flags, &qb, &kb, &wb);
    if (st != BCT_OK) return st;
    const Span in[] = {{"q", q, qb, false}, {"k", k, kb, false}, {"w_q", w_q, wb, true}, {"w_k", w_k, wb, true},
                       {"positions", rot_dim ? positions : nullptr, (size_t)n_tokens * 8, true},
                       {"freq", rot_dim ? freq : nullptr, (size_t)rot_dim * 4, true}};
    const Span outs[] = {{"q_out", q_out, qb, false}, {"k_out", k_out, kb, false}};
    const int in_place[] = {0, 1};
    if ((st = check_spans(in, 4)) != BCT_OK || (st = check_spans(outs, 2)) != BCT_OK) return st;
    if ((st = check_overlap(in, 6, outs, 2, in_place)) != BCT_OK) return st;
    const cudaError_t e = bct::launch_norm_rotate(n_tokens, n_q_heads, n_kv_heads, head_dim, dtype, q, k, w_q, w_k, eps,
                                                  positions, freq, rot_dim, (flags & BCT_ROTATE_INTERLEAVED) != 0, q_out,
                                                  k_out, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? BCT_OK : fail_cuda("norm_rotate launch", e);
}

bct_status_t bct_norm_rotate_scratch_bytes(int64_t n_tokens, int32_t head_dim, size_t* bytes) {
    if (n_tokens < 1 || n_tokens > bct::kMaxCallTokens || head_dim < 1 || bytes == nullptr)
        return fail(BCT_ERR_INVALID_ARG, "n_tokens must be in [1, 2^30], head_dim >= 1 and bytes not NULL");
    *bytes = round256((size_t)bct::norm_rotate_bwd_blocks(n_tokens) * 2 * head_dim * sizeof(float));
    return BCT_OK;
}

bct_status_t bct_norm_rotate_backward(int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                      int32_t dtype, const void* d_q_out, const void* d_k_out, const void* q, const void* k,
                                      const void* w_q, const void* w_k, float eps, const int64_t* positions,
                                      const double* freq, int32_t rot_dim, uint32_t flags, void* d_q, void* d_k, float* d_w_q,
                                      float* d_w_k, void* scratch, size_t scratch_bytes, void* cuda_stream) {
    size_t qb = 0, kb = 0, wb = 0;
    bct_status_t st = check_norm_rotate(n_tokens, n_q_heads, n_kv_heads, head_dim, dtype, eps, positions, freq, rot_dim,
                                        flags, &qb, &kb, &wb);
    if (st != BCT_OK) return st;
    size_t need = 0;
    if (d_w_q != nullptr || d_w_k != nullptr) {
        st = bct_norm_rotate_scratch_bytes(n_tokens, head_dim, &need);
        if (st == BCT_OK) st = check_scratch(scratch, scratch_bytes, need);
        if (st != BCT_OK) return st;
    }
    const Span in[] = {{"d_q_out", d_q_out, qb, false}, {"d_k_out", d_k_out, kb, false}, {"q", q, qb, false},
                       {"k", k, kb, false},             {"w_q", w_q, wb, true},          {"w_k", w_k, wb, true},
                       {"positions", rot_dim ? positions : nullptr, (size_t)n_tokens * 8, true},
                       {"freq", rot_dim ? freq : nullptr, (size_t)rot_dim * 4, true}};
    const size_t fw = (size_t)head_dim * sizeof(float);
    const Span outs[] = {{"d_q", d_q, qb, false},
                         {"d_k", d_k, kb, false},
                         {"d_w_q", d_w_q, fw, true},
                         {"d_w_k", d_w_k, fw, true},
                         {"scratch", need ? scratch : nullptr, need, true}};
    const int in_place[] = {0, 1, -1, -1, -1};
    if ((st = check_spans(in, 6)) != BCT_OK || (st = check_spans(outs, 5)) != BCT_OK) return st;
    if ((st = check_overlap(in, 8, outs, 5, in_place)) != BCT_OK) return st;
    const cudaError_t e = bct::launch_norm_rotate_bwd(
        n_tokens, n_q_heads, n_kv_heads, head_dim, dtype, d_q_out, d_k_out, q, k, w_q, w_k, eps, positions, freq, rot_dim,
        (flags & BCT_ROTATE_INTERLEAVED) != 0, d_q, d_k, d_w_q, d_w_k, static_cast<float*>(need ? scratch : nullptr),
        static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? BCT_OK : fail_cuda("norm_rotate backward launch", e);
}

}  // extern "C"
