// Host-side internals of the linear-attention calls: the roles of one launch, the segment plan and the
// launchers (bct_linear.cu: CUDA-core kernels, bct_linear_tc.cu: tensor-core kernel).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/bct.h"

namespace bct {

// Dynamic shared memory beyond 48 KiB has to be allowed once per kernel and device; `done` is the kernel's own record of
// the devices where it has been (a microsecond of every call otherwise).
inline cudaError_t allow_smem(const void* fn, int bytes, std::atomic<unsigned long long>& done) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 64 && (done.load(std::memory_order_relaxed) >> dev & 1)) return cudaSuccess;
    e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
    return e;
}

// One scan over the tokens of every (sequence, kv-head) unit.  All three passes of the backward have the
// forward's form, with other tensors in the three roles:
//     out_i = scale * ( sum_j lambda^|i-j| (a_i . b_j) c_j  +  lambda^(..) X a_i ),   j <= i, or j >= i in reverse
// X is the state outside the scan range, a [D][D] matrix with b's features in one axis and c's in the other.
//   forward  a = q,  b = k,  c = v   forward in time    state [b][c]
//   d_q      a = do, b = v,  c = k   forward in time    state [c][b]
//   d_k      a = v,  b = do, c = q   in reverse         state [c][b]
//   d_v      a = k,  b = q,  c = do  in reverse         state [b][c]
// States in memory always have the key's features in their rows and the value's in their columns, hence the
// two orders; state_t marks the second.
struct LinRole {
    const void* a;
    const void* b;
    const void* c;
    void* out;
    const float* state_in;  // [B][Hkv][D][D] or NULL (zeros)
    float* state_out;       // or NULL
    const float* seg;       // [U][nseg][D][D]: the state each segment starts from (only with nseg > 1)
    int Ga, Gb;             // heads per kv-head of (a, out) and of (b, c); one of the two is 1
    int reverse, state_t;
    float scale, in_mul, out_mul;  // of the output, the incoming and the outgoing state
};

struct LinArgs {
    LinRole role[3];
    const float* log_decay;  // [Hkv]
    const int* lens;         // [B] or NULL
    int n_roles;
    int B, Hkv, T;
    int nseg, seg_len;       // segments of the token axis, tokens per segment (a multiple of the chunk)
};

// The states that the segments start from: for each direction (0 forward in time, 1 reverse) what the
// segments before it add, then the running sum over them.
struct LinStates {
    const void* b[2];
    const void* c[2];
    float* seg[2];            // [U][nseg][D][D]; NULL: direction not needed
    const float* first[2];    // the state before the first segment, or NULL
    float in_mul[2];
    int G[2];
    // Not NULL (tensor path, reverse direction alone, G > 1): what every segment adds is formed by head, [B][Hkv * heads]
    // [nseg][D][D], and summed over the heads on the way; the state after the scan then goes to `last`, times last_mul.
    float* by_head;
    int heads;
    float* last;
    float last_mul;
};

struct LinPlan {
    int nseg, seg_len;
    size_t seg_bytes;  // one direction's states, 0 with one segment
    bool tensor;       // the tensor-core kernel serves the call
};

// One launch over the roles of `kind`: 0 forward, 1 backward (all three), 2 its d_q alone, 3 its d_k and d_v.  Depends on
// the sizes only (a B200's 148 SMs are assumed).
LinPlan lin_plan(const bct_linear_params_t& p, int64_t T, int kind);

cudaError_t launch_linear_step(const bct_linear_params_t& p, const void* q, const void* k, const void* v,
                               const float* log_decay, const float* state, float* state_out, void* out,
                               cudaStream_t stream);
// The whole scan: with more than one segment the segments' own contributions, their running sums, then every role.
cudaError_t launch_linear_scan(const bct_linear_params_t& p, const LinPlan& plan, const LinArgs& args,
                               const LinStates& states, cudaStream_t stream);
// The same on the tensor path (bct_linear_tc.cu): bfloat16.
// A launch has several heads on A's side in every role or in none.
cudaError_t launch_linear_tc(int D, const LinArgs& args, const LinStates& states, cudaStream_t stream);
// Running sums over the segments, in the order of the scan.
cudaError_t launch_linear_combine(int D, const LinArgs& args, const LinStates& states, cudaStream_t stream);
// The same over segments and heads (states.by_head).
cudaError_t launch_linear_combine_heads(int D, const LinArgs& args, const LinStates& states, cudaStream_t stream);

cudaError_t launch_norm_rotate(int64_t n_tokens, int Hq, int Hkv, int D, int dtype, const void* q, const void* k,
                               const void* w_q, const void* w_k, float eps, const int64_t* positions, const double* freq,
                               int rot, int interleaved, void* q_out, void* k_out, cudaStream_t stream);
int norm_rotate_bwd_blocks(int64_t n_tokens);   // rows of [2][D] floats that `partial` holds
cudaError_t launch_norm_rotate_bwd(int64_t n_tokens, int Hq, int Hkv, int D, int dtype, const void* d_q_out,
                                   const void* d_k_out, const void* q, const void* k, const void* w_q, const void* w_k,
                                   float eps, const int64_t* positions, const double* freq, int rot, int interleaved,
                                   void* d_q, void* d_k, float* d_w_q, float* d_w_k, float* partial, cudaStream_t stream);

}  // namespace bct
