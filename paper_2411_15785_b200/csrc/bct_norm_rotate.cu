// Norms of queries and keys for each head with the position rotation in the same pass, and the backward of both.
//
// Per head vector x [D] of a token at position p, with the weights w [D]:
//     r = 1 / sqrt(mean(x^2) + eps)      y = x r w      out = R(p) y
// R turns the pairs of the first `rot` features, (i, i + rot/2) or (2i, 2i + 1), by p * freq_i radians and leaves
// the rest.  Backward, for d = dL/dout:
//     g = R(p)^T d      dL/dw += g x r      n = g w      dL/dx = r (n - x r mean(n x r))
// Everything between the load and the one rounding at the end is fp32; the angle is formed in double, in turns,
// and only its fraction of a turn is handed to sincospi, so that far positions lose nothing.
//
// Bound by HBM: one load and one store per element (two loads and a store in the backward).  A lane holds 16
// bytes of a head, so a head is 8, 16 or 32 neighbouring lanes, the mean is a few shuffles, and the partner of a
// feature in the other half sits rot/2 features away in another lane at the same place (rot a multiple of 16).
// A block takes a few tokens at a time and all their heads: the sines of a token are formed once for all of them.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "bct_device.cuh"
#include "bct_internal.h"
#include "bct_linear.h"

namespace bct {
namespace {

constexpr int kNrThreads = 256;
constexpr int kNrMaxTok = 8;    // tokens a block works on at a time, at most

struct NrArgs {
    const void* x[2];        // q, k
    const void* w[2];        // weights or NULL (ones)
    const void* d[2];        // backward: gradients of the outputs
    void* y[2];              // outputs, or the gradients of q and k
    float* partial;          // backward: [blocks][2][D]
    const int64_t* positions;
    const double* freq;
    int64_t n_tokens;
    int H[2];
    int rot, interleaved;
    int tok;                 // tokens per turn of a block
    float eps;
};

template <typename T>
__device__ __forceinline__ uint4 ldg16(const T* p) {
    return *reinterpret_cast<const uint4*>(p);
}

// sin and cos of the tokens' angles; a position is one double product away from its angle in turns
__device__ __forceinline__ void fill_angles(float2 (*cs)[64], const NrArgs& a, int64_t t0, int nt) {
    const int half = a.rot >> 1;
    for (int i = threadIdx.x; i < nt * half; i += kNrThreads) {
        const int t = i / half, f = i - t * half;
        double turns = (double)a.positions[t0 + t] * (a.freq[f] * 0.15915494309189533577);
        turns -= rint(turns);
        float s, c;
        sincospif(2.f * (float)turns, &s, &c);
        cs[t][f] = make_float2(c, s);
    }
}

// Turn this lane's features (kE of them from feature e0 on) by the angles in cs, or back when dir = -1.
template <int kE>
__device__ __forceinline__ void turn(float* x, const float2* cs, int e0, int rot, bool interleaved, float dir) {
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < kE; i += 2) {
            if (e0 + i < rot) {
                const float2 a = cs[(e0 + i) >> 1];
                const float s = dir * a.y, u = x[i], v = x[i + 1];
                x[i] = u * a.x - v * s;
                x[i + 1] = u * s + v * a.x;
            }
        }
        return;
    }
    const int half = rot >> 1, lane = threadIdx.x & 31;
    const int hop = half / kE;                    // lanes between the two halves
    const bool first = e0 < half, in = e0 < rot;
    const int src = in ? (first ? lane + hop : lane - hop) : lane;
#pragma unroll
    for (int i = 0; i < kE; ++i) {
        const float other = __shfl_sync(0xffffffffu, x[i], src & 31);
        if (in) {
            const float2 a = cs[first ? e0 + i : e0 + i - half];
            const float s = first ? -dir * a.y : dir * a.y;
            x[i] = fmaf(other, s, x[i] * a.x);
        }
    }
}

template <typename T, int D, bool BWD>
__global__ void __launch_bounds__(kNrThreads) norm_rotate_kernel(const NrArgs a) {
    constexpr int kE = Chunk<T>::kElems;          // features of a lane
    constexpr int kLanes = D / kE;                // lanes of a head
    constexpr int kSlots = kNrThreads / kLanes;   // heads a block works on at a time
    __shared__ float2 cs[kNrMaxTok][64];
    const int lane = threadIdx.x % kLanes, slot = threadIdx.x / kLanes;
    const int e0 = lane * kE;
    const int H = a.H[0] + a.H[1];

    float w[2][kE];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        if (a.w[s] != nullptr) {
            Chunk<T>::unpack(ldg16(static_cast<const T*>(a.w[s]) + e0), w[s]);
        } else {
#pragma unroll
            for (int i = 0; i < kE; ++i) w[s][i] = 1.f;
        }
    }
    float dw[2][kE] = {};

    const int64_t turns = (a.n_tokens + a.tok - 1) / a.tok;
    for (int64_t tt = blockIdx.x; tt < turns; tt += gridDim.x) {
        const int64_t t0 = tt * a.tok;
        const int nt = (int)min((int64_t)a.tok, a.n_tokens - t0);
        __syncthreads();
        fill_angles(cs, a, t0, nt);
        __syncthreads();
        const int n = nt * H;
        for (int i0 = 0; i0 < n; i0 += kSlots) {
            const int i = min(i0 + slot, n - 1);      // (every lane takes part in the shuffles)
            const bool valid = i0 + slot < n;
            const int t = i / H, hh = i - t * H;
            const int s = hh >= a.H[0];
            const int h = s ? hh - a.H[0] : hh;
            const size_t off = ((size_t)(t0 + t) * a.H[s] + h) * D + e0;
            float x[kE];
            Chunk<T>::unpack(ldg16(static_cast<const T*>(a.x[s]) + off), x);
            float g[kE];
            if (BWD) {
                Chunk<T>::unpack(ldg16(static_cast<const T*>(a.d[s]) + off), g);
                turn<kE>(g, cs[t], e0, a.rot, a.interleaved != 0, -1.f);
            }
            float ss = 0.f;
#pragma unroll
            for (int j = 0; j < kE; ++j) ss = fmaf(x[j], x[j], ss);
#pragma unroll
            for (int m = kLanes / 2; m > 0; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
            const float r = rsqrtf(ss * (1.f / D) + a.eps);
            if (!BWD) {
#pragma unroll
                for (int j = 0; j < kE; ++j) x[j] = x[j] * r * (s ? w[1][j] : w[0][j]);
                turn<kE>(x, cs[t], e0, a.rot, a.interleaved != 0, 1.f);
            } else {
                float dot = 0.f;
#pragma unroll
                for (int j = 0; j < kE; ++j) {
                    x[j] *= r;
                    const float gx = g[j] * x[j];
                    if (valid) {
                        dw[0][j] += s ? 0.f : gx;
                        dw[1][j] += s ? gx : 0.f;
                    }
                    g[j] *= s ? w[1][j] : w[0][j];
                    dot = fmaf(g[j], x[j], dot);
                }
#pragma unroll
                for (int m = kLanes / 2; m > 0; m >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, m);
                dot *= 1.f / D;
#pragma unroll
                for (int j = 0; j < kE; ++j) x[j] = r * (g[j] - x[j] * dot);
            }
            if (valid) *reinterpret_cast<uint4*>(static_cast<T*>(a.y[s]) + off) = Chunk<T>::pack(x);
        }
    }
    if (BWD && a.partial != nullptr) {   // this block's share of dL/dw: its slots summed in order
        __shared__ float red[kNrThreads * kE];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kE; ++j) red[slot * D + e0 + j] = dw[s][j];
            __syncthreads();
            for (int e = threadIdx.x; e < D; e += kNrThreads) {
                float sum = 0.f;
                for (int k = 0; k < kSlots; ++k) sum += red[k * D + e];
                a.partial[((size_t)blockIdx.x * 2 + s) * D + e] = sum;
            }
        }
    }
}

// dL/dw: the blocks' shares in a fixed order, one block per weight vector, 1024 / D threads per element.
__global__ void __launch_bounds__(1024) norm_rotate_dw_kernel(const float* partial, int blocks, int D, float* dw_q,
                                                              float* dw_k) {
    __shared__ double red[1024];
    float* dst = blockIdx.x ? dw_k : dw_q;
    const int e = threadIdx.x % D, part = threadIdx.x / D, parts = 1024 / D;
    double sum = 0.;
    for (int b = part; b < blocks; b += parts) sum += (double)partial[((size_t)b * 2 + blockIdx.x) * D + e];
    red[threadIdx.x] = sum;
    __syncthreads();
    if (part == 0 && dst != nullptr) {
        for (int p = 1; p < parts; ++p) sum += red[p * D + e];
        dst[e] = (float)sum;
    }
}

int nr_tokens_per_turn(int64_t n_tokens) {
    // one token per block while that leaves SMs without work, more beyond (the sines of a turn fill the block)
    return n_tokens >= 148 * 4 * 4 ? 4 : 1;
}

int nr_grid(int64_t n_tokens, int tok, int per_sm) {
    const int64_t turns = (n_tokens + tok - 1) / tok;
    return (int)(turns < 148 * per_sm ? turns : 148 * per_sm);
}

template <bool BWD>
cudaError_t nr_launch(const NrArgs& a, int D, int dtype, int grid, cudaStream_t stream) {
    if (dtype == BCT_BF16) {
        if (D == 128)
            norm_rotate_kernel<__nv_bfloat16, 128, BWD><<<grid, kNrThreads, 0, stream>>>(a);
        else
            norm_rotate_kernel<__nv_bfloat16, 64, BWD><<<grid, kNrThreads, 0, stream>>>(a);
    } else {
        if (D == 128)
            norm_rotate_kernel<float, 128, BWD><<<grid, kNrThreads, 0, stream>>>(a);
        else
            norm_rotate_kernel<float, 64, BWD><<<grid, kNrThreads, 0, stream>>>(a);
    }
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_norm_rotate(int64_t n_tokens, int Hq, int Hkv, int D, int dtype, const void* q, const void* k,
                               const void* w_q, const void* w_k, float eps, const int64_t* positions, const double* freq,
                               int rot, int interleaved, void* q_out, void* k_out, cudaStream_t stream) {
    NrArgs a = {};
    a.x[0] = q, a.x[1] = k;
    a.w[0] = w_q, a.w[1] = w_k;
    a.y[0] = q_out, a.y[1] = k_out;
    a.positions = positions;
    a.freq = freq;
    a.n_tokens = n_tokens;
    a.H[0] = Hq, a.H[1] = Hkv;
    a.rot = rot;
    a.interleaved = interleaved;
    a.tok = nr_tokens_per_turn(n_tokens);
    a.eps = eps;
    return nr_launch<false>(a, D, dtype, nr_grid(n_tokens, a.tok, 8), stream);
}

int norm_rotate_bwd_blocks(int64_t n_tokens) { return nr_grid(n_tokens, nr_tokens_per_turn(n_tokens), 4); }

cudaError_t launch_norm_rotate_bwd(int64_t n_tokens, int Hq, int Hkv, int D, int dtype, const void* d_q_out,
                                   const void* d_k_out, const void* q, const void* k, const void* w_q, const void* w_k,
                                   float eps, const int64_t* positions, const double* freq, int rot, int interleaved,
                                   void* d_q, void* d_k, float* d_w_q, float* d_w_k, float* partial, cudaStream_t stream) {
    NrArgs a = {};
    a.x[0] = q, a.x[1] = k;
    a.w[0] = w_q, a.w[1] = w_k;
    a.d[0] = d_q_out, a.d[1] = d_k_out;
    a.y[0] = d_q, a.y[1] = d_k;
    const bool want_dw = d_w_q != nullptr || d_w_k != nullptr;
    a.partial = want_dw ? partial : nullptr;
    a.positions = positions;
    a.freq = freq;
    a.n_tokens = n_tokens;
    a.H[0] = Hq, a.H[1] = Hkv;
    a.rot = rot;
    a.interleaved = interleaved;
    a.tok = nr_tokens_per_turn(n_tokens);
    a.eps = eps;
    const int grid = norm_rotate_bwd_blocks(n_tokens);
    cudaError_t e = nr_launch<true>(a, D, dtype, grid, stream);
    if (e != cudaSuccess || !want_dw) return e;
    norm_rotate_dw_kernel<<<2, 1024, 0, stream>>>(partial, grid, D, d_w_q, d_w_k);
    return cudaGetLastError();
}

}  // namespace bct
