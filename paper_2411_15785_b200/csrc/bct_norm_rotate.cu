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
// Bound by HBM: one load and one store per element (two loads and a store in the backward).  A lane holds 16 bytes of
// a head, so a head is 8, 16 or 32 neighbouring lanes, the mean is a few shuffles, and the partner of a feature in the
// other half sits rot/2 features away in another lane at the same place (rot a multiple of 16).  A warp works alone on
// the heads of one token (or on a share of them, when there are few tokens): it forms the token's sines once, in its
// piece of shared memory, and the heads come as contiguous bulk copies into a ring of its own, three stages of 4 KiB.
// 192 KiB in flight per SM is what it takes: with the loads in registers (48 KiB in flight) 32768 tokens of 32 + 8
// heads of 128 took 150 us.  Measured: those (671 MB) 112 us back to back, 6.0 TB/s, 0.92 of the copy rate, 123 us with
// other calls between; the backward of 16384 tokens of 32 + 32 heads (805 MB) 150 and 160 us, where instructions are 60 %
// of the issue slots.  Three blocks of 64 KiB (four stages of 2 KiB a warp, 80 registers) instead of two of 96: 124 us.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "bct_device.cuh"
#include "bct_internal.h"
#include "bct_linear.h"

namespace bct {
namespace {

constexpr int kNrThreads = 256;
constexpr int kNrWarps = kNrThreads / 32;
constexpr int kNrStages = 3;
constexpr int kNrStageBytes = 4096;   // forward: 8 passes of heads; backward: 4, and their gradients
constexpr int kNrSmem = kNrWarps * kNrStages * kNrStageBytes;

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
    int parts;               // warps that share a token's heads
    float eps;
};

template <typename T>
__device__ __forceinline__ uint4 ldg16(const T* p) {
    return *reinterpret_cast<const uint4*>(p);
}

// 16 bytes as pairs of floats, and back
__device__ __forceinline__ void unpack2(const uint4& w, float2 (&x)[4]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = make_float2(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xffff0000u));
}
__device__ __forceinline__ void unpack2(const uint4& w, float2 (&x)[2]) {
    x[0] = make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
    x[1] = make_float2(__uint_as_float(w.z), __uint_as_float(w.w));
}
template <typename T>
__device__ __forceinline__ uint4 pack2s(const float2* x) {
    return Chunk<T>::pack(reinterpret_cast<const float*>(x));
}

template <typename T, int D, bool BWD, bool INTER>
__global__ void __launch_bounds__(kNrThreads, 2) norm_rotate_kernel(const NrArgs a) {
    constexpr int kE = Chunk<T>::kElems;          // features of a lane
    constexpr int kLanes = D / kE;                // lanes of a head
    constexpr int kHeads = 32 / kLanes;           // heads of a pass
    constexpr int kP = kNrStageBytes / 512 / (BWD ? 2 : 1);   // passes of a stage
    constexpr int kBatch = kHeads * kP;           // heads of a stage
    constexpr int kHeadBytes = D * (int)sizeof(T);
    extern __shared__ __align__(128) unsigned char nr_smem[];
    __shared__ float2 cs_all[kNrWarps][64];
    __shared__ uint64_t full_all[kNrWarps][kNrStages];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float2* cs = cs_all[warp];
    uint64_t* full = full_all[warp];
    unsigned char* ring = nr_smem + warp * (kNrStages * kNrStageBytes);
    const int e0 = (lane % kLanes) * kE, hl = lane / kLanes;
    const int half = a.rot >> 1;
    const bool in = e0 < a.rot, first = e0 < half;
    // where a feature's partner is: the next feature, or the same place of the lane half the rotated part away
    const int partner = !in || INTER ? lane : (first ? lane + half / kE : lane - half / kE);
    auto partners_of = [&](float2 x) {
        return INTER ? make_float2(x.y, x.x)
                     : make_float2(__shfl_sync(0xffffffffu, x.x, partner), __shfl_sync(0xffffffffu, x.y, partner));
    };

    // A warp's items: a token, or one of `parts` shares of it.  (With more than one part there are few tokens, so that
    // items count below 2^31 either way.)  An item's heads come in batches, those of q, then those of k.
    const int nbq = (a.H[0] + kBatch - 1) / kBatch, nb = nbq + (a.H[1] + kBatch - 1) / kBatch;
    const int items = (int)(a.n_tokens * a.parts), stride = (int)gridDim.x * kNrWarps;
    struct Cursor {
        int item, t, batch;
    };
    auto start = [&](int item) {
        Cursor c;
        c.item = item;
        c.t = a.parts == 1 ? item : item / a.parts;
        c.batch = a.parts == 1 ? 0 : item - c.t * a.parts;
        return c;
    };
    auto after = [&](const Cursor& c) {
        Cursor n = c;
        n.batch += a.parts;
        return n.batch < nb ? n : start(c.item + stride);
    };
    if (lane == 0) {
        for (int i = 0; i < kNrStages; ++i) mbar_init(&full[i], 1);
        fence_mbar_init_cluster();
    }
    __syncwarp();
    auto fetch = [&](const Cursor& c, int stage) {   // by one lane
        const bool k = c.batch >= nbq;
        const int H = k ? a.H[1] : a.H[0], h0 = (k ? c.batch - nbq : c.batch) * kBatch;
        const uint32_t bytes = (uint32_t)min(kBatch, H - h0) * kHeadBytes;
        const size_t off = ((size_t)c.t * H + h0) * kHeadBytes;
        unsigned char* dst = ring + stage * kNrStageBytes;
        mbar_arrive_expect_tx(&full[stage], BWD ? 2 * bytes : bytes);
        bulk_load(dst, static_cast<const char*>(k ? a.x[1] : a.x[0]) + off, bytes, &full[stage]);
        if (BWD) bulk_load(dst + kNrStageBytes / 2, static_cast<const char*>(k ? a.d[1] : a.d[0]) + off, bytes, &full[stage]);
    };
    Cursor cur = start((int)blockIdx.x * kNrWarps + warp), ahead = cur;
    for (int i = 0; i < kNrStages; ++i) {
        if (ahead.item < items) {
            if (lane == 0) fetch(ahead, i);
            ahead = after(ahead);
        }
    }

    double fr[2];   // this lane's share of the frequencies, in turns per position
#pragma unroll
    for (int i = 0; i < 2; ++i) fr[i] = lane + 32 * i < half ? a.freq[lane + 32 * i] * 0.15915494309189533577 : 0.;
    uint4 w_raw[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        if (a.w[s] != nullptr) {
            w_raw[s] = ldg16(static_cast<const T*>(a.w[s]) + e0);
        } else {
            float one[kE];
#pragma unroll
            for (int i = 0; i < kE; ++i) one[i] = 1.f;
            w_raw[s] = Chunk<T>::pack(one);
        }
    }
    float2 dw[2][kE / 2] = {};
    int64_t pos = cur.item < items && half > 0 ? a.positions[cur.t] : 0;
    int stage = 0;
    uint32_t phase = 0;

    while (cur.item < items) {
        const Cursor next_item = start(cur.item + stride);
        const int64_t pos1 = next_item.item < items && half > 0 ? a.positions[next_item.t] : 0;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 2; ++i) {   // sines of the token, formed once for all its heads
            if (lane + 32 * i < half) {
                double turns = (double)pos * fr[i];
                turns -= rint(turns);
                float sn, c;
                sincospif(2.f * (float)turns, &sn, &c);
                cs[lane + 32 * i] = make_float2(c, sn);
            }
        }
        __syncwarp();
        // The turn is one multiply-add per feature, x_i c_i + x_partner s_i with the partner's sign in s; features that
        // are not turned have c = 1, s = 0.  Forward, the weights are in both.  (Two features to an instruction throughout:
        // the backward is bound by the issue of instructions.)
        float2 tc[kE / 2], ts[kE / 2];
        int have = -1;
        for (; cur.batch < nb; cur.batch += a.parts) {
            const bool s = cur.batch >= nbq;
            const int h0 = (s ? cur.batch - nbq : cur.batch) * kBatch, H = s ? a.H[1] : a.H[0];
            float2 w[kE / 2];
            if (BWD || have != (int)s) unpack2(s ? w_raw[1] : w_raw[0], w);
            if (BWD ? have < 0 : have != (int)s) {
                have = s;
#pragma unroll
                for (int i = 0; i < kE / 2; ++i) {
                    const int f = first || INTER ? e0 + 2 * i : e0 + 2 * i - half;
                    const float2 u = in ? cs[INTER ? f >> 1 : f] : make_float2(1.f, 0.f);
                    const float2 v = INTER ? u : (in ? cs[f + 1] : make_float2(1.f, 0.f));
                    tc[i] = make_float2(u.x, v.x);
                    ts[i] = make_float2((INTER || first) != BWD ? -u.y : u.y, (!INTER && first) != BWD ? -v.y : v.y);
                    if (!BWD) {
                        tc[i] = __fmul2_rn(tc[i], w[i]);
                        ts[i] = __fmul2_rn(ts[i], partners_of(w[i]));
                    }
                }
            }
            const bool came = mbar_wait(&full[stage], phase);
            __syncwarp();
            const unsigned char* src = ring + stage * kNrStageBytes + lane * 16;
            T* ys = static_cast<T*>(s ? a.y[1] : a.y[0]) + ((size_t)cur.t * H + h0 + hl) * D + e0;
            const int passes = min(kP, (H - h0 + kHeads - 1) / kHeads);
#pragma unroll 2
            for (int p = 0; p < passes; ++p) {   // (lanes of heads past the last one work on zeros)
                const bool valid = h0 + p * kHeads + hl < H;
                float2 x[kE / 2], g[kE / 2], y[kE / 2];
                unpack2(valid ? *reinterpret_cast<const uint4*>(src + p * 512) : make_uint4(0, 0, 0, 0), x);
                if (BWD) unpack2(valid ? *reinterpret_cast<const uint4*>(src + kNrStageBytes / 2 + p * 512) : make_uint4(0, 0, 0, 0), g);
                float2 ss2 = make_float2(0.f, 0.f);
#pragma unroll
                for (int j = 0; j < kE / 2; ++j) ss2 = __ffma2_rn(x[j], x[j], ss2);
                float ss = ss2.x + ss2.y;
#pragma unroll
                for (int m = kLanes / 2; m > 0; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
                float r = rsqrtf(ss * (1.f / D) + a.eps);
                if (BWD && !valid) r = 0.f;   // (with eps = 0 their r is infinite, and 0 r not 0: it would enter dw)
                if (!came) r = __int_as_float(0x7fc00000);   // the copy never came: NaN, not old bytes
                const float2 rr = make_float2(r, r);
                const float2* v = BWD ? g : x;
#pragma unroll
                for (int j = 0; j < kE / 2; ++j) y[j] = __ffma2_rn(partners_of(v[j]), ts[j], __fmul2_rn(v[j], tc[j]));
                if (!BWD) {
#pragma unroll
                    for (int j = 0; j < kE / 2; ++j) y[j] = __fmul2_rn(y[j], rr);
                } else {
                    float2 d2 = make_float2(0.f, 0.f);
#pragma unroll
                    for (int j = 0; j < kE / 2; ++j) {
                        x[j] = __fmul2_rn(x[j], rr);
                        if (!s)
                            dw[0][j] = __ffma2_rn(y[j], x[j], dw[0][j]);
                        else
                            dw[1][j] = __ffma2_rn(y[j], x[j], dw[1][j]);
                        y[j] = __fmul2_rn(y[j], w[j]);
                        d2 = __ffma2_rn(y[j], x[j], d2);
                    }
                    float dot = d2.x + d2.y;
#pragma unroll
                    for (int m = kLanes / 2; m > 0; m >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, m);
                    dot *= -(1.f / D);
#pragma unroll
                    for (int j = 0; j < kE / 2; ++j) y[j] = __fmul2_rn(rr, __ffma2_rn(x[j], make_float2(dot, dot), y[j]));
                }
                if (valid) *reinterpret_cast<uint4*>(ys + (size_t)p * kHeads * D) = pack2s<T>(y);
            }
            __syncwarp();   // the stage has been read
            if (ahead.item < items) {
                if (lane == 0) fetch(ahead, stage);
                ahead = after(ahead);
            }
            if (++stage == kNrStages) stage = 0, phase ^= 1;
        }
        cur = next_item;
        pos = pos1;
    }
    if (BWD && a.partial != nullptr) {   // this block's share of dL/dw: its lanes' sums in a fixed order
        __shared__ float red[kNrThreads * kE];
        constexpr int kSlots = kNrThreads / kLanes;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kE / 2; ++j) *reinterpret_cast<float2*>(&red[(threadIdx.x / kLanes) * D + e0 + 2 * j]) = dw[s][j];
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

// Warps that share a token's heads: enough for about eight warps per SM in all, at most one to a batch.
int nr_parts(int64_t n_tokens, int Hq, int Hkv, int D, int dtype) {
    const int heads = kNrStageBytes / (D * (dtype == BCT_BF16 ? 2 : 4));   // of a batch
    const int most = (Hq + heads - 1) / heads + (Hkv + heads - 1) / heads;
    const int64_t parts = (148 * 8 + n_tokens - 1) / n_tokens;
    return (int)(parts > most ? most : parts);
}

int nr_grid(int64_t n_tokens, int parts, int per_sm) {
    const int64_t blocks = (n_tokens * parts + kNrWarps - 1) / kNrWarps;
    return (int)(blocks < 148 * per_sm ? blocks : 148 * per_sm);
}

template <typename T, int D, bool BWD, bool INTER>
cudaError_t nr_launch_kernel(const NrArgs& a, int grid, cudaStream_t stream) {
    auto fn = norm_rotate_kernel<T, D, BWD, INTER>;
    static std::atomic<unsigned long long> allowed{0};
    cudaError_t e = allow_smem(reinterpret_cast<const void*>(fn), kNrSmem, allowed);
    if (e != cudaSuccess) return e;
    fn<<<grid, kNrThreads, kNrSmem, stream>>>(a);
    return cudaGetLastError();
}
template <bool BWD, bool INTER>
cudaError_t nr_launch_as(const NrArgs& a, int D, int dtype, int grid, cudaStream_t stream) {
    if (dtype == BCT_BF16)
        return D == 128 ? nr_launch_kernel<__nv_bfloat16, 128, BWD, INTER>(a, grid, stream)
                        : nr_launch_kernel<__nv_bfloat16, 64, BWD, INTER>(a, grid, stream);
    return D == 128 ? nr_launch_kernel<float, 128, BWD, INTER>(a, grid, stream)
                    : nr_launch_kernel<float, 64, BWD, INTER>(a, grid, stream);
}
template <bool BWD>
cudaError_t nr_launch(const NrArgs& a, int D, int dtype, int grid, cudaStream_t stream) {
    return a.interleaved ? nr_launch_as<BWD, true>(a, D, dtype, grid, stream) : nr_launch_as<BWD, false>(a, D, dtype, grid, stream);
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
    a.parts = nr_parts(n_tokens, Hq, Hkv, D, dtype);
    a.eps = eps;
    return nr_launch<false>(a, D, dtype, nr_grid(n_tokens, a.parts, 2), stream);
}

// The backward keeps one warp to a token: a block's share of d_w costs as much however little it has summed.
int norm_rotate_bwd_blocks(int64_t n_tokens) { return nr_grid(n_tokens, 1, 2); }

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
    a.parts = 1;
    a.eps = eps;
    const int grid = norm_rotate_bwd_blocks(n_tokens);
    cudaError_t e = nr_launch<true>(a, D, dtype, grid, stream);
    if (e != cudaSuccess || !want_dw) return e;
    norm_rotate_dw_kernel<<<2, 1024, 0, stream>>>(partial, grid, D, d_w_q, d_w_k);
    return cudaGetLastError();
}

}  // namespace bct
