// Linear attention with a decay for each head on the CUDA cores: the single-token step, and the chunked scan in
// float (bfloat16 is the tensor-core kernel's).
//
//     S_t = lambda S_{t-1} + k_t^T v_t        o_t = scale q_t S_t         lambda = exp(log_decay[h])
//
// The scan takes the tokens in chunks of 32: inside a chunk the products (a_i . b_j) are formed for all pairs
// and weighted with lambda^|i-j|; what lies before the chunk comes out of the state, which is updated once per
// chunk.  Everything is fp32; the powers of lambda are formed in double (33 of them per block).
//
// One block holds one (sequence, kv-head) unit, one segment of the tokens and 32 of c's features: those columns of the
// state and of the output depend on nothing in the others, and only the 32 x 32 products are formed again for each 32.
// That trades an eighth more multiplications (head_dim 128) for four times the blocks, which is what the small calls
// in float want.  The state of the block lives in registers (its update reads b and c from shared memory) and is copied
// to shared memory once per chunk, where the next chunk's products with a read it; the next tiles come by
// asynchronous copies while this chunk is worked on.  Bound by latency at the sizes it is meant for (float prompts are
// tests and small models): the backward of 2 x 333 tokens, 8 heads of 64 over 2 states, takes 46 us with its three launches.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "bct_device.cuh"
#include "bct_internal.h"
#include "bct_linear.h"
#include "bct_tc.cuh"

namespace bct {
namespace {

constexpr int kCh = 32;         // tokens per chunk
constexpr int kScanThreads = 256;

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                       __uint_as_float(w.y & 0xffff0000u));
}
__device__ __forceinline__ void store4(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }
// 16 bytes into shared memory, asynchronously; zeros where `on` is false (nothing is read then)
__device__ __forceinline__ void copy16(float* dst, const float* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ float4 fma4(float s, float4 x, float4 acc) {
    return make_float4(fmaf(s, x.x, acc.x), fmaf(s, x.y, acc.y), fmaf(s, x.z, acc.z), fmaf(s, x.w, acc.w));
}
__device__ __forceinline__ float4 mul4(float s, float4 x) { return make_float4(s * x.x, s * x.y, s * x.z, s * x.w); }
__device__ __forceinline__ float dot4(float4 x, float4 y, float acc) {
    return fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, acc))));
}

constexpr int kNc = 32;         // columns of a block

template <int D>
struct ScanSmem {
    float a[2][kCh][D + 4];    // two buffers; rows 16 bytes apart modulo 128: neighbouring rows start in other banks
    float b[2][kCh][D + 4];
    float c[2][kCh][kNc];
    float p[kCh][kCh + 4];
    float s[D][kNc];
    float pw[kCh + 1];         // lambda^n
};

// lambda^n, n = 0..kCh
__device__ __forceinline__ void fill_powers(float* pw, float log_decay, int tid) {
    if (tid <= kCh) pw[tid] = tid == 0 ? 1.f : (float)exp((double)tid * (double)log_decay);
}

template <int D, bool STATE_ONLY>
__global__ void __launch_bounds__(kScanThreads, 2) linear_scan_kernel(const __grid_constant__ LinArgs args, const __grid_constant__ LinStates st) {
    extern __shared__ __align__(16) unsigned char scan_smem_raw[];
    ScanSmem<D>& sm = *reinterpret_cast<ScanSmem<D>*>(scan_smem_raw);
    constexpr int kCG = kNc / 4;                 // groups of four columns
    constexpr int kRG = kScanThreads / kCG;      // groups of rows: one output row each
    constexpr int kStateRows = D / kRG;          // state rows of a thread
    static_assert(kRG == kCh && (kStateRows == 2 || kStateRows == 4), "");

    const int tid = threadIdx.x;
    const int ncol = D / kNc;
    int idx = blockIdx.x;
    const int col0 = (idx % ncol) * kNc;
    idx /= ncol;
    const int seg = idx % args.nseg;
    const int u = idx / args.nseg;
    const int bi = u / args.Hkv, h = u - bi * args.Hkv;

    const int which = STATE_ONLY ? (st.seg[0] == nullptr ? 1 : (int)blockIdx.y) : (int)blockIdx.y;
    const LinRole& r = args.role[STATE_ONLY ? 0 : which];
    const int reverse = STATE_ONLY ? which : r.reverse;
    const int Ga = STATE_ONLY ? 1 : r.Ga, Gb = STATE_ONLY ? st.G[which] : r.Gb;
    // the last segment in the order of the scan feeds no other
    if (STATE_ONLY && seg == (reverse ? 0 : args.nseg - 1)) return;
    const float* ga = static_cast<const float*>(r.a);
    const float* gb = static_cast<const float*>(STATE_ONLY ? st.b[which] : r.b);
    const float* gc = static_cast<const float*>(STATE_ONLY ? st.c[which] : r.c);
    float* go = static_cast<float*>(r.out);

    const int len = args.lens ? min(max(args.lens[bi], 0), args.T) : args.T;
    const int t_begin = seg * args.seg_len;
    const int t_end = min(t_begin + args.seg_len, args.T);
    const int v_end = min(t_end, len);           // valid tokens of the segment end here
    const int n_chunks = v_end > t_begin ? (v_end - t_begin + kCh - 1) / kCh : 0;
    const int G = STATE_ONLY ? Gb : max(Ga, Gb), items = n_chunks * G;
    const size_t a_row = (size_t)args.Hkv * Ga * D, b_row = (size_t)args.Hkv * Gb * D;  // elements per token
    auto chunk_t0 = [&](int n) { return t_begin + (reverse ? n_chunks - 1 - n : n) * kCh; };

    // the tiles of item `it` (chunk it / G, head it % G): into the buffer of its tile count; rows behind the last valid
    // token are zeros
    auto fetch = [&](int it) {
        const int n = it / G, x = it - n * G, t0 = chunk_t0(n), nv = min(kCh, v_end - t0);
        const int na = Ga > 1 ? it : n, nb = Gb > 1 ? it : n;
        const bool new_b = x == 0 || Gb > 1, new_a = !STATE_ONLY && (x == 0 || Ga > 1);
        const size_t tok = (size_t)bi * args.T + t0;
        for (int i = tid; i < kCh * (D / 4); i += kScanThreads) {
            const int tr = i / (D / 4), q4 = i - tr * (D / 4);
            const size_t row = tok + min(tr, nv - 1);
            if (new_a) copy16(&sm.a[na & 1][tr][4 * q4], ga + row * a_row + (size_t)(h * Ga + (Ga > 1 ? x : 0)) * D + 4 * q4, tr < nv);
            if (new_b) copy16(&sm.b[nb & 1][tr][4 * q4], gb + row * b_row + (size_t)(h * Gb + (Gb > 1 ? x : 0)) * D + 4 * q4, tr < nv);
        }
        if (new_b) {
            const int tr = tid / kCG, q4 = tid - tr * kCG;
            const size_t row = tok + min(tr, nv - 1);
            copy16(&sm.c[nb & 1][tr][4 * q4], gc + row * b_row + (size_t)(h * Gb + (Gb > 1 ? x : 0)) * D + col0 + 4 * q4, tr < nv);
        }
        cp_async_commit();
    };
    if (items > 0) fetch(0);
    fill_powers(sm.pw, args.log_decay[h], tid);

    const int cg = tid % kCG, rg = tid / kCG;
    const int cc = col0 + 4 * cg;                // this thread's four columns
    float4 S[kStateRows];                        // rows rg * kStateRows ..
#pragma unroll
    for (int i = 0; i < kStateRows; ++i) S[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (!STATE_ONLY) {
        const bool from_seg = args.nseg > 1;
        const float* src = from_seg ? r.seg + ((size_t)u * args.nseg + seg) * D * D
                                    : (r.state_in ? r.state_in + (size_t)u * D * D : nullptr);
        const float mul = from_seg ? 1.f : r.in_mul;
        if (src != nullptr) {
#pragma unroll
            for (int i = 0; i < kStateRows; ++i) {
                const int k = rg * kStateRows + i;
                if (!r.state_t) {
                    S[i] = mul4(mul, *reinterpret_cast<const float4*>(src + (size_t)k * D + cc));
                } else {
                    S[i] = make_float4(mul * src[(size_t)cc * D + k], mul * src[(size_t)(cc + 1) * D + k],
                                       mul * src[(size_t)(cc + 2) * D + k], mul * src[(size_t)(cc + 3) * D + k]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kStateRows; ++i)
            *reinterpret_cast<float4*>(&sm.s[rg * kStateRows + i][4 * cg]) = S[i];
    }

    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int it = 0; it < items; ++it) {
        const int n = it / G, x = it - n * G;
        const int t0 = chunk_t0(n), nv = min(kCh, v_end - t0);
        const int na = Ga > 1 ? it : n, nb = Gb > 1 ? it : n;
        const bool new_b = x == 0 || Gb > 1, new_a = x == 0 || Ga > 1;
        cp_async_wait_all();
        __syncthreads();  // this item's tiles are here, the item before has been read, the state is in place
        if (it + 1 < items) fetch(it + 1);
        float (*ta)[D + 4] = sm.a[na & 1], (*tb)[D + 4] = sm.b[nb & 1], (*tc)[kNc] = sm.c[nb & 1];
        if (!STATE_ONLY) {
            {   // products of all pairs: this thread row i, columns j, j + 8, j + 16, j + 24
                const int i = tid >> 3, j = tid & 7;
                float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
                for (int kk = 0; kk < D; kk += 4) {
                    const float4 av = *reinterpret_cast<const float4*>(&ta[i][kk]);
#pragma unroll
                    for (int m = 0; m < 4; ++m) s[m] = dot4(av, *reinterpret_cast<const float4*>(&tb[j + 8 * m][kk]), s[m]);
                }
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const int jj = j + 8 * m;
                    const int dist = reverse ? jj - i : i - jj;
                    sm.p[i][jj] = dist >= 0 ? s[m] * sm.pw[dist] : 0.f;
                }
            }
            // the state's share, once per (chunk, head of a); this thread's output row is rg
            if (new_a) {
                float4 in = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                for (int kk = 0; kk < D; kk += 4) {
                    const float4 av = *reinterpret_cast<const float4*>(&ta[rg][kk]);
                    in = fma4(av.x, *reinterpret_cast<const float4*>(&sm.s[kk][4 * cg]), in);
                    in = fma4(av.y, *reinterpret_cast<const float4*>(&sm.s[kk + 1][4 * cg]), in);
                    in = fma4(av.z, *reinterpret_cast<const float4*>(&sm.s[kk + 2][4 * cg]), in);
                    in = fma4(av.w, *reinterpret_cast<const float4*>(&sm.s[kk + 3][4 * cg]), in);
                }
                acc = mul4(sm.pw[reverse ? max(nv - 1 - rg, 0) : rg + 1], in);   // the distance to the state's token
            }
            __syncwarp();     // a warp's rows of P are its own: rows 4 w .. 4 w + 3, as its output rows are
#pragma unroll 8
            for (int j = 0; j < kCh; ++j) acc = fma4(sm.p[rg][j], *reinterpret_cast<const float4*>(&tc[j][4 * cg]), acc);
            if ((Ga > 1 || x == G - 1) && rg < nv)
                store4(go + ((size_t)bi * args.T + t0 + rg) * a_row + (size_t)(h * Ga + (Ga > 1 ? x : 0)) * D + cc, mul4(r.scale, acc));
            __syncwarp();     // P has been read
        }
        if (new_b) {
            if (x == 0) {
                const float f = sm.pw[nv];
#pragma unroll
                for (int i = 0; i < kStateRows; ++i) S[i] = mul4(f, S[i]);
            }
#pragma unroll 4
            for (int j = 0; j < nv; ++j) {
                const float w = sm.pw[reverse ? j + 1 : nv - 1 - j];
                const float4 cv = mul4(w, *reinterpret_cast<const float4*>(&tc[j][4 * cg]));
#pragma unroll
                for (int i = 0; i < kStateRows; ++i) S[i] = fma4(tb[j][rg * kStateRows + i], cv, S[i]);
            }
        }
        if (!STATE_ONLY && x == G - 1) {
            __syncthreads();  // the state in shared memory has been read
#pragma unroll
            for (int i = 0; i < kStateRows; ++i)
                *reinterpret_cast<float4*>(&sm.s[rg * kStateRows + i][4 * cg]) = S[i];
        }
    }

    if (STATE_ONLY) {   // into the slot of the segment that it feeds
        float* dst = st.seg[which] + ((size_t)u * args.nseg + (reverse ? seg - 1 : seg + 1)) * D * D;
#pragma unroll
        for (int i = 0; i < kStateRows; ++i)
            *reinterpret_cast<float4*>(dst + (size_t)(rg * kStateRows + i) * D + cc) = S[i];
        return;
    }
    if (r.state_out != nullptr && seg == (reverse ? 0 : args.nseg - 1)) {
        float* dst = r.state_out + (size_t)u * D * D;
#pragma unroll
        for (int i = 0; i < kStateRows; ++i) {
            const int k = rg * kStateRows + i;
            const float4 o = mul4(r.out_mul, S[i]);
            if (!r.state_t) {
                *reinterpret_cast<float4*>(dst + (size_t)k * D + cc) = o;
            } else {
                dst[(size_t)cc * D + k] = o.x;
                dst[(size_t)(cc + 1) * D + k] = o.y;
                dst[(size_t)(cc + 2) * D + k] = o.z;
                dst[(size_t)(cc + 3) * D + k] = o.w;
            }
        }
    }
    // padding rows of this segment: zeros
    const int pad0 = max(v_end, t_begin);
    for (int t = pad0 + rg; t < t_end; t += kRG)
        for (int x = 0; x < Ga; ++x)
            store4(go + ((size_t)bi * args.T + t) * a_row + (size_t)(h * Ga + x) * D + cc, make_float4(0.f, 0.f, 0.f, 0.f));
}

// The state each segment starts from: slot s holds what the segment before it (in the order of the scan) adds;
// the running sum decays by that segment's valid tokens.  One thread walks four elements over the segments.
__global__ void __launch_bounds__(256) linear_combine_kernel(const LinArgs args, const LinStates st, int DD) {
    const int dir = st.seg[0] == nullptr ? 1 : (int)blockIdx.z;
    const int u = blockIdx.x;
    const int e = (blockIdx.y * 256 + threadIdx.x) * 4;
    if (e >= DD) return;
    const int bi = u / args.Hkv, h = u - bi * args.Hkv;
    const int len = args.lens ? min(max(args.lens[bi], 0), args.T) : args.T;
    const double g = (double)args.log_decay[h];
    const float f_whole = (float)exp((double)args.seg_len * g);
    float* base = st.seg[dir] + (size_t)u * args.nseg * DD + e;
    float4 run = make_float4(0.f, 0.f, 0.f, 0.f);
    if (st.first[dir] != nullptr) run = mul4(st.in_mul[dir], *reinterpret_cast<const float4*>(st.first[dir] + (size_t)u * DD + e));
    const int step = dir ? -1 : 1, s0 = dir ? args.nseg - 1 : 0;   // segments in the order of the scan
    *reinterpret_cast<float4*>(base + (size_t)s0 * DD) = run;
    constexpr int kAhead = 8;   // what the next segments add is asked for together: the walk is a chain of additions, not of loads
    for (int n0 = 1; n0 < args.nseg; n0 += kAhead) {
        float4 add[kAhead];
        const int m = min(kAhead, args.nseg - n0);
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (i < m) add[i] = *reinterpret_cast<const float4*>(base + (size_t)(s0 + step * (n0 + i)) * DD);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (i >= m) break;
            const int s = s0 + step * (n0 + i), prev = s - step;
            const int nv = min(max(len - prev * args.seg_len, 0), args.seg_len);
            const float f = nv == 0 ? 1.f : (nv == args.seg_len ? f_whole : (float)exp((double)nv * g));
            run = make_float4(fmaf(f, run.x, add[i].x), fmaf(f, run.y, add[i].y), fmaf(f, run.z, add[i].z), fmaf(f, run.w, add[i].w));
            *reinterpret_cast<float4*>(base + (size_t)s * DD) = run;
        }
    }
}

// What every segment adds comes by head (slot s of a head: what segment s adds): the running sum in reverse over the
// segments and, in each, over the heads that share the state, in fp32 and in a fixed order.  Slot s of `seg`, where there
// is one, gets what segment s starts from, `last` what comes out of the first token.
__global__ void __launch_bounds__(256) linear_combine_heads_kernel(const LinArgs args, const LinStates st, int DD) {
    const int u = blockIdx.x;
    const int e = (blockIdx.y * 256 + threadIdx.x) * 4;
    if (e >= DD) return;
    const int bi = u / args.Hkv, h = u - bi * args.Hkv;
    const int len = args.lens ? min(max(args.lens[bi], 0), args.T) : args.T;
    const double g = (double)args.log_decay[h];
    const float* add = st.by_head + (size_t)u * st.heads * args.nseg * DD + e;
    float4 run = make_float4(0.f, 0.f, 0.f, 0.f);
    if (st.first[1] != nullptr) run = mul4(st.in_mul[1], *reinterpret_cast<const float4*>(st.first[1] + (size_t)u * DD + e));
    for (int s = args.nseg - 1; s >= 0; --s) {
        if (st.seg[1] != nullptr) *reinterpret_cast<float4*>(st.seg[1] + ((size_t)u * args.nseg + s) * DD + e) = run;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int x = 0; x < st.heads; ++x) {
            const float4 y = *reinterpret_cast<const float4*>(add + ((size_t)x * args.nseg + s) * DD);
            sum = make_float4(sum.x + y.x, sum.y + y.y, sum.z + y.z, sum.w + y.w);
        }
        const int nv = min(max(len - s * args.seg_len, 0), args.seg_len);
        run = fma4(nv == 0 ? 1.f : (float)exp((double)nv * g), run, sum);
    }
    *reinterpret_cast<float4*>(st.last + (size_t)u * DD + e) = mul4(st.last_mul, run);
}

// One token for every unit: S' = lambda S + k^T v, o_g = scale q_g S'.  Bound by the state's bytes (read and
// written once).  A block holds 32 columns of one unit's state (128-byte row pieces): eight lanes per row, so
// that a thread's rows are all asked for before the first is used, and four blocks share a unit, which fills the
// machine from about forty units on.  64 sequences of 32 heads of 128 (270 MB): 44 us, 6.1 TB/s, 0.93 of the copy rate; one
// sequence: 10 us a call, all of it the call's (its bytes take 0.2 us).
template <typename T, int D>
__global__ void __launch_bounds__(128) linear_step_kernel(const T* __restrict__ q, const T* __restrict__ k,
                                                          const T* __restrict__ v, const float* __restrict__ log_decay,
                                                          const float* state, float* state_out, T* __restrict__ out,
                                                          int Hkv, int G, float scale) {
    constexpr int kRows = D / 16;   // state rows of a thread
    constexpr int kGq = 8;          // query heads per round
    __shared__ float sq[kGq][D];
    __shared__ float sk[D];
    __shared__ float red[4][kGq][32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int nb = D / 32;
    const int u = blockIdx.x / nb, col0 = (blockIdx.x - u * nb) * 32;
    const int h = u % Hkv;
    const int cg = lane & 7;                     // four columns
    const int r0 = warp * 4 + (lane >> 3);       // rows r0, r0 + 16, ...
    const float* src = state + (size_t)u * D * D + col0 + 4 * cg;
    float4 S[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) S[i] = *reinterpret_cast<const float4*>(src + (size_t)(r0 + 16 * i) * D);
    const float4 vv = load4(v + (size_t)u * D + col0 + 4 * cg);
    const float lam = expf(log_decay[h]);
    for (int i = tid; i < D; i += 128) sk[i] = (float)k[(size_t)u * D + i];
    for (int g0 = 0; g0 < G; g0 += kGq) {
        const int ng = min(kGq, G - g0);
        if (g0 > 0) __syncthreads();
        for (int i = tid; i < ng * D; i += 128) sq[i / D][i % D] = (float)q[((size_t)u * G + g0) * D + i];
        __syncthreads();
        if (g0 == 0) {
            float* dst = state_out + (size_t)u * D * D + col0 + 4 * cg;
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                S[i] = fma4(sk[r0 + 16 * i], vv, mul4(lam, S[i]));
                *reinterpret_cast<float4*>(dst + (size_t)(r0 + 16 * i) * D) = S[i];
            }
        }
        for (int g = 0; g < ng; ++g) {
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int i = 0; i < kRows; ++i) o = fma4(sq[g][r0 + 16 * i], S[i], o);
#pragma unroll
            for (int m = 8; m < 32; m <<= 1) {
                o.x += __shfl_xor_sync(0xffffffffu, o.x, m);
                o.y += __shfl_xor_sync(0xffffffffu, o.y, m);
                o.z += __shfl_xor_sync(0xffffffffu, o.z, m);
                o.w += __shfl_xor_sync(0xffffffffu, o.w, m);
            }
            if (lane < 8) *reinterpret_cast<float4*>(&red[warp][g][4 * lane]) = o;
        }
        __syncthreads();
        for (int i = tid; i < ng * 32; i += 128) {
            const int g = i >> 5, c = i & 31;
            const float o = (red[0][g][c] + red[1][g][c]) + (red[2][g][c] + red[3][g][c]);
            out[((size_t)u * G + g0 + g) * D + col0 + c] = (T)(scale * o);
        }
    }
}

template <int D, bool STATE_ONLY>
cudaError_t launch_scan(const LinArgs& args, const LinStates& st, int grid_y, cudaStream_t stream) {
    auto fn = linear_scan_kernel<D, STATE_ONLY>;
    const int smem = (int)sizeof(ScanSmem<D>);
    static std::atomic<unsigned long long> allowed{0};
    cudaError_t e = allow_smem(reinterpret_cast<const void*>(fn), smem, allowed);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)(args.B * args.Hkv * args.nseg * (D / kNc)), (unsigned)grid_y);
    fn<<<grid, kScanThreads, smem, stream>>>(args, st);
    return cudaGetLastError();
}

template <int D>
cudaError_t scan_all(const LinArgs& args, const LinStates& st, cudaStream_t stream) {
    if (args.nseg > 1) {
        const int dirs = (st.seg[0] != nullptr) + (st.seg[1] != nullptr);
        cudaError_t e = launch_scan<D, true>(args, st, dirs, stream);
        if (e == cudaSuccess) e = launch_linear_combine(D, args, st, stream);
        if (e != cudaSuccess) return e;
    }
    return launch_scan<D, false>(args, st, args.n_roles, stream);
}

}  // namespace

cudaError_t launch_linear_combine(int D, const LinArgs& args, const LinStates& st, cudaStream_t stream) {
    const int dirs = (st.seg[0] != nullptr) + (st.seg[1] != nullptr);
    const dim3 grid((unsigned)(args.B * args.Hkv), (unsigned)((D * D / 4 + 255) / 256), (unsigned)dirs);
    linear_combine_kernel<<<grid, 256, 0, stream>>>(args, st, D * D);
    return cudaGetLastError();
}

cudaError_t launch_linear_combine_heads(int D, const LinArgs& args, const LinStates& st, cudaStream_t stream) {
    const dim3 grid((unsigned)(args.B * args.Hkv), (unsigned)((D * D / 4 + 255) / 256));
    linear_combine_heads_kernel<<<grid, 256, 0, stream>>>(args, st, D * D);
    return cudaGetLastError();
}

LinPlan lin_plan(const bct_linear_params_t& p, int64_t T, int kind) {
    LinPlan plan;
    plan.tensor = p.dtype == BCT_BF16;
    // Blocks of one segment, blocks that the machine holds, and the tokens that segments are multiples of.
    const int64_t ncol = plan.tensor ? 1 : p.head_dim / kNc;
    const int64_t roles = kind == 1 ? 3 : (kind == 3 ? 2 : 1), dirs = kind == 1 ? 2 : 1;
    const int64_t units = (int64_t)p.batch * p.n_kv_heads * ncol;
    const int64_t slots = plan.tensor ? 148 : 148 * 2, step = plan.tensor ? 128 : kCh;
    const int64_t steps = (T + step - 1) / step;
    const double G = p.n_q_heads / p.n_kv_heads;
    // A block's time in units of one (chunk, head) of the full scan; a block starts in `start` of them.  A split adds the
    // pass that forms the segments' states (per chunk and head of k about half of the full one's) and two launches.
    const double start = plan.tensor ? 3.0 : 1.0, part = plan.tensor ? 0.6 : 0.4, launches = plan.tensor ? 1.5 : 2.0;
    int64_t best = 1;
    double best_cost = 0;
    for (int64_t n = 1; n <= steps && n <= 64; ++n) {
        const int64_t len = (steps + n - 1) / n;
        if ((steps + len - 1) / len != n) continue;
        const double rounds = (double)((units * roles * n + slots - 1) / slots);
        double cost = rounds * ((double)len * G + start);
        if (n > 1) {
            const double before = (double)((units * dirs * (n - 1) + slots - 1) / slots);
            cost += before * ((double)len * (kind == 1 || kind == 3 ? G : 1.0) * part + start) + launches;
        }
        if (n == 1 || cost < best_cost) {
            best = n;
            best_cost = cost;
        }
    }
    const int64_t len = (steps + best - 1) / best;
    plan.nseg = (int)best;
    plan.seg_len = (int)(len * step);
    plan.seg_bytes = best > 1 ? (size_t)p.batch * p.n_kv_heads * best * p.head_dim * p.head_dim * sizeof(float) : 0;
    return plan;
}

cudaError_t launch_linear_step(const bct_linear_params_t& p, const void* q, const void* k, const void* v,
                               const float* log_decay, const float* state, float* state_out, void* out,
                               cudaStream_t stream) {
    const int G = p.n_q_heads / p.n_kv_heads;
    const unsigned grid = (unsigned)(p.batch * p.n_kv_heads * (p.head_dim / 32));
#define BCT_STEP(T, D)                                                                                               \
    linear_step_kernel<T, D><<<grid, 128, 0, stream>>>(static_cast<const T*>(q), static_cast<const T*>(k),           \
                                                       static_cast<const T*>(v), log_decay, state, state_out,        \
                                                       static_cast<T*>(out), p.n_kv_heads, G, p.scale)
    if (p.dtype == BCT_BF16) {
        if (p.head_dim == 128)
            BCT_STEP(__nv_bfloat16, 128);
        else
            BCT_STEP(__nv_bfloat16, 64);
    } else {
        if (p.head_dim == 128)
            BCT_STEP(float, 128);
        else
            BCT_STEP(float, 64);
    }
#undef BCT_STEP
    return cudaGetLastError();
}

cudaError_t launch_linear_scan(const bct_linear_params_t& p, const LinPlan& plan, const LinArgs& args,
                               const LinStates& states, cudaStream_t stream) {
    if (plan.tensor) return launch_linear_tc(p.head_dim, args, states, stream);
    return p.head_dim == 128 ? scan_all<128>(args, states, stream) : scan_all<64>(args, states, stream);
}

}  // namespace bct
