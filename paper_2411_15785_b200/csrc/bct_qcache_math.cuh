// What the attention kernels of the 8-bit cache share on the device: what a row is and sees, codes and queries as fp16,
// scores.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "bct_device.cuh"
#include "bct_qcache.h"

namespace bct {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }
// a pair of bytes of `w` (each a code + 128), chosen by `sel`, as fp16
__device__ __forceinline__ uint32_t pair_of(uint32_t w, uint32_t sel) {
    const uint32_t u = prmt(w, 0x64646464u, sel);
    const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&u), __half2half2(__ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t half2_bits(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 half2_floats(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }
__device__ __forceinline__ void cp_async16_zfill(uint32_t dst, const void* src, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
// What a row sees: rows of a unit are (token, head), token-major.
struct Sees {
    int held, n, G;   // slots held, valid tokens
    int64_t R;        // (below 2^31)
    __device__ __forceinline__ int operator()(int64_t r) const {
        if (r >= R) return 0;
        const int i = (int)((unsigned)r / (unsigned)G);
        return i < n ? max(held - n + i + 1, 0) : 0;
    }
};
__device__ __forceinline__ Sees sees_of(const QcAttend& a, int b) {
    Sees s;
    s.held = min(max(a.c.state[b], 0), a.c.C);
    s.n = (int)(a.lens == nullptr ? a.T : min((int64_t)max(a.lens[b], 0), a.T));
    s.G = a.G;
    s.R = a.R;
    return s;
}
// B sequences have size_of(b) things each, per_seq times over.  Thing x of them all: its sequence, how many stand before that
// one, and the total, which x is made of by `where`; x = total has no sequence.  Up to 32 sequences are a warp's own affair; more are added up by the CTA, which then calls
// this with all its threads (upto: a word for each).
template <typename S, typename F>
__device__ __forceinline__ int64_t find_share(int B, S size_of, int64_t per_seq, int64_t* upto, F where, int64_t* x, int* seq,
                                              int64_t* before) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (B <= 32) {
        int64_t sum = lane < B ? size_of(lane) : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += y;
        }
        const int64_t total = __shfl_sync(0xffffffffu, sum, 31) * per_seq;
        *x = where(total);
        const int behind = __popc(__ballot_sync(0xffffffffu, sum * per_seq <= *x));   // sequences that end before it
        *seq = behind;
        *before = behind ? __shfl_sync(0xffffffffu, sum, behind - 1 & 31) * per_seq : 0;
        return total;
    }
    const int chunk = (B + blockDim.x - 1) / blockDim.x;
    int64_t sum = 0;
    for (int i = 0; i < chunk; ++i)
        if (tid * chunk + i < B) sum += size_of(tid * chunk + i);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += y;
    }
    __shared__ int64_t warps[32];
    if (lane == 31) warps[warp] = sum;
    __syncthreads();
    for (int i = 0; i < warp; ++i) sum += warps[i];
    upto[tid] = sum;
    __syncthreads();
    const int64_t total = upto[blockDim.x - 1] * per_seq;
    *x = where(total);
    if (*x >= total) return total;
    int lo = 0, hi = blockDim.x - 1;               // first thread's share that ends behind x
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (upto[mid] * per_seq > *x) hi = mid; else lo = mid + 1;
    }
    *seq = lo * chunk;
    *before = (lo ? upto[lo - 1] : 0) * per_seq;
    for (;;) {
        const int64_t nb = size_of(*seq);
        if (*before + nb * per_seq > *x) break;
        *before += nb * per_seq;
        ++*seq;
    }
    return total;
}
template <typename T>
__device__ __forceinline__ const T* row_of(const QcAttend& a, const void* base, int b, int h, int64_t r) {
    const unsigned i = (unsigned)r / (unsigned)a.G, head = (unsigned)h * a.G + ((unsigned)r - i * a.G);
    return static_cast<const T*>(base) + (((int64_t)b * a.T + i) * ((int64_t)a.c.Hkv * a.G) + head) * a.c.D;
}

// The power of two that brings a row whose largest magnitude is `top` into [2^14, 2^15), from 2^-113 to 2^126, and its
// inverse; rows of zeros, infinities or NaN are left as they are.
__device__ __forceinline__ void row_scale(float top, float* by, float* back) {
    const int e = (int)(__float_as_uint(top) >> 23) - 127;
    const int up = e > -127 && e < 128 ? min(14 - e, 126) : 0;
    *by = __uint_as_float((uint32_t)(up + 127) << 23);
    *back = __uint_as_float((uint32_t)(127 - up) << 23);
}
// what a row's products are multiplied with, besides the block's scale
__device__ __forceinline__ float row_factor(const QcAttend& a, float mul) {
    return a.cap > 0.f ? mul * (a.scale / a.cap) : mul * (a.scale * kLog2e);
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}

// tanh.  Up to 1, x times a polynomial in x^2 whose largest relative error is least (5e-8; fitted to tanh(x) / x by weighted
// least squares; with its roundings 1.6e-7); beyond, (e - 1) / (e + 1) with e = exp(2 |x|), where nothing cancels.  Scores are
// rarely that close to the cap, so that warps ask once for many of them whether all are up to 1.
__device__ __forceinline__ float tanh_near(float x) {
    const float y = x * x;
    float p = fmaf(y, 0.001041022245772183f, -0.006203378085047007f);
    p = fmaf(y, p, 0.020289979875087738f);
    p = fmaf(y, p, -0.05345702916383743f);
    p = fmaf(y, p, 0.13325203955173492f);
    p = fmaf(y, p, -0.33332839608192444f);
    return x * fmaf(y, p, 0.9999999403953552f);
}
// two at a time (there are instructions for pairs of floats)
__device__ __forceinline__ uint64_t f2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ void tanh_near2(float& a, float& b) {
    auto both = [](float c) { return f2(c, c); };
    const uint64_t x = f2(a, b), y = mul2(x, x);
    uint64_t p = fma2(y, both(0.001041022245772183f), both(-0.006203378085047007f));
    p = fma2(y, p, both(0.020289979875087738f));
    p = fma2(y, p, both(-0.05345702916383743f));
    p = fma2(y, p, both(0.13325203955173492f));
    p = fma2(y, p, both(-0.33332839608192444f));
    p = mul2(x, fma2(y, p, both(0.9999999403953552f)));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p));
}
__device__ __forceinline__ float tanh_any(float x) {
    if (!(fabsf(x) > 1.f)) return tanh_near(x);   // (a NaN too)
    const float e = ex2(fminf(fabsf(x), 16.f) * (2.f * kLog2e));
    return copysignf(__fdividef(e - 1.f, e + 1.f), x);
}

}  // namespace bct
