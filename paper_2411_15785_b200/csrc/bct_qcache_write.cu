// The 8-bit cache: quantised append, and eviction by accumulated attention weight.
//
// A block of 32 slots of a head has one scale s for its keys and one for its values; a code c stands for c s.
//   - A block that holds nothing takes s = amax / 127, rounded to float once, of what comes in: half a step off at most.
//   - A block that holds something keeps its s while amax <= 127.5 s (127.5 s still rounds to the code 127, half a step
//     off).  Otherwise s grows by the smallest power of two that makes room, and the codes held are divided by it: their
//     distance from the value halves before the new rounding, so that it stays below one step however often s grows.
//     (With s = amax / 127 at every growth each one adds up to half a step.)
// Codes are the correctly rounded x / s, ties to the even code: whatever computes them finds the same ones.
//
// Bound by HBM: an append reads and writes each token once, an eviction reads 8 bytes per slot and moves the slots that
// survive behind the new end into the holes before it, which is the least that can move: evicting n of C slots moves
// n (C - n) / C of them when they are spread evenly, an order-preserving compaction all that follow the first hole.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "bct_device.cuh"
#include "bct_internal.h"
#include "bct_qcache.h"

namespace bct {
namespace {

constexpr int kQwThreads = 256;   // four warps for the keys of a block, four for its values, eight slots a warp
constexpr int kQwRows = kQcBlock / 4;

// round((x + lo) / s) in -127..127, ties to the even code; |lo| is at most half an ulp of x.  q is off by one at most
// where x / s is next to a half; r = x - q s is exact there (multiples of s's ulp, or of half of it where q is 0 or 1,
// below s), and so are the differences from half a step that decide.
__device__ __forceinline__ float code_of(float x, float lo, float s, float inv) {
    float q = rintf(x * inv);
    const float r = fmaf(-q, s, x), half = 0.5f * s;
    const bool odd = (static_cast<int>(q) & 1) != 0;
    const float up = (r - half) + lo, down = (r + half) + lo;
    if (up > 0.f || (up == 0.f && odd)) q += 1.f;
    else if (down < 0.f || (down == 0.f && odd)) q -= 1.f;
    return fminf(fmaxf(q, -127.f), 127.f);
}

// The scale of a block that takes values up to amax, and the factor by which the codes it holds are multiplied.
__device__ __forceinline__ float grown(float s, double amax, bool fresh, float* shrink) {
    *shrink = 1.f;
    if (fresh || s == 0.f)
        return amax > 0. ? fmaxf((float)(amax / 127.), 1.17549435e-38f) : (float)amax;   // (a NaN stays one)
    const double top = 127.5 * (double)s;
    if (!(amax > top)) return amax == amax ? s : (float)amax;
    int e;
    const double m = frexp(amax / top, &e);
    if (!(m > 0.5)) --e;
    *shrink = ldexpf(1.f, -e);
    return ldexpf(s, e);
}

template <typename T, int N>
struct Row;   // N features of a lane
template <int N>
struct Row<float, N> {
    float x[N];
    __device__ __forceinline__ void load(const float* p) {
        if constexpr (N == 4) {
            const float4 w = *reinterpret_cast<const float4*>(p);
            x[0] = w.x, x[1] = w.y, x[2] = w.z, x[3] = w.w;
        } else {
            const float2 w = *reinterpret_cast<const float2*>(p);
            x[0] = w.x, x[1] = w.y;
        }
    }
};
template <int N>
struct Row<__nv_bfloat16, N> {
    float x[N];
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        uint32_t w[N / 2];
        if constexpr (N == 4) {
            const uint2 u = *reinterpret_cast<const uint2*>(p);
            w[0] = u.x, w[1] = u.y;
        } else {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        }
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
};

// N codes of a lane, as the N bytes of a word
template <int N>
__device__ __forceinline__ uint32_t load_codes(const int8_t* p) {
    if constexpr (N == 4) return *reinterpret_cast<const uint32_t*>(p);
    else return *reinterpret_cast<const uint16_t*>(p);
}
template <int N>
__device__ __forceinline__ void store_codes(int8_t* p, const float* c) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) w |= (uint32_t)(uint8_t)(int8_t)(int)c[i] << (8 * i);
    if constexpr (N == 4) *reinterpret_cast<uint32_t*>(p) = w;
    else *reinterpret_cast<uint16_t*>(p) = (uint16_t)w;
}
__device__ __forceinline__ float code_at(uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); }

// Largest magnitude of a plane's four warps (64 bits: a code times a scale has 31); a NaN or an infinity in any of them
// makes it a NaN.
__device__ __forceinline__ double plane_amax(double mine, bool odd_one, double (*share)[4], int plane, int part) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine = fmax(mine, __shfl_xor_sync(0xffffffffu, mine, o));
    if (__any_sync(0xffffffffu, odd_one)) mine = nan("");
    if ((threadIdx.x & 31) == 0) share[plane][part] = mine;
    __syncthreads();
    double amax = 0.;
    bool is_nan = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const double m = share[plane][i];
        is_nan |= m != m;
        amax = fmax(amax, m);
    }
    return is_nan ? nan("") : amax;
}
__device__ __forceinline__ bool not_finite(float x) { return !(fabsf(x) <= 3.402823466e38f); }

// ---- append -----------------------------------------------------------------------------------------------------
// A CTA per (sequence, head, block of the cache that the new tokens may touch).  The last CTA of a sequence moves its
// length on: all of them have read it by then.
template <typename T, int D>
__global__ void __launch_bounds__(kQwThreads) qc_append_kernel(const QcAppend a) {
    constexpr int kN = D / 32;
    __shared__ double share[2][4];
    const int w = blockIdx.x % a.W, unit = blockIdx.x / a.W, b = unit / a.c.Hkv, h = unit - b * a.c.Hkv;
    const int C = a.c.C;
    const int held = min(max(a.c.state[b], 0), C), seen = a.c.state[a.c.B + b];
    const int64_t want = a.lens == nullptr ? a.T : min((int64_t)max(a.lens[b], 0), a.T);
    const int n = (int)min(want, (int64_t)(C - held));
    const int blk = held / kQcBlock + w, lo = blk * kQcBlock;
    if (lo < held + n && n > 0) {
        const int plane = threadIdx.x >> 7, part = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31;
        const int first = max(held, lo), last = min(held + n, lo + kQcBlock);   // the new slots of this block
        int8_t* codes = a.c.codes[plane] + (size_t)unit * C * D;
        float* scale = a.c.scale[plane] + (size_t)unit * a.c.NB + blk;
        const T* x = static_cast<const T*>(a.x[plane]);
        Row<T, kN> row[kQwRows];
        float top = 0.f;
        bool odd_one = false;
#pragma unroll
        for (int i = 0; i < kQwRows; ++i) {
            const int slot = lo + part * kQwRows + i;
            if (slot < first || slot >= last) continue;
            row[i].load(x + (((size_t)b * a.T + (slot - held)) * a.c.Hkv + h) * D + lane * kN);
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                top = fmaxf(top, fabsf(row[i].x[j]));
                odd_one |= not_finite(row[i].x[j]);
            }
        }
        const float old = *scale;
        // (all have read the old scale when its barrier lets them go)
        const double amax = plane_amax(top, odd_one, share, plane, part);
        float shrink;
        const float s = grown(old, amax, first == lo, &shrink), inv = s > 0.f ? 1.f / s : 0.f;
#pragma unroll
        for (int i = 0; i < kQwRows; ++i) {
            const int slot = lo + part * kQwRows + i;
            int8_t* p = codes + (size_t)slot * D + lane * kN;
            float c[kN];
            if (slot >= first && slot < last) {
#pragma unroll
                for (int j = 0; j < kN; ++j) c[j] = s > 0.f ? code_of(row[i].x[j], 0.f, s, inv) : 0.f;
                store_codes<kN>(p, c);
            } else if (slot < first && shrink != 1.f) {
                const uint32_t word = load_codes<kN>(p);
#pragma unroll
                for (int j = 0; j < kN; ++j) c[j] = rintf(code_at(word, j) * shrink);
                store_codes<kN>(p, c);
            }
        }
        if (part == 0 && lane == 0) *scale = s;
        if (plane == 0 && part == 0) {
            const int slot = lo + lane;
            if (slot >= first && slot < last) {
                a.c.weight[(size_t)unit * C + slot] = 0.f;
                a.c.position[(size_t)unit * C + slot] = seen + (slot - held);
            }
        }
    }
    __syncthreads();   // (all of this CTA have read the sequence's state)
    if (threadIdx.x == 0) {
        __threadfence();
        int* done = reinterpret_cast<int*>(a.c.state + 2 * a.c.B + b);
        if (atomicAdd(done, 1) == a.W * a.c.Hkv - 1) {
            a.c.state[b] = held + n;
            a.c.state[a.c.B + b] = seen + n;
            *done = 0;
        }
    }
}

// ---- eviction ---------------------------------------------------------------------------------------------------
constexpr int kQsThreads = 1024;
constexpr int kQsWarps = kQsThreads / 32;
constexpr int kQsBins = 2048;          // 11 bits of a key at a time
constexpr int kQsKeys = 40960;         // keys that are kept in shared memory; those behind are formed anew

// Floats in their order, as integers; slots that stay in any case come last.
__device__ __forceinline__ uint32_t worth_key(float w, bool stays) {
    if (stays || w != w) return stays ? 0xffffffffu : 0xfffffffeu;
    const uint32_t u = __float_as_uint(w + 0.f);   // (-0 is 0)
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

// Inclusive sum over the CTA's threads in order, and the total.  share: kQsWarps + 1 words.
__device__ __forceinline__ int cta_scan(int x, int* share, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) share[warp] = x;
    __syncthreads();
    if (warp == 0) {
        int y = share[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int z = __shfl_up_sync(0xffffffffu, y, o);
            if (lane >= o) y += z;
        }
        share[lane] = y;
    }
    __syncthreads();
    *total = share[kQsWarps - 1];
    return x + (warp ? share[warp - 1] : 0);
}

// A CTA per unit finds the n least keys: 11 + 11 + 10 bits of the n-th one, by counting; then one pass in the slots'
// order, in which a warp is a block, lists the blocks with holes and the slots that move.
__global__ void __launch_bounds__(kQsThreads) qc_select_kernel(const QcEvict a) {
    extern __shared__ uint32_t keys[];
    __shared__ int bins[kQsBins];
    __shared__ int share[kQsWarps + 1];
    __shared__ int found[2];
    const int unit = blockIdx.x, b = unit / a.c.Hkv, C = a.c.C, tid = threadIdx.x, lane = tid & 31;
    const int held = min(max(a.c.state[b], 0), C), from = a.c.state[a.c.B + b] - a.recent;
    const int n = held - a.keep;
    if (n <= 0) {
        if (tid == 0) a.n_out[unit] = a.n_blocks[unit] = 0;
        return;
    }
    const float* weight = a.c.weight + (size_t)unit * C;
    const int32_t* position = a.c.position + (size_t)unit * C;
    const int kept_keys = min(held, kQsKeys);
    for (int j = tid; j < kept_keys; j += kQsThreads) keys[j] = worth_key(weight[j], position[j] >= from);
    auto key_at = [&](int j) { return j < kQsKeys ? keys[j] : worth_key(weight[j], position[j] >= from); };

    uint32_t prefix = 0, mask = 0;
    int left = n;                          // of the keys that share the prefix, so many go
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
        bins[tid] = bins[tid + kQsThreads] = 0;
        __syncthreads();
        for (int j = tid; j < held; j += kQsThreads) {
            const uint32_t k = key_at(j);
            if ((k & mask) == prefix) atomicAdd(&bins[(k >> shift) & ((1u << width) - 1)], 1);
        }
        __syncthreads();
        const int c0 = bins[2 * tid], c1 = bins[2 * tid + 1];
        int total;
        const int upto = cta_scan(c0 + c1, share, &total), before = upto - c0 - c1;
        if (before < left && left <= upto) {
            const bool second = left > before + c0;
            found[0] = 2 * tid + second;
            found[1] = left - before - (second ? c0 : 0);
        }
        __syncthreads();
        prefix |= (uint32_t)found[0] << shift;
        left = found[1];
        mask |= ((1u << width) - 1) << shift;
        __syncthreads();
    }

    int4* blocks = a.blocks + (size_t)unit * a.max_blocks;
    int32_t* movers = a.movers + (size_t)unit * a.max_moves;
    int ties = 0, n_holes = 0, n_movers = 0, n_blocks = 0;
    for (int base = 0; base < held; base += kQsThreads) {
        const int j = base + tid;
        const uint32_t k = j < held ? key_at(j) : 0xffffffffu;
        const bool tie = j < held && k == prefix;
        int total;
        const int tie_no = ties + cta_scan(tie, share, &total) - 1;
        ties += total;
        const bool out = j < held && (k < prefix || (tie && tie_no < left));
        const bool hole = out && j < a.keep, mover = !out && j >= a.keep && j < held;
        // what comes before, of both kinds: a slot is one of them at most
        const int no = cta_scan(hole ? 1 : mover ? 1 << 16 : 0, share, &total);
        if (mover) movers[n_movers + (no >> 16) - 1] = j;
        const unsigned holes = __ballot_sync(0xffffffffu, hole);
        const int hole_no = n_holes + (__shfl_sync(0xffffffffu, no, 31) & 0xffff) - __popc(holes);
        n_holes += total & 0xffff;
        n_movers += total >> 16;
        const int blk_no = n_blocks + cta_scan(lane == 0 && holes != 0, share, &total) - 1;
        if (lane == 0 && holes != 0) blocks[blk_no] = make_int4(j / kQcBlock, hole_no, (int)holes, 0);
        n_blocks += total;
    }
    if (tid < 2 && a.keep < C) a.cut_scale[2 * unit + tid] = a.c.scale[tid][(size_t)unit * a.c.NB + a.keep / kQcBlock];
    if (tid == 0) {
        a.n_out[unit] = n;
        a.n_blocks[unit] = n_blocks;
    }
}

// A CTA per block with holes: the slots that move in come with the codes and scale of where they were.
template <int D>
__global__ void __launch_bounds__(kQwThreads) qc_move_kernel(const QcEvict a, int ctas) {
    constexpr int kN = D / 32;
    __shared__ double share[2][4];
    const int no = blockIdx.x % ctas, unit = blockIdx.x / ctas, C = a.c.C;
    if (no == 0 && unit % a.c.Hkv == 0 && threadIdx.x == 0 && a.n_out[unit] > 0) a.c.state[unit / a.c.Hkv] = a.keep;
    if (no >= a.n_blocks[unit]) return;
    const int4 e = a.blocks[(size_t)unit * a.max_blocks + no];
    const int lo = e.x * kQcBlock;
    const unsigned holes = (unsigned)e.z;
    const int32_t* movers = a.movers + (size_t)unit * a.max_moves + e.y;
    const int plane = threadIdx.x >> 7, part = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31;
    int8_t* codes = a.c.codes[plane] + (size_t)unit * C * D;
    float* scales = a.c.scale[plane] + (size_t)unit * a.c.NB;
    // (the block that the new end cuts takes slots in and gives some away: its scale is the one before)
    auto scale_of = [&](int src) { return src / kQcBlock == a.keep / kQcBlock ? a.cut_scale[2 * unit + plane] : scales[src / kQcBlock]; };
    const int kept = min(kQcBlock, a.keep - lo);
    const bool fresh = holes == (kept == kQcBlock ? 0xffffffffu : (1u << kept) - 1u);

    uint32_t word[kQwRows];
    float from[kQwRows];
    double amax = 0.;
    bool odd_one = false;
#pragma unroll
    for (int i = 0; i < kQwRows; ++i) {
        const int at = part * kQwRows + i;
        if (!((holes >> at) & 1)) continue;
        const int src = movers[__popc(holes & ((1u << at) - 1u))];
        from[i] = scale_of(src);
        word[i] = load_codes<kN>(codes + (size_t)src * D + lane * kN);
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < kN; ++j) top = fmaxf(top, fabsf(code_at(word[i], j)));
        amax = fmax(amax, (double)top * (double)from[i]);
        odd_one |= not_finite(from[i]);
    }
    const float old = scales[e.x];
    amax = plane_amax(amax, odd_one, share, plane, part);
    float shrink;
    const float s = grown(old, amax, fresh, &shrink), inv = s > 0.f ? 1.f / s : 0.f;
#pragma unroll
    for (int i = 0; i < kQwRows; ++i) {
        const int at = part * kQwRows + i, slot = lo + at;
        if (at >= kept) continue;
        int8_t* p = codes + (size_t)slot * D + lane * kN;
        float c[kN];
        if ((holes >> at) & 1) {
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                const float code = code_at(word[i], j), x = code * from[i];
                c[j] = s > 0.f ? code_of(x, fmaf(code, from[i], -x), s, inv) : 0.f;
            }
            store_codes<kN>(p, c);
        } else if (shrink != 1.f) {
            const uint32_t held = load_codes<kN>(p);
#pragma unroll
            for (int j = 0; j < kN; ++j) c[j] = rintf(code_at(held, j) * shrink);
            store_codes<kN>(p, c);
        }
    }
    if (part == 0 && lane == 0) scales[e.x] = s;
    if (plane == 0 && part == 0 && ((holes >> lane) & 1)) {
        const int src = movers[__popc(holes & ((1u << lane) - 1u))];
        const size_t u = (size_t)unit * C;
        a.c.weight[u + lo + lane] = a.c.weight[u + src];
        a.c.position[u + lo + lane] = a.c.position[u + src];
    }
}

}  // namespace

cudaError_t qc_append(const QcAppend& a, int dtype, cudaStream_t s) {
    const unsigned grid = (unsigned)((int64_t)a.c.B * a.c.Hkv * a.W);
    if (dtype == BCT_BF16) {
        if (a.c.D == 128) qc_append_kernel<__nv_bfloat16, 128><<<grid, kQwThreads, 0, s>>>(a);
        else qc_append_kernel<__nv_bfloat16, 64><<<grid, kQwThreads, 0, s>>>(a);
    } else {
        if (a.c.D == 128) qc_append_kernel<float, 128><<<grid, kQwThreads, 0, s>>>(a);
        else qc_append_kernel<float, 64><<<grid, kQwThreads, 0, s>>>(a);
    }
    return cudaGetLastError();
}

cudaError_t qc_evict(const QcEvict& a, cudaStream_t s) {
    const int units = a.c.B * a.c.Hkv;
    const int smem = (a.c.C < kQsKeys ? a.c.C : kQsKeys) * 4;
    cudaError_t e = cudaFuncSetAttribute(qc_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kQsKeys * 4);
    if (e != cudaSuccess) return e;
    qc_select_kernel<<<units, kQsThreads, smem, s>>>(a);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    const int ctas = a.max_blocks > 0 ? a.max_blocks : 1;
    const unsigned grid = (unsigned)((int64_t)units * ctas);
    if (a.c.D == 128) qc_move_kernel<128><<<grid, kQwThreads, 0, s>>>(a, ctas);
    else qc_move_kernel<64><<<grid, kQwThreads, 0, s>>>(a, ctas);
    return cudaGetLastError();
}

}  // namespace bct
