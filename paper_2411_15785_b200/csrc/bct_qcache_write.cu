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

#include <algorithm>

#include "bct_device.cuh"
#include "bct_internal.h"
#include "bct_qcache.h"
#include "bct_qcache.cuh"

namespace bct {
namespace {

constexpr int kQwThreads = 256;   // four warps for the keys of a block, four for its values, eight slots a warp
constexpr int kQwRows = kQcBlock / 4;

// round((x + lo) / s) in -127..127, ties to the even code; |lo| is at most half an ulp of x.  q is off by one at most
// where x / s is next to a half; r = x - q s is exact there (multiples of s's ulp, or of half of it where q is 0 or 1,
// below s), and so are the differences of 2 r from s that decide (half of s is no float where s is among the smallest).
__device__ __forceinline__ int exact_code(float x, float lo, float s, float inv) {
    float q = rintf(x * inv);
    const float r = fmaf(-q, s, x);
    const bool odd = (static_cast<int>(q) & 1) != 0;
    const float up = fmaf(2.f, lo, fmaf(2.f, r, -s)), down = fmaf(2.f, lo, fmaf(2.f, r, s));
    if (up > 0.f || (up == 0.f && odd)) q += 1.f;
    else if (down < 0.f || (down == 0.f && odd)) q -= 1.f;
    return static_cast<int>(fminf(fmaxf(q, -127.f), 127.f));
}
__device__ __forceinline__ uint32_t packed(const uint32_t (&u)[4]) {   // the low bytes
    return __byte_perm(__byte_perm(u[0], u[1], 0x0040), __byte_perm(u[2], u[3], 0x0040), 0x5410);
}
// Four codes as the bytes of a word.  Adding 1.5 2^23 rounds x / s to an integer, whose low byte is the code; *far is the
// largest distance from it: only next to a half can it be the wrong one.  x, a code times a scale, and inv are rounded, 2^-24 of
// themselves each, so that x inv is off by 127.5 2^-23 = 1.52e-5 at most, and the distance by 2^-25 more: up to kNextToHalf =
// 0.5 - 2e-5 the integer is the right one.  127 too is the largest then: a quotient is 127.5 at most, where 128 is further off.
__device__ __forceinline__ uint32_t codes_of(const float* x, float inv, float* far) {
    constexpr float kMagic = 12582912.f;
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float m = fmaf(x[i], inv, kMagic);
        u[i] = __float_as_uint(m);
        *far = fmaxf(*far, fabsf(fmaf(x[i], inv, kMagic - m)));
    }
    return packed(u);
}
// Four codes of x itself.  With q the rounded x inv, r = x - q s is exact next to half a step (multiples of s's ulp or of half
// of it): 2 r against s decides whether the neighbour is right, which is one apart.  `edge` is s, or infinity where it is 0.
__device__ __forceinline__ uint32_t new_codes(const float* x, float inv, float s, float edge) {
    constexpr float kMagic = 12582912.f;
    float m[4], far = 0.f;
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = fmaf(x[i], inv, kMagic);
        u[i] = __float_as_uint(m[i]);
        far = fmaxf(far, fabsf(fmaf(kMagic - m[i], s, x[i])));
    }
    if (2.f * far >= edge) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float r = fmaf(kMagic - m[i], s, x[i]), over = fmaf(2.f, fabsf(r), -s);
            if (over > 0.f || (over == 0.f && (u[i] & 1))) u[i] += r > 0.f ? 1 : -1;
            u[i] = min(max(u[i], 0x4b400000u - 127u), 0x4b400000u + 127u);   // 127.5 s would be 128
        }
    }
    return packed(u);
}
// The exact ones of x + lo (out of the way of the loops that rarely need them).
__device__ __noinline__ uint32_t exact_codes(float4 x, float4 lo, float s, float inv) {
    const uint32_t u[4] = {(uint32_t)exact_code(x.x, lo.x, s, inv), (uint32_t)exact_code(x.y, lo.y, s, inv),
                           (uint32_t)exact_code(x.z, lo.z, s, inv), (uint32_t)exact_code(x.w, lo.w, s, inv)};
    return packed(u);
}
constexpr float kNextToHalf = 0.49998f;
// Code i of a word as a float (and no conversion, of which there are few to a clock): the byte + 128 under the exponent of 2^23
__device__ __forceinline__ float code_at(uint32_t w, int i) {
    return __uint_as_float(__byte_perm(w ^ 0x80808080u, 0x4b000000u, 0x7440 | i)) - 8388736.f;
}
// The largest magnitude of the codes of a word, -127..127.
__device__ __forceinline__ unsigned top_code(uint32_t w) {
    const uint32_t minus = (w >> 7) & 0x01010101u, a = (w ^ (minus * 0xffu)) + minus;
    const uint32_t two = __vmaxu2(a & 0x00ff00ffu, (a >> 8) & 0x00ff00ffu);
    return max(two & 0xffffu, two >> 16);
}
// Four codes divided by a power of two, ties to the even one.
__device__ __forceinline__ uint32_t shrunk(uint32_t w, float by) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(fmaf(code_at(w, i), by, 12582912.f));
    return packed(u);
}

// The scale of a block that takes values up to amax, and the factor by which the codes it holds are multiplied.  64 bits
// only where they decide: in a block that starts afresh from products of codes and scales, and where a scale grows.
template <typename F>
__device__ __forceinline__ float grown(float s, F amax, bool fresh, float* shrink) {
    *shrink = 1.f;
    if (fresh || s == 0.f) return amax > F(0) ? fmaxf((float)(amax / F(127)), 1.17549435e-38f) : (float)amax;   // (a NaN stays one)
    if ((float)amax < 127.4f * s) return s;
    const double top = 127.5 * (double)s;
    if (!((double)amax > top)) return amax == amax ? s : (float)amax;
    int e;
    const double m = frexp((double)amax / top, &e);
    if (!(m > 0.5)) --e;
    *shrink = ldexpf(1.f, -e);
    return ldexpf(s, e);
}

// Eight lanes share a row.  Of the features of new tokens a lane has 16 bytes in each 128 of the row (kE of them, whose codes
// it stores together); of a row of codes, D / 8.
template <typename T>
struct Piece {
    static constexpr int kE = 16 / (int)sizeof(T);
    uint4 w;
    // the largest magnitude, as the bits of a float (which are in its order; a NaN's and an infinity's come last); of
    // bfloat16 in both halves of the word
    __device__ __forceinline__ uint32_t top(uint32_t so_far) const {
        if constexpr (sizeof(T) == 4)
            return max(max(so_far, w.x & 0x7fffffffu), max(w.y & 0x7fffffffu, max(w.z & 0x7fffffffu, w.w & 0x7fffffffu)));
        else
            return __vmaxu2(__vmaxu2(so_far, w.x & 0x7fff7fffu), __vmaxu2(w.y & 0x7fff7fffu, __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu)));
    }
    __device__ __forceinline__ static uint32_t top_of(uint32_t t) { return sizeof(T) == 4 ? t : max(t << 16, t & 0xffff0000u); }
};
template <int N>
__device__ __forceinline__ void load_words(const int8_t* p, uint32_t (&w)[N]) {
    if constexpr (N == 4) {
        const uint4 u = *reinterpret_cast<const uint4*>(p);
        w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
    } else if constexpr (N == 2) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        w[0] = u.x, w[1] = u.y;
    } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
}
template <int N>
__device__ __forceinline__ void store_words(int8_t* p, const uint32_t (&w)[N]) {
    if constexpr (N == 4) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else if constexpr (N == 2) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(p) = w[0];
}

// Largest magnitude (its bits) of a plane's four warps, as a float; a NaN or an infinity in any of them makes it a NaN.
__device__ __forceinline__ float plane_amax(uint32_t mine, uint32_t (*share)[4], int plane, int part) {
    mine = __reduce_max_sync(0xffffffffu, mine);
    if ((threadIdx.x & 31) == 0) share[plane][part] = mine;
    __syncthreads();
    const uint32_t amax = max(max(share[plane][0], share[plane][1]), max(share[plane][2], share[plane][3]));
    return __uint_as_float(amax < 0x7f800000u ? amax : 0x7fffffffu);
}

// ---- append -----------------------------------------------------------------------------------------------------
// A few CTAs per (sequence, head) go through the blocks that its new tokens touch, the next block's tokens on their way while
// this one's are worked on.  The last CTA of a sequence to have read its length moves it on.
// A fill of 8 sequences by up to 4096 tokens of 8 heads of 128: 39 us = 3.3 TB/s, half of a copy's rate.  What it spends is
// instructions (some 17 for a value, of which the codes 8) more than bytes.  A warp to a plane of a block instead of four needs
// a third fewer, but all of the registers, and took 46 us; two warps 38.
constexpr int kQwResident = 4;    // CTAs on an SM
template <typename T, int D>
__global__ void __launch_bounds__(kQwThreads, sizeof(T) == 2 ? kQwResident : 2) qc_append_kernel(const QcAppend a) {
    constexpr int kE = Piece<T>::kE, kC = D * (int)sizeof(T) / 128;   // pieces of a lane in a row
    constexpr int kTurns = kQwRows / 4, kW = D / 32;                  // turns of four rows; words of a lane in a row of codes
    __shared__ uint32_t share[2][2][4];
    pdl_wait();
    pdl_open();
    // the heads of a block of tokens run side by side: they stand side by side in memory
    const int h = blockIdx.x % a.c.Hkv, bw = blockIdx.x / a.c.Hkv, w0 = bw % a.ctas, b = bw / a.ctas, unit = b * a.c.Hkv + h;
    const int C = a.c.C;
    const int held = min(max(a.c.state[b], 0), C), seen = a.c.state[a.c.B + b];
    const int64_t want = a.lens == nullptr ? a.T : min((int64_t)max(a.lens[b], 0), a.T);
    const int n = (int)min(want, (int64_t)(C - held)), end = held + n;
    const int plane = threadIdx.x >> 7, part = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31, l8 = lane & 7;
    const int blk_end = n > 0 ? (end - 1) / kQcBlock + 1 : 0;
    __syncthreads();          // all of this CTA have the sequence's state (their bounds are made of it)

    const int row_in = part * kQwRows + (lane >> 3);          // the lane's rows of a block: this one, and 4 further on at each turn
    const int64_t step = 4 * (int64_t)a.c.Hkv * D;
    const T* const x0 = static_cast<const T*>(a.x[plane]) + ((int64_t)b * a.T * a.c.Hkv + h) * D + l8 * kE;
    float* const scales = a.c.scale[plane] + (size_t)unit * a.c.NB;
    Piece<T> ahead[kTurns][kC];
    float old_ahead = 0.f;
    auto fetch = [&](int blk) {
        if (blk >= blk_end) return;
        const int row0 = blk * kQcBlock + row_in;
        const T* x = x0 + (int64_t)(row0 - held) * a.c.Hkv * D;
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const bool there = row0 + 4 * i >= held && row0 + 4 * i < end;
#pragma unroll
            for (int c = 0; c < kC; ++c)
                ahead[i][c].w = there ? *reinterpret_cast<const uint4*>(x + i * step + c * 8 * kE) : make_uint4(0, 0, 0, 0);
        }
        old_ahead = scales[blk];
    };
    int turn = 0;
    int blk = held / kQcBlock + w0;
    fetch(blk);
    // (a ticket orders nothing by itself: the fences put every CTA's reading of the state before the last one's writing.  Taken
    // while the first tokens are on their way: a fill of 8 x 4096 39 us, 40.5 in front of their loads)
    int ticket = 0;
    if (threadIdx.x == 0) {
        __threadfence();
        ticket = atomicAdd(reinterpret_cast<int*>(a.c.state + 2 * a.c.B + b), 1);
    }
    for (; blk < blk_end; blk += a.ctas, turn ^= 1) {
        const int lo = blk * kQcBlock, first = max(held, lo), last = min(end, lo + kQcBlock), row0 = lo + row_in;
        int8_t* codes = a.c.codes[plane] + ((size_t)unit * C + row0) * D;
        auto is_new = [&](int i) { return row0 + 4 * i >= first && row0 + 4 * i < last; };
        Piece<T> in[kTurns][kC];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < kTurns; ++i)
#pragma unroll
            for (int c = 0; c < kC; ++c) {
                in[i][c] = ahead[i][c];
                top = in[i][c].top(top);
            }
        const float old = old_ahead;
        fetch(blk + a.ctas);
        const float amax = plane_amax(Piece<T>::top_of(top), share[turn], plane, part);
        float shrink;
        const float s = grown(old, amax, first == lo, &shrink), inv = s > 0.f ? 1.f / s : 0.f, edge = s > 0.f ? s : INFINITY;
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            if (!is_new(i)) continue;
#pragma unroll
            for (int c = 0; c < kC; ++c) {
                float y[kE];
                Chunk<T>::unpack(in[i][c].w, y);
                uint32_t out[kE / 4];
#pragma unroll
                for (int k = 0; k < kE / 4; ++k) out[k] = s > 0.f ? new_codes(y + 4 * k, inv, s, edge) : 0;
                store_words(codes + i * 4 * D + (c * 8 + l8) * kE, out);
            }
        }
        if (shrink != 1.f) {                                // (what stands behind the new end too: a block's codes have one scale)
#pragma unroll
            for (int i = 0; i < kTurns; ++i) {
                if (is_new(i) || row0 + 4 * i >= C) continue;
                uint32_t w[kW];
                int8_t* p = codes + i * 4 * D + l8 * (D / 8);
                load_words(p, w);
#pragma unroll
                for (int k = 0; k < kW; ++k) w[k] = shrunk(w[k], shrink);
                store_words(p, w);
            }
        }
        // (the plane's warps have read the old scale: the barrier above came after their loads of it were used or not, and
        // no other block of this loop has the same)
        if (part == 0 && lane == 0) scales[blk] = s;
        if (plane == 0 && part == 0) {
            const int slot = lo + lane;
            if (slot >= first && slot < last) {
                a.c.weight[(size_t)unit * C + slot] = 0.f;
                a.c.position[(size_t)unit * C + slot] = seen + (slot - held);
            }
        }
    }
    if (threadIdx.x == 0 && ticket == a.ctas * a.c.Hkv - 1) {
        __threadfence();
        a.c.state[b] = end;
        a.c.state[a.c.B + b] = seen + n;
        a.c.state[2 * a.c.B + b] = 0;
    }
}

// ---- eviction ---------------------------------------------------------------------------------------------------
constexpr int kQsBins = 2048;          // 11 bits of a key at a time
constexpr int kQsKeys = 40960;         // keys that are kept in shared memory; those behind are formed anew

// Floats in their order, as integers; slots that stay in any case come last.
__device__ __forceinline__ uint32_t worth_key(float w, bool stays) {
    if (stays || w != w) return stays ? 0xffffffffu : 0xfffffffeu;
    const uint32_t u = __float_as_uint(w + 0.f);   // (-0 is 0)
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

// Sum of the words of the warps before this thread's, and of all.  share: two sets of 32 words, used in turn, so that one
// barrier is enough; `x` is the same in all of a warp.
template <int WARPS>
__device__ __forceinline__ uint32_t warps_before(uint32_t x, uint32_t (*share)[32], int* turn, uint32_t* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t* s = share[*turn];
    *turn ^= 1;
    if (lane == 0) s[warp] = x;
    __syncthreads();
    uint32_t y = lane < WARPS ? s[lane] : 0;
#pragma unroll
    for (int o = 1; o < WARPS; o <<= 1) {
        const uint32_t z = __shfl_up_sync(0xffffffffu, y, o);
        if (lane >= o) y += z;
    }
    *total = __shfl_sync(0xffffffffu, y, WARPS - 1);
    const uint32_t before = __shfl_sync(0xffffffffu, y, warp ? warp - 1 : 0);
    return warp ? before : 0;
}

// A CTA per unit finds the n least keys: 11 + 11 + 10 bits of the n-th one, by counting (one slot alone: the least pair
// of key and slot); then one pass in the slots' order, in which a warp is a block, lists the blocks with holes and the
// slots that move.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) qc_select_kernel(const QcEvict a) {
    constexpr int kWarps = THREADS / 32, kBinsEach = kQsBins / THREADS;
    extern __shared__ uint32_t keys[];
    __shared__ int bins[kQsBins];
    __shared__ uint32_t share[2][32];
    __shared__ unsigned long long least[kWarps];
    __shared__ int found[3];
    const int unit = blockIdx.x, b = unit / a.c.Hkv, C = a.c.C, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    pdl_open();
    const int held = min(max(a.c.state[b], 0), C), from = a.c.state[a.c.B + b] - a.recent;
    const int n = held - a.keep;
    if (n <= 0) {
        if (tid == 0) a.n_out[unit] = a.n_blocks[unit] = 0;
        return;
    }
    const float* weight = a.c.weight + (size_t)unit * C;
    const int32_t* position = a.c.position + (size_t)unit * C;
    int4* blocks = a.blocks + (size_t)unit * a.max_blocks;
    int32_t* movers = a.movers + (size_t)unit * a.max_moves;
    if (tid < 2 && a.keep < C) a.cut_scale[2 * unit + tid] = a.c.scale[tid][(size_t)unit * a.c.NB + a.keep / kQcBlock];

    if (n == 1) {
        unsigned long long best = ~0ull;
#pragma unroll 4
        for (int j = tid; j < held; j += THREADS) {
            const unsigned long long k = ((unsigned long long)worth_key(weight[j], position[j] >= from) << 32) | (unsigned)j;
            best = k < best ? k : best;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const unsigned long long k = __shfl_xor_sync(0xffffffffu, best, o);
            best = k < best ? k : best;
        }
        if (lane == 0) least[warp] = best;
        __syncthreads();
        if (tid != 0) return;
        for (int i = 1; i < kWarps; ++i) best = least[i] < best ? least[i] : best;
        const int j = (int)(unsigned)best;
        const bool moves = j < a.keep;         // or the slot behind the new end is itself the one
        if (moves) {
            movers[0] = held - 1;
            blocks[0] = make_int4(j / kQcBlock, 0, (int)(1u << (j % kQcBlock)), 0);
        }
        a.n_out[unit] = 1;
        a.n_blocks[unit] = moves;
        return;
    }

    const int kept_keys = min(held, kQsKeys);
#pragma unroll 4
    for (int j = tid; j < kept_keys; j += THREADS) keys[j] = worth_key(weight[j], position[j] >= from);
    auto key_at = [&](int j) { return j < kQsKeys ? keys[j] : worth_key(weight[j], position[j] >= from); };

    uint32_t prefix = 0, mask = 0, total;
    int left = n, turn = 0;                // of the keys that share the prefix, so many go
    bool ties = false;                     // and others with the very same key stay
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
#pragma unroll
        for (int i = 0; i < kBinsEach; ++i) bins[tid + i * THREADS] = 0;
        __syncthreads();
        for (int j = tid; j < held; j += THREADS) {
            const uint32_t k = key_at(j);
            if ((k & mask) == prefix) atomicAdd(&bins[(k >> shift) & ((1u << width) - 1)], 1);
        }
        __syncthreads();
        int mine[kBinsEach], sum = 0;
#pragma unroll
        for (int i = 0; i < kBinsEach; ++i) sum += mine[i] = bins[kBinsEach * tid + i];
        int upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += y;
        }
        upto += (int)warps_before<kWarps>((uint32_t)__shfl_sync(0xffffffffu, upto, 31), share, &turn, &total);
        int before = upto - sum;
        if (before < left && left <= upto) {
#pragma unroll
            for (int i = 0; i < kBinsEach; ++i) {
                if (before < left && left <= before + mine[i]) {
                    found[0] = kBinsEach * tid + i;
                    found[1] = left - before;
                    found[2] = mine[i];
                }
                before += mine[i];
            }
        }
        __syncthreads();
        prefix |= (uint32_t)found[0] << shift;
        left = found[1];
        ties = found[2] != left;
        mask |= ((1u << width) - 1) << shift;
        __syncthreads();
    }

    int tied = 0, n_holes = 0, n_movers = 0, n_blocks = 0;
    const unsigned below = (1u << lane) - 1u;
    for (int base = 0; base < held; base += THREADS) {
        const int j = base + tid;
        const uint32_t k = j < held ? key_at(j) : 0xffffffffu;
        const bool tie = j < held && k == prefix;
        bool out = j < held && k <= prefix;
        if (ties) {                        // the lower slots go
            const unsigned t = __ballot_sync(0xffffffffu, tie);
            const int no = tied + (int)warps_before<kWarps>(__popc(t), share, &turn, &total) + __popc(t & below);
            if (tie) out = no < left;
            tied += (int)total;
        }
        const unsigned holes = __ballot_sync(0xffffffffu, out && j < a.keep);
        const unsigned moves = __ballot_sync(0xffffffffu, !out && j >= a.keep && j < held);
        // of all warps, up to 1024 of each, 32 blocks
        const uint32_t before = warps_before<kWarps>(__popc(holes) | (__popc(moves) << 11) | ((holes != 0) << 22), share, &turn, &total);
        if ((moves >> lane) & 1) movers[n_movers + ((before >> 11) & 0x7ff) + __popc(moves & below)] = j;
        if (lane == 0 && holes != 0)
            blocks[n_blocks + (before >> 22)] = make_int4(j / kQcBlock, n_holes + (int)(before & 0x7ff), (int)holes, 0);
        n_holes += total & 0x7ff;
        n_movers += (total >> 11) & 0x7ff;
        n_blocks += total >> 22;
    }
    if (tid == 0) {
        a.n_out[unit] = n;
        a.n_blocks[unit] = n_blocks;
    }
}

// A warp per block with holes and plane: the slots that move in come with the codes and scale of where they were, four
// rows at a time.  (Four warps to a block, as an append has, would be idle where a block has a few holes.)  What a block
// needs is found in steps that wait for one another, list, slots, codes, so a warp goes from block to block and looks up the
// next one's slots while this one's codes are on their way.
constexpr int kQmResident = 5;   // CTAs on an SM
template <int D>
__global__ void __launch_bounds__(kQwThreads, kQmResident) qc_move_kernel(const QcEvict a, int per_unit, int64_t items) {
    constexpr int kW = D / 32;   // words of a lane in a row of codes
    const int lane = threadIdx.x & 31, plane = (threadIdx.x >> 5) & 1, C = a.c.C;
    const int64_t stride = (int64_t)gridDim.x * (kQwThreads / 64);
    pdl_wait();
    pdl_open();
    struct Item {
        int unit;
        bool some;               // a block with holes
        int4 e;                  // block, first hole's number, mask of holes
        int src;                 // lane i: the slot that moves into the i-th hole
        float old;               // the block's scale
    };
    auto look = [&](int64_t at) {
        Item t = {};
        if (at >= items) return t;
        t.unit = (int)((unsigned)at / (unsigned)per_unit);
        const int no = (int)((unsigned)at - (unsigned)t.unit * per_unit);
        const int n_blocks = a.n_blocks[t.unit];
        if (a.max_blocks > 0) t.e = a.blocks[(size_t)t.unit * a.max_blocks + no];
        if (no == 0 && plane == 0 && t.unit % a.c.Hkv == 0 && lane == 0 && a.n_out[t.unit] > 0) a.c.state[t.unit / a.c.Hkv] = a.keep;
        t.some = no < n_blocks;
        return t;
    };
    auto find = [&](Item& t) {
        if (!t.some) return;
        t.src = lane < __popc(t.e.z) ? a.movers[(size_t)t.unit * a.max_moves + t.e.y + lane] : 0;
        t.old = a.c.scale[plane][(size_t)t.unit * a.c.NB + t.e.x];
    };
    int64_t at = (int64_t)blockIdx.x * (kQwThreads / 64) + (threadIdx.x >> 6);
    Item next = look(at);
    find(next);
    for (; at < items; at += stride) {
        const Item now = next;
        next = look(at + stride);
        if (!now.some) {
            find(next);
            continue;
        }
        const int unit = now.unit, lo = now.e.x * kQcBlock, src = now.src;
        const float old = now.old;
        const unsigned holes = (unsigned)now.e.z;
        const int count = __popc(holes);
        int8_t* codes = a.c.codes[plane] + (size_t)unit * C * D + (lane & 7) * (D / 8);
        float* scales = a.c.scale[plane] + (size_t)unit * a.c.NB;
        const int kept = min(kQcBlock, a.keep - lo);
        const unsigned all = kept == kQcBlock ? 0xffffffffu : (1u << kept) - 1u;
        const bool fresh = holes == all;

        // four rows at a time, eight lanes to each: the lane's is the (i0 + lane / 8)-th
        uint32_t w[kW];
        auto load = [&](int i0) {
            const int no = i0 + (lane >> 3), slot = __shfl_sync(0xffffffffu, src, no & 31);
            if (no < count) load_words(codes + (size_t)slot * D, w);
        };
        load(0);
        // (the block that the new end cuts takes slots in and gives some away: its scale is the one before)
        float from = 0.f;
        if (lane < count) from = src / kQcBlock == a.keep / kQcBlock ? a.cut_scale[2 * unit + plane] : scales[src / kQcBlock];
        find(next);
        int dst = lo;            // lane i: the i-th hole
        for (unsigned m = holes, i = 0; m != 0; m &= m - 1, ++i)
            if (i == (unsigned)lane) dst = lo + __ffs(m) - 1;
        // the largest |code| of a row: its product with the row's scale is exact in 64 bits
        double amax = 0.;
        for (int i0 = 0;;) {
            const int no = i0 + (lane >> 3);
            unsigned top = 0;
            if (no < count) {
#pragma unroll
                for (int k = 0; k < kW; ++k) top = max(top, top_code(w[k]));
            }
            amax = fmax(amax, (double)top * (double)__shfl_sync(0xffffffffu, from, no & 31));
            if ((i0 += 4) >= count) break;
            load(i0);
        }
        if (__any_sync(0xffffffffu, !(fabsf(from) <= 3.402823466e38f))) amax = nan("");
        const unsigned bits = __reduce_max_sync(0xffffffffu, __float_as_uint((float)amax) & 0x7fffffffu);
        float s = old, shrink = 1.f;
        if (fresh || old == 0.f || !(__uint_as_float(bits) < 127.4f * old)) {   // (or not a number)
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) amax = fmax(amax, __shfl_xor_sync(0xffffffffu, amax, o));
            s = grown(old, bits < 0x7f800000u ? amax : nan(""), fresh, &shrink);
        }
        const float inv = s > 0.f ? 1.f / s : 0.f;
        if (count > 4) load(0);
        for (int i0 = 0;;) {
            const int no = i0 + (lane >> 3);
            const float f = __shfl_sync(0xffffffffu, from, no & 31);
            const int to = __shfl_sync(0xffffffffu, dst, no & 31);
            if (no < count) {
#pragma unroll
                for (int k = 0; k < kW; ++k) {
                    float x[4], far = 0.f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = code_at(w[k], j) * f;
                    uint32_t c = s > 0.f ? codes_of(x, inv, &far) : 0;
                    if (far > kNextToHalf) {
                        float rest[4];                       // what the products lost
#pragma unroll
                        for (int j = 0; j < 4; ++j) rest[j] = fmaf(code_at(w[k], j), f, -x[j]);
                        c = exact_codes(make_float4(x[0], x[1], x[2], x[3]), make_float4(rest[0], rest[1], rest[2], rest[3]), s, inv);
                    }
                    w[k] = c;
                }
                store_words(codes + (size_t)to * D, w);
            }
            if ((i0 += 4) >= count) break;
            load(i0);
        }
        if (shrink != 1.f) {
            const unsigned stay = all & ~holes;
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                uint32_t v[4][kW];
                const unsigned mine = stay >> (16 * half + (lane >> 3));
                int8_t* p = codes + (size_t)(lo + 16 * half + (lane >> 3)) * D;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if ((mine >> (4 * i)) & 1) load_words(p + 4 * i * D, v[i]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (!((mine >> (4 * i)) & 1)) continue;
#pragma unroll
                    for (int k = 0; k < kW; ++k) v[i][k] = shrunk(v[i][k], shrink);
                    store_words(p + 4 * i * D, v[i]);
                }
            }
        }
        if (lane == 0) scales[now.e.x] = s;
        if (plane == 0 && lane < count) {
            const size_t u = (size_t)unit * C;
            a.c.weight[u + dst] = a.c.weight[u + src];
            a.c.position[u + dst] = a.c.position[u + src];
        }
    }
}

}  // namespace

cudaError_t qc_append(const QcAppend& args, int dtype, cudaStream_t s) {
    QcAppend a = args;
    const int64_t units = (int64_t)a.c.B * a.c.Hkv;
    // As many CTAs as run side by side, where there are as many blocks; four blocks to each at most, so that sequences of
    // unlike lengths even out.
    a.ctas = (int)std::max<int64_t>(std::min<int64_t>(a.W, 148 * kQwResident / units), (a.W + 3) / 4);
    const unsigned grid = (unsigned)(units * a.ctas);
    if (dtype == BCT_BF16)
        return a.c.D == 128 ? pdl_launch(qc_append_kernel<__nv_bfloat16, 128>, grid, kQwThreads, 0, s, a)
                            : pdl_launch(qc_append_kernel<__nv_bfloat16, 64>, grid, kQwThreads, 0, s, a);
    return a.c.D == 128 ? pdl_launch(qc_append_kernel<float, 128>, grid, kQwThreads, 0, s, a)
                        : pdl_launch(qc_append_kernel<float, 64>, grid, kQwThreads, 0, s, a);
}

cudaError_t qc_evict(const QcEvict& a, cudaStream_t s) {
    const int units = a.c.B * a.c.Hkv;
    // Many units fill the SMs with small CTAs, whose barriers cost less; few units need their threads, and so do long ones, of
    // whose keys an SM holds few.  An eviction of C / 16 slots with 256 / 1024 threads to a CTA: 64 units of 4096 slots 23 / 18 us, 256
    // 38 / 35, 320 45 / 46, 512 60 / 64, 1024 107 / 114; 512 of 8192 108 / 111, of 16384 259 / 207, of 32768 594 / 414.  Of one slot: 256 of
    // 4096 8.2 / 9.2, 512 9.7 / 12.1; 512 of 8192 11.8 / 14.1, of 16384 18.8 / 17.9, of 32768 95 / 55.
    const bool small = units >= 296 && a.c.C <= 8192;
    const auto kernel = small ? qc_select_kernel<256> : qc_select_kernel<1024>;
    const int smem = (a.c.C < kQsKeys ? a.c.C : kQsKeys) * 4;
    cudaError_t e;
    static std::atomic<uint64_t> done[2];
    if (smem > 32768 && (e = allow_smem(kernel, kQsKeys * 4, &done[small])) != cudaSuccess) return e;
    if ((e = pdl_launch(kernel, units, small ? 256 : 1024, smem, s, a)) != cudaSuccess) return e;
    const int per_unit = a.max_blocks > 0 ? a.max_blocks : 1;
    const int64_t items = (int64_t)units * per_unit, ctas = (items + kQwThreads / 64 - 1) / (kQwThreads / 64);
    const unsigned grid = (unsigned)std::min<int64_t>(ctas, 148 * kQmResident);
    return a.c.D == 128 ? pdl_launch(qc_move_kernel<128>, grid, kQwThreads, 0, s, a, per_unit, items)
                        : pdl_launch(qc_move_kernel<64>, grid, kQwThreads, 0, s, a, per_unit, items);
}

}  // namespace bct
