// Attention over the 8-bit cache, few rows to a unit: decode steps and drafted tokens (bct_qcache_prompt.cu has prompts).
//
// Per (sequence, kv-head) unit, with its R = T G rows q_r and slots j < sees_r:
//     s_rj = scale q_r . k_j  (cap tanh(s / cap) where the call says so)      p_rj = exp(s_rj - max_j s_rj)
//     o_r  = sum_j p_rj v_j / sum_j p_rj                                       weight_j += sum_r p_rj / sum_j p_rj
//
// Bound by HBM: 2 d bytes of codes per slot, which every row of the unit shares.  A warp works alone on blocks of 32 slots
// (the block of a scale), which come by 16-byte asynchronous copies into a ring of its own; the blocks of all units, in
// their order, are dealt to the warps in equal runs, whatever the sequences' lengths.  What a warp has of a unit that
// others share (at most two such per warp) goes to scratch and is joined by qc_join_kernel, which then gives each slot its
// weight from the stored scores (4 R bytes a slot written and read, against 2 d for reading the keys again).
//
// Products are mma.sync m16n8k16 with the slots in M and eight rows in N: rows are few, and an 8-bit code has to be
// turned into 16 bits in registers on its way in any case, so there is nothing for tcgen05 to read from shared memory; the
// tensor cores are idle most of the time here.  Codes become fp16 exactly (two instructions for a pair: the byte under the
// exponent of 1024, less 1152).  A query is scaled by a power of two to below 2^15 and is fp16 as it is if it is bfloat16
// (terms below 2^-39 of the row's largest apart); a float query is two such terms.  Scores are thus exact products with
// fp32 sums.  The probabilities enter the second product as fp16 times 2^15 (off by 2^-11 of each, and by 2^-40 in any case),
// for float results as two terms (2^-22).  Each block's V product starts from zero and is added with the block's scale in
// fp32, so scales may differ by any factor.
//
// Fragments need no shuffling of codes: the order of features in the first product's sum, and of slots in the second's, is
// free.  Lane (g, t) = (lane / 4, lane % 4) reads for slot 8 (g / 2) + 4 (g % 2) + i, i < 4, the features 16 t .. 16 t + 15
// (and 64 + 16 t ..), and for the slots 8 t + i, 8 t + 4 + i the features 16 g .. 16 g + 15 of V; what it computes for the
// former is, transposed 8 x 8 at a time by movmatrix, the other operand of the latter.  16-byte chunks of a slot are stored
// at chunk ^ x(slot), with which both readings are free of bank conflicts.
//
// Measured (bfloat16, d 128): one row of 64 sequences x 32 heads x 2048 slots 174 us = 6.4 TB/s of codes and scales, 0.97 of a
// copy's rate; of 37 sequences of up to 16384 slots x 8 heads 94 us = 5.6 TB/s; of one of 131071 50 us = 5.5 TB/s, joined in 16
// to 20 more.  20 rows of 16 x 4001 slots x 8 heads under a cap: 78 us + 28; three tiles of rows take 255 registers, so eight
// warps of an SM wait for their own results (issue slots 42 % used).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "bct_device.cuh"
#include "bct_internal.h"
#include "bct_qcache.h"
#include "bct_qcache.cuh"
#include "bct_qcache_math.cuh"
#include "bct_tc.cuh"

namespace bct {
namespace {

constexpr int kQaWarps = 8;
constexpr int kQaThreads = kQaWarps * 32;
// Two tiles of rows or more leave no registers for their queries: those stand in shared memory then, in place of a stage (16
// rows of 64 x 2048 slots x 8 heads 124 -> 118 us, 24 rows 198 -> 187).
template <int NT>
constexpr bool kQueriesShared = NT >= 2;
template <int NT>
constexpr int kQaStages = kQueriesShared<NT> ? 2 : 3;
template <int D, int NT, int TERMS>
constexpr int kQaQueries = kQueriesShared<NT> ? NT * TERMS * (D / 16) * 32 * 8 : 0;   // bytes of a warp
constexpr int kQaScored = kQcScoredRows;
constexpr int kQjThreads = 128;
constexpr int kQjResident = 8;        // CTAs of the joining kernel on an SM
constexpr int kQjSlots = 4 * kQjThreads;   // slots that one of them takes at a time
constexpr float kPBack = 32768.f;     // 2^15
constexpr float kPShift = 15.f;       // of a probability on its way into fp16, in powers of two

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Where the 16-byte chunk of a slot stands in its block's tile.
template <int D>
__device__ __forceinline__ int tile_at(int slot, int chunk) {
    const int x = (((slot >> 3) & 3) << 1) ^ (((slot >> 2) & 1) << 2);
    if constexpr (D == 128) return slot * 128 + ((chunk ^ x) << 4);
    else return (slot >> 1) * 128 + (((((slot & 1) << 2) | chunk) ^ x) << 4);
}

// Blocks of a sequence.
__device__ __forceinline__ int blocks_of(const QcAttend& a, int b) {
    return (min(max(a.c.state[b], 0), a.c.C) + kQcBlock - 1) / kQcBlock;
}
// The warp whose run has block x of `total` in all, of n runs (n <= total).
__device__ __forceinline__ int run_of(int64_t x, int64_t total, int n) { return (int)(((x + 1) * n - 1) / total); }

// The queries of eight rows as fragments: lane (g, t) has row g.  `mul`: what the row was divided by.
template <typename T, int D>
constexpr int kQueryWords = D / 4 / Chunk<T>::kElems;
template <typename T, int D>
__device__ __forceinline__ void fetch_queries(const T* row, bool real, uint4 (&w)[kQueryWords<T, D>]) {
    constexpr int kE = Chunk<T>::kElems, kEach = 16 / kE;
#pragma unroll
    for (int i = 0; i < kQueryWords<T, D>; ++i) {
        w[i] = make_uint4(0, 0, 0, 0);
        if (real) w[i] = *reinterpret_cast<const uint4*>(row + 64 * (i / kEach) + 16 * (threadIdx.x & 3) + i % kEach * kE);
    }
}
template <typename T, int D, int TERMS>
__device__ __forceinline__ void make_queries(const uint4 (&w)[kQueryWords<T, D>], uint32_t (&f)[TERMS][D / 16][2], float* mul) {
    float x[D / 4];
#pragma unroll
    for (int i = 0; i < kQueryWords<T, D>; ++i) Chunk<T>::unpack(w[i], x + i * Chunk<T>::kElems);
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < D / 4; ++i) top = fmaxf(top, fabsf(x[i]));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    float by;
    row_scale(top, &by, mul);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const float u = x[4 * ks + 2 * p] * by, v = x[4 * ks + 2 * p + 1] * by;
            f[0][ks][p] = half2_bits(u, v);
            if constexpr (TERMS == 2) {
                const float2 b = half2_floats(f[0][ks][p]);
                f[1][ks][p] = half2_bits(u - b.x, v - b.y);
            }
        }
    }
}

template <typename T, int D, int TERMS>
__device__ __forceinline__ void load_queries(const T* row, bool real, uint32_t (&f)[TERMS][D / 16][2], float* mul) {
    uint4 w[kQueryWords<T, D>];
    fetch_queries<T, D>(row, real, w);
    make_queries<T, D, TERMS>(w, f, mul);
}

// The codes of a block's keys as fragments: [i][word] pairs, i the lane's slots, word four features.
template <int D>
__device__ __forceinline__ void load_keys(const unsigned char* tile, int g, int t, uint32_t (&w)[4][D / 16]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int slot = 8 * (g >> 1) + 4 * (g & 1) + i;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            const uint4 u = *reinterpret_cast<const uint4*>(tile + tile_at<D>(slot, t + 4 * j));
            w[i][4 * j] = u.x ^ 0x80808080u, w[i][4 * j + 1] = u.y ^ 0x80808080u;
            w[i][4 * j + 2] = u.z ^ 0x80808080u, w[i][4 * j + 3] = u.w ^ 0x80808080u;
        }
    }
}

// Products of a block's keys with eight rows: s[mt][..] for the slots i = 2 mt (c0, c1: rows 2t, 2t + 1), 2 mt + 1 (c2, c3).
// q(tile, term, step) is a lane's fragment of the queries.
template <int D, int TERMS, int NT, typename Q>
__device__ __forceinline__ void score_products(const uint32_t (&w)[4][D / 16], Q q, float (&s)[NT][2][4]) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[nt][i >> 2][i & 3] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            const uint32_t u = w[2 * mt][ks], v = w[2 * mt + 1][ks];
            const uint32_t a0 = pair_of(u, 0x4140), a1 = pair_of(v, 0x4140), a2 = pair_of(u, 0x4342), a3 = pair_of(v, 0x4342);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int term = 0; term < TERMS; ++term) {
                    const uint2 f = q(nt, term, ks);
                    mma16816(s[nt][mt], a0, a1, a2, a3, f.x, f.y);
                }
        }
    }
}

// Scores in powers of two from products: `mul` has the block's scale and the row's.
__device__ __forceinline__ void to_scores(float (&s)[2][4], float mul0, float mul1, float cap) {
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i >> 2][i & 3] *= i & 1 ? mul1 : mul0;
    if (cap > 0.f) {
        const float to = cap * kLog2e;
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(s[i >> 2][i & 3]));
        if (__any_sync(0xffffffffu, top > 1.f)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i >> 2][i & 3] = to * tanh_any(s[i >> 2][i & 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i >> 2][i & 3] = to * tanh_near(s[i >> 2][i & 3]);
        }
    }
}
template <typename T, int D, int NT, int TERMS>
__global__ void __launch_bounds__(kQaThreads, 1) qc_attend_kernel(const QcAttend a) {
    constexpr int kTile = kQcBlock * D;
    constexpr int kMt = D / 16;                    // tiles of 16 features
    constexpr int kRows = 8 * NT;
    extern __shared__ __align__(128) unsigned char qa_smem[];
    __shared__ int64_t upto[kQaThreads];
    constexpr int kStages = kQaStages<NT>;
    constexpr bool kShared = kQueriesShared<NT>;
    __shared__ float2 scales_all[kQaWarps][kStages];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    unsigned char* ring = qa_smem + warp * (kStages * 2 * kTile + kQaQueries<D, NT, TERMS>);
    uint2* shared_q = reinterpret_cast<uint2*>(ring + kStages * 2 * kTile) + lane;   // [tile][term][step][lane]
    const float2* scales = scales_all[warp];

    pdl_wait();
    pdl_open();
    // where the run begins: its sequence, then the unit and row group within
    const int64_t per_seq = (int64_t)a.c.Hkv * a.n_groups;
    const int run = warp * gridDim.x + blockIdx.x;
    int n_runs, b;
    int64_t x, before;    // blocks of the sequences before b, times per_seq
    const int64_t total = find_share(a.c.B, [&](int i) { return blocks_of(a, i); }, per_seq, upto,
                                     [&](int64_t all) {
                                         n_runs = (int)min((int64_t)a.n_warps, all);
                                         return run < n_runs ? all * run / n_runs : all;
                                     },
                                     &x, &b, &before);
    if (run >= n_runs) return;
    const int64_t end = total * (run + 1) / n_runs;

    // Where the run stands: its blocks are fetched two ahead of those that are worked on, across units.
    struct Place {
        int b, nb, unit_in, blk;   // sequence, its blocks, h * n_groups + group, block
    };
    auto next_unit = [&](Place& p, bool more) {
        p.blk = 0;
        if (++p.unit_in == (int)per_seq && more) {
            p.unit_in = 0;
            do p.nb = blocks_of(a, ++p.b);
            while (p.nb == 0);
        }
    };
    Place now;
    now.b = b;
    now.nb = blocks_of(a, b);
    now.unit_in = (int)((x - before) / now.nb);
    now.blk = (int)((x - before) - (int64_t)now.unit_in * now.nb);

    Place ahead = now;
    int64_t fetched = x;
    const int8_t *kp = nullptr, *vp = nullptr;      // the fetched unit's, for this lane
    const float *ksp = nullptr, *vsp = nullptr;
    constexpr int kChunks = D / 16, kPer = 32 / kChunks;   // chunks of a slot, slots of an instruction
    auto unit_of = [&](const Place& p) { return (int64_t)p.b * a.c.Hkv + p.unit_in / (int)a.n_groups; };
    auto at_unit = [&]() {
        const int64_t u = unit_of(ahead);
        kp = a.c.codes[0] + (size_t)u * a.c.C * D + lane * 16;
        vp = a.c.codes[1] + (size_t)u * a.c.C * D + lane * 16;
        ksp = a.c.scale[0] + (size_t)u * a.c.NB;
        vsp = a.c.scale[1] + (size_t)u * a.c.NB;
    };
    at_unit();
    const uint32_t lane_at = smem_u32(ring) + tile_at<D>(lane / kChunks, lane % kChunks);
    auto fetch = [&](int stage) {
        if (fetched < end) {
            const uint32_t dst = lane_at + stage * 2 * kTile;
            const int left = a.c.C - ahead.blk * kQcBlock - lane / kChunks;      // slots of the lane that exist
            const size_t from = (size_t)ahead.blk * kTile;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int8_t* src = (p ? vp : kp) + from;
#pragma unroll
                for (int i = 0; i < kQcBlock / kPer; ++i) {   // (the swizzle of slot i * kPer + .. is that of i * kPer, in bits 4..6)
                    const uint32_t to = (dst ^ (uint32_t)(tile_at<D>(i * kPer, 0) & 0x70)) + (p * kTile + i * kPer * D);
                    if ((ahead.blk + 1) * kQcBlock <= a.c.C) cp_async16_zfill(to, src + i * kPer * D, true);
                    else cp_async16_zfill(to, i * kPer < left ? src + i * kPer * D : kp, i * kPer < left);
                }
            }
            if (lane < 2)
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4;"
                             ::"r"(smem_u32(scales + stage) + lane * 4), "l"((lane ? vsp : ksp) + ahead.blk) : "memory");
            ++fetched;
            if (++ahead.blk == ahead.nb && fetched < end) {
                next_unit(ahead, true);
                at_unit();
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) fetch(s);
    int stage = 0;

    while (x < end) {
        const int nb = now.nb, unit_in = now.unit_in;
        b = now.b;
        const int h = unit_in / (int)a.n_groups;
        const int64_t group = unit_in - h * (int)a.n_groups;
        const int64_t unit = (int64_t)b * a.c.Hkv + h, r0 = group * kRows;
        const int first = now.blk, last = (int)min((int64_t)nb, first + (end - x));   // this piece's blocks
        const Sees sees = sees_of(a, b);

        // rows 2t, 2t + 1 of each tile of eight are this lane's in the scores and outputs, row g in the queries
        uint32_t q[kShared ? 1 : NT][TERMS][D / 16][2];
        float mul[NT][2];
        int lim[NT][2];
        int lim_max = 0, lim_min = 0x7fffffff;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int64_t r = r0 + nt * 8 + g;
            float m;
            load_queries<T, D, TERMS>(row_of<T>(a, a.q, b, h, r < a.R ? r : 0), r < a.R && sees(r) > 0, q[kShared ? 0 : nt], &m);
            if constexpr (kShared) {
#pragma unroll
                for (int i = 0; i < TERMS * (D / 16); ++i) {
                    const uint32_t(&f)[2] = q[0][i / (D / 16)][i % (D / 16)];
                    shared_q[(nt * TERMS * (D / 16) + i) * 32] = make_uint2(f[0], f[1]);
                }
            }
            m = row_factor(a, m);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                mul[nt][e] = __shfl_sync(0xffffffffu, m, (2 * t + e) * 4);
                lim[nt][e] = sees(r0 + nt * 8 + 2 * t + e);
                lim_max = max(lim_max, lim[nt][e]);
                lim_min = min(lim_min, lim[nt][e]);
            }
        }
        lim_max = __reduce_max_sync(0xffffffffu, lim_max);
        lim_min = __reduce_min_sync(0xffffffffu, lim_min);
        const int stop = min(last, (lim_max + kQcBlock - 1) / kQcBlock);   // blocks behind it are hidden from all rows

        float o[NT][kMt][4], m_run[NT][2], l_run[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < kMt * 4; ++i) o[nt][i >> 2][i & 3] = 0.f;
            m_run[nt][0] = m_run[nt][1] = -INFINITY;
            l_run[nt][0] = l_run[nt][1] = 0.f;
        }
        for (int i = first; i < last; ++i) {
            cp_async_wait<kStages - 2>();
            __syncwarp();
            fetch(stage == 0 ? kStages - 1 : stage - 1);
            const unsigned char* tile = ring + stage * 2 * kTile;
            const float ks = scales[stage].x;
            float vs = scales[stage].y;
            if (++stage == kStages) stage = 0;
            if (i >= stop) {
                __syncwarp();
                continue;
            }

            float s[NT][2][4];
            {
                uint32_t w[4][D / 16];
                load_keys<D>(tile, g, t, w);
                score_products<D, TERMS, NT>(w, [&](int nt, int term, int ks) {
                    if constexpr (kShared) return shared_q[((nt * TERMS + term) * (D / 16) + ks) * 32];
                    else return make_uint2(q[nt][term][ks][0], q[nt][term][ks][1]);
                }, s);
            }
            const int slot0 = i * kQcBlock + 8 * (g >> 1) + 4 * (g & 1);
            const bool all = (i + 1) * kQcBlock <= lim_min;
            uint32_t pf[NT][TERMS][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float top[2] = {-INFINITY, -INFINITY};
                to_scores(s[nt], ks * mul[nt][0], ks * mul[nt][1], a.cap);
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float& v = s[nt][j >> 1][2 * (j & 1) + e];
                        if (!all && slot0 + j >= lim[nt][e]) v = -INFINITY;
                        top[e] = fmaxf(top[e], v);
                    }
                if (a.scores != nullptr) {                    // rows of whole blocks: a lane's four slots side by side
                    float* to = a.scores + ((size_t)unit * a.R + r0 + nt * 8 + 2 * t) * a.Cs + slot0;
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (r0 + nt * 8 + 2 * t + e < a.R)
                            *reinterpret_cast<float4*>(to + (size_t)e * a.Cs) =
                                make_float4(s[nt][0][e], s[nt][0][2 + e], s[nt][1][e], s[nt][1][2 + e]);
                }
                bool higher = false;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int o_ = 4; o_ < 32; o_ <<= 1) top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], o_));
                    higher |= top[e] > m_run[nt][e];
                }
                if (__any_sync(0xffffffffu, higher)) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float m = fmaxf(m_run[nt][e], top[e]);
                        const float by = m == -INFINITY ? 1.f : ex2(m_run[nt][e] - m);
                        m_run[nt][e] = m;
                        l_run[nt][e] *= by;
#pragma unroll
                        for (int f = 0; f < kMt; ++f) o[nt][f][e] *= by, o[nt][f][2 + e] *= by;
                    }
                }
                // P, and its sum, times 2^15 until the piece is done
                float less[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) less[e] = (m_run[nt][e] == -INFINITY ? 0.f : m_run[nt][e]) - kPShift;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float p[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        p[e] = ex2(s[nt][j >> 1][2 * (j & 1) + e] - less[e]);
                        l_run[nt][e] += p[e];
                    }
                    const uint32_t hi = half2_bits(p[0], p[1]);
                    pf[nt][0][j] = transposed(hi);
                    if constexpr (TERMS == 2) {
                        const float2 b2 = half2_floats(hi);
                        pf[nt][1][j] = transposed(half2_bits(p[0] - b2.x, p[1] - b2.y));
                    }
                }
            }

            if (vs != vs) {                                   // spoilt values: the rows that see the block have them, no others
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (lim[nt][e] > i * kQcBlock) {
#pragma unroll
                            for (int f = 0; f < kMt; ++f) o[nt][f][e] = o[nt][f][2 + e] = vs;
                        }
                vs = 0.f;
            }
            // V: for the slots 8 t + i (e = 0) and 8 t + 4 + i (e = 1) the lane's D / 8 features, 16 or 8 from 16 g or 8 g on
            const unsigned char* vt = tile + kTile;
#pragma unroll
            for (int half = 0; half < D / 64; ++half) {       // 8 bytes of each slot at a time
                uint2 w[2][4];
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int slot = 8 * t + 4 * e + j;
                        const int at = D == 128 ? tile_at<D>(slot, g) + 8 * half : tile_at<D>(slot, g >> 1) + 8 * (g & 1);
                        w[e][j] = *reinterpret_cast<const uint2*>(vt + at);
                    }
#pragma unroll
                for (int wd = 0; wd < 2; ++wd) {
                    uint32_t lo[4], hi[4];            // slots 8t + j and 8t + 4 + j, two features
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t u = (wd ? w[0][j].y : w[0][j].x) ^ 0x80808080u, v = (wd ? w[1][j].y : w[1][j].x) ^ 0x80808080u;
                        lo[j] = prmt(u, v, 0x5140);
                        hi[j] = prmt(u, v, 0x7362);
                    }
#pragma unroll
                    for (int hm = 0; hm < 2; ++hm) {
                        const int f = half * 4 + wd * 2 + hm;   // features 2 f, 2 f + 1 of the lane's
                        uint32_t A[4][2];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t u = hm ? hi[j] : lo[j];
                            A[j][0] = pair_of(u, 0x4140);
                            A[j][1] = pair_of(u, 0x4342);
                        }
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int term = 0; term < TERMS; ++term)
#pragma unroll
                                for (int k2 = 0; k2 < 2; ++k2)
                                    mma16816(acc, A[2 * k2][0], A[2 * k2][1], A[2 * k2 + 1][0], A[2 * k2 + 1][1],
                                             pf[nt][term][2 * k2], pf[nt][term][2 * k2 + 1]);
#pragma unroll
                            for (int c = 0; c < 4; ++c) o[nt][f][c] = fmaf(acc[c], vs, o[nt][f][c]);
                        }
                    }
                }
            }
            __syncwarp();   // the stage may be filled again
        }
        // the piece's sums; a whole unit is done, a part goes to scratch
        const bool whole = first == 0 && last == nb;
        if (first == 0 && lane == 0)    // for who joins them: the first and last run that have blocks of these rows
            a.spans[unit * a.n_groups + group] = make_int2(run, whole ? run : run_of(x + nb - 1, total, n_runs));
        const int64_t slot_no = first == 0 ? 2 * (int64_t)run + 1 : 2 * (int64_t)run;
        constexpr int kE = D / 8;     // features of a lane
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float l = l_run[nt][e];
#pragma unroll
                for (int o_ = 4; o_ < 32; o_ <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o_);
                const int row = nt * 8 + 2 * t + e;
                const int64_t r = r0 + row;
                if (r >= a.R) continue;
                if (whole) {
                    const float inv = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
                    T* to = const_cast<T*>(row_of<T>(a, a.out, b, h, r)) + g * kE;
                    float y[kE];
#pragma unroll
                    for (int f = 0; f < kMt; ++f) y[2 * f] = o[nt][f][e] * inv, y[2 * f + 1] = o[nt][f][2 + e] * inv;
#pragma unroll
                    for (int c = 0; c < kE / Chunk<T>::kElems; ++c)
                        *reinterpret_cast<uint4*>(to + c * Chunk<T>::kElems) = Chunk<T>::pack(y + c * Chunk<T>::kElems);
                    if (g == 0) a.ml[unit * a.R + r] = make_float2(m_run[nt][e], inv * kPBack);
                } else {
                    float* to = a.part_o + (slot_no * kRows + row) * D + g * kE;
#pragma unroll
                    for (int f = 0; f < kMt; f += 2)
                        *reinterpret_cast<float4*>(to + 2 * f) = make_float4(o[nt][f][e], o[nt][f][2 + e], o[nt][f + 1][e], o[nt][f + 1][2 + e]);
                    if (g == 0) a.part_ml[slot_no * kRows + row] = make_float2(m_run[nt][e], l);   // (both times 2^15)
                }
            }

        x += last - first;
        now.blk = last;
        if (last == nb && x < end) next_unit(now, true);
    }
    cp_async_wait<0>();
}

// Joins what several warps have of a unit, writes the zeros of an empty cache's rows, and adds the weights from the stored
// scores (SCORED).  A CTA for some of a unit's slots, or, without scores, per unit and 8 of its rows; the rows that
// a unit's CTAs join are shared out among them, and a row's parts, up to two for each warp that the call has, among the
// CTA's threads.  ONE: one row to a unit.
template <typename T, int D, bool SCORED, bool ONE>
__global__ void __launch_bounds__(kQjThreads, kQjResident) qc_join_kernel(const QcAttend a, int ctas, int group_rows, int share, int ml_lanes, int rows_each) {
    // outputs are joined by pieces of 32 features, four of a lane, whose parts are shared out among groups of lanes
    constexpr int kLanes = 8, kGroups = kQjThreads / kLanes, kPieces = D / 32;
    __shared__ float2 row_ml[SCORED ? kQaScored : 8];
    __shared__ int row_sees[SCORED ? kQaScored : 1];
    __shared__ float4 sums[kGroups][kLanes];
    const unsigned unit = blockIdx.x / (unsigned)ctas;
    const int part = (int)(blockIdx.x - unit * ctas);
    const int b = (int)(unit / (unsigned)a.c.Hkv), h = (int)unit - b * a.c.Hkv, tid = threadIdx.x;
    const int lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    pdl_open();
    const Sees sees = sees_of(a, b);
    const int nb = (sees.held + kQcBlock - 1) / kQcBlock;
    // The CTA's slots, kQjSlots at a time.  What a CTA does takes a few steps that wait for one another, so everything that can
    // be loaded before it is known to be needed is (it exists in any case).
    const int seen = sees.n > 0 ? sees.held : 0, chunks = (a.c.C + kQjSlots - 1) / kQjSlots;
    const int chunk0 = SCORED ? chunks * part / ctas : 0, chunk1 = SCORED ? chunks * (part + 1) / ctas : 0;
    float* weight = a.c.weight + (size_t)unit * a.c.C;
    const float* scores = a.scores + (size_t)unit * a.R * a.Cs;
    const bool quads = (a.c.C & 3) == 0;                       // a thread has four slots side by side
    auto load_weights = [&](int j, float (&w)[4]) {
        if (quads && j < a.c.C) {
            const float4 v = *reinterpret_cast<const float4*>(weight + j);
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = j + i < a.c.C ? weight[j + i] : 0.f;
        }
    };
    auto load_scores = [&](int r, int j) {
        return j < a.c.C ? *reinterpret_cast<const float4*>(scores + (size_t)r * a.Cs + j) : make_float4(0.f, 0.f, 0.f, 0.f);
    };
    // A turn: a chunk with its first four rows, or four chunks of one row; all of it on its way at once, the first turn's
    // while the rows' sums are formed.
    constexpr int kDeep = ONE ? 4 : 1;
    float before[kDeep][4];
    float4 early[4];
    auto load_turn = [&](int c) {
#pragma unroll
        for (int i = 0; i < kDeep; ++i)
            if (c + i < chunk1) load_weights((c + i) * kQjSlots + 4 * tid, before[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (ONE ? c + i < chunk1 : i < (int)a.R) early[i] = load_scores(ONE ? 0 : i, (c + (ONE ? i : 0)) * kQjSlots + 4 * tid);
    };
    if constexpr (SCORED)
        if (chunk0 < chunk1) load_turn(chunk0);

    // A row's group, the runs that have it (2 first + 1, then 2 run are their places), and its place in theirs.
    struct Row {
        unsigned group, in;
        int first, last;
    };
    auto row_at = [&](int64_t r) {
        Row w;
        w.group = (unsigned)r / (unsigned)group_rows;
        w.in = (unsigned)r - w.group * group_rows;
        const int2 span = a.spans[(size_t)unit * a.n_groups + w.group];
        w.first = nb > 0 ? span.x : 0, w.last = nb > 0 ? span.y : 0;
        return w;
    };
    auto place = [&](const Row& w, int run) { return (2u * run + (run == w.first)) * group_rows + w.in; };
    // Maximum and 1 / sum of a row, by ml_lanes lanes (8, or 32 where a row has many parts).  All lanes of a warp call it.
    const int ml_at = tid & (ml_lanes - 1), ml_group = tid / ml_lanes, ml_groups = kQjThreads / ml_lanes;
    auto join = [&](bool real, int64_t r, const Row& w) {
        const float2 whole = real ? a.ml[(size_t)unit * a.R + r] : make_float2(0.f, 0.f);
        float m = -INFINITY, l = 0.f;
        constexpr int kAt = 6;                                       // parts of a lane on their way together
        const int last = real && nb > 0 && w.first < w.last ? w.last : -1;
        for (int i0 = w.first + ml_at; i0 <= last; i0 += ml_lanes * kAt) {
            float2 p[kAt];
            float top = m;
#pragma unroll
            for (int i = 0; i < kAt; ++i)
                p[i] = i0 + ml_lanes * i <= last ? a.part_ml[place(w, i0 + ml_lanes * i)] : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int i = 0; i < kAt; ++i) top = fmaxf(top, p[i].x);
            const float ref = top == -INFINITY ? 0.f : top;          // (a part without slots: minus infinity and 0, or a NaN)
            l *= ex2(m - ref);
#pragma unroll
            for (int i = 0; i < kAt; ++i) l += p[i].x == -INFINITY ? p[i].y : p[i].y * ex2(p[i].x - ref);
            m = top;
        }
        float top = m;
        for (int o = 1; o < ml_lanes; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (top != -INFINITY && m != -INFINITY) l *= ex2(m - top);
        for (int o = 1; o < ml_lanes; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        if (nb == 0) return make_float2(-INFINITY, 0.f);
        return last >= 0 ? make_float2(top, l > 0.f ? kPBack / l : (l == l ? 0.f : l)) : whole;
    };

    if constexpr (SCORED) {                        // every row's, for the weights (R <= kQaScored)
        for (int r0 = 0; r0 < (int)a.R; r0 += ml_groups) {
            const int r = r0 + ml_group;
            const float2 v = join(r < (int)a.R, r, row_at(min(r, (int)a.R - 1)));
            if (ml_at == 0 && r < (int)a.R) {
                row_ml[r] = v;
                row_sees[r] = v.y == 0.f ? 0 : sees(r);
            }
        }
        __syncthreads();
#pragma unroll 1
        for (int c = chunk0; c < chunk1 && c * kQjSlots < seen; c += kDeep) {
            if (c > chunk0) load_turn(c);
            auto add = [&](float (&w)[4], const float4& v, int r, int j) {
                const float2 ml = row_ml[r];
                const int lim = row_sees[r] - j;
                if (lim > 0) w[0] += ex2(v.x - ml.x) * ml.y;
                if (lim > 1) w[1] += ex2(v.y - ml.x) * ml.y;
                if (lim > 2) w[2] += ex2(v.z - ml.x) * ml.y;
                if (lim > 3) w[3] += ex2(v.w - ml.x) * ml.y;
            };
            const int j0 = c * kQjSlots + 4 * tid;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (ONE ? c + i < chunk1 : i < (int)a.R) add(before[ONE ? i : 0], early[i], ONE ? 0 : i, j0 + (ONE ? i * kQjSlots : 0));
            if constexpr (!ONE) {
                for (int r = 4; r < (int)a.R; r += 4) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (r + i < (int)a.R) early[i] = load_scores(r + i, j0);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (r + i < (int)a.R) add(before[0], early[i], r + i, j0);
                }
            }
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                const int j = j0 + i * kQjSlots;
                if (c + i >= chunk1 || j >= seen) continue;
                if (quads) {                                   // (what stands behind the slots held stays as it was)
                    *reinterpret_cast<float4*>(weight + j) = make_float4(before[i][0], before[i][1], before[i][2], before[i][3]);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (j + k < seen) weight[j + k] = before[i][k];
                }
            }
        }
    }
    // Outputs.  The CTA's pieces of rows side by side, `share` groups of lanes to each.
    const int64_t r_first = SCORED ? 0 : (int64_t)part * rows_each;
    const int rows = SCORED ? (int)a.R : (int)min((int64_t)rows_each, a.R - r_first), step = SCORED ? ctas : 1;
    if constexpr (!SCORED) {
        for (int i0 = 0; i0 < rows; i0 += ml_groups) {
            const int i = i0 + ml_group;
            const Row w = row_at(r_first + min(i, rows - 1));
            const float2 v = join(i < rows, r_first + i, w);
            if (ml_at == 0 && i < rows) {
                row_ml[i] = v;
                if (nb == 0 || w.first != w.last) a.ml[(size_t)unit * a.R + r_first + i] = v;
            }
        }
        __syncthreads();
    }
    const int from = SCORED ? part : 0, pieces = (rows * kPieces - from + step - 1) / step;
    const int group = tid / kLanes, f = tid % kLanes, slice = group % share;
    for (int base = 0; base < pieces; base += kGroups / share) {
        const int no = base + group / share, piece = from + no * step, row = piece / kPieces, at_f = piece % kPieces * 32 + 4 * f;
        const int64_t r = r_first + row;
        bool mine = no < pieces;
        Row w = {};
        float2 ml = make_float2(-INFINITY, 0.f);
        if (mine) {
            w = row_at(r);
            ml = row_ml[row];
            mine = nb == 0 || w.first != w.last;                // (a whole one was written by its warp)
        }
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
        if (mine && nb > 0) {
            for (int i0 = w.first + slice; i0 <= w.last; i0 += 4 * share) {   // four parts on their way together
                float m[4];
                float4 o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned at = place(w, i0 + i * share);
                    const bool there = i0 + i * share <= w.last;
                    m[i] = there ? a.part_ml[at].x : -INFINITY;
                    o[i] = there ? *reinterpret_cast<const float4*>(a.part_o + (size_t)at * D + at_f) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float by = m[i] == -INFINITY ? 0.f : ex2(m[i] - ml.x - kPShift) * ml.y;
                    y.x = fmaf(o[i].x, by, y.x), y.y = fmaf(o[i].y, by, y.y), y.z = fmaf(o[i].z, by, y.z), y.w = fmaf(o[i].w, by, y.w);
                }
            }
        }
        sums[group][f] = y;
        __syncthreads();
        if (mine && slice == 0) {
            for (int i = 1; i < share; ++i) {
                const float4 o = sums[group + i][f];
                y.x += o.x, y.y += o.y, y.z += o.z, y.w += o.w;
            }
            if (ml.y != ml.y) y = make_float4(ml.y, ml.y, ml.y, ml.y);
            T* to = const_cast<T*>(row_of<T>(a, a.out, b, h, r)) + at_f;
            if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(to) = y;
            else *reinterpret_cast<uint2*>(to) = make_uint2(Chunk<T>::pack2(y.x, y.y), Chunk<T>::pack2(y.z, y.w));
        }
        __syncthreads();
    }
}

// The weights from the keys again, for float calls with many rows: a CTA per block of slots, whose warps share the rows that
// see it, the next ones' queries on their way, and add up in their order.  There are few blocks in such calls, so it is the
// chain of a warp's turns that counts: of 333 tokens x 8 heads of 2 sequences of 640, 34 us with 8 warps, 22 with 16, 19 with the
// queries asked for ahead.  (As many as the registers allow: 122 of a thread with d 64, 168 with 128.)
template <int D>
constexpr int kQwWarps = D == 64 ? 16 : 12;
template <typename T, int D, int TERMS>
__global__ void __launch_bounds__(32 * kQwWarps<D>) qc_weights_kernel(const QcAttend a) {
    __shared__ __align__(128) unsigned char tile[kQcBlock * D];
    __shared__ float sums[kQwWarps<D>][kQcBlock];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const unsigned unit = blockIdx.x / (unsigned)a.c.NB;
    const int blk = (int)(blockIdx.x - unit * a.c.NB);
    const int b = (int)(unit / (unsigned)a.c.Hkv), h = (int)unit - b * a.c.Hkv;
    pdl_wait();
    const Sees sees = sees_of(a, b);
    const int slot0 = blk * kQcBlock;
    if (slot0 >= sees.held || sees.n == 0) return;
    {
        const int8_t* kp = a.c.codes[0] + (size_t)unit * a.c.C * D;
        constexpr int kChunks = D / 16;
        if (tid < kQcBlock * kChunks) {
            const int s = tid / kChunks, c = tid % kChunks;
            const bool real = slot0 + s < sees.held;
            cp_async16_zfill(smem_u32(tile + tile_at<D>(s, c)), kp + (size_t)(real ? slot0 + s : 0) * D + c * 16, real);
        }
        cp_async_commit();
        cp_async_wait<0>();
        __syncthreads();
    }
    const float ks = a.c.scale[0][(size_t)unit * a.c.NB + blk];
    uint32_t w[4][D / 16];
    load_keys<D>(tile, g, t, w);
    // the first token that sees the block's first slot
    const int i0 = max(0, slot0 - (sees.held - sees.n));
    const int mine = 8 * (g >> 1) + 4 * (g & 1);
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    uint4 next[kQueryWords<T, D>];
    float2 next_ml[2];
    auto ask = [&](int64_t r0) {                     // eight rows, an iteration ahead
        const int64_t r = r0 + g;
        const bool valid = r < (int64_t)sees.n * a.G;             // (rows behind the lengths are not read)
        fetch_queries<T, D>(row_of<T>(a, a.q, b, h, valid ? r : 0), valid, next);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int64_t re = r0 + 2 * t + e;
            next_ml[e] = re < a.R ? a.ml[(size_t)unit * a.R + re] : make_float2(0.f, 0.f);
        }
    };
    int64_t r0 = (int64_t)i0 * a.G / 8 * 8 + warp * 8;
    ask(r0);
    for (; r0 < (int64_t)sees.n * a.G; r0 += 8 * kQwWarps<D>) {
        uint32_t q[1][TERMS][D / 16][2];
        float m;
        make_queries<T, D, TERMS>(next, q[0], &m);
        m = row_factor(a, m);
        const float2 ml[2] = {next_ml[0], next_ml[1]};
        ask(r0 + 8 * kQwWarps<D>);
        float s[1][2][4];
        score_products<D, TERMS, 1>(w, [&](int, int term, int ks) { return make_uint2(q[0][term][ks][0], q[0][term][ks][1]); }, s);
        to_scores(s[0], __shfl_sync(0xffffffffu, m, 8 * t) * ks, __shfl_sync(0xffffffffu, m, 8 * t + 4) * ks, a.cap);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int lim = sees(r0 + 2 * t + e);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (slot0 + mine + j < lim && ml[e].y != 0.f) sum[j] += ex2(s[0][j >> 1][2 * (j & 1) + e] - ml[e].x) * ml[e].y;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 1);
        sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 2);
        if (t == 0) sums[warp][mine + j] = sum[j];
    }
    __syncthreads();
    if (tid < kQcBlock && slot0 + tid < sees.held) {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < kQwWarps<D>; ++i) x += sums[i][tid];
        a.c.weight[(size_t)unit * a.c.C + slot0 + tid] += x;
    }
}

template <typename T, int D, int NT, int TERMS>
cudaError_t attend_with(const QcAttend& a, cudaStream_t s) {
    constexpr int smem = kQaWarps * (kQaStages<NT> * 2 * kQcBlock * D + kQaQueries<D, NT, TERMS>);
    static std::atomic<uint64_t> done{0};
    if (const cudaError_t e = allow_smem(qc_attend_kernel<T, D, NT, TERMS>, smem, &done)) return e;
    return pdl_launch(qc_attend_kernel<T, D, NT, TERMS>, (a.n_warps + kQaWarps - 1) / kQaWarps, kQaThreads, smem, s, a);
}

template <typename T, int D, int TERMS>
cudaError_t attend_of(const QcAttend& a, const QcPlan& p, cudaStream_t s) {
    cudaError_t e = cudaErrorInvalidValue;
    if (p.tiles == 1) e = attend_with<T, D, 1, TERMS>(a, s);
    else if (p.tiles == 2) e = attend_with<T, D, 2, TERMS>(a, s);
    else if constexpr (TERMS == 1) e = attend_with<T, D, 3, TERMS>(a, s);
    if (e != cudaSuccess) return e;
    const int64_t units = (int64_t)a.c.B * a.c.Hkv;
    // With scores: a CTA for each kQjSlots slots, or for each four pieces of the outputs, but no more than run side by side.
    // Without: eight rows to a CTA, or one where they are few.
    const int64_t even = (148 * kQjResident + units - 1) / units;
    const int64_t most = std::max<int64_t>((a.c.C + kQjSlots - 1) / kQjSlots, a.R <= 4 ? a.R * (D / 32) : a.R * (D / 32) / 4);
    const int rows_each = units * a.R <= 148 * kQjResident ? 1 : 8;
    const int ctas = (int)(p.by_scores ? std::min(most, even) : (a.R + rows_each - 1) / rows_each);
    // Groups of lanes for a row's parts, four parts to each, and lanes for their sums: by the arguments alone, as is the order
    // of the sums then.
    const int64_t parts = a.n_warps / (units * a.n_groups) + 1;
    int share = 1;
    while (share < 16 && share * 4 < parts) share *= 2;
    const int ml_lanes = parts > 48 ? 32 : 8;
    const auto kernel = !p.by_scores ? qc_join_kernel<T, D, false, false> : a.R == 1 ? qc_join_kernel<T, D, true, true> : qc_join_kernel<T, D, true, false>;
    e = pdl_launch(kernel, (unsigned)(units * ctas), kQjThreads, 0, s, a, ctas, p.rows, share, ml_lanes, rows_each);
    if constexpr (TERMS == 2) {   // (many bfloat16 rows are the tensor path's)
        if (e == cudaSuccess && a.accumulate != 0 && !p.by_scores)
            e = pdl_launch(qc_weights_kernel<T, D, TERMS>, (unsigned)(units * a.c.NB), 32 * kQwWarps<D>, 0, s, a);
    }
    return e;
}

}  // namespace

int qc_attend_max_warps() { return 148 * kQaWarps; }

cudaError_t qc_attend(const QcAttend& a, const QcPlan& p, int dtype, cudaStream_t s) {
    if (dtype == BCT_BF16)
        return a.c.D == 128 ? attend_of<__nv_bfloat16, 128, 1>(a, p, s) : attend_of<__nv_bfloat16, 64, 1>(a, p, s);
    return a.c.D == 128 ? attend_of<float, 128, 2>(a, p, s) : attend_of<float, 64, 2>(a, p, s);
}

}  // namespace bct
