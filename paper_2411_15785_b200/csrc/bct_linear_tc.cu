// Linear attention with a decay for each head on the sm_100a tensor path: the chunked scan for bfloat16 (the forward, and
// the three scans of the backward; bct_linear.h names the roles a, b, c).
//
// Per (sequence, kv-head) unit and chunk of 128 tokens, X being the state outside the chunk:
//     W     = A B^T                                 products of all pairs   [i][j]
//     P_ij  = W_ij lambda^|i-j| / f_i               j <= i (j >= i in reverse), bfloat16
//     O     = A X + P C                             [i][feature of c]
//     out_i = scale f_i O_i                         f_i = lambda^(distance of i to X's token)
//     X    <- lambda^n X + (w o B)^T C              w_j = lambda^(distance of j to the new X's token)
// all as tcgen05.mma with M = 128 and N = 128 (64 columns of results with head_dim 64) and fp32 accumulators in tensor
// memory.  What bounds it is the traffic of shared memory (operands, tiles, results at 128 bytes a clock: some 4400 of a
// chunk's 6400 clocks), so operands are kept in tensor memory where they can be:
//  - W's columns are reused for P once its rows have been read.
//  - B^T comes into tensor memory as a product with a 16 x 16 unit matrix, is multiplied with w there and split into
//    three bfloat16 terms in place: 24 bits, so that the fp32 state is as good as one of fp32 sums.  (Two terms leave
//    2.8e-6 of it; they took 220 instead of 249 us for 8 x 4096 tokens of 32 heads.)  Weighted in shared memory it took
//    2300 clocks of traffic a chunk instead of 800.
//  - The state accumulates in tensor memory, b's features in the lanes.  Once per chunk it is read, written to shared
//    memory in bfloat16 as the operand X, and scaled.  Where a slow decay would let the sums' cut-off show in a float
//    state, only what X leaves out stays in tensor memory (by_parts, below).
//  - f_i multiplies the whole row at the end instead of A's row, so A goes into both products as it is.  It is
//    floored at 2^-64.  That is off by 2^-64 of the state's share at most, and leaves W and the results a range of 2^63: O
//    is up to 2^64 times too large.  (Both come out of the one accumulator that A X and P C share, so that a floor divides
//    fp32's range between them; at 2^-40 a state 2^40 times what the tokens add stayed visible under a strong decay.)
//  - P and X are each rounded to bfloat16 once, where they enter a product with bfloat16 results.
// Roles: warp 0 issues the products of the outputs (W, A X, P C), warp 3 those of the state (B^T and its terms with C, a
// quarter tile at a time; one warp for both waited for one while the other was ready, 300 instead of 249 us), warp 1 loads
// (TMA), warp 2 stores (TMA); warps 4-11 turn W into P, warps 12-19 weight and split B^T, warps 20-27 keep the state and
// write the outputs, over the A tile that has been read.  With several heads of A to a state, whose W and P also use the
// place of B^T, warp 0 issues everything: W, A X, the state's products while P is formed, P C.  With more than one
// segment, the same kernel without A, W and P forms what every segment adds.  Every wait is bounded; a timeout ends the
// work and fills the block's outputs with NaN.
//
// Measured, decays spread over the heads from exp(-0.84) to exp(-0.004): 8 x 4096 tokens of 32 heads of 128 (1.11 GB)
// 259 us at full clock, 4.3 TB/s, 0.66 of the copy rate (244 before the slow quarter of the heads kept their states in two
// parts); the backward of 4 x 4096 (three scans) 372 us; 16384 tokens of one sequence, 32 heads over 8 states, 127 us (state
// pass 25, segments' states 5, outputs 88 to 97).  With one head to a state a chunk takes some 6400 clocks, of which the
// state's chain (its products 4600, the turn 1600, 1000 more in two parts) is the longest; the tensor cores are busy 44 %
// and the issue slots 49 % of the time.  With four heads of A to a state the state is formed once for four of them, and a
// (chunk, head) still takes 5100 to 5700 clocks: the warps that form P are busy 1300 of them, those that write outputs 1200,
// the tensor cores 2000; warp 0, which issues everything, waits for 1200 and is in its own loop for the rest.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "bct_internal.h"
#include "bct_linear.h"
#include "bct_tc.cuh"

namespace bct {
namespace {

constexpr int kLtThreads = 896;
constexpr int kLtCh = 128;                    // tokens per chunk
constexpr int kLtHalf = 128 * 128;            // 64 columns (128 bytes) x 128 rows
constexpr float kLtHuge = 8.507059173023462e37f;   // 2^126
// tensor-memory columns
constexpr int kLtColW = 0;     // W, then P (bfloat16 pairs) in the first half of each of its 64-column halves
constexpr int kLtColO = 128;
constexpr int kLtColS = 256;   // the state [feature of b][feature of c]
constexpr int kLtColT = 384;   // two places of 64 columns for B^T [feature of b][j] of a quarter tile, 32 columns; of every
                               // 16 of them 8 then hold the first terms, 8 the second, and 16 columns behind them the third.
                               // With several heads of A to a state also every other head's W and P

struct LtArgs {
    CUtensorMap in[4];    // forward: q, k, v;  backward: d_out, q, k, v
    CUtensorMap out[3];   // per role
    LinArgs s;
    LinStates st;
    int map_a[3], map_b[3], map_c[3];     // which of `in` a role reads
    int st_map_b[2], st_map_c[2];
};

template <int D, bool STATE_ONLY>
struct LtSmem {   // two buffers of every tile (three without A); everything else is kept small enough for that
    static constexpr int kLtTile = D / 64 * kLtHalf;   // bytes of a tile
    static constexpr int kBc = STATE_ONLY ? 3 : 2;     // buffers of B and of C
    static constexpr int b = 0;
    static constexpr int c = b + kBc * kLtTile;
    static constexpr int a = c + kBc * kLtTile;
    static constexpr int x = a + (STATE_ONLY ? 0 : 2 * kLtTile);   // the state as an operand: rows = features of b
    static constexpr int unit = x + (STATE_ONLY ? 0 : D * D * 2);  // 16 x 16 unit matrix
    static constexpr int bars = unit + 512;
    static constexpr int pt = bars + 38 * 8;           // [256]: lambda^(i - j) at 127 + j - i, reverse lambda^(j - i); else 0
    static constexpr int total = pt + 256 * 4 + 1024;  // slack to align the base to 1024 bytes
};

// The products are issued by a whole warp, one lane of which is elected: descriptors and addresses then stay in uniform
// registers.  A product of N = 128 takes 64 clocks; issued by one thread among 27 warps (a register move for every word of
// its descriptors) it took 95 to 170.  Several go out under one election.
#define LT_UMMA "tcgen05.mma.cta_group::1.kind::f16 "
// D (+)= A B over four steps of 16, whose descriptors are DA and DB apart
template <int DA, int DB>
__device__ __forceinline__ void umma4_warp(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, bool accum) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q " LT_UMMA "[%0], %1, %2, %3, p;\n\t"
        "setp.eq.b32 p, 0, 0;\n\t"
        "add.s64 a, %1, %5;\n\tadd.s64 b, %2, %6;\n\t"
        "@q " LT_UMMA "[%0], a, b, %3, p;\n\t"
        "add.s64 a, %1, %7;\n\tadd.s64 b, %2, %8;\n\t"
        "@q " LT_UMMA "[%0], a, b, %3, p;\n\t"
        "add.s64 a, %1, %9;\n\tadd.s64 b, %2, %10;\n\t"
        "@q " LT_UMMA "[%0], a, b, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"((uint32_t)accum),
          "n"(DA), "n"(DB), "n"(2 * DA), "n"(2 * DB), "n"(3 * DA), "n"(3 * DB)
        : "memory");
}
// D += A B over four steps with A (bfloat16 pairs, 8 columns a step) in tensor memory
template <int DB>
__device__ __forceinline__ void umma4_warp_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b32 a;\n\t.reg .b64 b;\n\t"
        "setp.eq.b32 p, 0, 0;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q " LT_UMMA "[%0], [%1], %2, %3, p;\n\t"
        "add.s32 a, %1, 8;\n\tadd.s64 b, %2, %4;\n\t"
        "@q " LT_UMMA "[%0], [a], b, %3, p;\n\t"
        "add.s32 a, %1, 16;\n\tadd.s64 b, %2, %5;\n\t"
        "@q " LT_UMMA "[%0], [a], b, %3, p;\n\t"
        "add.s32 a, %1, 24;\n\tadd.s64 b, %2, %6;\n\t"
        "@q " LT_UMMA "[%0], [a], b, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "n"(DB), "n"(2 * DB), "n"(3 * DB)
        : "memory");
}
// D (+)= (the three terms of a quarter tile) C: two steps of 16 tokens, `step` apart in C's descriptor, the small terms first
__device__ __forceinline__ void umma_terms_warp(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, int64_t step, uint32_t idesc,
                                                bool accum) {
    asm volatile(
        "{\n\t.reg .pred p, q, c;\n\t.reg .b32 a;\n\t.reg .b64 b;\n\t"
        "setp.eq.b32 p, 0, 0;\n\t"
        "setp.ne.b32 c, %5, 0;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "add.s32 a, %1, 32;\n\t"
        "@q " LT_UMMA "[%0], [a], %2, %3, c;\n\t"
        "add.s32 a, %1, 8;\n\t"
        "@q " LT_UMMA "[%0], [a], %2, %3, p;\n\t"
        "@q " LT_UMMA "[%0], [%1], %2, %3, p;\n\t"
        "add.s32 a, %1, 40;\n\tadd.s64 b, %2, %4;\n\t"
        "@q " LT_UMMA "[%0], [a], b, %3, p;\n\t"
        "add.s32 a, %1, 24;\n\t"
        "@q " LT_UMMA "[%0], [a], b, %3, p;\n\t"
        "add.s32 a, %1, 16;\n\t"
        "@q " LT_UMMA "[%0], [a], b, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "l"(step), "r"((uint32_t)accum)
        : "memory");
}
// A quarter of B^T: two steps of 16 tokens, `step` apart in B's descriptor and 16 columns in the result
__device__ __forceinline__ void umma_transpose_warp(uint32_t tmem_d, uint64_t adesc, int64_t step, uint64_t unit, uint32_t idesc,
                                                    uint64_t* bar) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b32 d;\n\t.reg .b64 a;\n\t"
        "setp.ne.b32 p, 0, 0;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q " LT_UMMA "[%0], %1, %2, %3, p;\n\t"
        "add.s32 d, %0, 16;\n\tadd.s64 a, %1, %5;\n\t"
        "@q " LT_UMMA "[d], a, %2, %3, p;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%4];\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(unit), "r"(idesc), "r"(smem_u32(bar)), "l"(step)
        : "memory");
}
__device__ __forceinline__ void umma_commit_warp(uint64_t* bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void tmem_st8u(uint32_t taddr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void tmem_st16u(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tma_store_4d(const CUtensorMap* map, int x, int y, int z, int w, const void* src) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%1, %2, %3, %4}], [%5];"
                 ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(src))
                 : "memory");
}

// eight bfloat16 numbers as pairs of floats
__device__ __forceinline__ void unpack4(const uint4& w, float2 (&x)[4]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = make_float2(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xffff0000u));
}

// Bounded wait.  try_wait is given a suspend time, since most of the warps wait here at any time and every poll takes an
// issue slot; the limit is four seconds of the global timer, a thousandth of that once a wait has failed.
__device__ __forceinline__ void lt_wait_slow(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
    const unsigned long long limit = *abort_flag ? 4000000ull : 4000000000ull;
    for (;;) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 20000;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(smem_u32(bar)), "r"(parity)
            : "memory");
        if (ok) return;
        asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
        if (t - t0 > limit) {
            *abort_flag = 1;
            return;
        }
    }
}
__device__ __forceinline__ void lt_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    if (!mbar_try_wait(bar, parity)) lt_wait_slow(bar, parity, abort_flag);
}

// One look at a barrier, without a wait.
__device__ __forceinline__ bool mbar_test_wait(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok;
}

// MULTI_A: every role has several heads on A's side (and one on B's).
template <int D, bool STATE_ONLY, bool MULTI_A>
__global__ void __launch_bounds__(kLtThreads, 1) linear_tc_kernel(const __grid_constant__ LtArgs args) {
    using L = LtSmem<D, STATE_ONLY>;
    constexpr int kLtTile = L::kLtTile, kHalves = D / 64;
    extern __shared__ unsigned char lt_smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(lt_smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::bars);
    uint64_t* full_a = bars;             // [3]
    uint64_t* empty_a = bars + 3;        // [3] the output that took A's place has been read out
    uint64_t* out_full = bars + 6;       // [3] the output is in A's place
    uint64_t* full_b = STATE_ONLY ? bars : bars + 9;        // [2] (without A: [3], in the place of the three above)
    uint64_t* empty_b = STATE_ONLY ? bars + 3 : bars + 11;
    uint64_t* full_c = bars + 13;        // [2]
    uint64_t* empty_c = STATE_ONLY ? bars + 6 : bars + 15;
    // padding rows of B and C are zeros, by padded tiles in turn: [2].  Two warps look at it and only one of them paces the
    // warps that arrive, so that one barrier could go through two phases between two looks of the other warp, which would
    // then wait for good; a phase that is two tiles on needs a buffer that both have given back.
    auto clean = [&](int n) { return bars + (n & 1 ? 37 : 17); };
    uint64_t* bt_full = bars + 18;       // [4] a quarter of B^T complete, by places
    uint64_t* terms_full = bars + 22;    // [4] its terms in place
    uint64_t* w_full = bars + 26;        // [2] W complete, by items in turn
    uint64_t* p_full = bars + 28;        // [2] P in place
    uint64_t* kv_done = w_full;          // [4] without W and P: a quarter's products with C complete, by places
    uint64_t* o_full = bars + 30;
    uint64_t* o_empty = bars + 31;
    uint64_t* s_full = bars + 32;        // the state holds the chunk
    uint64_t* x_full = bars + 33;        // X in place, the state scaled
    uint64_t* x_empty = bars + 34;       // the products with X complete
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 35);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 36);
    float* pt = reinterpret_cast<float*>(smem + L::pt);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const LinArgs& s = args.s;
    const int seg = blockIdx.x % s.nseg;
    const int u = blockIdx.x / s.nseg;
    const int bi = u / s.Hkv, h = u - bi * s.Hkv;
    const int which = STATE_ONLY ? (args.st.seg[0] == nullptr ? 1 : (int)blockIdx.y) : (int)blockIdx.y;
    const LinRole& r = s.role[STATE_ONLY ? 0 : which];
    const int reverse = STATE_ONLY ? which : r.reverse;
    const int Ga = MULTI_A ? r.Ga : 1, Gb = MULTI_A ? 1 : (STATE_ONLY ? args.st.G[which] : r.Gb);
    const bool by_head = STATE_ONLY && args.st.by_head != nullptr;   // (s.Hkv counts the heads of b then)
    if (STATE_ONLY && !by_head && seg == (reverse ? 0 : s.nseg - 1)) return;   // feeds no other segment
    const CUtensorMap* map_a = &args.in[STATE_ONLY ? 0 : args.map_a[which]];
    const CUtensorMap* map_b = &args.in[STATE_ONLY ? args.st_map_b[which] : args.map_b[which]];
    const CUtensorMap* map_c = &args.in[STATE_ONLY ? args.st_map_c[which] : args.map_c[which]];

    const int len = s.lens ? min(max(s.lens[bi], 0), s.T) : s.T;
    const int t_begin = seg * s.seg_len;
    const int t_end = min(t_begin + s.seg_len, s.T);
    const int v_end = min(t_end, len);
    const int n_chunks = v_end > t_begin ? (v_end - t_begin + kLtCh - 1) / kLtCh : 0;
    const int G = MULTI_A ? Ga : Gb;
    auto chunk_t0 = [&](int n) { return t_begin + (reverse ? n_chunks - 1 - n : n) * kLtCh; };
    auto chunk_nv = [&](int t0) { return min(kLtCh, v_end - t0); };

    // The state is read in two rounds by the threads that keep it; here it is asked for into L2.
    const float* state_src = nullptr;
    if (!STATE_ONLY) state_src = s.nseg > 1 ? r.seg + ((size_t)u * s.nseg + seg) * (D * D) : (r.state_in ? r.state_in + (size_t)u * (D * D) : nullptr);
    if (state_src != nullptr && tid < D * D / 32) asm volatile("prefetch.global.L2 [%0];" ::"l"(state_src + tid * 32));
    if (tid == 0) {
        for (int i = 0; i < 3; ++i) {
            mbar_init(&full_a[i], 1);
            mbar_init(&empty_a[i], 1);
            mbar_init(&out_full[i], STATE_ONLY ? 1 : 8);
        }
        for (int i = 0; i < 2; ++i) {
            if (!STATE_ONLY) {
                mbar_init(&full_b[i], 1);
                mbar_init(&empty_b[i], MULTI_A ? 1 : 2);   // (two warps issue products that read it)
                mbar_init(&full_c[i], 1);
                mbar_init(&empty_c[i], MULTI_A ? 1 : 2);
            }
            mbar_init(&w_full[i], 1);
            mbar_init(&p_full[i], STATE_ONLY ? 1 : 8);
        }
        mbar_init(clean(0), 8);
        mbar_init(clean(1), 8);
        for (int i = 0; i < 4; ++i) {
            mbar_init(&bt_full[i], 1);
            mbar_init(&terms_full[i], 8);
        }
        mbar_init(o_full, 1);
        mbar_init(o_empty, 8);
        mbar_init(s_full, 1);
        mbar_init(x_full, 8);
        mbar_init(x_empty, 1);
        *abort_flag = 0;
        fence_mbar_init_cluster();
    }
    if (warp == 0) tmem_alloc(tmem_slot, 512);
    const float log_decay = s.log_decay[by_head ? h / args.st.heads : h];
    if (tid < 256) {   // the powers in double, rounded once
        const int d = reverse ? tid - 127 : 127 - tid;
        pt[tid] = d < 0 ? 0.f : (d == 0 ? 1.f : (float)exp((double)log_decay * d));
    } else if (tid < 512) {
        const int n = (tid - 256) >> 4, k = tid & 15;   // blocks of 8 rows x 16 bytes
        reinterpret_cast<unsigned short*>(smem + L::unit)[(n >> 3) * 128 + (k >> 3) * 64 + (n & 7) * 8 + (k & 7)] = n == k ? 0x3f80 : 0;
    }
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    // lambda^e, 0 <= e <= 128
    auto lam = [&](int e) { return reverse ? pt[127 + e] : (e < 128 ? pt[127 - e] : pt[0] * pt[126]); };
    // f of row i in a chunk of nv valid tokens
    auto f_of = [&](int i, int nv) { return fmaxf(lam(reverse ? max(nv - 1 - i, 0) : i + 1), 5.421010862427522e-20f); };   // 2^-64
    const int nv_last = n_chunks > 0 ? (v_end - t_begin - 1) % kLtCh + 1 : kLtCh;   // of the one chunk that may be shorter
#define LT_WAIT(bar, parity) lt_wait(bar, (parity) & 1, abort_flag);

// for a whole warp that goes on together
#define LT_WAIT_WARP(bar, parity)    \
    {                                \
        LT_WAIT(bar, parity);        \
        __syncwarp();                \
    }
// for padded tile n, and n counted on
#define LT_WAIT_CLEAN(n)                     \
    {                                        \
        LT_WAIT_WARP(clean(n), (n) >> 1);    \
        ++(n);                               \
    }

    // Where the qb-th quarter tile of B is transposed.  (All four quarters' terms at once have no room beside W, O and the
    // state; in two halves that took turns in one place the state waited for them, 6450 clocks a chunk.)  Where nothing but
    // the state is formed, W's place makes two more.
    constexpr int kPlaces = STATE_ONLY ? 4 : 2;
    auto t_place = [&](int qb) { return (STATE_ONLY && (qb & 2) ? kLtColW : kLtColT) + (qb & 1) * 64; };

    // (Loops are kept short where that costs nothing: 28 warps of seven roles share the instruction caches, and straight-line
    // code that is run once per chunk is fetched anew each time.)
    const int items = n_chunks * G;   // (chunk, head) in turn: head x of the side that has G of them
    // Buffers: two of every tile; with several heads on A's side, whose tiles then turn over fastest, B's second one is a
    // third of A's.
    constexpr int n_a = MULTI_A ? 3 : 2, n_b = MULTI_A ? 1 : L::kBc;
    struct Ring {   // a place in a ring of buffers and the parity of its turn
        int s = 0;
        uint32_t turn = 0;
        __device__ __forceinline__ void next(int n) {
            if (++s == n) s = 0, turn ^= 1;
        }
    };
    auto a_at = [&](int st) { return st < 2 ? L::a + st * kLtTile : L::b + kLtTile; };
    if (warp == 1) {
        // =========================== loads ===========================
        if (lane == 0) {
            auto copy = [&](const CUtensorMap* map, int head, int t0, unsigned char* dst, uint64_t* bar) {
                for (int hf = 0; hf < kHalves; ++hf) tma_load_4d(dst + hf * kLtHalf, map, hf * 64, head, t0, bi, bar);
            };
            auto load = [&](const CUtensorMap* map, int head, int t0, unsigned char* dst, uint64_t* bar) {
                mbar_arrive_expect_tx(bar, kLtTile);
                copy(map, head, t0, dst, bar);
            };
            Ring ra, rb, rc;
            for (int n = 0; n < n_chunks; ++n) {
                const int t0 = chunk_t0(n);
                for (int x = 0; x < G; ++x) {
                    const bool new_b = x == 0 || Gb > 1, new_a = !STATE_ONLY && (x == 0 || Ga > 1);
                    const int hb = h * Gb + (Gb > 1 ? x : 0);
                    if (!MULTI_A) {   // one barrier for B and C: every wait costs the warp that issues the products
                        uint64_t* full = &full_b[rb.s];
                        LT_WAIT(&empty_b[rb.s], rb.turn ^ 1);
                        mbar_arrive_expect_tx(full, 2 * kLtTile);
                        copy(map_b, hb, t0, smem + L::b + rb.s * kLtTile, full);
                        LT_WAIT(&empty_c[rb.s], rb.turn ^ 1);
                        copy(map_c, hb, t0, smem + L::c + rb.s * kLtTile, full);
                        rb.next(n_b);
                        if (new_a) {   // (A's buffer is the last to be free: the output goes out of it)
                            LT_WAIT(&empty_a[ra.s], ra.turn ^ 1);
                            load(map_a, h, t0, smem + L::a + ra.s * kLtTile, &full_a[ra.s]);
                            ra.next(n_a);
                        }
                        continue;
                    }
                    if (new_b) {
                        LT_WAIT(&empty_b[rb.s], rb.turn ^ 1);
                        load(map_b, hb, t0, smem + L::b + rb.s * kLtTile, &full_b[rb.s]);
                        rb.next(n_b);
                    }
                    if (new_a) {
                        LT_WAIT(&empty_a[ra.s], ra.turn ^ 1);
                        load(map_a, h * Ga + (Ga > 1 ? x : 0), t0, smem + a_at(ra.s), &full_a[ra.s]);
                        ra.next(n_a);
                    }
                    if (new_b) {
                        LT_WAIT(&empty_c[rc.s], rc.turn ^ 1);
                        load(map_c, hb, t0, smem + L::c + rc.s * kLtTile, &full_c[rc.s]);
                        rc.next(2);
                    }
                }
            }
        }
        __syncwarp();
    } else if (warp == 0 || (!MULTI_A && warp == 3)) {
        // =========================== products ===========================
        constexpr uint32_t id_kk = instr_desc_mn(128, 128, false, false);
        constexpr uint32_t id_kn = instr_desc_mn(128, D, false, true);
        constexpr uint32_t id_t = instr_desc_mn(128, 16, true, false);
        const DescKind dk(smem_desc(0, 16, 1024)), dmn(smem_desc(0, kLtHalf, 1024));
        const uint32_t base16 = desc_addr16(smem_u32(smem)), x16 = base16 + L::x / 16;
        // the unit matrix is not swizzled: blocks of 8 rows x 16 bytes, 128 bytes apart along k, 256 along its rows
        const uint64_t unit = (smem_desc(0, 128, 256) & ~((uint64_t)7 << 61)) + base16 + L::unit / 16;
        constexpr uint32_t h16 = kLtHalf / 16;
        const int n_short = nv_last == kLtCh ? -1 : (reverse ? 0 : n_chunks - 1);   // the chunk with padding rows
        int n_clean = 0, n_t = 0;   // padded tiles, and quarter tiles of B transposed so far
        Ring ra, rb, rt, rc;   // A and B as W takes them, B as its transposition does, C
        uint32_t a_w = 0, b_w = 0, c_now = 0;
        int c_slot = 0;
        // The tensor cores' sums are cut off, not rounded, at every 16 tokens of a term (2^-25 of the sum on average, always
        // towards zero), so a chunk's tokens enter the state in the order of their weights, the largest last: from the last
        // 16 to the first in reverse.  128 tokens of lambda = 0.95 then leave a state 1.5e-7 off, in the other order 6.7e-7.
        auto first_of = [&](int quarter) { return reverse ? 896 - 256 * quarter : 256 * quarter; };   // 16-byte units
        const int64_t step_t = reverse ? -128 : 128;
        // B^T of the next quarter tile of B, which belongs to chunk n.  (With head_dim 64 the upper 64 rows of this product,
        // and of the state's, come from what lies behind the tile; nothing reads them.)
        auto transpose = [&](int n) {
            const int quarter = n_t & 3;
            if (quarter == 0) {
                LT_WAIT_WARP(&full_b[rt.s], rt.turn);
                if (n == n_short) LT_WAIT_CLEAN(n_clean);
            }
            tc_fence_after();
            const uint32_t ba = base16 + (L::b + rt.s * kLtTile) / 16 + first_of(quarter);
            umma_transpose_warp(tmem + t_place(n_t), dmn.at(ba), step_t, unit, id_t, &bt_full[n_t % kPlaces]);
            if (quarter == 3) {
                if (!MULTI_A) umma_commit_warp(&empty_b[rt.s]);
                rt.next(n_b);
            }
            ++n_t;
        };
        // With several heads on A's side every other one's W goes where B^T was, which is free from the chunk's share of
        // the state until the next chunk: the next head's W then does not wait for this one's P.
        auto w_col = [&](int x) { return MULTI_A && (x & 1) ? kLtColT : kLtColW; };
        auto w_products = [&](int it, int x) {
            if (x == 0 || Ga > 1) {
                LT_WAIT_WARP(&full_a[ra.s], ra.turn);
                a_w = base16 + a_at(ra.s) / 16;
                ra.next(n_a);
            }
            const bool new_b = x == 0 || Gb > 1;
            if (new_b) {
                LT_WAIT_WARP(&full_b[rb.s], rb.turn);
                b_w = rb.s;
                rb.next(n_b);
            }
            tc_fence_after();
            const uint32_t col = tmem + w_col(x), ba = base16 + (L::b + b_w * kLtTile) / 16;
#pragma unroll
            for (int hf = 0; hf < kHalves; ++hf) umma4_warp<2, 2>(col, dk.at(a_w + hf * h16), dk.at(ba + hf * h16), id_kk, hf > 0);
            umma_commit_warp(&w_full[it & 1]);
            if (Gb > 1 || x == G - 1) umma_commit_warp(&empty_b[b_w]);
        };
        auto state_products = [&](int qb, uint32_t ca, bool accum = true) {   // a quarter tile's share of the state
            LT_WAIT_WARP(&terms_full[qb % kPlaces], qb / kPlaces);
            tc_fence_after();
            umma_terms_warp(tmem + kLtColS, tmem + t_place(qb), dmn.at(ca + first_of(qb & 3)), step_t, id_kn, accum);
        };
        auto ready = [&](uint64_t* bar, uint32_t parity) { return (bool)__all_sync(0xffffffffu, mbar_test_wait(bar, parity & 1)); };
        if constexpr (STATE_ONLY) {
            // (An item's C has come with its B.)  One warp transposes, up to four quarters ahead, the other adds to the state:
            // with both in one, 5200 instead of 4200 clocks a chunk went by in issuing them in turn.  (What is left is the chain
            // of the products and the turn; the idle warps of W and P beside those that weight B^T changed nothing.)
            int x = 0;
            if (warp == 3) {
                for (int n = 0, qb = 0; qb < 4 * items; ++qb) {
                    if (qb >= kPlaces) LT_WAIT_WARP(&kv_done[qb % kPlaces], qb / kPlaces - 1);
                    transpose(n);
                    if ((qb & 3) == 3 && ++x == G) x = 0, ++n;
                }
            } else {
                for (int n = 0, it = 0; it < items; ++it) {
                    const uint32_t ca = base16 + (L::c + rc.s * kLtTile) / 16;
                    if (x == 0) LT_WAIT_WARP(x_full, n);
#pragma unroll 1
                    for (int qb = 4 * it; qb < 4 * it + 4; ++qb) {
                        state_products(qb, ca, x > 0 || (qb & 3) > 0);
                        umma_commit_warp(&kv_done[qb % kPlaces]);
                    }
                    umma_commit_warp(&empty_c[rc.s]);
                    rc.next(n_b);
                    if (++x == G) {
                        umma_commit_warp(s_full);
                        x = 0, ++n;
                    }
                }
            }
        } else if (!MULTI_A && warp == 3) {
            // The state: quarters are transposed as far ahead of their products as there are places.  (An item's C has come
            // with its B.)
            int x = 0, xt = 0, nt = 0;   // xt, nt: of the next tile to be transposed
            for (int n = 0, it = 0; it < items; ++it) {
                const uint32_t ca = base16 + (L::c + rc.s * kLtTile) / 16;
#pragma unroll 1
                for (int qb = 4 * it; qb < 4 * it + 4; ++qb) {
                    while (n_t < 4 * items && n_t < qb + kPlaces && (n_t <= qb || (n_t & 3) != 0 || ready(&full_b[rt.s], rt.turn))) {
                        transpose(nt);
                        if ((n_t & 3) == 0 && ++xt == G) xt = 0, ++nt;
                    }
                    if (qb == 4 * it && x == 0) LT_WAIT_WARP(x_full, n);
                    state_products(qb, ca);
                }
                umma_commit_warp(&empty_c[rc.s]);
                rc.next(n_b);
                if (++x == G) {
                    umma_commit_warp(s_full);
                    x = 0, ++n;
                }
            }
        } else if constexpr (!MULTI_A) {
            // The outputs.
            int x = 0;
            for (int n = 0, it = 0; it < items; ++it) {
                const uint32_t aa = base16 + (L::a + (n & 1) * kLtTile) / 16, ba = base16 + (L::b + rb.s * kLtTile) / 16;
                const uint32_t ca = base16 + (L::c + rb.s * kLtTile) / 16;
                LT_WAIT_WARP(&full_b[rb.s], rb.turn);
                if (x == 0) LT_WAIT_WARP(&full_a[n & 1], n >> 1);
                tc_fence_after();
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf)
                    umma4_warp<2, 2>(tmem + kLtColW, dk.at(aa + hf * h16), dk.at(ba + hf * h16), id_kk, hf > 0);
                umma_commit_warp(&w_full[it & 1]);
                umma_commit_warp(&empty_b[rb.s]);
                if (x == 0) {             // the state's share
                    LT_WAIT_WARP(x_full, n);
                    if (n > 0) LT_WAIT_WARP(o_empty, n - 1);
                    tc_fence_after();
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf)
                        umma4_warp<2, 128>(tmem + kLtColO, dk.at(aa + hf * h16), dmn.at(x16 + hf * 512), id_kn, hf > 0);
                    umma_commit_warp(x_empty);
                }
                if (n == n_short) LT_WAIT_CLEAN(n_clean);
                LT_WAIT_WARP(&p_full[it & 1], it >> 1);
                tc_fence_after();
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
                    umma4_warp_ts<128>(tmem + kLtColO, tmem + kLtColW + hf * 64, dmn.at(ca + hf * 512), id_kn);
                umma_commit_warp(&empty_c[rb.s]);
                rb.next(n_b);
                if (++x == G) {
                    umma_commit_warp(o_full);
                    x = 0, ++n;
                }
            }
        } else {
        bool w_ahead = false;
        int n = 0, x = 0, na = 0, nb = 0;
        if (items > 0) transpose(0), transpose(0);
        for (int it = 0; it < items; ++it) {
            const bool new_b = x == 0 || Gb > 1, new_a = x == 0 || Ga > 1, last = x == G - 1, more = it + 1 < items;
            const int n1 = last ? n + 1 : n, x1 = last ? 0 : x + 1;      // the next item
            if (!w_ahead) w_products(it, x);
            w_ahead = false;
            if (x == 0) LT_WAIT_WARP(x_full, n);
            if (new_a) {   // the state's share
                if (na > 0) LT_WAIT_WARP(o_empty, na - 1);
                tc_fence_after();
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf)
                    umma4_warp<2, 128>(tmem + kLtColO, dk.at(a_w + hf * h16), dmn.at(x16 + hf * 512), id_kn, hf > 0);
                if (Gb > 1 || last) umma_commit_warp(x_empty);
            }
            if (new_b) {
                LT_WAIT_WARP(&full_c[rc.s], rc.turn);
                c_now = base16 + (L::c + rc.s * kLtTile) / 16;
                c_slot = rc.s;
                rc.next(2);
            }
            int add = new_b ? 4 : 0;                 // quarters of the chunk's share of the state
            bool put = true;                         // this item's last product
            int next_b = (Gb > 1 || last) && more ? 2 : 0;   // quarters of B that the next chunk's first item begins with
            while (add || put || next_b) {
                // with several heads of A, P may well be there before B^T has been weighted
                if (add && !(put && ready(&p_full[it & 1], it >> 1))) {
                    state_products(4 * nb + 4 - add, c_now);
                    if (--add >= 2) transpose(n);   // the third and the fourth
                    if (add == 0) umma_commit_warp(s_full);
                    continue;
                }
                // the next tile's transposition before this item's last product, if the tile is there and its place free
                if (next_b && !add && (!put || (w_col(x) != kLtColT && ((n_t & 3) != 0 || ready(&full_b[rt.s], rt.turn))))) {
                    transpose(n1);
                    --next_b;
                    continue;
                }
                // and the next item's W, if it has a place of its own
                if (put && more && !add && !w_ahead && w_col(x1) != w_col(x) &&
                    __all_sync(0xffffffffu, mbar_try_wait(&full_a[ra.s], ra.turn) &&
                                                (x1 != 0 || mbar_try_wait(&full_b[rb.s], rb.turn)))) {
                    w_products(it + 1, x1);
                    w_ahead = true;
                }
                if (put) {
                    LT_WAIT_WARP(&p_full[it & 1], it >> 1);
                    tc_fence_after();
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf)
                        umma4_warp_ts<128>(tmem + kLtColO, tmem + w_col(x) + hf * 64, dmn.at(c_now + hf * 512), id_kn);
                    if (Ga > 1 || last) umma_commit_warp(o_full);
                    if (Gb > 1 || last) umma_commit_warp(&empty_c[c_slot]);
                    put = false;
                }
            }
            na += new_a;
            nb += new_b;
            x = x1;
            n = n1;
        }
        }
        __syncwarp();
    } else if (warp < 4) {
        // =========================== stores ===========================
        if (!STATE_ONLY && warp == 2 && lane == 0) {
            const CUtensorMap* map_o = &args.out[which];
            Ring ra;
            for (int n = 0; n < n_chunks; ++n) {
                const int t0 = chunk_t0(n);
                for (int x = 0; x < Ga; ++x) {
                    const unsigned char* src = smem + a_at(ra.s);
                    LT_WAIT(&out_full[ra.s], ra.turn);
                    for (int hf = 0; hf < kHalves; ++hf) tma_store_4d(map_o, hf * 64, h * Ga + x, t0, bi, src + hf * kLtHalf);
                    bulk_commit();
                    bulk_wait_read();
                    mbar_arrive(&empty_a[ra.s]);
                    ra.next(n_a);
                }
            }
            bulk_wait_all();
        }
        __syncwarp();
    } else if (warp < 12) {
        // =========================== W -> P: two threads per row i, 64 columns each ===========
        if (!STATE_ONLY) {
            const int q = warp & 3, half = (warp - 4) >> 2, i = q * 32 + lane;
            const uint32_t lane_w = tmem + ((uint32_t)(q * 32) << 16) + half * 64;
            const float* pti = pt + 127 - i;
            const float inv_full = 1.f / f_of(i, kLtCh), inv_last = 1.f / f_of(i, nv_last);
            int it = 0;
            for (int n = 0; n < n_chunks; ++n) {
                const int nv = chunk_nv(chunk_t0(n));
                const float inv_f = nv < kLtCh ? inv_last : inv_full;
                for (int x = 0; x < G; ++x, ++it) {
                    const uint32_t lane_base = lane_w + (MULTI_A && (x & 1) ? kLtColT : kLtColW);
                    LT_WAIT(&w_full[it & 1], it >> 1);
                    tc_fence_after();
#pragma unroll 1
                    for (int e = 0; e < 2; ++e) {   // 32 columns; P takes the place of columns read before
                        const int cb = half * 2 + e, j0 = cb * 32;
                        float v[32];
                        if (reverse ? cb < q : cb > q) {   // the mask leaves nothing
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = 0.f;
                        } else {
                            tmem_ld32(lane_base + e * 32, v);
                            if (cb == q) {   // the mask's edge runs through this block
#pragma unroll
                                for (int j = 0; j < 32; ++j) {
                                    const float w = pti[j0 + j];
                                    v[j] = w > 0.f ? v[j] * (w * inv_f) : 0.f;
                                }
                            } else {         // a power for the row and the block, one for the column
                                const float wr = lam(reverse ? j0 - i - 1 : i - j0 - 31) * inv_f;
#pragma unroll
                                for (int j = 0; j < 32; j += 4) {
                                    const float4 wc = *reinterpret_cast<const float4*>(pt + (reverse ? 128 : 96) + j);
                                    const float2 y = __fmul2_rn(__fmul2_rn(make_float2(v[j], v[j + 1]), make_float2(wc.x, wc.y)),
                                                                make_float2(wr, wr));
                                    const float2 z = __fmul2_rn(__fmul2_rn(make_float2(v[j + 2], v[j + 3]), make_float2(wc.z, wc.w)),
                                                                make_float2(wr, wr));
                                    v[j] = y.x, v[j + 1] = y.y, v[j + 2] = z.x, v[j + 3] = z.y;
                                }
                            }
                            if (nv < kLtCh) {   // products with padding rows, which hold anything
#pragma unroll
                                for (int j = 0; j < 32; ++j) v[j] = j0 + j < nv ? v[j] : 0.f;
                            }
                        }
#pragma unroll
                        for (int hf = 0; hf < 2; ++hf) {
                            uint32_t pk[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) pk[j] = Chunk<__nv_bfloat16>::pack2(v[16 * hf + 2 * j], v[16 * hf + 2 * j + 1]);
                            tmem_st8u(lane_base + e * 16 + hf * 8, pk);
                        }
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_full[it & 1]);
                }
            }
            // padding rows behind the last chunk
            constexpr int kRow = D * 2 / 16;   // 16-byte pieces of a row
            char* out = static_cast<char*>(r.out) + ((size_t)bi * s.T * s.Hkv + h) * Ga * (D * 2);
            const long long end = (long long)t_end * kRow;
            for (long long j = (long long)(t_begin + n_chunks * kLtCh) * kRow + tid - 128; j < end; j += 256)
                for (int x = 0; x < Ga; ++x)
                    reinterpret_cast<uint4*>(out + ((size_t)(j / kRow) * s.Hkv * Ga + x) * (D * 2))[j % kRow] = make_uint4(0, 0, 0, 0);
        }
    } else if (warp < 20) {
        // =========================== w o B^T in three terms: two threads per feature of b ===========
        const int q = warp & 3, part = (warp - 12) >> 2, wt = tid & 127;
        const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
        int nb = 0, n_clean = 0;
        Ring rb;
        for (int n = 0; n < n_chunks; ++n) {
            const int nv = chunk_nv(chunk_t0(n));
            const float* w = pt + (reverse ? 128 : kLtCh - nv);   // w_j = w[j], 0 behind the last valid token
            const bool aligned = reverse || (nv & 3) == 0;
            for (int x = 0; x < Gb; ++x, ++nb) {
                if (nv < kLtCh) {   // padding rows hold anything: zeros in B (this half of the warps) and in C (the other)
                    LT_WAIT(&full_b[rb.s], rb.turn);
                    if (MULTI_A) LT_WAIT(&full_c[nb & 1], nb >> 1);
                    if (wt >= nv) {
                        uint4* z = reinterpret_cast<uint4*>(smem + (part ? L::c + (MULTI_A ? nb & 1 : rb.s) * kLtTile : L::b + rb.s * kLtTile) + wt * 128);
#pragma unroll
                        for (int j = 0; j < 8 * kHalves; ++j) z[(j & 7) + (j >> 3) * (kLtHalf / 16)] = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(clean(n_clean));
                    ++n_clean;
                }
#pragma unroll 1
                for (int qb = 4 * nb; qb < 4 * nb + 4; ++qb) {
                    LT_WAIT(&bt_full[qb % kPlaces], qb / kPlaces);
                    tc_fence_after();
                    const uint32_t place = lane_base + t_place(qb), t_col = place + part * 16;
                    const float* wp = w + (reverse ? 112 - (qb & 3) * 32 - part * 16 : (qb & 3) * 32 + part * 16);
                    if (q * 32 < D) {   // (lanes without a feature only take part in the barriers)
                        float v[16];
                        tmem_ld16(t_col, v);
                        uint32_t o[16], o3[8];
#pragma unroll
                        for (int j = 0; j < 16; j += 4) {
                            const float4 wj = aligned ? *reinterpret_cast<const float4*>(wp + j)
                                                      : make_float4(wp[j], wp[j + 1], wp[j + 2], wp[j + 3]);
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                float2 y = __fmul2_rn(make_float2(v[j + 2 * k], v[j + 2 * k + 1]),
                                                      k ? make_float2(wj.z, wj.w) : make_float2(wj.x, wj.y));
#pragma unroll
                                for (int t = 0; t < 3; ++t) {
                                    const uint32_t term = Chunk<__nv_bfloat16>::pack2(y.x, y.y);
                                    (t < 2 ? o[8 * t + (j >> 1) + k] : o3[(j >> 1) + k]) = term;
                                    // what the term leaves out, exactly
                                    y = __ffma2_rn(make_float2(__uint_as_float(term << 16), __uint_as_float(term & 0xffff0000u)),
                                                   make_float2(-1.f, -1.f), y);
                                }
                            }
                        }
                        tmem_st16u(t_col, o);
                        tmem_st8u(place + 32 + part * 8, o3);
                        tmem_wait_st();
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&terms_full[qb % kPlaces]);
                }
                rb.next(n_b);
            }
        }
    } else {
        // =========================== the state and the outputs ===========================
        const int q = warp & 3, hs = (warp - 20) >> 2;   // lanes 32q.., columns 64 hs..
        const int c = q * 32 + lane;                      // this thread's feature of b; of the outputs, its row
        const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
        constexpr int kCols = D / 2;                      // columns of a thread, from hs * kCols on
        const bool has_row = q * 32 < D;                  // (head_dim 64: half of the lanes hold no row of the state)
        const uint32_t s_col = lane_base + kLtColS + hs * kCols;
        const uint32_t keep_col = lane_base + (STATE_ONLY ? kLtColO : kLtColS) + hs * kCols;   // where the state is at the end
        unsigned char* x_row = smem + L::x + (hs * kCols / 64) * (D * 128) + c * 128;
        constexpr int kPiece = kHalves == 2 ? 0 : 4;      // 16-byte pieces of a 128-byte row before hs = 1's
        // The state passes through X's place, kVia columns at a time, and every warp keeps to the bytes of X that it writes
        // itself (another warp may be a step ahead): piece `piece` of the warp's row `row`.
        constexpr int kVia = D / 4;
        auto via = [&](int row, int piece) { return x_row + (row - lane) * 128 + (((hs * kPiece + piece) ^ (row & 7)) * 16); };
        float* dst = nullptr;   // where the state goes
        if (STATE_ONLY)         // into the slot of the segment that it feeds (by head: its own), key's features in the rows
            dst = args.st.seg[which] + ((size_t)u * s.nseg + (by_head ? seg : (reverse ? seg - 1 : seg + 1))) * (D * D);
        else if (r.state_out != nullptr && seg == (reverse ? 0 : s.nseg - 1))
            dst = r.state_out + (size_t)u * (D * D);   // (never transposed)
        if (has_row) {
            const float* src = state_src;
            const float mul = STATE_ONLY || s.nseg > 1 ? 1.f : r.in_mul;
#pragma unroll 1
            for (int k = 0; k < kCols / kVia; ++k) {
                float v[kVia];
#pragma unroll
                for (int i = 0; i < kVia; ++i) v[i] = 0.f;
                if (!STATE_ONLY && src != nullptr) {
                    if (r.state_t) {
#pragma unroll
                        for (int i = 0; i < kVia; ++i) v[i] = src[(hs * kCols + k * kVia + i) * D + c];
                    } else {
                        // A thread's row is D * 4 bytes from its neighbour's: read so, the loads held up the whole SM's
                        // shared-memory pipe for 10 us.  Whole lines come into shared memory, then every thread its row.
#pragma unroll
                        for (int i = 0; i < kVia / 4; ++i) {
                            const int row = i * (128 / kVia) + lane / (kVia / 4), piece = lane % (kVia / 4);
                            cp_async16(via(row, piece), src + (q * 32 + row) * D + hs * kCols + k * kVia + piece * 4);
                        }
                        cp_async_commit();
                        cp_async_wait_all();
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < kVia / 4; ++i) {
                            const float4 x = *reinterpret_cast<const float4*>(via(lane, i));
                            v[4 * i] = x.x, v[4 * i + 1] = x.y, v[4 * i + 2] = x.z, v[4 * i + 3] = x.w;
                        }
                        __syncwarp();
                    }
#pragma unroll
                    for (int i = 0; i < kVia; ++i) v[i] *= mul;
                }
#pragma unroll
                for (int i = 0; i < kVia; i += 16) tmem_st16u(keep_col + k * kVia + i, reinterpret_cast<const uint32_t*>(v + i));
            }
            tmem_wait_st();
        }
        // The tensor cores cut their sums off towards zero, three times for 16 tokens, so that a state that stays under their
        // sum loses some 4e-7 of itself with every chunk and, a chunk leaving a share of L of it, 4e-7 / (1 - L) in all:
        // 1.2e-5 after 4096 tokens without a decay to speak of, in one call or in many.  Where that would be seen in a float
        // state (L > 1/4 over a chunk, or over the tokens of a shorter call) the state is kept in two parts: X, the operand,
        // and under the sum only what X leaves out, 2^-8 of it at most; X times the decay is added at the turn, with
        // rounding.  That makes a turn 1000 clocks longer (8 x 4096 tokens of 32 heads, all of them slow: 271 instead of
        // 244 us), so a scan whose state is only seen in bfloat16 does it from 64 chunks on, where the loss comes to a
        // hundredth of that rounding.  Without X there is room for the state beside the sum, for every decay.
        const bool by_parts = !STATE_ONLY && lam(n_chunks > 1 ? kLtCh : nv_last) > 0.25f && (dst != nullptr || n_chunks > 64);
        auto x_at = [&](int piece) { return reinterpret_cast<uint4*>(x_row + (((hs * kPiece + piece) ^ (c & 7)) * 16)); };
        if (by_parts && has_row) {   // X holds nothing yet
#pragma unroll
            for (int i = 0; i < kCols / 8; ++i) *x_at(i) = make_uint4(0, 0, 0, 0);
        }
        // The state, times g, and the last chunk's share.
        auto add_share = [&](float g) {
#pragma unroll 1
            for (int k = 0; k < kCols / 16; ++k) {
                float x[16], y[16];
                tmem_ld16(s_col + k * 16, x);
                if (STATE_ONLY) {
                    tmem_ld16(keep_col + k * 16, y);
                } else {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float2 hi[4];
                        unpack4(*x_at(2 * k + e), hi);
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[8 * e + 2 * i] = hi[i].x, y[8 * e + 2 * i + 1] = hi[i].y;
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float2 z = __ffma2_rn(make_float2(y[i], y[i + 1]), make_float2(g, g), make_float2(x[i], x[i + 1]));
                    x[i] = z.x, x[i + 1] = z.y;
                }
                tmem_st16u(keep_col + k * 16, reinterpret_cast<const uint32_t*>(x));
            }
            tmem_wait_st();
        };
        // Before chunk n: the state as chunk n's operand, and scaled for what chunk n adds.
        auto turn = [&](int n) {
            const float f = lam(chunk_nv(chunk_t0(n)));
            if (n > 0) {
                LT_WAIT(s_full, n - 1);
                if (!STATE_ONLY) LT_WAIT(x_empty, n - 1);
                tc_fence_after();
            }
            if (STATE_ONLY) {
                if (n > 0 && has_row) add_share(lam(chunk_nv(chunk_t0(n - 1))));
            } else if (by_parts) {
                const float g = n > 0 ? lam(chunk_nv(chunk_t0(n - 1))) : 1.f;
#pragma unroll 1
                for (int k = has_row ? 0 : kCols / 8; k < kCols / 8; ++k) {
                    float x[8];
                    float2 hi[4];
                    tmem_ld8(s_col + k * 8, x);
                    unpack4(*x_at(k), hi);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 y = __ffma2_rn(hi[i], make_float2(g, g), make_float2(x[2 * i], x[2 * i + 1]));
                        x[2 * i] = y.x, x[2 * i + 1] = y.y;
                    }
                    const uint4 p = Chunk<__nv_bfloat16>::pack(x);
                    *x_at(k) = p;
                    unpack4(p, hi);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 y = __fmul2_rn(__ffma2_rn(hi[i], make_float2(-1.f, -1.f), make_float2(x[2 * i], x[2 * i + 1])), make_float2(f, f));
                        // (what an infinity leaves out of itself is no number; a finite one leaves it as it is)
                        x[2 * i] = fmaxf(y.x, -kLtHuge), x[2 * i + 1] = fmaxf(y.y, -kLtHuge);
                    }
                    tmem_st8u(s_col + k * 8, reinterpret_cast<const uint32_t*>(x));
                }
            } else {
#pragma unroll 1
                for (int k = has_row ? 0 : kCols / 16; k < kCols / 16; ++k) {
                    float x[16];
                    tmem_ld16(s_col + k * 16, x);
                    *x_at(2 * k) = Chunk<__nv_bfloat16>::pack(x);
                    *x_at(2 * k + 1) = Chunk<__nv_bfloat16>::pack(x + 8);
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const float2 y = __fmul2_rn(make_float2(x[i], x[i + 1]), make_float2(f, f));
                        x[i] = y.x, x[i + 1] = y.y;
                    }
                    tmem_st16u(s_col + k * 16, reinterpret_cast<const uint32_t*>(x));
                }
            }
            tmem_wait_st();
            if (!STATE_ONLY) fence_proxy_async_smem();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(x_full);
        };
        const float f_full = STATE_ONLY ? 0.f : f_of(c, kLtCh) * r.scale, f_last = STATE_ONLY ? 0.f : f_of(c, nv_last) * r.scale;
        int na = 0;
        Ring ra;
        if (n_chunks > 0) turn(0);
        for (int n = 0; n < n_chunks; ++n) {
            if (STATE_ONLY) {
                if (n + 1 < n_chunks) turn(n + 1);
                continue;
            }
            const int nv = chunk_nv(chunk_t0(n));
            const float f = nv < kLtCh ? f_last : f_full;
            for (int x = 0; x < Ga; ++x, ++na) {
                // The chunk's last output and the state's turn: what is complete first goes first.  (The output has to leave
                // A's place before the tile after the next can be loaded; the next chunk's products wait for the state.)
                const bool turns = x == Ga - 1 && n + 1 < n_chunks;
                const bool out_first = !turns || __all_sync(0xffffffffu, mbar_test_wait(o_full, na & 1));
                if (!out_first) turn(n + 1);
                LT_WAIT(o_full, na);
                tc_fence_after();
                unsigned char* dst = smem + a_at(ra.s) + (hs * kCols / 64) * kLtHalf + c * 128;
#pragma unroll 1
                for (int k = 0; k < kCols / 16; ++k) {
                    float o[16];
                    tmem_ld16(lane_base + kLtColO + hs * kCols + k * 16, o);
                    if (k == kCols / 16 - 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(o_empty);
                    }
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const float2 y = __fmul2_rn(make_float2(o[i], o[i + 1]), make_float2(f, f));
                        o[i] = y.x, o[i + 1] = y.y;
                    }
                    uint4 lo = Chunk<__nv_bfloat16>::pack(o), hi = Chunk<__nv_bfloat16>::pack(o + 8);
                    if (c >= nv) lo = hi = make_uint4(0, 0, 0, 0);   // padding rows
                    const int pc = hs * kPiece + 2 * k;
                    *reinterpret_cast<uint4*>(dst + ((pc ^ (c & 7)) * 16)) = lo;
                    *reinterpret_cast<uint4*>(dst + (((pc + 1) ^ (c & 7)) * 16)) = hi;
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&out_full[ra.s]);
                ra.next(n_a);
                if (turns && out_first) turn(n + 1);
            }
        }
        if (n_chunks > 0) {
            LT_WAIT(s_full, n_chunks - 1);
            tc_fence_after();
            if ((STATE_ONLY || by_parts) && has_row && dst != nullptr) add_share(lam(chunk_nv(chunk_t0(n_chunks - 1))));
        }
        const float poison = *abort_flag ? __int_as_float(0x7fc00000) : 0.f, mul = STATE_ONLY ? 1.f : r.out_mul;
        if (dst != nullptr && has_row) {
#pragma unroll 1
            for (int k = 0; k < kCols / 16; ++k) {
                float x[16];
                tmem_ld16(keep_col + k * 16, x);
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = x[i] * mul + poison;
                if (STATE_ONLY) {   // (no X there, and nothing beside this)
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        *reinterpret_cast<float4*>(dst + c * D + hs * kCols + k * 16 + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
                } else {            // whole lines again, 16 columns at a time
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<float4*>(via(lane, i)) = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int row = i * 8 + lane / 4, piece = lane % 4;
                        *reinterpret_cast<float4*>(dst + (q * 32 + row) * D + hs * kCols + k * 16 + piece * 4) =
                            *reinterpret_cast<const float4*>(via(row, piece));
                    }
                    __syncwarp();
                }
            }
        }
    }
#undef LT_WAIT
#undef LT_WAIT_WARP
#undef LT_WAIT_CLEAN
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (!STATE_ONLY && *abort_flag != 0) {   // after a timeout everything is NaN
        constexpr int kRow = D * 2 / 16;
        char* out = static_cast<char*>(r.out) + ((size_t)bi * s.T * s.Hkv + h) * Ga * (D * 2);
        const long long end = (long long)t_end * kRow;
        for (long long i = (long long)t_begin * kRow + tid; i < end; i += kLtThreads)
            for (int x = 0; x < Ga; ++x)
                reinterpret_cast<uint4*>(out + ((size_t)(i / kRow) * s.Hkv * Ga + x) * (D * 2))[i % kRow] =
                    make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
    }
}

// [B][T][H][D] bfloat16 as (feature, head, token, sequence); one box is 64 features of one head for 128 tokens;
// tokens past T read as zeros and are not written.
bool lt_map(CUtensorMap* map, const void* base, int B, int T, int H, int D) {
    TensorMapEncodeFn fn = tensor_map_encode_fn();
    if (fn == nullptr) return false;
    const cuuint64_t row = (cuuint64_t)D * 2;
    const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)H, (cuuint64_t)T, (cuuint64_t)B};
    const cuuint64_t strides[3] = {row, (cuuint64_t)H * row, (cuuint64_t)T * H * row};
    const cuuint32_t box[4] = {64, 1, (cuuint32_t)kLtCh, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool STATE_ONLY, bool MULTI_A>
cudaError_t lt_launch(const LtArgs& a, int grid_y, cudaStream_t stream) {
    auto fn = linear_tc_kernel<D, STATE_ONLY, MULTI_A>;
    const int smem = LtSmem<D, STATE_ONLY>::total;
    static_assert(LtSmem<D, STATE_ONLY>::total <= 232448, "shared memory of a block");
    static std::atomic<unsigned long long> allowed{0};
    cudaError_t e = allow_smem(reinterpret_cast<const void*>(fn), smem, allowed);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)(a.s.B * a.s.Hkv * a.s.nseg), (unsigned)grid_y);
    fn<<<grid, kLtThreads, smem, stream>>>(a);
    return cudaGetLastError();
}

template <int D, bool MULTI_A>
cudaError_t launch_all(const LinArgs& args, const LinStates& states, cudaStream_t stream) {
    LtArgs a;
    a.s = args;
    a.st = states;
    int n_in = 0;
    const void* base[4] = {};
    int base_heads[4] = {};
    auto map_of = [&](const void* p, int heads) -> int {   // one map per tensor
        for (int i = 0; i < n_in; ++i)
            if (base[i] == p && base_heads[i] == heads) return i;
        if (n_in == 4 || !lt_map(&a.in[n_in], p, args.B, args.T, args.Hkv * heads, D)) return -1;
        base[n_in] = p;
        base_heads[n_in] = heads;
        return n_in++;
    };
    for (int i = 0; i < args.n_roles; ++i) {
        const LinRole& r = args.role[i];
        a.map_a[i] = map_of(r.a, r.Ga);
        a.map_b[i] = map_of(r.b, r.Gb);
        a.map_c[i] = map_of(r.c, r.Gb);
        if (a.map_a[i] < 0 || a.map_b[i] < 0 || a.map_c[i] < 0) return cudaErrorInvalidValue;
        if (!lt_map(&a.out[i], r.out, args.B, args.T, args.Hkv * r.Ga, D)) return cudaErrorInvalidValue;
    }
    if (states.by_head != nullptr) {
        // A state that G heads add to, G tiles to a chunk, would be off by G times what the cutting off of the tensor
        // cores' sums leaves (2.6e-6 with four heads); by head it is as exact as with one.
        a.st_map_b[1] = map_of(states.b[1], states.heads);
        a.st_map_c[1] = map_of(states.c[1], states.heads);
        if (a.st_map_b[1] < 0 || a.st_map_c[1] < 0) return cudaErrorInvalidValue;
        LtArgs x = a;
        x.s.Hkv = args.Hkv * states.heads;
        x.st.G[1] = 1;
        x.st.seg[0] = nullptr, x.st.seg[1] = states.by_head;
        cudaError_t e = lt_launch<D, true, false>(x, 1, stream);
        if (e == cudaSuccess) e = launch_linear_combine_heads(D, args, states, stream);
        if (e != cudaSuccess) return e;
    } else if (args.nseg > 1) {
        for (int d = 0; d < 2; ++d) {
            if (states.seg[d] == nullptr) continue;
            a.st_map_b[d] = map_of(states.b[d], states.G[d]);
            a.st_map_c[d] = map_of(states.c[d], states.G[d]);
            if (a.st_map_b[d] < 0 || a.st_map_c[d] < 0) return cudaErrorInvalidValue;
        }
        const int dirs = (states.seg[0] != nullptr) + (states.seg[1] != nullptr);
        cudaError_t e = lt_launch<D, true, false>(a, dirs, stream);
        if (e == cudaSuccess) e = launch_linear_combine(D, args, states, stream);
        if (e != cudaSuccess) return e;
    }
    return lt_launch<D, false, MULTI_A>(a, args.n_roles, stream);
}

}  // namespace

cudaError_t launch_linear_tc(int D, const LinArgs& args, const LinStates& states, cudaStream_t stream) {
    if (args.role[0].Ga > 1)   // (in every role then)
        return D == 128 ? launch_all<128, true>(args, states, stream) : launch_all<64, true>(args, states, stream);
    return D == 128 ? launch_all<128, false>(args, states, stream) : launch_all<64, false>(args, states, stream);
}

}  // namespace bct
