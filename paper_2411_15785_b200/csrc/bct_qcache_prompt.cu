// Attention over the 8-bit cache on the sm_100a tensor path: bfloat16 calls with many rows to a unit (prompts).
//
// The formulas are those of bct_qcache_attend.cu; a unit's rows are its (token, head) pairs, token-major.  A CTA has 256 of
// them, two tiles of 128, and goes through the slots that they see, 128 at a time:
//     S = Q K^T  (M = 128 rows, N = 128 slots)     P = exp2(S - m), fp16, into S's place     O += P V  (N = d)
// as tcgen05.mma with fp32 accumulators in tensor memory; P is read from there.  Warps 0-3 and 4-7 form P of the two
// tiles, a row to a thread; warps 8-10 turn codes into fp16 operands (exactly), which both tiles use; warp 11 issues the
// products, so that one tile's products run while the other's P is formed.
//  - A query is fp16 after a power of two that brings its row below 2^15, which is exact (terms below 2^-39 of the row's
//    largest apart), and codes are fp16 exactly: scores are exact products with fp32 sums.
//  - The running maximum m moves only when a score passes it by 2^6: P is 2^9 p, below 2^15, and O is rarely scaled.
//  - The blocks' value scales multiply P, relative to one that follows the loudest block of a tile (vref below), so that one
//    product covers four blocks; the accumulators are in units of it.
// With few rows the slots are dealt to several CTAs, whose results qc_prompt_join_kernel joins.  The weights come from a
// second pass in the transposed form, S^T = K Q^T with the slots in the lanes: with each row's maximum and sum known, a
// thread adds up exp2(S - m) / sum over the rows, in their order, without atomics.
//
// Bound by the exponentials and what surrounds them: of 4300 clocks that a tile of 128 slots takes for 256 rows, d 128, the
// products are 2048 and forming P 2300 (its exponentials alone 2048, 16 a clock), in a chain from one to the other; a CTA's
// beginning and end are some 14000 beside them.  Measured: 2048 tokens of 2 sequences, 32 heads over 8 of 128: 119 us = 0.58
// PFLOP/s (0.35 of the measured bf16 rate), the weights 66 more; 777 tokens of 5 sequences of up to 2477, 8 heads of 64, under a
// cap 84 us, the weights 56.
//
// Every wait is bounded; a timeout ends the work and fills what the CTA writes with NaN.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <type_traits>

#include "bct_device.cuh"
#include "bct_internal.h"
#include "bct_qcache.h"
#include "bct_qcache.cuh"
#include "bct_qcache_math.cuh"
#include "bct_tc.cuh"

namespace bct {
namespace {

constexpr int kQpRows = 256;                 // rows of a CTA
constexpr int kQpSlots = 128;                // slots of a tile
constexpr int kQpThreads = 12 * 32;         // (three warps to a quarter of an SM: 168 registers, for 64 columns of S and P of 32)
constexpr int kQpMakers = 96;               // threads that turn codes into operands
constexpr int kQpHalf = 128 * 128;           // bytes of 128 rows x 64 fp16 columns
constexpr float kQpPScale = 512.f;           // 2^9
constexpr float kQpSlack = 6.f;              // m may be passed by as many powers of two

#define QP_UMMA "tcgen05.mma.cta_group::1.kind::f16 "
// D (+)= A B over four steps of 16, both K-major (32 bytes a step)
__device__ __forceinline__ void umma4_kk(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, bool accum) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q " QP_UMMA "[%0], %1, %2, %3, p;\n\t"
        "setp.eq.b32 p, 0, 0;\n\t"
        "add.s64 a, %1, 2;\n\tadd.s64 b, %2, 2;\n\t"
        "@q " QP_UMMA "[%0], a, b, %3, p;\n\t"
        "add.s64 a, %1, 4;\n\tadd.s64 b, %2, 4;\n\t"
        "@q " QP_UMMA "[%0], a, b, %3, p;\n\t"
        "add.s64 a, %1, 6;\n\tadd.s64 b, %2, 6;\n\t"
        "@q " QP_UMMA "[%0], a, b, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"((uint32_t)accum)
        : "memory");
}
// D (+)= A B over four steps with A (fp16 pairs, 8 columns a step) in tensor memory, B MN-major (16 rows of 128 bytes a step)
__device__ __forceinline__ void umma4_tm(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, bool accum) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b32 a;\n\t.reg .b64 b;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q " QP_UMMA "[%0], [%1], %2, %3, p;\n\t"
        "setp.eq.b32 p, 0, 0;\n\t"
        "add.s32 a, %1, 8;\n\tadd.s64 b, %2, 128;\n\t"
        "@q " QP_UMMA "[%0], [a], b, %3, p;\n\t"
        "add.s32 a, %1, 16;\n\tadd.s64 b, %2, 256;\n\t"
        "@q " QP_UMMA "[%0], [a], b, %3, p;\n\t"
        "add.s32 a, %1, 24;\n\tadd.s64 b, %2, 384;\n\t"
        "@q " QP_UMMA "[%0], [a], b, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"((uint32_t)accum)
        : "memory");
}
__device__ __forceinline__ void commit_warp(uint64_t* bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar))
        : "memory");
}
// fp16 x fp16 -> fp32
__host__ __device__ constexpr uint32_t idesc_f16(uint32_t M, uint32_t N, bool b_mn_major) {
    return instr_desc_mn(M, N, false, b_mn_major) & ~((7u << 7) | (7u << 10));
}
__device__ __forceinline__ void tmem_ld32_raw(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
// until loads are complete; names the destination so that no use of it moves ahead
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                   "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                   "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :
                 : "memory");
}
// The 128 columns of this thread's lane, 32 at a time: use(c, x) for c = 0..3, the next ones on their way meanwhile.  (A
// loop: with all of it unrolled, masks and caps in every copy, the kernels missed the instruction cache and took twice as
// long.)
template <typename F>
__device__ __forceinline__ void by_chunks(uint32_t taddr, F use) {
    uint32_t x[32], y[32];
    tmem_ld32_raw(taddr, x);
#pragma unroll 1
    for (int c = 0; c < 4; c += 2) {
        tmem_wait_ld(x);
        tmem_ld32_raw(taddr + 32 * c + 32, y);
        use(c, x);
        tmem_wait_ld(y);
        if (c == 0) tmem_ld32_raw(taddr + 64, x);
        use(c + 1, y);
    }
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    tmem_st16(taddr, r);
    tmem_st16(taddr + 16, r + 16);
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// tanh of 32 numbers, some of them beyond 1 (rare: out of the way, through local memory)
__device__ __noinline__ void tanh_far(float* s) {
#pragma unroll 1
    for (int j = 0; j < 32; ++j) s[j] = tanh_any(s[j]);
}
// tanh of 32 scores that have their factors
__device__ __forceinline__ void tanh32(float (&s)[32]) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 32; j += 2) top = max3(top, fabsf(s[j]), fabsf(s[j + 1]));
    if (__any_sync(0xffffffffu, top > 1.f)) {
        float far[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) far[j] = s[j];
        tanh_far(far);
#pragma unroll
        for (int j = 0; j < 32; ++j) s[j] = far[j];
    } else {
#pragma unroll
        for (int j = 0; j < 32; j += 2) tanh_near2(s[j], s[j + 1]);
    }
}

// A bounded wait of a warp: two seconds of the global timer, a thousandth of that once a wait has failed.  try_wait is given
// a suspend time: warps wait here most of the time, and every poll takes issue slots from those that work.
__device__ __noinline__ void qp_wait_slow(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
    const unsigned long long limit = *abort_flag ? 2000000ull : 2000000000ull;
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
__device__ __forceinline__ void qp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    if (!mbar_try_wait(bar, parity & 1)) qp_wait_slow(bar, parity & 1, abort_flag);
    __syncwarp();
}
// Where 16-byte chunk c (8 fp16 columns) of a row stands in an operand tile: halves of 64 columns, 128-byte swizzle.
__device__ __forceinline__ int operand_at(int row, int c) { return (c >> 3) * kQpHalf + row * 128 + (((c & 7) ^ (row & 7)) << 4); }

// THREADS threads turn a tile of codes into an fp16 operand: raw[i] are the 16-byte pieces of a thread.  Its rows are
// multiples of four apart, so that their swizzles are two, and all addresses constants away from two.
template <int D, int THREADS>
struct Codes {
    static constexpr int kPer = D / 16, kAll = 128 * kPer;              // 16-byte pieces of a slot, of the tile
    static constexpr int kRaw = (kAll + THREADS - 1) / THREADS, kStep = THREADS / kPer;
    static_assert(THREADS % kPer == 0 && kStep % 4 == 0, "a thread's rows are multiples of four apart");
    uint4 raw[kRaw];
    __device__ __forceinline__ void load(const int8_t* unit, int slot0, int end, int t) {
        const uint4* from = reinterpret_cast<const uint4*>(unit + (size_t)slot0 * D) + t;
        const int most = (end - slot0) * kPer - t;
        if ((end - slot0) >= 128) {
#pragma unroll
            for (int i = 0; i < kRaw; ++i)
                if ((i + 1) * THREADS <= kAll || i * THREADS + t < kAll) raw[i] = from[i * THREADS];
        } else {
#pragma unroll
            for (int i = 0; i < kRaw; ++i) raw[i] = i * THREADS < most ? from[i * THREADS] : make_uint4(0, 0, 0, 0);
        }
    }
    // asks for a tile that comes later to be brought into L2
    __device__ __forceinline__ static void ahead(const int8_t* unit, int slot0, int end, int t) {
        const int lines = min(128, end - slot0) * D / 128;
        for (int i = t; i < lines; i += THREADS) asm volatile("prefetch.global.L2 [%0];" ::"l"(unit + (size_t)slot0 * D + i * 128));
    }
    __device__ __forceinline__ void store(unsigned char* tile, int t) const {
        const int row = t / kPer, c = t % kPer * 2;
        // (the lanes of the second half of a row begin with the other chunk: no two lanes at the same banks)
        const bool second = (c >> 3) != 0;
        unsigned char* const to[2] = {tile + operand_at(row, c + second), tile + operand_at(row, c + !second)};
        unsigned char* const to4[2] = {tile + operand_at(row ^ 4, c + second) + (row - (row ^ 4)) * 128,
                                       tile + operand_at(row ^ 4, c + !second) + (row - (row ^ 4)) * 128};
#pragma unroll
        for (int i = 0; i < kRaw; ++i) {
            if ((i + 1) * THREADS > kAll && i * THREADS + t >= kAll) break;
            const uint32_t w[4] = {(second ? raw[i].z : raw[i].x) ^ 0x80808080u, (second ? raw[i].w : raw[i].y) ^ 0x80808080u,
                                   (second ? raw[i].x : raw[i].z) ^ 0x80808080u, (second ? raw[i].y : raw[i].w) ^ 0x80808080u};
#pragma unroll
            for (int k = 0; k < 2; ++k)
                *reinterpret_cast<uint4*>(((kStep * i) & 4 ? to4[k] : to[k]) + kStep * i * 128) =
                    make_uint4(pair_of(w[2 * k], 0x4140), pair_of(w[2 * k], 0x4342), pair_of(w[2 * k + 1], 0x4140),
                               pair_of(w[2 * k + 1], 0x4342));
        }
    }
};

// For the pass that forms the weights, of each tile of 128 rows: the queries as that operand, and a record of the rows'
// terms: {factor, factor, -log, -log} for each pair of rows (what the row's products are multiplied with; the logarithm of
// its sum of powers of two, infinity for a row that adds nothing), then how many slots each row sees.
constexpr int kQpRecord = 128 * 8 + 128 * 4;
__device__ __forceinline__ float* terms_of(const QcPrompt& pr, size_t tile, int row) {
    return reinterpret_cast<float*>(pr.records + tile * kQpRecord) + (row >> 1) * 4 + (row & 1);
}
__device__ __forceinline__ int* limits_of(const QcPrompt& pr, size_t tile) {
    return reinterpret_cast<int*>(pr.records + tile * kQpRecord + 1024);
}

// Where rows stand in q and out, `step` rows on at a time.
struct RowWalk {
    int64_t at, token_step, head_step;
    int head, G, heads_on;
    __device__ __forceinline__ RowWalk(const QcAttend& a, int b, int h, int64_t r, int step) {
        const unsigned i = (unsigned)r / (unsigned)a.G;
        const int64_t token = (int64_t)a.c.Hkv * a.G * a.c.D;
        G = a.G;
        head = (int)((unsigned)r - i * a.G);
        at = ((int64_t)b * a.T + i) * token + (int64_t)(h * a.G + head) * a.c.D;
        int tokens_on = 0;
        for (heads_on = step; heads_on >= G; heads_on -= G) ++tokens_on;   // (step is a few rows)
        head_step = tokens_on * token + (int64_t)heads_on * a.c.D;
        token_step = token - (int64_t)G * a.c.D;       // a token on, and the heads of a group back
    }
    __device__ __forceinline__ void next() {
        head += heads_on;
        at += head_step;
        if (head >= G) head -= G, at += token_step;
    }
};

template <int D>
struct QpSmem {
    static constexpr int kTile = D / 64 * kQpHalf;    // an operand tile of 128 rows
    static constexpr int q = 0;                       // two
    static constexpr int k = q + 2 * kTile;           // two stages
    static constexpr int v = k + 2 * kTile;           // two stages
    static constexpr int bars = v + 2 * kTile;
    static constexpr int total = bars + 256 + 1024;   // (1024 to align the base)
};

template <int D, bool CAP>
__global__ void __launch_bounds__(kQpThreads, 1) qc_prompt_kernel(const QcAttend a, const QcPrompt pr) {
    using L = QpSmem<D>;
    extern __shared__ unsigned char qp_smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(qp_smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::bars);
    uint64_t *k_full = bars, *k_empty = bars + 2, *v_full = bars + 4, *v_empty = bars + 6;   // [2] by stages
    uint64_t *q_full = bars + 8, *s_full = bars + 10, *p_full = bars + 12, *o_full = bars + 14;   // [2] by tiles of rows
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 16);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 17);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // (unit, rows, split): the rows that see most come first
    const unsigned units = (unsigned)(a.c.B * a.c.Hkv);
    unsigned idx = blockIdx.x;
    const unsigned split = idx % pr.splits;
    idx /= pr.splits;
    const unsigned unit = idx % units;
    const int64_t r0 = (int64_t)(pr.tiles - 1 - (int)(idx / units)) * kQpRows;
    const int b = (int)(unit / a.c.Hkv), h = (int)(unit - b * a.c.Hkv);
    pdl_wait();
    const Sees sees = sees_of(a, b);
    const int64_t valid = (int64_t)sees.n * a.G;                        // rows of valid tokens
    const int rows = (int)max((int64_t)0, min((int64_t)kQpRows, valid - r0));
    const int lim_max = rows > 0 ? sees(r0 + rows - 1) : 0, lim_min = rows > 0 ? sees(r0) : 0;
    const int all_tiles = (lim_max + kQpSlots - 1) / kQpSlots;
    const int lo = (int)((int64_t)all_tiles * split / pr.splits), hi = (int)((int64_t)all_tiles * (split + 1) / pr.splits);
    // Two tiles of rows, or, where a unit has one, its tiles of slots in turn to each of two sets of accumulators.
    const bool by_slots = pr.by_slots != 0;
    const int N = hi - lo, subs = rows > 128 ? 2 : 1;
    const int8_t* kp = a.c.codes[0] + (size_t)unit * a.c.C * D;
    const int8_t* vp = a.c.codes[1] + (size_t)unit * a.c.C * D;

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&k_full[i], kQpMakers / 32);
            mbar_init(&k_empty[i], 1);
            mbar_init(&v_full[i], kQpMakers / 32);
            mbar_init(&v_empty[i], 1);
            mbar_init(&q_full[i], 4);
            mbar_init(&s_full[i], 1);
            mbar_init(&p_full[i], 4);
            mbar_init(&o_full[i], 1);
        }
        *abort_flag = 0;
        fence_mbar_init_cluster();
    }
    if (warp == 11) tmem_alloc(tmem_slot, 512);

    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_open();
    const uint32_t tmem = *tmem_slot;

    if (warp == 11) {
        // =========================== products ===========================
        constexpr uint32_t id_s = idesc_f16(128, 128, false), id_o = idesc_f16(128, D, true);
        const DescKind dk(smem_desc(0, 16, 1024)), dmn(smem_desc(0, kQpHalf, 1024));
        const uint32_t base16 = desc_addr16(smem_u32(smem));
        auto scores = [&](int n, int g) {
            const uint32_t qa = base16 + (L::q + g * L::kTile) / 16, ka = base16 + (L::k + (n & 1) * L::kTile) / 16;
#pragma unroll
            for (int hf = 0; hf < D / 64; ++hf)
                umma4_kk(tmem + g * 128, dk.at(qa + hf * (kQpHalf / 16)), dk.at(ka + hf * (kQpHalf / 16)), id_s, hf > 0);
            commit_warp(&s_full[g]);
            if (by_slots || g == subs - 1) commit_warp(&k_empty[n & 1]);
        };
        auto outputs = [&](int n, int g, int turn) {
            const uint32_t va = base16 + (L::v + (n & 1) * L::kTile) / 16;
            qp_wait(&p_full[g], turn, abort_flag);
            tc_fence_after();
            umma4_tm(tmem + 256 + g * D, tmem + g * 128, dmn.at(va), id_o, turn > 0);
            umma4_tm(tmem + 256 + g * D, tmem + g * 128 + 32, dmn.at(va + 512), id_o, true);
            commit_warp(&o_full[g]);
            if (by_slots || g == subs - 1) commit_warp(&v_empty[n & 1]);
        };
        auto wait_k = [&](int n) {
            qp_wait(&k_full[n & 1], n >> 1, abort_flag);
            tc_fence_after();
        };
        if (by_slots) {
            for (int n = 0; n < min(N, 2); ++n) {
                qp_wait(&q_full[n], 0, abort_flag);
                wait_k(n);
                scores(n, n);
            }
            for (int n = 0; n < N; ++n) {
                qp_wait(&v_full[n & 1], n >> 1, abort_flag);
                outputs(n, n & 1, n >> 1);
                if (n + 2 < N) {
                    wait_k(n + 2);
                    scores(n + 2, n & 1);          // (after the product that reads P from its place)
                }
            }
        } else {
            if (N > 0) {
                wait_k(0);
                for (int g = 0; g < subs; ++g) {
                    qp_wait(&q_full[g], 0, abort_flag);
                    tc_fence_after();
                    scores(0, g);
                }
            }
            for (int n = 0; n < N; ++n) {
                for (int g = 0; g < subs; ++g) {
                    if (g == 0) qp_wait(&v_full[n & 1], n >> 1, abort_flag);
                    outputs(n, g, n);
                    if (n + 1 < N) {
                        if (g == 0) wait_k(n + 1);
                        scores(n + 1, g);
                    }
                }
            }
        }
    } else if (warp >= 8) {
        // =========================== codes to operands ===========================
        const int t = tid - 256;
        Codes<D, kQpMakers> k, v;
        if (N > 0) {
            k.load(kp, lo * kQpSlots, lim_max, t);
            v.load(vp, lo * kQpSlots, lim_max, t);
        }
        constexpr int kAhead = 4;      // (a tile's loads are one tile ahead, which DRAM takes longer than)
        for (int n = 1; n < min(N, kAhead); ++n) {
            k.ahead(kp, (lo + n) * kQpSlots, lim_max, t);
            v.ahead(vp, (lo + n) * kQpSlots, lim_max, t);
        }
        for (int n = 0; n < N; ++n) {
            const int st = n & 1;
            if (n + kAhead < N) {
                k.ahead(kp, (lo + n + kAhead) * kQpSlots, lim_max, t);
                v.ahead(vp, (lo + n + kAhead) * kQpSlots, lim_max, t);
            }
            if (n >= 2) qp_wait(&k_empty[st], (n >> 1) - 1, abort_flag);
            k.store(smem + L::k + st * L::kTile, t);
            if (n + 1 < N) k.load(kp, (lo + n + 1) * kQpSlots, lim_max, t);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&k_full[st]);
            if (n >= 2) qp_wait(&v_empty[st], (n >> 1) - 1, abort_flag);
            v.store(smem + L::v + st * L::kTile, t);
            if (n + 1 < N) v.load(vp, (lo + n + 1) * kQpSlots, lim_max, t);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&v_full[st]);
        }
    } else {
        // =========================== queries, softmax ===========================
        const int sub = warp >> 2;                                          // of warps 0-7: the tile of rows
        const int my_row = (warp & 3) * 32 + lane;
        const int64_t r = r0 + (by_slots ? 0 : sub * 128) + my_row;
        const size_t tile128 = ((size_t)unit * pr.tiles + (size_t)(r0 / kQpRows)) * 2 + sub;
        const bool keep_q = pr.q_tiles != nullptr && split == 0 && !(by_slots && sub == 1);            // for the pass that forms the weights
        float factor = 0.f;                                                 // what the row's products are multiplied with
        int lim = 0;
        // The warp's rows, as an operand: kLanes lanes to a row, 16 bytes each.
        constexpr int kLanes = D / 8, kEach = 32 / kLanes, kTurns = 32 / kEach;
        const int part = lane % kLanes;
        uint4 w[kTurns];
        RowWalk walk(a, b, h, r - lane + lane / kLanes, kEach);
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            w[i] = make_uint4(0, 0, 0, 0);
            if (r - lane + i * kEach + lane / kLanes < valid)
                w[i] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + walk.at + 8 * part);
            walk.next();
        }
        // (magnitudes in their order as 16-bit integers, two at a time; all rows at once, since a row's shuffles wait for one
        // another)
        uint32_t two[kTurns];
#pragma unroll
        for (int i = 0; i < kTurns; ++i)
            two[i] = __vmaxu2(__vmaxu2(w[i].x & 0x7fff7fffu, w[i].y & 0x7fff7fffu), __vmaxu2(w[i].z & 0x7fff7fffu, w[i].w & 0x7fff7fffu));
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1)
#pragma unroll
            for (int i = 0; i < kTurns; ++i) two[i] = __vmaxu2(two[i], __shfl_xor_sync(0xffffffffu, two[i], o));
        // the lane's own row
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const uint32_t t = __shfl_sync(0xffffffffu, two[i], lane % kEach * kLanes);
            if (i == lane / kEach) top = t;
        }
        float unused;
        row_scale(__uint_as_float(max(top << 16, top & 0xffff0000u)), &unused, &factor);
        factor = row_factor(a, factor);
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            float by, back, x[8];
            row_scale(__uint_as_float(max(two[i] << 16, two[i] & 0xffff0000u)), &by, &back);
            Chunk<__nv_bfloat16>::unpack(w[i], x);
            const uint4 o = make_uint4(half2_bits(x[0] * by, x[1] * by), half2_bits(x[2] * by, x[3] * by),
                                       half2_bits(x[4] * by, x[5] * by), half2_bits(x[6] * by, x[7] * by));
            const int at = operand_at((warp & 3) * 32 + i * kEach + lane / kLanes, part);
            *reinterpret_cast<uint4*>(smem + L::q + sub * L::kTile + at) = o;
            if (keep_q) *reinterpret_cast<uint4*>(pr.q_tiles + tile128 * L::kTile + at) = o;
        }
        const bool real = r < valid;
        lim = real ? sees(r) : 0;
        if (keep_q) {
            float* terms = terms_of(pr, tile128, my_row);
            terms[0] = real ? factor : 0.f;
            terms[2] = -INFINITY;
            limits_of(pr, tile128)[my_row] = lim;
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&q_full[sub]);

        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);      // (32 lanes further in bits 16 and up)
        const uint32_t s_col = lanes + sub * 128, o_col = lanes + 256 + sub * D;
        const float* ksp = a.c.scale[0] + (size_t)unit * a.c.NB;
        const float* vsp = a.c.scale[1] + (size_t)unit * a.c.NB;
        const int blocks = (lim_max + kQcBlock - 1) / kQcBlock;
        const bool idle = (warp & 3) * 32 + (by_slots ? 0 : sub * 128) >= rows;   // none of the warp's rows is a valid token's
        float m = -INFINITY, vref = 0.f, vmost = 0.f;
        const float cap = a.cap * kLog2e;
        float l = 0.f;
        bool spoilt = false;
        // lane c (of four) has the scales of a tile's block c, a tile ahead
        float ks_next = 0.f, vs_next = 0.f;
        auto load_scales = [&](int n) {
            const int blk = (lo + n) * (kQpSlots / kQcBlock) + (lane & 3);
            ks_next = vs_next = 0.f;
            if (n < N && blk < blocks) ks_next = ksp[blk], vs_next = vsp[blk];
        };
        // the tiles of slots of this warp's accumulators: from n0 on, n_step apart
        const int n0 = by_slots ? sub : 0, n_step = by_slots ? 2 : 1, turns = by_slots ? (N + 1 - sub) / 2 : sub < subs ? N : 0;
        load_scales(n0);
        if (turns > 0) {
            auto tile = [&](int turn, auto hide) {               // hide: some row does not see all of it
                constexpr bool kHide = decltype(hide)::value;
                const int n = n0 + turn * n_step, slot0 = (lo + n) * kQpSlots;
                const float ks = ks_next, vs = vs_next;
                load_scales(n + n_step);
                float vt = fmaxf(vs, __shfl_xor_sync(0xffffffffu, vs, 1));
                vt = fmaxf(0.f, fmaxf(vt, __shfl_xor_sync(0xffffffffu, vt, 2)));
                // the scale that the values are relative to follows the loudest block of the tile: above it, so that it moves rarely,
                // by 8 at most, so that P's last place, 2^-25 of 2^9, is 2^-31 of the tile's largest value; but not below 2^-60 of
                // the loudest so far
                float by_v = 1.f;
                vmost = fmaxf(vmost, vt);
                if (vt > vref || vt < vref * 0.125f) {
                    const float to = 4.f * fmaxf(vt, vmost * 8.67361738e-19f);
                    if (vref > 0.f && to > 0.f) by_v = vref / to;
                    if (to > 0.f) vref = to;
                }
                // P's factor of the lane's block, as a power of two and inverted; a block of zeros has any, and one of spoilt values,
                // which the rows that see it are given at the end
                const float v_rel = vs > 0.f ? fmaxf(__fdividef(vs, vref > 0.f ? vref : 1.f), 8.67361738e-19f) * kQpPScale : kQpPScale;
                if (const unsigned bad = __ballot_sync(0xffffffffu, vs != vs) & 15u) spoilt |= lim > slot0 + 32 * (__ffs(bad) - 1);
                const float v_log = __log2f(v_rel), v_inv = __fdividef(1.f, v_rel);
                qp_wait(&s_full[sub], turn, abort_flag);
                tc_fence_after();
                if (idle) {
                    if (lane == 0) mbar_arrive(&p_full[sub]);
                    return;
                }

                float top = -INFINITY;
                by_chunks(s_col, [&](int c, const uint32_t (&x)[32]) {
                    const float k = __shfl_sync(0xffffffffu, ks, c) * factor;
                    const int see = lim - (slot0 + 32 * c);   // slots of this block that the row sees
                    float part[2] = {-INFINITY, -INFINITY};
                    if constexpr (kHide) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) part[j & 1] = fmaxf(part[j & 1], j < see ? __uint_as_float(x[j]) : -INFINITY);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            part[0] = max3(part[0], __uint_as_float(x[j]), __uint_as_float(x[j + 1]));
                            part[1] = max3(part[1], __uint_as_float(x[j + 2]), __uint_as_float(x[j + 3]));
                        }
                    }
                    if (!kHide || see > 0) top = fmaxf(top, fmaxf(part[0], part[1]) * k);
                });
                if constexpr (CAP) top = top == -INFINITY ? top : cap * tanh_any(top);
                float by = by_v;
                if (top > m + kQpSlack || (m == -INFINITY && top > m)) {
                    const float keep = ex2(m - top);           // (0 the first time)
                    by *= keep;
                    l *= keep;
                    m = top;
                }
                if (turn > 0 && __any_sync(0xffffffffu, by != 1.f)) {
                    qp_wait(&o_full[sub], turn - 1, abort_flag);
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        uint32_t x[32];
                        tmem_ld32_raw(o_col + c, x);
                        tmem_wait_ld(x);
#pragma unroll
                        for (int j = 0; j < 32; ++j) x[j] = __float_as_uint(__uint_as_float(x[j]) * by);
                        tmem_st32(o_col + c, x);
                    }
                }
                const float m0 = m == -INFINITY ? 0.f : m;
                // (P of 32 slots goes into 16 columns of what has been read: by_chunks is 32 ahead at most)
                by_chunks(s_col, [&](int c, const uint32_t (&x)[32]) {
                    const float k = __shfl_sync(0xffffffffu, ks, c) * factor;
                    const float bias = __shfl_sync(0xffffffffu, v_log, c) - m0, v_back = __shfl_sync(0xffffffffu, v_inv, c);
                    const int see = lim - (slot0 + 32 * c);
                    float e[32], sum[4] = {0.f, 0.f, 0.f, 0.f};
                    uint32_t p[16];
#pragma unroll
                    for (int j = 0; j < 32; ++j) e[j] = CAP ? __uint_as_float(x[j]) * k : fmaf(__uint_as_float(x[j]), k, bias);
                    if constexpr (CAP) {
                        tanh32(e);
#pragma unroll
                        for (int j = 0; j < 32; ++j) e[j] = fmaf(e[j], cap, bias);
                    }
#pragma unroll
                    for (int j = 0; j < 32; ++j) e[j] = ex2(e[j]);
                    if constexpr (kHide) {                    // hidden slots give nothing, whatever their scales
#pragma unroll
                        for (int j = 0; j < 32; ++j) e[j] = j < see ? e[j] : 0.f;
                    }
#pragma unroll
                    for (int j = 0; j < 32; ++j) sum[j & 3] += e[j];
                    if (!kHide || see > 0) l = fmaf((sum[0] + sum[1]) + (sum[2] + sum[3]), v_back, l);
#pragma unroll
                    for (int j = 0; j < 16; ++j) p[j] = half2_bits(e[2 * j], e[2 * j + 1]);
                    tmem_st16(s_col + 16 * c, p);
                });
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[sub]);
            };
            const int seen = min(max(lim_min / kQpSlots - lo, 0), N);   // tiles that every row sees
            const int seen_turns = by_slots ? (seen + 1 - sub) / 2 : seen;
#pragma unroll 1
            for (int t = 0; t < seen_turns; ++t) tile(t, std::false_type());
#pragma unroll 1
            for (int t = seen_turns; t < turns; ++t) tile(t, std::true_type());
        }
        // results: the accumulators are in units of vref / 2^9
        const bool mine = turns > 0;
        if (mine) {
            qp_wait(&o_full[sub], turns - 1, abort_flag);
            tc_fence_after();
        }
        if (lim == 0) l = 0.f;                                // (a padding row in a tile that others see through)
        if (*abort_flag) l = __uint_as_float(0x7fffffffu);
        float mul = vref * (1.f / kQpPScale);
        const bool there = r < a.R;
        const float inv = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
        if (pr.parts == 1) mul = l == l ? mul * inv : l;
        if (spoilt) mul = __uint_as_float(0x7fffffffu);
        const int64_t at = ((int64_t)unit * a.R + r) * pr.parts + (by_slots ? 2 * split + sub : split);
        // (through the warp's part of the queries' tile, which is free by now, so that rows are written in one piece)
        unsigned char* stage = smem + L::q + sub * L::kTile + (warp & 3) * (32 * D * 2);
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
            uint32_t x[32];
            if (mine) {                                       // (the whole warp)
                tmem_ld32_raw(o_col + c, x);
                tmem_wait_ld(x);
            }
            float y[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) y[j] = mine && (l != 0.f) ? __uint_as_float(x[j]) * mul : 0.f;
            if (pr.parts == 1) {
#pragma unroll
                for (int j = 0; j < 32; j += 8)
                    *reinterpret_cast<uint4*>(stage + lane * (D * 2) + ((((c + j) >> 3) ^ (lane & 7)) << 4)) = Chunk<__nv_bfloat16>::pack(y + j);
            } else if (there) {
#pragma unroll
                for (int j = 0; j < 32; j += 4)
                    *reinterpret_cast<float4*>(a.part_o + at * D + c + j) = make_float4(y[j], y[j + 1], y[j + 2], y[j + 3]);
            }
            __syncwarp();
        }
        if (pr.parts == 1) {
            constexpr int kLanes = D / 8, kEach = 32 / kLanes;
            RowWalk walk(a, b, h, r - lane + lane / kLanes, kEach);
#pragma unroll 4
            for (int i = 0; i < 32; i += kEach) {
                const int row = i + lane / kLanes, part = lane % kLanes;
                const uint4 v = *reinterpret_cast<const uint4*>(stage + row * (D * 2) + ((part ^ (row & 7)) << 4));
                if (r - lane + row < a.R) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + walk.at + 8 * part) = v;
                walk.next();
            }
        }
        if (there) {
            if (pr.parts > 1) a.part_ml[at] = make_float2(m, l);
            else if (keep_q && inv != 0.f) terms_of(pr, tile128, my_row)[2] = log2f(inv) - m;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 11) tmem_dealloc(tmem, 512);
}

// Joins the splits of a row: a warp to a row.
template <int D>
__global__ void __launch_bounds__(256) qc_prompt_join_kernel(const QcAttend a, const QcPrompt pr) {
    const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), rows = (int64_t)a.c.B * a.c.Hkv * a.R;
    const int lane = threadIdx.x & 31;
    pdl_wait();
    pdl_open();
    if (row >= rows) return;
    const int64_t unit = row / a.R, r = row - unit * a.R;
    const float2* ml = a.part_ml + row * pr.parts;
    float m = -INFINITY, l = 0.f;
    for (int i = 0; i < pr.parts; ++i) m = fmaxf(m, ml[i].x);
    for (int i = 0; i < pr.parts; ++i) l += m == -INFINITY ? ml[i].y : ml[i].y * ex2(ml[i].x - m);
    const float inv = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
    constexpr int kN = D / 32;
    float y[kN] = {};
    for (int i = 0; i < pr.parts; ++i) {
        const float by = ml[i].x == -INFINITY ? 0.f : ex2(ml[i].x - m) * inv;
#pragma unroll
        for (int j = 0; j < kN; ++j) y[j] = fmaf(a.part_o[(row * pr.parts + i) * D + lane * kN + j], by, y[j]);
    }
    const int b = (int)(unit / a.c.Hkv), h = (int)(unit - (int64_t)b * a.c.Hkv);
    __nv_bfloat16* to = const_cast<__nv_bfloat16*>(row_of<__nv_bfloat16>(a, a.out, b, h, r)) + lane * kN;
#pragma unroll
    for (int j = 0; j < kN; j += 2)
        *reinterpret_cast<uint32_t*>(to + j) = l == l ? Chunk<__nv_bfloat16>::pack2(y[j], y[j + 1]) : 0x7fff7fffu;
    if (lane == 0 && pr.q_tiles != nullptr && inv != 0.f)
        terms_of(pr, ((size_t)unit * pr.tiles + (size_t)(r / kQpRows)) * 2 + (size_t)(r % kQpRows) / 128, (int)(r % 128))[2] = log2f(inv) - m;
}

// ---- the weights ------------------------------------------------------------------------------------------------
constexpr int kQwtStages = 4;                          // of query tiles, and of products in tensor memory
constexpr int kQwtThreads = 10 * 32;                   // eight warps that add up, one that loads, one for the products
template <int D>
struct QwtSmem {
    static constexpr int kTile = D / 64 * kQpHalf;
    static constexpr int k = 0;
    static constexpr int q = k + kTile;
    static constexpr int rows = q + kQwtStages * kTile;   // the rows' records
    static constexpr int bars = rows + kQwtStages * kQpRecord;
    static constexpr int total = bars + 256 + 1024;
};

// What 32 rows give a thread's slot, from their products with its key.
template <bool CAP>
__device__ __forceinline__ void add_weights(const uint32_t (&x)[32], const float* row, const int* lims, float ks, float cap, int slot,
                                            bool masked, float (&acc)[4]) {
    float e[32];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const float4 t = *reinterpret_cast<const float4*>(row + 4 * j);
        const float u = __uint_as_float(x[2 * j]) * ks, v = __uint_as_float(x[2 * j + 1]) * ks;
        e[2 * j] = CAP ? u * t.x : fmaf(u, t.x, t.z);
        e[2 * j + 1] = CAP ? v * t.y : fmaf(v, t.y, t.w);
    }
    if constexpr (CAP) {
        tanh32(e);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float2 t = *reinterpret_cast<const float2*>(row + 4 * j + 2);
            e[2 * j] = fmaf(e[2 * j], cap, t.x);
            e[2 * j + 1] = fmaf(e[2 * j + 1], cap, t.y);
        }
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) e[j] = ex2(e[j]);
    if (masked) {
#pragma unroll
        for (int j = 0; j < 32; ++j) e[j] = slot < lims[j] ? e[j] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) acc[j & 3] += e[j];
}

template <int D, bool CAP>
__global__ void __launch_bounds__(kQwtThreads, 1) qc_prompt_weights_kernel(const QcAttend a, const QcPrompt pr) {
    using L = QwtSmem<D>;
    constexpr int kSt = kQwtStages;
    extern __shared__ unsigned char qp_smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(qp_smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::bars);
    uint64_t *q_full = bars, *q_empty = bars + kSt, *s_full = bars + 2 * kSt, *s_empty = bars + 3 * kSt;   // [kSt]
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 4 * kSt);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 4 * kSt + 1);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned units = (unsigned)(a.c.B * a.c.Hkv);
    const unsigned unit = blockIdx.x % units;
    const int slot0 = (int)(blockIdx.x / units) * kQpSlots;             // the slots that most rows see come first
    const int b = (int)(unit / a.c.Hkv), h = (int)(unit - b * a.c.Hkv);
    pdl_wait();
    const Sees sees = sees_of(a, b);
    if (slot0 >= sees.held || sees.n == 0) return;
    const int64_t valid = (int64_t)sees.n * a.G;
    const int i0 = max(0, slot0 - (sees.held - sees.n));                // the first token that sees the first slot
    const int64_t first = (int64_t)i0 * a.G / 128 * 128;
    const int N = (int)((valid - first + 127) / 128);

    if (tid == 0) {
        for (int i = 0; i < kSt; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 5);                                  // the products and the four warps that read the rows' terms
            mbar_init(&s_full[i], 1);
            mbar_init(&s_empty[i], 4);
        }
        *abort_flag = 0;
        fence_mbar_init_cluster();
    }
    if (warp == 9) tmem_alloc(tmem_slot, 512);
    if (warp < 8) {
        Codes<D, 256> k;
        k.load(a.c.codes[0] + (size_t)unit * a.c.C * D, slot0, sees.held, tid);
        k.store(smem + L::k, tid);
    }
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    float sum = 0.f;

    if (warp == 9) {
        constexpr uint32_t id_s = idesc_f16(128, 128, false);
        const DescKind dk(smem_desc(0, 16, 1024));
        const uint32_t base16 = desc_addr16(smem_u32(smem));
        for (int n = 0; n < N; ++n) {
            const int st = n % kSt;
            qp_wait(&q_full[st], n / kSt, abort_flag);
            if (n >= kSt) qp_wait(&s_empty[st], n / kSt - 1, abort_flag);
            tc_fence_after();
            const uint32_t ka = base16 + L::k / 16, qa = base16 + (L::q + st * L::kTile) / 16;
#pragma unroll
            for (int hf = 0; hf < D / 64; ++hf)
                umma4_kk(tmem + st * 128, dk.at(ka + hf * (kQpHalf / 16)), dk.at(qa + hf * (kQpHalf / 16)), id_s, hf > 0);
            commit_warp(&s_full[st]);
            commit_warp(&q_empty[st]);
        }
    } else if (warp == 8) {
        // =========================== queries and their rows' terms ===========================
        const size_t tile0 = (size_t)unit * pr.tiles * 2 + (size_t)(first / 128);
        for (int n = 0; n < N; ++n) {
            const int st = n % kSt;
            if (n >= kSt) qp_wait(&q_empty[st], n / kSt - 1, abort_flag);
            if (lane == 0) {
                mbar_arrive_expect_tx(&q_full[st], L::kTile + kQpRecord);
                bulk_load(smem + L::q + st * L::kTile, pr.q_tiles + (tile0 + n) * L::kTile, L::kTile, &q_full[st]);
                bulk_load(smem + L::rows + st * kQpRecord, pr.records + (tile0 + n) * kQpRecord, kQpRecord, &q_full[st]);
            }
            __syncwarp();
        }
        // (the copies end before the CTA does: the products of the last tile wait for them)
    } else {
        // =========================== a slot to a thread; warps 0-3 and 4-7 take the row tiles in turn ===========================
        const int g = warp >> 2, my = (warp & 3) * 32 + lane, slot = slot0 + my;
        const int blk = slot / kQcBlock;
        const float ks = slot < sees.held ? a.c.scale[0][(size_t)unit * a.c.NB + blk] : 0.f;
        const float cap = a.cap * kLog2e;
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        for (int n = g; n < N; n += 2) {
            const int st = n % kSt;
            const float* rows = reinterpret_cast<const float*>(smem + L::rows + st * kQpRecord);
            const int* lims = reinterpret_cast<const int*>(rows + 256);
            qp_wait(&q_full[st], n / kSt, abort_flag);                  // (the rows' terms)
            qp_wait(&s_full[st], n / kSt, abort_flag);
            tc_fence_after();
            const bool masked = slot0 + kQpSlots > lims[0];             // (a tile's first row sees least of its valid ones)
            by_chunks(tmem + ((uint32_t)(warp & 3) << 21) + st * 128, [&](int c, const uint32_t (&x)[32]) {
                add_weights<CAP>(x, rows + 64 * c, lims + 32 * c, ks, cap, slot, masked, acc);
            });
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s_empty[st]);
            __syncwarp();
            if (lane == 0) mbar_arrive(&q_empty[st]);
        }
        sum = (acc[0] + acc[1]) + (acc[2] + acc[3]);
    }
    tc_fence_before();
    __syncthreads();
    float* share = reinterpret_cast<float*>(smem + L::rows);
    if (warp >= 4 && warp < 8) share[tid - 128] = sum;
    __syncthreads();
    if (warp < 4 && slot0 + tid < sees.held) {
        sum += share[tid];
        if (*abort_flag) sum = __uint_as_float(0x7fffffffu);
        a.c.weight[(size_t)unit * a.c.C + slot0 + tid] += sum;
    }
    if (warp == 9) tmem_dealloc(tmem, 512);
}

// The same for few rows, where a tile of slots is little work: CTAs go through runs of 256-slot pieces that are of equal work,
// whatever the sequences' lengths, with the queries in place until the unit changes (R <= 256, two tiles at most) or, STREAM,
// through two places in turn.  Warps 0-3 have a
// piece's first 128 slots, 4-7 its others; warps 8-9 turn codes into operands, a piece ahead; warp 10 loads queries, warp 11
// issues the products.
constexpr int kQwfMakers = 64;
template <int D>
struct QwfSmem {
    static constexpr int kTile = D / 64 * kQpHalf;
    static constexpr int k = 0;                        // [2 stages][2 halves of a piece]
    static constexpr int q = k + 4 * kTile;            // two
    static constexpr int rows = q + 2 * kTile;         // their records
    static constexpr int bars = rows + 2 * kQpRecord;
    static constexpr int total = bars + 256 + 1024;
};

template <int D, bool CAP, bool STREAM>
__global__ void __launch_bounds__(kQpThreads, 1) qc_prompt_few_weights_kernel(const QcAttend a, const QcPrompt pr) {
    using L = QwfSmem<D>;
    extern __shared__ unsigned char qp_smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(qp_smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::bars);
    uint64_t *k_full = bars, *k_empty = bars + 4;      // [stage][half]
    uint64_t *s_full = bars + 8, *s_empty = bars + 12; // [half][turn]
    uint64_t *q_full = bars + 16, *q_empty = bars + 18;   // the units' queries, by turns; STREAM: [place]
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 20);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 21);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_wait();

    if (tid == 0) {
        for (int i = 0; i < 4; ++i) {
            mbar_init(&k_full[i], kQwfMakers / 32);
            mbar_init(&k_empty[i], 1);
            mbar_init(&s_full[i], 1);
            mbar_init(&s_empty[i], 4);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 9);                 // the products and the eight warps that read the rows' terms
        }
        *abort_flag = 0;
        fence_mbar_init_cluster();
    }
    if (warp == 11) tmem_alloc(tmem_slot, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    // A piece's work is the tiles of rows that see its first slot (STREAM; all tiles otherwise), and one more for its slots.
    auto tiles_of = [&](const Sees& sees) { return (int)(((int64_t)sees.n * a.G + 127) / 128); };
    auto first_tile = [&](const Sees& sees, int slot0) {
        return STREAM ? (int)((int64_t)max(0, slot0 - (sees.held - sees.n)) * a.G / 128) : 0;
    };
    auto pieces_of = [&](const Sees& sees) { return sees.n > 0 ? (sees.held + 255) / 256 : 0; };
    // pieces that all the tiles see: the first ones
    auto full_of = [&](const Sees& sees) {
        return !STREAM ? pieces_of(sees) : sees.held < sees.n ? 0 : min(pieces_of(sees), (sees.held - sees.n) / 256 + 1);
    };
    auto work_of = [&](int b) {
        const Sees sees = sees_of(a, b);
        const int N = tiles_of(sees), P = pieces_of(sees), full = full_of(sees);
        int64_t work = (int64_t)full * (N + 1);
        for (int p = full; p < P; ++p) work += N + 1 - first_tile(sees, p * 256);
        return work;
    };
    // The run: from the first piece whose work starts at x0 or behind it, as work is counted through all units, to x1.
    int64_t x0 = 0, x1 = 0, before = 0;
    int seq = a.c.B;
    find_share(a.c.B, work_of, a.c.Hkv, reinterpret_cast<int64_t*>(smem),
               [&](int64_t all) {
                   x1 = all * (blockIdx.x + 1) / gridDim.x;
                   return all * blockIdx.x / gridDim.x;
               },
               &x0, &seq, &before);
    __syncthreads();                                                    // (the words are the operands' place)
    // Every role walks through the run alike: walk(visit) for each piece, `fresh` where it is the run's first of a unit.
    auto walk = [&](auto&& visit) {
        if (x0 >= x1) return 0;
        int done = 0, units = 0, b = seq;
        int64_t at = before;
        for (;; ++b) {
            if (b >= a.c.B) return units;
            const Sees sees = sees_of(a, b);
            const int N = tiles_of(sees), P = pieces_of(sees), full = full_of(sees);
            if (P == 0) continue;
            int h = 0, p = 0;
            if (at < x0) {                                              // the run's first sequence
                const int64_t work = work_of(b);
                h = (int)((x0 - at) / work);
                at += h * work;
                p = (int)min((int64_t)full, (x0 - at + N) / (N + 1));
                at += (int64_t)p * (N + 1);
                for (; p < P && at < x0; ++p) at += N + 1 - first_tile(sees, p * 256);
            }
            for (; h < a.c.Hkv; ++h, p = 0) {
                bool fresh = true;
                for (; p < P; ++p) {
                    if (at >= x1) return units;
                    if (fresh) ++units;
                    visit(b * a.c.Hkv + h, p * 256, sees, done++, units - 1, fresh);
                    fresh = false;
                    at += N + 1 - first_tile(sees, p * 256);
                }
            }
        }
    };

    if (warp == 11) {
        // =========================== products ===========================
        constexpr uint32_t id_s = idesc_f16(128, 128, false);
        const DescKind dk(smem_desc(0, 16, 1024));
        const uint32_t base16 = desc_addr16(smem_u32(smem));
        int turns = 0;                                                  // products of a half so far
        auto product = [&](int st, int h, int place, int turn) {
            if (turn >= 2) qp_wait(&s_empty[2 * h + (turn & 1)], (turn >> 1) - 1, abort_flag);
            tc_fence_after();
            const uint32_t ka = base16 + (L::k + (2 * st + h) * L::kTile) / 16, qa = base16 + (L::q + place * L::kTile) / 16;
#pragma unroll
            for (int hf = 0; hf < D / 64; ++hf)
                umma4_kk(tmem + (2 * h + (turn & 1)) * 128, dk.at(ka + hf * (kQpHalf / 16)), dk.at(qa + hf * (kQpHalf / 16)), id_s, hf > 0);
            commit_warp(&s_full[2 * h + (turn & 1)]);
        };
        walk([&](int, int slot0, const Sees& sees, int no, int unit_no, bool fresh) {
            const int N = tiles_of(sees), st = no & 1;
            if constexpr (STREAM) {
                for (int h = 0; h < 2; ++h) qp_wait(&k_full[2 * st + h], no >> 1, abort_flag);
                for (int n = first_tile(sees, slot0); n < N; ++n, ++turns) {
                    qp_wait(&q_full[turns & 1], turns >> 1, abort_flag);
                    for (int h = 0; h < 2; ++h) product(st, h, turns & 1, turns);
                    commit_warp(&q_empty[turns & 1]);
                }
                for (int h = 0; h < 2; ++h) commit_warp(&k_empty[2 * st + h]);
            } else {
                if (fresh) {
                    if (unit_no > 0) commit_warp(q_empty);
                    qp_wait(q_full, unit_no, abort_flag);
                }
                for (int h = 0; h < 2; ++h) {
                    qp_wait(&k_full[2 * st + h], no >> 1, abort_flag);
                    for (int n = 0; n < N; ++n) product(st, h, n, turns + n);
                    commit_warp(&k_empty[2 * st + h]);
                }
                turns += N;
            }
        });
    } else if (warp == 10) {
        // =========================== queries and their rows' terms ===========================
        int turns = 0;
        auto load = [&](int unit, int n, int place, uint64_t* bar) {
            const size_t tile = (size_t)unit * pr.tiles * 2 + n;
            bulk_load(smem + L::q + place * L::kTile, pr.q_tiles + tile * L::kTile, L::kTile, bar);
            bulk_load(smem + L::rows + place * kQpRecord, pr.records + tile * kQpRecord, kQpRecord, bar);
        };
        walk([&](int unit, int slot0, const Sees& sees, int, int unit_no, bool fresh) {
            const int N = tiles_of(sees);
            if constexpr (STREAM) {
                for (int n = first_tile(sees, slot0); n < N; ++n, ++turns) {
                    if (turns >= 2) qp_wait(&q_empty[turns & 1], (turns >> 1) - 1, abort_flag);
                    if (lane == 0) {
                        mbar_arrive_expect_tx(&q_full[turns & 1], L::kTile + kQpRecord);
                        load(unit, n, turns & 1, &q_full[turns & 1]);
                    }
                    __syncwarp();
                }
            } else if (fresh) {
                if (unit_no > 0) qp_wait(q_empty, unit_no - 1, abort_flag);
                if (lane == 0) {
                    mbar_arrive_expect_tx(q_full, N * (L::kTile + kQpRecord));
                    for (int n = 0; n < N; ++n) load(unit, n, n, q_full);
                }
                __syncwarp();
            }
        });
    } else if (warp >= 8) {
        // =========================== codes to operands ===========================
        const int t = tid - 256;
        Codes<D, kQwfMakers> raw;
        int ready_unit = -1, ready_slot = -1;                           // what `raw` has: a half that was asked for ahead
        walk([&](int unit, int slot0, const Sees& sees, int no, int, bool) {
            const int8_t* kp = a.c.codes[0] + (size_t)unit * a.c.C * D;
            const int st = no & 1;
            for (int h = 0; h < 2; ++h) {
                const int at = slot0 + 128 * h;
                if (ready_unit != unit || ready_slot != at) raw.load(kp, at, max(sees.held, at), t);
                if (no >= 2) qp_wait(&k_empty[2 * st + h], (no >> 1) - 1, abort_flag);
                raw.store(smem + L::k + (2 * st + h) * L::kTile, t);
                ready_unit = unit, ready_slot = at + 128;
                if (at + 6 * 128 < sees.held) raw.ahead(kp, at + 6 * 128, sees.held, t);
                if (at + 128 < sees.held) raw.load(kp, at + 128, sees.held, t);
                else ready_unit = -1;
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&k_full[2 * st + h]);
            }
        });
    } else {
        // =========================== a slot to a thread ===========================
        const int h = warp >> 2, my = h * 128 + (warp & 3) * 32 + lane;
        const float cap = a.cap * kLog2e;
        int turns = 0;
        walk([&](int unit, int slot0, const Sees& sees, int, int unit_no, bool fresh) {
            const int slot = slot0 + my;
            const bool there = slot < sees.held;
            const int64_t valid = (int64_t)sees.n * a.G;
            const int N = tiles_of(sees);
            const float ks = there ? a.c.scale[0][(size_t)unit * a.c.NB + slot / kQcBlock] : 0.f;
            float* weight = a.c.weight + (size_t)unit * a.c.C + slot;
            const float before = there ? *weight : 0.f;
            if (!STREAM && fresh) {
                if (unit_no > 0) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(q_empty);
                }
                qp_wait(q_full, unit_no, abort_flag);
            }
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
            for (int n = first_tile(sees, slot0); n < N; ++n) {
                const int turn = turns++;
                const float* rows = reinterpret_cast<const float*>(smem + L::rows + (STREAM ? turn & 1 : n) * kQpRecord);
                if constexpr (STREAM) qp_wait(&q_full[turn & 1], turn >> 1, abort_flag);
                const int* lims = reinterpret_cast<const int*>(rows + 256);
                qp_wait(&s_full[2 * h + (turn & 1)], turn >> 1, abort_flag);
                tc_fence_after();
                const bool masked = slot0 + 256 > lims[0];
                const int chunks = (int)min((int64_t)4, (valid - (int64_t)n * 128 + 31) / 32);   // rows by 32
                const uint32_t col = tmem + ((uint32_t)(warp & 3) << 21) + (2 * h + (turn & 1)) * 128;
#pragma unroll 1
                for (int c = 0; c < chunks; ++c) {
                    uint32_t x[32];
                    tmem_ld32_raw(col + 32 * c, x);
                    tmem_wait_ld(x);
                    add_weights<CAP>(x, rows + 64 * c, lims + 32 * c, ks, cap, slot, masked, acc);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&s_empty[2 * h + (turn & 1)]);
                    if constexpr (STREAM) mbar_arrive(&q_empty[turn & 1]);
                }
            }
            float sum = (acc[0] + acc[1]) + (acc[2] + acc[3]);
            if (*abort_flag) sum = __uint_as_float(0x7fffffffu);
            if (there) *weight = before + sum;
        });
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 11) tmem_dealloc(tmem, 512);
}

template <int D, bool CAP>
cudaError_t prompt_with(const QcAttend& a, const QcPrompt& pr, cudaStream_t s) {
    static std::atomic<uint64_t> done[4];
    const int64_t units = (int64_t)a.c.B * a.c.Hkv;
    cudaError_t e = allow_smem(qc_prompt_kernel<D, CAP>, QpSmem<D>::total, &done[0]);
    if (e != cudaSuccess) return e;
    e = pdl_launch(qc_prompt_kernel<D, CAP>, (unsigned)(units * pr.tiles * pr.splits), kQpThreads, QpSmem<D>::total, s, a, pr);
    if (e != cudaSuccess) return e;
    if (pr.parts > 1 && (e = pdl_launch(qc_prompt_join_kernel<D>, (unsigned)((units * a.R + 7) / 8), 256, 0, s, a, pr)) != cudaSuccess)
        return e;
    if (!a.accumulate) return cudaSuccess;
    // Runs of slots even out when there are many pieces, each of little work; otherwise a tile of slots gets a CTA of its own.
    // The whole call by runs / by tiles, 8 heads of 4 queries to a sequence: 4 x 8192, 512 rows 182 / 220 us; 16 x 4096, 4096
    // rows 2030 / 2096; 4 x 2048, 2048 rows 178 / 177; 5 ragged sequences of up to 2500, 777 rows of 8 heads 147 / 140.
    const int64_t pieces = units * ((a.c.C + 255) / 256);
    if (a.R <= 256 || (pieces >= 4 * 148 && a.R <= 4 * pieces)) {
        const bool stream = a.R > 256;
        const auto kernel = stream ? qc_prompt_few_weights_kernel<D, CAP, true> : qc_prompt_few_weights_kernel<D, CAP, false>;
        if ((e = allow_smem(kernel, QwfSmem<D>::total, &done[2 + stream])) != cudaSuccess) return e;
        return pdl_launch(kernel, (unsigned)std::min<int64_t>(148, pieces), kQpThreads, QwfSmem<D>::total, s, a, pr);
    }
    if ((e = allow_smem(qc_prompt_weights_kernel<D, CAP>, QwtSmem<D>::total, &done[1])) != cudaSuccess) return e;
    return pdl_launch(qc_prompt_weights_kernel<D, CAP>, (unsigned)(units * ((a.c.C + kQpSlots - 1) / kQpSlots)), kQwtThreads,
                      QwtSmem<D>::total, s, a, pr);
}

}  // namespace

cudaError_t qc_prompt(const QcAttend& a, const QcPrompt& pr, cudaStream_t s) {
    if (a.c.D == 128) return a.cap > 0.f ? prompt_with<128, true>(a, pr, s) : prompt_with<128, false>(a, pr, s);
    return a.cap > 0.f ? prompt_with<64, true>(a, pr, s) : prompt_with<64, false>(a, pr, s);
}

}  // namespace bct
