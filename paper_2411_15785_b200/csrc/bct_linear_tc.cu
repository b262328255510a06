// Linear attention with a decay for each head on the sm_100a tensor path: the chunked scan for bfloat16 and
// head_dim 128 (the forward, and the three scans of the backward; bct_linear.h names the roles a, b, c).
//
// Per (sequence, kv-head) unit and chunk of 128 tokens, X being the state outside the chunk:
//     W     = A B^T                                 products of all pairs   [i][j]
//     P_ij  = W_ij lambda^|i-j| / f_i               j <= i (j >= i in reverse), bfloat16
//     O     = A X + P C                             [i][feature of c]
//     out_i = scale f_i O_i                         f_i = lambda^(distance of i to X's token)
//     X    <- lambda^n X + (w o B)^T C              w_j = lambda^(distance of j to the new X's token)
// all as tcgen05.mma with M = N = 128 and fp32 accumulators in tensor memory:
//  - W's columns are reused for P (a tensor-memory operand) once its rows have been read.
//  - The state is kept in fp32 in tensor memory, transposed (c's features in the lanes); what a chunk adds is formed
//    beside it and added in registers, rounded to nearest.  Once per chunk it goes to shared memory in bfloat16, as an
//    operand.
//  - f_i multiplies the whole row at the end instead of A's row, so A goes into both products as it is.  It is
//    floored at 2^-40, which keeps P_ij in range: below that the state's share, as it is and as it is then taken,
//    is under the rounding of what the row's own token adds.
//  - w o B is split into two bfloat16 terms, 16 bits, as this library keeps the bounded cache's MV: what a token adds
//    to the state is off by at most 2^-16 of it.  A third term made it exact to fp32 and cost 8 more products and half
//    as much splitting again.
//  - P and the state are each rounded to bfloat16 once where they enter a product with bfloat16 results.
// Roles (27 warps): warps 0-7 turn W into P, warps 8-15 split w o B into a ring of 16-row steps, warps 16-23 keep the
// state and write the outputs, over the A tile that has been read; warp 24 loads (TMA), warp 25 issues the products,
// warp 26 stores (TMA).  The products of a chunk go out as W, A X, w o B C, P C: each waits for something that was
// started at least one product earlier.  There is room for one tile of B and of C; their next tiles are brought into L2
// two chunks ahead, so that the reload is short.  With more than one segment, the same kernel without A, W and P
// forms what every segment adds.  Every wait is bounded; a timeout ends the work and fills the block's outputs with NaN.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "bct_internal.h"
#include "bct_linear.h"
#include "bct_tc.cuh"

namespace bct {
namespace {

constexpr int kLtThreads = 864;
constexpr int kLtCh = 128;                    // tokens per chunk
constexpr int kLtHalf = 128 * 128;            // 64 columns (128 bytes) x 128 rows
constexpr int kLtTile = 2 * kLtHalf;
constexpr int kLtStep = 16;                   // rows of w o B per ring slot (one K step)
constexpr int kLtTerms = 2;
constexpr int kLtTermBytes = kLtStep * 256;   // two halves of 16 rows x 128 bytes
constexpr int kLtSlotBytes = kLtTerms * kLtTermBytes;
constexpr int kLtSlots = 7;
// tensor-memory columns
constexpr int kLtColW = 0;     // W, then P (bfloat16 pairs) in the first half of each of its 64-column halves
constexpr int kLtColO = 128;
constexpr int kLtColD = 256;   // what the chunk adds to the state, [feature of c][feature of b]
constexpr int kLtColS = 384;   // the state

struct LtArgs {
    CUtensorMap in[4];    // forward: q, k, v;  backward: d_out, q, k, v
    CUtensorMap out[3];   // per role
    LinArgs s;
    LinStates st;
    int map_a[3], map_b[3], map_c[3];     // which of `in` a role reads
    int st_map_b[2], st_map_c[2];
};

template <bool STATE_ONLY>
struct LtSmem {
    static constexpr int kBc = STATE_ONLY ? 2 : 1;     // buffers of B and of C
    static constexpr int b = 0;
    static constexpr int c = b + kBc * kLtTile;
    static constexpr int a = c + kBc * kLtTile;        // two buffers
    static constexpr int x = a + (STATE_ONLY ? 0 : 2 * kLtTile);   // the state as an operand: rows = features of c
    static constexpr int slots = x + (STATE_ONLY ? 0 : kLtTile);
    static constexpr int bars = slots + kLtSlots * kLtSlotBytes;
    static constexpr int pw = bars + 64 * 8;           // lambda^n, n = 0..128
    static constexpr int pt = pw + 132 * 4;            // [256]: lambda^|j - i| at 127 + j - i, 0 where the mask is
    // by the token's place in its chunk, for a full chunk and for the one that ends early:
    static constexpr int pc = pt + 256 * 4;            // [32]: lambda^(31 - j), in reverse lambda^j
    static constexpr int fo = pc + 32 * 4;           // [2][128] scale f_i
    static constexpr int fi = fo + 256 * 4;            // [2][128] 1 / f_i
    static constexpr int wb = fi + 256 * 4;            // [2][128] w_j, 0 behind the last valid token
    static constexpr int total = wb + 256 * 4 + 1024;  // slack to align the base to 1024 bytes
};

// D (+)= A B with A (bfloat16 pairs) in tensor memory
__device__ __forceinline__ void umma_bf16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, bool accum) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"((uint32_t)accum)
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
// 16 columns from each of two places, one wait.
__device__ __forceinline__ void tmem_ld16_two(uint32_t ta, float* x, uint32_t tb, float* y) {
    uint32_t a[16], b[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]), "=r"(a[4]), "=r"(a[5]), "=r"(a[6]), "=r"(a[7]), "=r"(a[8]),
          "=r"(a[9]), "=r"(a[10]), "=r"(a[11]), "=r"(a[12]), "=r"(a[13]), "=r"(a[14]), "=r"(a[15])
        : "r"(ta));
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(b[0]), "=r"(b[1]), "=r"(b[2]), "=r"(b[3]), "=r"(b[4]), "=r"(b[5]), "=r"(b[6]), "=r"(b[7]), "=r"(b[8]),
          "=r"(b[9]), "=r"(b[10]), "=r"(b[11]), "=r"(b[12]), "=r"(b[13]), "=r"(b[14]), "=r"(b[15])
        : "r"(tb));
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(a[0]), "+r"(a[1]), "+r"(a[2]), "+r"(a[3]), "+r"(a[4]), "+r"(a[5]), "+r"(a[6]), "+r"(a[7]),
                   "+r"(a[8]), "+r"(a[9]), "+r"(a[10]), "+r"(a[11]), "+r"(a[12]), "+r"(a[13]), "+r"(a[14]), "+r"(a[15])
                 :
                 : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(b[0]), "+r"(b[1]), "+r"(b[2]), "+r"(b[3]), "+r"(b[4]), "+r"(b[5]), "+r"(b[6]), "+r"(b[7]),
                   "+r"(b[8]), "+r"(b[9]), "+r"(b[10]), "+r"(b[11]), "+r"(b[12]), "+r"(b[13]), "+r"(b[14]), "+r"(b[15])
                 :
                 : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(a[i]), y[i] = __uint_as_float(b[i]);
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tma_store_4d(const CUtensorMap* map, int x, int y, int z, int w, const void* src) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%1, %2, %3, %4}], [%5];"
                 ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(src))
                 : "memory");
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

__device__ __forceinline__ void tma_prefetch_4d(const CUtensorMap* map, int x, int y, int z, int w) {
    asm volatile("cp.async.bulk.prefetch.tensor.4d.L2.global.tile [%0, {%1, %2, %3, %4}];"
                 ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(w)
                 : "memory");
}

template <bool STATE_ONLY>
__global__ void __launch_bounds__(kLtThreads, 1) linear_tc_kernel(const __grid_constant__ LtArgs args) {
    using L = LtSmem<STATE_ONLY>;
    extern __shared__ unsigned char lt_smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(lt_smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::bars);
    uint64_t* full_a = bars;             // [2]
    uint64_t* empty_a = bars + 2;        // [2] the output that took A's place has been read out
    uint64_t* out_full = bars + 4;       // [2] the output is in A's place
    uint64_t* full_b = bars + 6;         // [2]
    uint64_t* empty_b = bars + 8;        // [2]
    uint64_t* full_c = bars + 10;        // [2]
    uint64_t* empty_c = bars + 12;       // [2]
    uint64_t* slot_full = bars + 14;     // [kLtSlots], at most 8
    uint64_t* slot_empty = bars + 22;    // [kLtSlots]
    uint64_t* w_full = bars + 30;        // W complete
    uint64_t* p_full = bars + 31;        // P in place, W read
    uint64_t* o_full = bars + 33;
    uint64_t* o_empty = bars + 34;
    uint64_t* d_full = bars + 35;        // the chunk's addition to the state complete
    uint64_t* d_empty = bars + 36;
    uint64_t* x_full = bars + 37;        // the state operand in place
    uint64_t* x_empty = bars + 38;       // the products with the state operand complete
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 40);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 41);
    float* pw = reinterpret_cast<float*>(smem + L::pw);
    float* pt = reinterpret_cast<float*>(smem + L::pt);
    float* pc = reinterpret_cast<float*>(smem + L::pc);
    float* fo = reinterpret_cast<float*>(smem + L::fo);
    float* fi = reinterpret_cast<float*>(smem + L::fi);
    float* wb = reinterpret_cast<float*>(smem + L::wb);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const LinArgs& s = args.s;
    const int seg = blockIdx.x % s.nseg;
    const int u = blockIdx.x / s.nseg;
    const int bi = u / s.Hkv, h = u - bi * s.Hkv;
    const int which = STATE_ONLY ? (args.st.seg[0] == nullptr ? 1 : (int)blockIdx.y) : (int)blockIdx.y;
    const LinRole& r = s.role[STATE_ONLY ? 0 : which];
    const int reverse = STATE_ONLY ? which : r.reverse;
    const int Ga = STATE_ONLY ? 1 : r.Ga, Gb = STATE_ONLY ? args.st.G[which] : r.Gb;
    if (STATE_ONLY && seg == (reverse ? 0 : s.nseg - 1)) return;   // feeds no other segment
    const CUtensorMap* map_a = &args.in[STATE_ONLY ? 0 : args.map_a[which]];
    const CUtensorMap* map_b = &args.in[STATE_ONLY ? args.st_map_b[which] : args.map_b[which]];
    const CUtensorMap* map_c = &args.in[STATE_ONLY ? args.st_map_c[which] : args.map_c[which]];

    const int len = s.lens ? min(max(s.lens[bi], 0), s.T) : s.T;
    const int t_begin = seg * s.seg_len;
    const int t_end = min(t_begin + s.seg_len, s.T);
    const int v_end = min(t_end, len);
    const int n_chunks = v_end > t_begin ? (v_end - t_begin + kLtCh - 1) / kLtCh : 0;
    const int G = Ga > Gb ? Ga : Gb;
    auto chunk_t0 = [&](int n) { return t_begin + (reverse ? n_chunks - 1 - n : n) * kLtCh; };
    auto chunk_nv = [&](int t0) { return min(kLtCh, v_end - t0); };

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&full_a[i], 1);
            mbar_init(&empty_a[i], 1);
            mbar_init(&out_full[i], 8);
            mbar_init(&full_b[i], 1);
            mbar_init(&empty_b[i], STATE_ONLY ? 8 : 9);   // the splitting warps, and the products with B
            mbar_init(&full_c[i], 1);
            mbar_init(&empty_c[i], 1);
        }
        for (int i = 0; i < kLtSlots; ++i) {
            mbar_init(&slot_full[i], 4);
            mbar_init(&slot_empty[i], 1);
        }
        mbar_init(w_full, 1);
        mbar_init(p_full, 8);
        mbar_init(o_full, 1);
        mbar_init(o_empty, 8);
        mbar_init(d_full, 1);
        mbar_init(d_empty, 8);
        mbar_init(x_full, 8);
        mbar_init(x_empty, 1);
        *abort_flag = 0;
        fence_mbar_init_cluster();
    }
    if (warp == 25) tmem_alloc(tmem_slot, 512);
    const float log_decay = s.log_decay[h];
    for (int i = tid; i < 132; i += kLtThreads) {   // the powers in double, rounded once
        const double g = (double)log_decay;
        pw[i] = i == 0 ? 1.f : (float)exp(g * i);
    }
    for (int i = tid; i < 256; i += kLtThreads) {
        const int t = i & 127, nv = i < 128 ? 128 : (n_chunks > 0 ? (v_end - t_begin - 1) % kLtCh + 1 : 1);
        const int to_end = max(nv - 1 - t, 0), from_start = t + 1;
        const double g = (double)log_decay;
        const int ef = reverse ? to_end : from_start, ew = reverse ? from_start : to_end;
        const float f = ef == 0 ? 1.f : fmaxf((float)exp(g * ef), 9.094947017729282e-13f);   // 2^-40
        if (!STATE_ONLY) {
            fo[i] = f * r.scale;
            fi[i] = 1.f / f;
        }
        const int dist = reverse ? i - 127 : 127 - i;
        pt[i] = dist < 0 ? 0.f : (dist == 0 ? 1.f : (float)exp(g * dist));
        if (i < 32) {
            const int e = reverse ? i : 31 - i;
            pc[i] = e == 0 ? 1.f : (float)exp(g * e);
        }
        wb[i] = t >= nv ? 0.f : (ew == 0 ? 1.f : (float)exp(g * ew));
    }
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

#define LT_WAIT(bar, parity) lt_wait(bar, (parity) & 1, abort_flag);

    const int items = n_chunks * G;   // (chunk, head) in turn: head x of the side that has G of them
    if (warp == 24) {
        // =========================== loads ===========================
        if (lane == 0) {
            auto load = [&](const CUtensorMap* map, int head, int t0, unsigned char* dst, uint64_t* bar) {
                mbar_arrive_expect_tx(bar, kLtTile);
                tma_load_4d(dst, map, 0, head, t0, bi, bar);
                tma_load_4d(dst + kLtHalf, map, 64, head, t0, bi, bar);
            };
            auto load_a = [&](int it) {
                const int n = it / G, x = it - n * G, na = Ga > 1 ? it : n;
                if (STATE_ONLY || (x > 0 && Ga == 1)) return;
                if (na > 1) LT_WAIT(&empty_a[na & 1], (na >> 1) - 1);
                load(map_a, h * Ga + (Ga > 1 ? x : 0), chunk_t0(n), smem + L::a + (na & 1) * kLtTile, &full_a[na & 1]);
            };
            auto load_b = [&](int it) {
                const int n = it / G, x = it - n * G, nb = Gb > 1 ? it : n, st = nb % L::kBc;
                if (x > 0 && Gb == 1) return;
                if (nb >= L::kBc) LT_WAIT(&empty_b[st], nb / L::kBc - 1);
                load(map_b, h * Gb + (Gb > 1 ? x : 0), chunk_t0(n), smem + L::b + st * kLtTile, &full_b[st]);
            };
            auto load_c = [&](int it) {
                const int n = it / G, x = it - n * G, nb = Gb > 1 ? it : n, st = nb % L::kBc;
                if (x > 0 && Gb == 1) return;
                if (nb >= L::kBc) LT_WAIT(&empty_c[st], nb / L::kBc - 1);
                load(map_c, h * Gb + (Gb > 1 ? x : 0), chunk_t0(n), smem + L::c + st * kLtTile, &full_c[st]);
            };
            auto prefetch = [&](int it) {
                const int n = it / G, x = it - n * G, t0 = chunk_t0(n);
                if (!STATE_ONLY && (x == 0 || Ga > 1)) {
                    tma_prefetch_4d(map_a, 0, h * Ga + (Ga > 1 ? x : 0), t0, bi);
                    tma_prefetch_4d(map_a, 64, h * Ga + (Ga > 1 ? x : 0), t0, bi);
                }
                if (x == 0 || Gb > 1) {
                    const int head = h * Gb + (Gb > 1 ? x : 0);
                    tma_prefetch_4d(map_b, 0, head, t0, bi);
                    tma_prefetch_4d(map_b, 64, head, t0, bi);
                    tma_prefetch_4d(map_c, 0, head, t0, bi);
                    tma_prefetch_4d(map_c, 64, head, t0, bi);
                }
            };
            if (items > 0) {
                load_b(0);
                load_a(0);
            }
            if (items > 1) prefetch(1);
            for (int it = 0; it < items; ++it) {   // in the order in which the tiles before them are free
                load_c(it);
                if (it + 2 < items) prefetch(it + 2);
                if (it + 1 < items) {
                    load_a(it + 1);
                    load_b(it + 1);
                }
            }
        }
        __syncwarp();
    } else if (warp == 25) {
        // =========================== products ===========================
        if (lane == 0) {
            constexpr uint32_t id_kk = instr_desc_mn(128, 128, false, false);
            constexpr uint32_t id_kn = instr_desc_mn(128, 128, false, true);
            constexpr uint32_t id_nn = instr_desc_mn(128, 128, true, true);
            const DescKind dk(smem_desc(0, 16, 1024)), dmn(smem_desc(0, kLtHalf, 1024)),
                dslot(smem_desc(0, kLtStep * 128, 1024));
            const uint32_t a16 = desc_addr16(smem_u32(smem + L::a)), b16 = desc_addr16(smem_u32(smem + L::b)),
                           c16 = desc_addr16(smem_u32(smem + L::c)), x16 = desc_addr16(smem_u32(smem + L::x)),
                           s16 = desc_addr16(smem_u32(smem + L::slots));
            constexpr uint32_t t16 = kLtTile / 16, h16 = kLtHalf / 16;
            // (Loops here and in the other roles are kept short: 27 warps of six roles share the instruction caches, and
            // straight-line code that is run once per chunk is fetched anew each time.)
            auto product_kk = [&](uint32_t d, uint32_t xa, uint32_t ya) {   // D = X Y^T, both with k along their rows
#pragma unroll 1
                for (int hf = 0; hf < 2; ++hf, xa += h16, ya += h16) {
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) umma_bf16(d, dk.at(xa + 2 * kk), dk.at(ya + 2 * kk), id_kk, hf > 0 || kk > 0);
                }
            };
            int sl = 0;          // ring slot and the parity of its turn
            uint32_t turn = 0;
            for (int it = 0; it < items; ++it) {
                const int n = it / G, x = it - n * G;
                const int na = Ga > 1 ? it : n, nb = Gb > 1 ? it : n, sb = nb % L::kBc;
                const bool new_b = x == 0 || Gb > 1, new_a = x == 0 || Ga > 1, last = x == G - 1;
                const uint32_t aa = a16 + (na & 1) * t16, ba = b16 + sb * t16, ca = c16 + sb * t16;
                if (!STATE_ONLY) {
                    LT_WAIT(&full_a[na & 1], na >> 1);
                    LT_WAIT(&full_b[sb], nb / L::kBc);
                    tc_fence_after();
                    product_kk(tmem + kLtColW, aa, ba);
                    umma_commit(w_full);
                    if (Gb > 1 || last) umma_commit(&empty_b[sb]);
                    if (new_a) {   // the state's share
                        if (x == 0) LT_WAIT(x_full, n);
                        if (na > 0) LT_WAIT(o_empty, na - 1);
                        tc_fence_after();
                        product_kk(tmem + kLtColO, aa, x16);
                        if (Gb > 1 || last) umma_commit(x_empty);
                    }
                }
                if (new_b) {   // the chunk's addition to the state
                    if (x == 0 && n > 0) LT_WAIT(d_empty, n - 1);
                    LT_WAIT(&full_c[sb], nb / L::kBc);
#pragma unroll 1
                    for (int st = 0; st < kLtCh / kLtStep; ++st) {
                        LT_WAIT(&slot_full[sl], turn);
                        tc_fence_after();
                        const uint64_t cd = dmn.at(ca + st * 128);
                        const uint32_t sa = s16 + sl * (kLtSlotBytes / 16);
#pragma unroll
                        for (int t = 0; t < kLtTerms; ++t)
                            umma_bf16(tmem + kLtColD, cd, dslot.at(sa + t * (kLtTermBytes / 16)), id_nn, t > 0 || st > 0 || x > 0);
                        umma_commit(&slot_empty[sl]);
                        if (++sl == kLtSlots) sl = 0, turn ^= 1;
                    }
                    if (Gb == 1 || last) umma_commit(d_full);
                    if (STATE_ONLY) umma_commit(&empty_c[sb]);
                }
                if (!STATE_ONLY) {
                    LT_WAIT(p_full, it);
                    tc_fence_after();
#pragma unroll 1
                    for (int hf = 0; hf < 2; ++hf) {
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            umma_bf16_ts(tmem + kLtColO, tmem + kLtColW + hf * 64 + kk * 8, dmn.at(ca + hf * 512 + kk * 128), id_kn, true);
                    }
                    if (Ga > 1 || last) umma_commit(o_full);
                    if (Gb > 1 || last) umma_commit(&empty_c[sb]);
                }
            }
        }
        __syncwarp();
    } else if (warp == 26) {
        // =========================== stores ===========================
        if (!STATE_ONLY && lane == 0) {
            const CUtensorMap* map_o = &args.out[which];
            int na = 0;
            for (int n = 0; n < n_chunks; ++n) {
                const int t0 = chunk_t0(n);
                for (int x = 0; x < Ga; ++x, ++na) {
                    const unsigned char* src = smem + L::a + (na & 1) * kLtTile;
                    LT_WAIT(&out_full[na & 1], na >> 1);
                    tma_store_4d(map_o, 0, h * Ga + x, t0, bi, src);
                    tma_store_4d(map_o, 64, h * Ga + x, t0, bi, src + kLtHalf);
                    bulk_commit();
                    bulk_wait_read();
                    mbar_arrive(&empty_a[na & 1]);
                }
            }
            bulk_wait_all();
        }
        __syncwarp();
    } else if (warp < 8) {
        // =========================== W -> P: two threads per row i, 64 columns each ===========
        if (!STATE_ONLY) {
            const int q = warp & 3, half = warp >> 2, i = q * 32 + lane;
            const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16) + kLtColW + half * 64;
            const float* pti = pt + 127 - i;
            int it = 0;
            for (int n = 0; n < n_chunks; ++n) {
                const int nv = chunk_nv(chunk_t0(n));
                const float inv_f = fi[(nv < kLtCh ? 128 : 0) + i];
                for (int x = 0; x < G; ++x, ++it) {
                    LT_WAIT(w_full, it);
                    tc_fence_after();
#pragma unroll 1
                    for (int e = 0; e < 4; ++e) {   // 16 columns; P takes the place of columns read before
                        const int j0 = half * 64 + e * 16, cb = j0 >> 5;
                        float v[16];
                        if (reverse ? cb < q : cb > q) {   // the mask leaves nothing
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[j] = 0.f;
                        } else {
                            tmem_ld16(lane_base + e * 16, v);
                            if (cb == q) {   // the mask's edge runs through this block
#pragma unroll
                                for (int j = 0; j < 16; ++j) {
                                    const float w = pti[j0 + j];
                                    v[j] = w > 0.f ? v[j] * (w * inv_f) : 0.f;
                                }
                            } else {         // a power for the row and the block, one for the column
                                const float wr = pw[reverse ? cb * 32 - i : i - cb * 32 - 31] * inv_f;
#pragma unroll
                                for (int j = 0; j < 16; j += 4) {
                                    const float4 wc = *reinterpret_cast<const float4*>(pc + (e & 1) * 16 + j);
                                    const float2 y = __fmul2_rn(__fmul2_rn(make_float2(v[j], v[j + 1]), make_float2(wc.x, wc.y)),
                                                                make_float2(wr, wr));
                                    const float2 z = __fmul2_rn(__fmul2_rn(make_float2(v[j + 2], v[j + 3]), make_float2(wc.z, wc.w)),
                                                                make_float2(wr, wr));
                                    v[j] = y.x, v[j + 1] = y.y, v[j + 2] = z.x, v[j + 3] = z.y;
                                }
                            }
                            if (nv < kLtCh) {   // products with padding rows, which hold anything
#pragma unroll
                                for (int j = 0; j < 16; ++j) v[j] = j0 + j < nv ? v[j] : 0.f;
                            }
                        }
                        uint32_t pk[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) pk[j] = Chunk<__nv_bfloat16>::pack2(v[2 * j], v[2 * j + 1]);
                        tmem_st8u(lane_base + e * 8, pk);
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full);
                }
            }
        }
    } else if (warp < 16) {
        // =========================== w o B in three terms, 16 rows at a time ===========================
        const int group = (warp - 8) >> 2, wt = tid & 127;   // two groups of four warps: even and odd steps
        const int row = wt >> 3, c8 = wt & 7;
        const int place = row * 128 + ((c8 ^ (row & 7)) * 16);
        int nb = 0;
        for (int n = 0; n < n_chunks; ++n) {
            const int nv = chunk_nv(chunk_t0(n));
            for (int x = 0; x < Gb; ++x, ++nb) {
                const int st = nb % L::kBc, use = nb / L::kBc;
                const unsigned char* bt = smem + L::b + st * kLtTile;
                LT_WAIT(&full_b[st], use);
                if (nv < kLtCh && group == 0) {   // padding rows of C hold anything: zero, before the first product reads them
                    LT_WAIT(&full_c[st], use);
                    if (wt >= nv) {
                        uint4* z = reinterpret_cast<uint4*>(smem + L::c + st * kLtTile + wt * 128);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            z[j] = make_uint4(0, 0, 0, 0);
                            z[j + kLtHalf / 16] = make_uint4(0, 0, 0, 0);
                        }
                    }
                }
#pragma unroll 1
                for (int t = group; t < kLtCh / kLtStep; t += 2) {
                    const int ks = nb * (kLtCh / kLtStep) + t, sl = ks % kLtSlots;
                    const int j = t * kLtStep + row;
                    const float w = wb[(nv < kLtCh ? 128 : 0) + j];
                    if (ks >= kLtSlots) LT_WAIT(&slot_empty[sl], ks / kLtSlots - 1);
                    const unsigned char* src = bt + t * kLtStep * 128 + place;
                    unsigned char* dst = smem + L::slots + sl * kLtSlotBytes + place;
#pragma unroll 1
                    for (int hf = 0; hf < 2; ++hf, src += kLtHalf, dst += kLtStep * 128) {
                        uint4 raw = *reinterpret_cast<const uint4*>(src);
                        if (j >= nv) raw = make_uint4(0, 0, 0, 0);   // (padding may hold NaN)
                        const uint32_t rw[4] = {raw.x, raw.y, raw.z, raw.w};
                        uint32_t o[kLtTerms][4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float2 v = __fmul2_rn(make_float2(__uint_as_float(rw[e] << 16), __uint_as_float(rw[e] & 0xffff0000u)),
                                                  make_float2(w, w));
#pragma unroll
                            for (int tm = 0; tm < kLtTerms; ++tm) {
                                const uint32_t pk = Chunk<__nv_bfloat16>::pack2(v.x, v.y);
                                o[tm][e] = pk;
                                if (tm + 1 < kLtTerms)   // what the term leaves out, exactly
                                    v = __fadd2_rn(v, make_float2(-__uint_as_float(pk << 16), -__uint_as_float(pk & 0xffff0000u)));
                            }
                        }
#pragma unroll
                        for (int tm = 0; tm < kLtTerms; ++tm)
                            *reinterpret_cast<uint4*>(dst + tm * kLtTermBytes) = make_uint4(o[tm][0], o[tm][1], o[tm][2], o[tm][3]);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(&slot_full[sl]);
                        if (t >= kLtCh / kLtStep - 2) mbar_arrive(&empty_b[st]);   // this group has read its rows of B
                    }
                }
            }
        }
    } else {
        // =========================== the state and the outputs ===========================
        const int q = warp & 3, hs = (warp - 16) >> 2;   // lanes 32q.., columns 64 hs..
        const int c = q * 32 + lane;                      // this thread's feature of c; of the outputs, its row
        const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
        const uint32_t s_col = lane_base + kLtColS + hs * 64, d_col = lane_base + kLtColD + hs * 64;
        {
            const bool from_seg = !STATE_ONLY && s.nseg > 1;
            const float* src = STATE_ONLY ? nullptr
                               : from_seg ? r.seg + ((size_t)u * s.nseg + seg) * 16384
                                          : (r.state_in ? r.state_in + (size_t)u * 16384 : nullptr);
            const float mul = from_seg || STATE_ONLY ? 1.f : r.in_mul;
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {
                float v[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = 0.f;
                if (src != nullptr) {
                    if (!r.state_t) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] = mul * src[(hs * 64 + k * 16 + i) * 128 + c];
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float4 x = *reinterpret_cast<const float4*>(src + c * 128 + hs * 64 + k * 16 + 4 * i);
                            v[4 * i] = mul * x.x, v[4 * i + 1] = mul * x.y, v[4 * i + 2] = mul * x.z, v[4 * i + 3] = mul * x.w;
                        }
                    }
                }
                tmem_st16u(s_col + k * 16, reinterpret_cast<const uint32_t*>(v));
            }
            tmem_wait_st();
        }
        unsigned char* x_row = smem + L::x + hs * kLtHalf + c * 128;
        // Before chunk n: take in what chunk n - 1 adds, and write the operand for chunk n's products.
        auto turn = [&](int n) {
            const bool add = n > 0, put = !STATE_ONLY && n < n_chunks;
            const float f = add ? pw[chunk_nv(chunk_t0(n - 1))] : 1.f;
            if (add) {
                LT_WAIT(d_full, n - 1);
                if (put) LT_WAIT(x_empty, n - 1);
                tc_fence_after();
            }
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {
                float x[16], d[16];
                tmem_ld16_two(s_col + k * 16, x, d_col + k * 16, d);
                if (add) {
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const float2 y = __ffma2_rn(make_float2(x[i], x[i + 1]), make_float2(f, f), make_float2(d[i], d[i + 1]));
                        x[i] = y.x, x[i + 1] = y.y;
                    }
                    tmem_st16u(s_col + k * 16, reinterpret_cast<const uint32_t*>(x));
                }
                if (put) {
                    *reinterpret_cast<uint4*>(x_row + (((2 * k) ^ (c & 7)) * 16)) = Chunk<__nv_bfloat16>::pack(x);
                    *reinterpret_cast<uint4*>(x_row + (((2 * k + 1) ^ (c & 7)) * 16)) = Chunk<__nv_bfloat16>::pack(x + 8);
                }
            }
            tmem_wait_st();
            if (put) fence_proxy_async_smem();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (add) mbar_arrive(d_empty);
                if (put) mbar_arrive(x_full);
            }
        };
        int na = 0;
        if (n_chunks > 0) turn(0);
        for (int n = 0; n < n_chunks; ++n) {
            if (STATE_ONLY) {
                turn(n + 1);
                continue;
            }
            const int nv = chunk_nv(chunk_t0(n));
            const float f = fo[(nv < kLtCh ? 128 : 0) + c];
            for (int x = 0; x < Ga; ++x, ++na) {
                if (x == Ga - 1) turn(n + 1);   // complete before the chunk's last output, and the next chunk's products wait for it
                LT_WAIT(o_full, na);
                tc_fence_after();
                unsigned char* dst = smem + L::a + (na & 1) * kLtTile + hs * kLtHalf + c * 128;
#pragma unroll 1
                for (int k = 0; k < 4; ++k) {
                    float o[16];
                    tmem_ld16(lane_base + kLtColO + hs * 64 + k * 16, o);
                    if (k == 3) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(o_empty);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] = c < nv ? o[i] * f : 0.f;   // padding rows: zeros
                    *reinterpret_cast<uint4*>(dst + (((2 * k) ^ (c & 7)) * 16)) = Chunk<__nv_bfloat16>::pack(o);
                    *reinterpret_cast<uint4*>(dst + (((2 * k + 1) ^ (c & 7)) * 16)) = Chunk<__nv_bfloat16>::pack(o + 8);
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&out_full[na & 1]);
            }
        }
        const float poison = *abort_flag ? __int_as_float(0x7fc00000) : 0.f;
        float* dst = nullptr;
        float mul = 1.f;
        if (STATE_ONLY) {   // into the slot of the segment that it feeds, key's features in the rows
            dst = args.st.seg[which] + ((size_t)u * s.nseg + (reverse ? seg - 1 : seg + 1)) * 16384;
        } else if (r.state_out != nullptr && seg == (reverse ? 0 : s.nseg - 1)) {
            dst = r.state_out + (size_t)u * 16384;   // (never transposed)
            mul = r.out_mul;
        }
        if (dst != nullptr) {
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {
                float x[16];
                tmem_ld16(s_col + k * 16, x);
#pragma unroll
                for (int i = 0; i < 16; ++i) dst[(hs * 64 + k * 16 + i) * 128 + c] = x[i] * mul + poison;
            }
        }
    }
#undef LT_WAIT
    tc_fence_before();
    __syncthreads();
    if (warp == 25) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (!STATE_ONLY) {   // padding rows behind the last chunk: zeros; after a timeout everything is NaN
        const bool bad = *abort_flag != 0;
        const int first = bad ? t_begin : t_begin + n_chunks * kLtCh;
        const uint32_t fill = bad ? 0x7fc07fc0u : 0u;
        char* out = static_cast<char*>(r.out);
        for (int i = tid; (long long)first + i / 16 < t_end; i += kLtThreads) {
            const size_t row = (size_t)bi * s.T + first + i / 16;
            for (int x = 0; x < Ga; ++x)
                reinterpret_cast<uint4*>(out + (row * s.Hkv * Ga + (size_t)h * Ga + x) * 256)[i & 15] =
                    make_uint4(fill, fill, fill, fill);
        }
    }
}

// [B][T][H][128] bfloat16 as (feature, head, token, sequence); one box is 64 features of one head for 128 tokens;
// tokens past T read as zeros and are not written.
bool lt_map(CUtensorMap* map, const void* base, int B, int T, int H) {
    TensorMapEncodeFn fn = tensor_map_encode_fn();
    if (fn == nullptr) return false;
    const cuuint64_t dims[4] = {128, (cuuint64_t)H, (cuuint64_t)T, (cuuint64_t)B};
    const cuuint64_t strides[3] = {256, (cuuint64_t)H * 256, (cuuint64_t)T * H * 256};
    const cuuint32_t box[4] = {64, 1, (cuuint32_t)kLtCh, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool STATE_ONLY>
cudaError_t lt_launch(const LtArgs& a, int grid_y, cudaStream_t stream) {
    auto fn = linear_tc_kernel<STATE_ONLY>;
    const int smem = LtSmem<STATE_ONLY>::total;
    static_assert(LtSmem<STATE_ONLY>::total <= 232448, "shared memory of a block");
    cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(fn), cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)(a.s.B * a.s.Hkv * a.s.nseg), (unsigned)grid_y);
    fn<<<grid, kLtThreads, smem, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_linear_tc(const LinArgs& args, const LinStates& states, cudaStream_t stream) {
    LtArgs a;
    a.s = args;
    a.st = states;
    int n_in = 0;
    const void* base[4] = {};
    auto map_of = [&](const void* p, int heads) -> int {   // one map per tensor
        for (int i = 0; i < n_in; ++i)
            if (base[i] == p) return i;
        if (n_in == 4 || !lt_map(&a.in[n_in], p, args.B, args.T, args.Hkv * heads)) return -1;
        base[n_in] = p;
        return n_in++;
    };
    for (int i = 0; i < args.n_roles; ++i) {
        const LinRole& r = args.role[i];
        a.map_a[i] = map_of(r.a, r.Ga);
        a.map_b[i] = map_of(r.b, r.Gb);
        a.map_c[i] = map_of(r.c, r.Gb);
        if (a.map_a[i] < 0 || a.map_b[i] < 0 || a.map_c[i] < 0) return cudaErrorInvalidValue;
        if (!lt_map(&a.out[i], r.out, args.B, args.T, args.Hkv * r.Ga)) return cudaErrorInvalidValue;
    }
    if (args.nseg > 1) {
        for (int d = 0; d < 2; ++d) {
            if (states.seg[d] == nullptr) continue;
            a.st_map_b[d] = map_of(states.b[d], states.G[d]);
            a.st_map_c[d] = map_of(states.c[d], states.G[d]);
            if (a.st_map_b[d] < 0 || a.st_map_c[d] < 0) return cudaErrorInvalidValue;
        }
        const int dirs = (states.seg[0] != nullptr) + (states.seg[1] != nullptr);
        cudaError_t e = lt_launch<true>(a, dirs, stream);
        if (e == cudaSuccess) e = launch_linear_combine(128, args, states, stream);
        if (e != cudaSuccess) return e;
    }
    return lt_launch<false>(a, args.n_roles, stream);
}

}  // namespace bct
