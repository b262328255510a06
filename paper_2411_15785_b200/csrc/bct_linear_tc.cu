// Linear attention with a decay for each head on the sm_100a tensor path: the chunked scan for bfloat16 and
// head_dim 128 (the forward, and the three scans of the backward; bct_linear.h names the roles a, b, c).
//
// Per (sequence, kv-head) unit and chunk of 128 tokens, X being the state outside the chunk:
//     W    = A B^T                                  products of all pairs            [i][j]
//     P_ij = W_ij lambda^|i-j| / f_i                j <= i (j >= i in reverse)       bfloat16
//     O    = C^T P^T + X A^T                        transposed: [feature of c][i]
//     out_i = scale f_i O_i                         f_i = lambda^(distance of i to X's token)
//     X   <- lambda^n X + C^T (w o B)               w_j = lambda^(distance of j to the new X's token)
// all as tcgen05.mma with M = N = 128 and fp32 accumulators in tensor memory.
//  - O is formed with its tokens in the columns so that the state can be the tensor-memory operand of the second
//    product: X lives with c's features in its lanes and b's in its columns, in registers (two threads per lane, 64
//    columns each) in fp32; per chunk it is rounded to bfloat16 once, into tensor memory, for the product with A.
//  - f_i multiplies the whole column at the end instead of A's row, so A goes into both products as it is.  It is
//    floored at 2^-40, which keeps P_ij in range: below that the state's share, as it is and as it is then taken,
//    is under the rounding of what the column's own token adds.
//  - w o B is split into three bfloat16 terms (24 bits), so what enters the state is exact to fp32: 3 of the 6.6
//    products of a chunk, hidden behind the loads.
//  - P's columns (rows of the product) that the mask empties are left out of the product: 0.56 of the full one.
//  - P and the state are each rounded to bfloat16 once where they enter a product with bfloat16 results.
// Roles (19 warps): warps 0-3 turn W into P, warps 4-7 split w o B into a ring of 16-row steps, warps 8-15 keep the
// state and write the outputs, over the A tile that has been read; warp 16 loads (TMA), warp 17 issues the products,
// warp 18 stores (TMA).  With more than one segment, the same kernel without A, W and P forms what every segment adds.
// Every wait is bounded; a timeout ends the work and fills the block's outputs with NaN.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "bct_internal.h"
#include "bct_linear.h"
#include "bct_tc.cuh"

namespace bct {
namespace {

constexpr int kLtThreads = 608;
constexpr int kLtCh = 128;                    // tokens per chunk
constexpr int kLtHalf = 128 * 128;            // 64 columns (128 bytes) x 128 rows
constexpr int kLtTile = 2 * kLtHalf;
constexpr int kLtStep = 16;                   // rows of w o B per ring slot (one K step)
constexpr int kLtTerms = 3;
constexpr int kLtTermBytes = kLtStep * 256;   // two halves of 16 rows x 128 bytes
constexpr int kLtSlotBytes = kLtTerms * kLtTermBytes;
constexpr int kLtSlots = 5;
// tensor-memory columns
constexpr int kLtColW = 0;
constexpr int kLtColO = 128;
constexpr int kLtColD = 256;   // what the chunk adds to the state
constexpr int kLtColX = 384;   // the state as an operand: 64 columns of bfloat16 pairs

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
    static constexpr int p = a + (STATE_ONLY ? 0 : 2 * kLtTile);
    static constexpr int slots = p + (STATE_ONLY ? 0 : kLtTile);
    static constexpr int bars = slots + kLtSlots * kLtSlotBytes;
    static constexpr int pw = bars + 64 * 8;           // lambda^n, n = 0..128
    static constexpr int pt = pw + 132 * 4;            // [256]: lambda^|j - i| at 127 + j - i, 0 where the mask is
    // by the token's place in its chunk, for a full chunk and for the one that ends early:
    static constexpr int fo = pt + 256 * 4;           // [2][128] scale f_i
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
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
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
    uint64_t* slot_full = bars + 14;     // [kLtSlots]
    uint64_t* slot_empty = bars + 20;    // [kLtSlots]
    uint64_t* w_full = bars + 26;        // W complete
    uint64_t* p_full = bars + 27;        // P in place, W read
    uint64_t* p_empty = bars + 28;       // the product with P complete
    uint64_t* o_full = bars + 29;
    uint64_t* o_empty = bars + 30;
    uint64_t* d_full = bars + 31;        // the chunk's addition to the state complete
    uint64_t* d_empty = bars + 32;
    uint64_t* x_full = bars + 33;        // the state operand in place
    uint64_t* x_empty = bars + 34;       // the products with the state operand complete
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 36);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 37);
    float* pw = reinterpret_cast<float*>(smem + L::pw);
    float* pt = reinterpret_cast<float*>(smem + L::pt);
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
            mbar_init(&empty_b[i], STATE_ONLY ? 4 : 5);   // the splitting warps, and the products with B
            mbar_init(&full_c[i], 1);
            mbar_init(&empty_c[i], 1);
        }
        for (int i = 0; i < kLtSlots; ++i) {
            mbar_init(&slot_full[i], 4);
            mbar_init(&slot_empty[i], 1);
        }
        mbar_init(w_full, 1);
        mbar_init(p_full, 4);
        mbar_init(p_empty, 1);
        mbar_init(o_full, 1);
        mbar_init(o_empty, 8);
        mbar_init(d_full, 1);
        mbar_init(d_empty, 8);
        mbar_init(x_full, 8);
        mbar_init(x_empty, 1);
        *abort_flag = 0;
        fence_mbar_init_cluster();
    }
    if (warp == 17) tmem_alloc(tmem_slot, 512);
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
        wb[i] = t >= nv ? 0.f : (ew == 0 ? 1.f : (float)exp(g * ew));
    }
    if (!STATE_ONLY)   // what the mask empties of P is never written again
        for (int i = tid; i < kLtTile / 16; i += kLtThreads) reinterpret_cast<uint4*>(smem + L::p)[i] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

#define LT_WAIT(bar, parity) \
    if (!mbar_wait_abortable(bar, (parity) & 1, abort_flag)) *abort_flag = 1;

    if (warp == 16) {
        // =========================== loads ===========================
        if (lane == 0) {
            int na = 0, nb = 0;
            for (int n = 0; n < n_chunks; ++n) {
                const int t0 = chunk_t0(n);
                for (int x = 0; x < G; ++x) {
                    const bool new_b = x == 0 || Gb > 1, new_a = !STATE_ONLY && (x == 0 || Ga > 1);
                    if (new_b) {
                        const int st = nb % L::kBc, use = nb / L::kBc, head = h * Gb + (Gb > 1 ? x : 0);
                        unsigned char* dst = smem + L::b + st * kLtTile;
                        if (use > 0) LT_WAIT(&empty_b[st], use - 1);
                        mbar_arrive_expect_tx(&full_b[st], kLtTile);
                        tma_load_4d(dst, map_b, 0, head, t0, bi, &full_b[st]);
                        tma_load_4d(dst + kLtHalf, map_b, 64, head, t0, bi, &full_b[st]);
                    }
                    if (new_a) {
                        const int st = na & 1, use = na >> 1, head = h * Ga + (Ga > 1 ? x : 0);
                        unsigned char* dst = smem + L::a + st * kLtTile;
                        if (use > 0) LT_WAIT(&empty_a[st], use - 1);
                        mbar_arrive_expect_tx(&full_a[st], kLtTile);
                        tma_load_4d(dst, map_a, 0, head, t0, bi, &full_a[st]);
                        tma_load_4d(dst + kLtHalf, map_a, 64, head, t0, bi, &full_a[st]);
                        ++na;
                    }
                    if (new_b) {
                        const int st = nb % L::kBc, use = nb / L::kBc, head = h * Gb + (Gb > 1 ? x : 0);
                        unsigned char* dst = smem + L::c + st * kLtTile;
                        if (use > 0) LT_WAIT(&empty_c[st], use - 1);
                        mbar_arrive_expect_tx(&full_c[st], kLtTile);
                        tma_load_4d(dst, map_c, 0, head, t0, bi, &full_c[st]);
                        tma_load_4d(dst + kLtHalf, map_c, 64, head, t0, bi, &full_c[st]);
                        ++nb;
                    }
                }
            }
        }
        __syncwarp();
    } else if (warp == 17) {
        // =========================== products ===========================
        if (lane == 0) {
            constexpr uint32_t id_kk = instr_desc_mn(128, 128, false, false);
            constexpr uint32_t id_nn = instr_desc_mn(128, 128, true, true);
            const DescKind dk(smem_desc(0, 16, 1024)), dmn(smem_desc(0, kLtHalf, 1024)),
                dslot(smem_desc(0, kLtStep * 128, 1024));
            const uint32_t a16 = desc_addr16(smem_u32(smem + L::a)), b16 = desc_addr16(smem_u32(smem + L::b)),
                           c16 = desc_addr16(smem_u32(smem + L::c)), p16 = desc_addr16(smem_u32(smem + L::p)),
                           s16 = desc_addr16(smem_u32(smem + L::slots));
            constexpr uint32_t t16 = kLtTile / 16, h16 = kLtHalf / 16;
            const int items = n_chunks * G;
            int ks = 0;   // slots used so far
            // W of item `it` = chunk n, head x
            auto w_products = [&](int it) {
                const int n = it / G, x = it - n * G;
                const int na = Ga > 1 ? it : n, nb = Gb > 1 ? it : n;
                LT_WAIT(&full_a[na & 1], na >> 1);
                LT_WAIT(&full_b[nb % L::kBc], nb / L::kBc);
                tc_fence_after();
                const uint32_t xa = a16 + (na & 1) * t16, ya = b16 + (nb % L::kBc) * t16;
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    const uint32_t o = (kk >> 2) * h16 + (kk & 3) * 2;
                    umma_bf16(tmem + kLtColW, dk.at(xa + o), dk.at(ya + o), id_kk, kk > 0);
                }
                umma_commit(w_full);
                if (Gb > 1 || x == G - 1) umma_commit(&empty_b[nb % L::kBc]);
            };
            if (!STATE_ONLY && items > 0) w_products(0);
            for (int it = 0; it < items; ++it) {
                const int n = it / G, x = it - n * G;
                const int na = Ga > 1 ? it : n, nb = Gb > 1 ? it : n;
                const bool new_b = x == 0 || Gb > 1, new_a = x == 0 || Ga > 1;
                const uint32_t ca = c16 + (nb % L::kBc) * t16;
                if (new_b) {   // the chunk's addition to the state
                    if (x == 0 && n > 0) LT_WAIT(d_empty, n - 1);
                    LT_WAIT(&full_c[nb % L::kBc], nb / L::kBc);
                    for (int st = 0; st < kLtCh / kLtStep; ++st, ++ks) {
                        const int sl = ks % kLtSlots;
                        LT_WAIT(&slot_full[sl], ks / kLtSlots);
                        tc_fence_after();
#pragma unroll
                        for (int t = 0; t < kLtTerms; ++t)
                            umma_bf16(tmem + kLtColD, dmn.at(ca + st * 128),
                                      dslot.at(s16 + (sl * kLtSlotBytes + t * kLtTermBytes) / 16), id_nn,
                                      t > 0 || st > 0 || x > 0);
                        umma_commit(&slot_empty[sl]);
                    }
                    if (Gb == 1 || x == G - 1) umma_commit(d_full);
                    if (STATE_ONLY) umma_commit(&empty_c[nb % L::kBc]);
                }
                if (STATE_ONLY) continue;
                if (new_a) {   // the state's share
                    if (x == 0) LT_WAIT(x_full, n);
                    if (na > 0) LT_WAIT(o_empty, na - 1);
                    tc_fence_after();
                    const uint32_t xa = a16 + (na & 1) * t16;
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        umma_bf16_ts(tmem + kLtColO, tmem + kLtColX + kk * 8, dk.at(xa + (kk >> 2) * h16 + (kk & 3) * 2),
                                     id_kk, kk > 0);
                    if (Gb > 1 || x == G - 1) umma_commit(x_empty);
                }
                LT_WAIT(p_full, it);
                tc_fence_after();
                // the next item's W before this one's last product, if its tiles are there
                bool next_done = it + 1 >= items;
                if (!next_done) {
                    const int it1 = it + 1, n1 = it1 / G;
                    const int na1 = Ga > 1 ? it1 : n1, nb1 = Gb > 1 ? it1 : n1;
                    if (mbar_try_wait(&full_a[na1 & 1], (na1 >> 1) & 1) &&
                        mbar_try_wait(&full_b[nb1 % L::kBc], (nb1 / L::kBc) & 1)) {
                        w_products(it1);
                        next_done = true;
                    }
                }
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {   // rows i of P that step kk of the tokens j reaches
                    const int i0 = reverse ? 0 : 16 * kk, ni = reverse ? 16 * (kk + 1) : 128 - 16 * kk;
                    const uint32_t id = instr_desc_mn(128, 0, true, false) | ((uint32_t)(ni >> 3) << 17);
                    umma_bf16(tmem + kLtColO + i0, dmn.at(ca + kk * 128),
                              dk.at(p16 + (kk >> 2) * h16 + (kk & 3) * 2 + i0 * 8), id, true);
                }
                umma_commit(p_empty);
                if (Ga > 1 || x == G - 1) umma_commit(o_full);
                if (Gb > 1 || x == G - 1) umma_commit(&empty_c[nb % L::kBc]);
                if (!next_done) w_products(it + 1);
            }
        }
        __syncwarp();
    } else if (warp == 18) {
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
    } else if (warp < 4) {
        // =========================== W -> P: one thread per row i ===========================
        if (!STATE_ONLY) {
            const int q = warp & 3, i = q * 32 + lane;
            const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16) + kLtColW;
            unsigned char* prow = smem + L::p + i * 128;
            const float* pti = pt + 127 - i;
            int it = 0;
            for (int n = 0; n < n_chunks; ++n) {
                const int nv = chunk_nv(chunk_t0(n));
                const float inv_f = fi[(nv < kLtCh ? 128 : 0) + i];
                for (int x = 0; x < G; ++x, ++it) {
                    LT_WAIT(w_full, it);
                    tc_fence_after();
                    bool waited = it == 0;
                    // blocks of 32 columns that the mask leaves something of
                    for (int cb = reverse ? q : 0; cb <= (reverse ? 3 : q); ++cb) {
                        float v[32];
                        tmem_ld32(lane_base + cb * 32, v);
                        uint32_t pk[16];
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const float w = pti[cb * 32 + j];
                            v[j] = w > 0.f ? v[j] * (w * inv_f) : 0.f;
                        }
                        if (nv < kLtCh) {   // products with padding rows, which hold anything
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = cb * 32 + j < nv ? v[j] : 0.f;
                        }
#pragma unroll
                        for (int j = 0; j < 16; ++j) pk[j] = Chunk<__nv_bfloat16>::pack2(v[2 * j], v[2 * j + 1]);
                        if (!waited) LT_WAIT(p_empty, it - 1);
                        waited = true;
                        unsigned char* dst = prow + (cb >> 1) * kLtHalf;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            *reinterpret_cast<uint4*>(dst + ((((cb & 1) * 4 + j) ^ (i & 7)) * 16)) =
                                make_uint4(pk[4 * j], pk[4 * j + 1], pk[4 * j + 2], pk[4 * j + 3]);
                    }
                    fence_proxy_async_smem();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full);
                }
            }
        }
    } else if (warp < 8) {
        // =========================== w o B in three terms, 16 rows at a time ===========================
        const int wt = tid - 128;
        const int row = wt >> 3, c8 = wt & 7;
        const int place = row * 128 + ((c8 ^ (row & 7)) * 16);
        int nb = 0, ks = 0;
        for (int n = 0; n < n_chunks; ++n) {
            const int nv = chunk_nv(chunk_t0(n));
            for (int x = 0; x < Gb; ++x, ++nb) {
                const int st = nb % L::kBc, use = nb / L::kBc;
                const unsigned char* bt = smem + L::b + st * kLtTile;
                LT_WAIT(&full_b[st], use);
                if (nv < kLtCh) {   // padding rows of C hold anything: zero, before the first product reads them
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
                for (int t = 0; t < kLtCh / kLtStep; ++t, ++ks) {
                    const int j = t * kLtStep + row;
                    const float w = wb[(nv < kLtCh ? 128 : 0) + j];
                    uint32_t o[2][kLtTerms][4];
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        const uint4 raw = *reinterpret_cast<const uint4*>(bt + hf * kLtHalf + t * kLtStep * 128 + place);
                        float v[8];
                        Chunk<__nv_bfloat16>::unpack(raw, v);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = j < nv ? v[e] * w : 0.f;
#pragma unroll
                        for (int tm = 0; tm < kLtTerms; ++tm) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const uint32_t pk = Chunk<__nv_bfloat16>::pack2(v[2 * e], v[2 * e + 1]);
                                o[hf][tm][e] = pk;
                                if (tm + 1 < kLtTerms) {   // what the term leaves out, exactly
                                    v[2 * e] -= __uint_as_float(pk << 16);
                                    v[2 * e + 1] -= __uint_as_float(pk & 0xffff0000u);
                                }
                            }
                        }
                    }
                    const int sl = ks % kLtSlots;
                    if (ks >= kLtSlots) LT_WAIT(&slot_empty[sl], ks / kLtSlots - 1);
                    unsigned char* dst = smem + L::slots + sl * kLtSlotBytes + place;
#pragma unroll
                    for (int tm = 0; tm < kLtTerms; ++tm)
#pragma unroll
                        for (int hf = 0; hf < 2; ++hf)
                            *reinterpret_cast<uint4*>(dst + tm * kLtTermBytes + hf * (kLtStep * 128)) =
                                make_uint4(o[hf][tm][0], o[hf][tm][1], o[hf][tm][2], o[hf][tm][3]);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(&slot_full[sl]);
                        if (t == kLtCh / kLtStep - 1) mbar_arrive(&empty_b[st]);
                    }
                }
            }
        }
    } else {
        // =========================== the state and the outputs ===========================
        const int q = warp & 3, hs = (warp - 8) >> 2;   // lanes 32q.., columns 64 hs..
        const int c = q * 32 + lane;                      // this thread's feature of c
        const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
        float S[64];                                      // [feature of b - 64 hs]
#pragma unroll
        for (int i = 0; i < 64; ++i) S[i] = 0.f;
        if (!STATE_ONLY) {
            const bool from_seg = s.nseg > 1;
            const float* src = from_seg ? r.seg + ((size_t)u * s.nseg + seg) * 16384
                                        : (r.state_in ? r.state_in + (size_t)u * 16384 : nullptr);
            const float mul = from_seg ? 1.f : r.in_mul;
            if (src != nullptr) {
                if (!r.state_t) {
#pragma unroll
                    for (int i = 0; i < 64; ++i) S[i] = mul * src[(hs * 64 + i) * 128 + c];
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float4 v = *reinterpret_cast<const float4*>(src + c * 128 + hs * 64 + 4 * i);
                        S[4 * i] = mul * v.x, S[4 * i + 1] = mul * v.y, S[4 * i + 2] = mul * v.z, S[4 * i + 3] = mul * v.w;
                    }
                }
            }
        }
        auto update = [&](int n) {   // after chunk n
            const float f = pw[chunk_nv(chunk_t0(n))];
            LT_WAIT(d_full, n);
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float d[16];
                tmem_ld16(lane_base + kLtColD + hs * 64 + k * 16, d);
#pragma unroll
                for (int i = 0; i < 16; ++i) S[k * 16 + i] = fmaf(f, S[k * 16 + i], d[i]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(d_empty);
        };
        const int c_place = (c >> 6) * kLtHalf + (c & 7) * 2, c16 = (c & 63) >> 3;
        int na = 0;
        for (int n = 0; n < n_chunks; ++n) {
            if (n > 0) update(n - 1);
            if (STATE_ONLY) continue;
            const int nv = chunk_nv(chunk_t0(n));
            if (n > 0) LT_WAIT(x_empty, n - 1);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uint32_t pk[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) pk[i] = Chunk<__nv_bfloat16>::pack2(S[k * 32 + 2 * i], S[k * 32 + 2 * i + 1]);
                tmem_st16(lane_base + kLtColX + hs * 32 + k * 16, pk);
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(x_full);
            for (int x = 0; x < Ga; ++x, ++na) {
                LT_WAIT(o_full, na);
                tc_fence_after();
                unsigned char* dst = smem + L::a + (na & 1) * kLtTile + c_place;
#pragma unroll 1
                for (int k = 0; k < 4; ++k) {   // 16 tokens of this feature
                    float o[16];
                    tmem_ld16(lane_base + kLtColO + hs * 64 + k * 16, o);
                    if (k == 3) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(o_empty);
                    }
                    const float4* fp = reinterpret_cast<const float4*>(fo + (nv < kLtCh ? 128 : 0) + hs * 64 + k * 16);
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) {
                        const float4 f = fp[i4];
                        const int t = hs * 64 + k * 16 + 4 * i4;
                        o[4 * i4] = t < nv ? o[4 * i4] * f.x : 0.f;
                        o[4 * i4 + 1] = t + 1 < nv ? o[4 * i4 + 1] * f.y : 0.f;
                        o[4 * i4 + 2] = t + 2 < nv ? o[4 * i4 + 2] * f.z : 0.f;
                        o[4 * i4 + 3] = t + 3 < nv ? o[4 * i4 + 3] * f.w : 0.f;
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        *reinterpret_cast<__nv_bfloat16*>(dst + (hs * 64 + k * 16 + i) * 128 + ((c16 ^ (i & 7)) * 16)) =
                            __float2bfloat16_rn(o[i]);
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&out_full[na & 1]);
            }
        }
        if (n_chunks > 0) update(n_chunks - 1);
        const float poison = *abort_flag ? __int_as_float(0x7fc00000) : 0.f;
        if (STATE_ONLY) {   // into the slot of the segment that it feeds, key's features in the rows
            float* dst = args.st.seg[which] + ((size_t)u * s.nseg + (reverse ? seg - 1 : seg + 1)) * 16384;
#pragma unroll
            for (int i = 0; i < 64; ++i) dst[(hs * 64 + i) * 128 + c] = S[i] + poison;
        } else if (r.state_out != nullptr && seg == (reverse ? 0 : s.nseg - 1)) {
            float* dst = r.state_out + (size_t)u * 16384;
#pragma unroll
            for (int i = 0; i < 64; ++i) dst[(hs * 64 + i) * 128 + c] = S[i] * r.out_mul + poison;   // (never transposed)
        }
    }
#undef LT_WAIT
    tc_fence_before();
    __syncthreads();
    if (warp == 17) {
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
