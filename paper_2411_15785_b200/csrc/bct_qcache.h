// The 8-bit cache with eviction by accumulated attention weight: what its API file and its kernels share.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "bct.h"

namespace bct {

constexpr int kQcBlock = BCT_QCACHE_BLOCK;   // slots that share a scale
constexpr int kQcScoredRows = 32;            // rows of a unit up to which the weights come from stored scores

// The caller's cache, resolved: planes by (sequence, kv-head) unit, state by sequence.
struct QcView {
    int8_t* codes[2];      // k, v   [B][Hkv][C][d]
    float* scale[2];       //        [B][Hkv][NB]
    float* weight;         //        [B][Hkv][C]
    int32_t* position;     //        [B][Hkv][C]
    int32_t* state;        // [3][B]: slots held, tokens seen, CTAs of an append that are done
    int B, Hkv, D, C, NB;
};

struct QcAppend {
    QcView c;
    const void* x[2];      // k, v   [B][T][Hkv][d]
    const int32_t* lens;   // or NULL
    int64_t T;
    int W;                 // blocks of a cache that T tokens touch at most
    int ctas;              // that share a unit's blocks (set by qc_append)
};
cudaError_t qc_append(const QcAppend& a, int dtype, cudaStream_t s);

// Scratch of an eviction: what the selection hands to the moves.
struct QcEvict {
    QcView c;
    int keep, recent;
    int max_moves, max_blocks;   // per unit
    int32_t* n_out;        // [units] slots evicted
    int32_t* n_blocks;     // [units] blocks with holes
    float* cut_scale;      // [units][2]: the scales of the block that the new end cuts, as they were
    int4* blocks;          // [units][max_blocks]: block, first hole's number, mask of holes
    int32_t* movers;       // [units][max_moves]: slots that move, ascending
};
cudaError_t qc_evict(const QcEvict& a, cudaStream_t s);

// Attention of T >= 1 tokens.  A unit's rows are its (token, head of the group) pairs, token-major: R = T G.
struct QcAttend {
    QcView c;
    const void* q;         // [B][T][Hq][d]
    void* out;
    const int32_t* lens;   // or NULL
    int64_t T;
    int G;
    int64_t R;             // rows of a unit
    int64_t n_groups;      // row groups of a unit
    float scale;           // of the scores
    float cap;             // > 0: scores are cap * tanh(score / cap)
    int accumulate;
    // scratch
    int n_warps;           // warps that share the blocks of all units
    float* part_o;         // [2 n_warps][rows of a group][d]: what a warp has of a unit that it shares with others
    float2* part_ml;       // [2 n_warps][rows of a group]: running maximum (in powers of two) and sum
    int2* spans;           // [units][row groups]: the first and last warp that have blocks of them
    float2* ml;            // [units][R]: maximum, 1 / sum
    float* scores;         // [units][R][Cs], powers of two; NULL where the weights are formed from the keys again
    int Cs;                // C, rounded up to whole blocks
};
// The tensor path's share of such a call (bct_qcache_prompt.cu).
struct QcPrompt {
    int tiles;             // of 256 rows, per unit
    int splits;            // CTAs that share the slots of a tile of rows
    int by_slots;          // one tile of 128 rows to a unit: a CTA's two sets of accumulators share its slots
    int parts;             // partial results of a row
    unsigned char* q_tiles;   // [units][2 tiles] of 128 rows: queries as operands; NULL without weights
    unsigned char* records;   // their rows' terms
};
// Which kernels serve a call, and its scratch: offsets into the caller's buffer, by the arguments alone.
struct QcPlan {
    bool prompt;           // the tensor path: bfloat16, more than kQcScoredRows rows
    QcPrompt pr;
    int rows;              // otherwise: rows of a group
    int tiles;             // of 8 rows each
    bool by_scores;        // the weights come from stored scores
    int n_warps;
    int64_t n_groups;
    size_t part_o, part_ml, spans, ml, scores, q_tiles, records, total;
};
cudaError_t qc_attend(const QcAttend& a, const QcPlan& p, int dtype, cudaStream_t s);
cudaError_t qc_prompt(const QcAttend& a, const QcPrompt& pr, cudaStream_t s);
int qc_attend_max_warps();

}  // namespace bct
