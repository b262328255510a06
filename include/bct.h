/*
 * bct.h: C ABI of the bounded-cache attention library for NVIDIA B200 (sm_100a).
 *
 * One attention layer of a Bounded-Cache Transformer keeps, per (sequence, kv-head)
 * "unit", a key vector sequence MK and a key-value vector sequence MV of a predefined
 * number of slots M (Method, "Model Structure"); here M is called `capacity` (C).
 * Per token, every query head of the unit reads the resident slots with softmax
 * attention, and the update rule of the paper then rewrites MV in place
 * (Method step 4, Algorithm 1, Illustration step 3):
 *
 *     read :  o_g  = softmax(read_scale  * q_g . MK^T) . MV_{t-1}       g = 0..G-1
 *     write:  MV_t = MV_{t-1} + softmax(write_scale * k_t . MK^T)^T . v_t
 *
 * q_g are the token's read queries (G = n_q_heads / n_kv_heads per unit), k_t is the
 * paper's write query wq_t and v_t its write key-value vector wv_t; the projections
 * that produce them (Algorithm 1, first two statements of the loop) are upstream of
 * this library.  MK is never assigned by Algorithm 1 and is frozen once resident.
 * While fewer than `capacity` slots are resident (a cache created with
 * init_len < capacity), a token's (k_t, v_t) is appended at slot `len`, the read covers
 * the len+1 resident slots, and no soft write happens.
 *
 * General conventions
 *  - Every pointer marked DEVICE is a device address on the current CUDA device,
 *    16-byte aligned, in memory the caller owns.  Pointers marked HOST are host
 *    addresses (pinned memory makes the copies asynchronous).
 *  - The library never allocates or frees device memory: all device storage is the
 *    caller's workspace given to bct_cache_create.
 *  - Every call validates its arguments on the host before enqueuing anything and
 *    returns a bct_status_t.  A call refused with BCT_ERR_INVALID_ARG, BCT_ERR_UNSUPPORTED
 *    or BCT_ERR_STATE has enqueued nothing and leaves the cache as it was.  BCT_ERR_CUDA
 *    means the CUDA runtime refused a launch or a copy: a call that covers several
 *    launches (bct_prefill_stream and the calls built on it split T tokens into chunk
 *    and single-token launches) may then have enqueued a prefix of its tokens; that
 *    prefix is applied in full, bct_cache_len and the token counters describe exactly
 *    the tokens enqueued, and the cache stays consistent and usable.
 *    bct_last_error() gives a thread-local message for the last failure.
 *  - Work is enqueued on the `cuda_stream` argument (a cudaStream_t passed as void*;
 *    NULL is the default stream) and the call returns without synchronising, except
 *    where stated.
 *  - A handle is not thread-safe; different handles are independent.  The library keeps a
 *    mutex-guarded list of its live handles, so that a handle passed in after
 *    bct_cache_destroy is answered with BCT_ERR_STATE without being dereferenced.
 *  - No environment variable is read.
 *  - `len` (resident slots) is the same for every sequence of the batch.
 */
#ifndef BCT_H_
#define BCT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum bct_status {
    BCT_OK = 0,
    BCT_ERR_INVALID_ARG = 1, /* NULL / misaligned pointer, out-of-range size */
    BCT_ERR_UNSUPPORTED = 2, /* a shape or flag the library has no kernel for */
    BCT_ERR_STATE = 3,       /* destroyed or corrupted handle */
    BCT_ERR_CUDA = 4,        /* a CUDA runtime call failed; see bct_last_error() */
    BCT_ERR_TIMEOUT = 5      /* a bounded device-side wait gave up (bct_cache_status) */
} bct_status_t;

typedef enum bct_dtype {
    BCT_F32 = 0, /* cache planes and step vectors in float */
    BCT_BF16 = 1 /* cache planes and step vectors in bfloat16, fp32 accumulation;
                    MV additionally carries a bfloat16 residual plane so that the
                    accumulated state keeps about 16 significand bits */
    ,
    BCT_BF16_PAIR = 2 /* checkpoint format of a bfloat16 cache's MV only (export / import):
                         one 32-bit word per element, value plane bits in the high half,
                         residual plane bits in the low half; lossless */
} bct_dtype_t;

/* flags */
#define BCT_FLAG_SKIP_FIRST_WRITE 1u /* Algorithm 1's literal "if t = 1": the first
                                        full-phase token leaves MV unchanged */
#define BCT_FLAG_WRITE_THEN_READ 2u  /* the token's read sees its own write */
#define BCT_FLAG_DENSE_WRITE 4u      /* rewrite every slot, whatever its write weight */
#define BCT_FLAG_PRECISE_READ 16u     /* bfloat16 cache: the read uses MV's value plus its
                                        residual (one more plane streamed per token; in the
                                        chunked stream kernel one more product per tile); for
                                        states whose magnitude makes a bfloat16 ulp matter */
#define BCT_FLAG_CUDA_CORES 32u       /* keep every decode step on the CUDA-core kernel (the
                                        tensor-core kernel serves bfloat16, head_dim 128,
                                        G <= 15, C >= 128 by default) */
#define BCT_FLAG_OUT_F32 8u          /* `out` is float (the fp32 accumulator, unrounded)
                                        whatever the cache dtype */

typedef struct bct_params {
    int32_t batch;      /* B  >= 1 sequences */
    int32_t n_q_heads;  /* Hq >= 1, a multiple of n_kv_heads; G = Hq / Hkv <= 8 on the CUDA-core
                           kernel, <= 15 on the tensor-core kernel */
    int32_t n_kv_heads; /* Hkv >= 1; one (MK, MV) memory per (sequence, kv-head) */
    int32_t head_dim;   /* d in {64, 128} */
    int32_t capacity;   /* C >= 1: the paper's predefined number of slots M */
    int32_t dtype;      /* bct_dtype_t */
    float read_scale;   /* <= 0 selects 1/sqrt(head_dim) */
    float write_scale;  /* <= 0 selects 1.0 (Algorithm 1 prints no scale) */
    int32_t init_len;   /* resident slots at create, 0..C; C is the paper's full-size MV_0 */
    uint32_t flags;     /* BCT_FLAG_* */
    float write_eps;    /* a slot whose write weight ww_j is below this is not rewritten
                           (its increment ww_j * v_t is dropped), in every entry point:
                           decode steps, stream chunks and bct_update_kv alike;
                           <= 0 selects 2^-24.  Ignored with BCT_FLAG_DENSE_WRITE.  With
                           BCT_FLAG_WRITE_THEN_READ the token's own read sees the slots
                           actually rewritten (the tensor-core decode kernel adds the
                           dropped slots' share as well: at most write_eps * |eta_t v_t|). */
    int32_t max_stream; /* largest T a later bct_prefill_stream_host call may pass;
                           sizes the staging area of the host-buffer entry points.
                           <= 0 selects 1. */
} bct_params_t;

typedef struct bct_cache bct_cache_t; /* opaque, host-side */

/* Library version as major*10000 + minor*100 + patch. */
int32_t bct_version(void);

/* Message of the calling thread's last failed call ("" if none).  Never NULL. */
const char *bct_last_error(void);

/*
 * Size and alignment of the device workspace a cache with these parameters needs
 * (Method, "Model Structure": MK and MV of M slots each, per unit; plus the bfloat16
 * residual plane, the status words, one progress word per (sequence, kv-head) unit and the staging
 * area of the *_host entry points).
 * The size depends on the parameters only and never grows afterwards, which is the
 * bounded-memory property of the method ("Fixed-Length Cache").
 */
bct_status_t bct_cache_bytes(const bct_params_t *params, size_t *bytes, size_t *align);

/*
 * Build a cache over caller-owned device memory and import its initial state.
 *   workspace  DEVICE, `bytes` >= bct_cache_bytes, aligned as bct_cache_bytes says;
 *              owned by the caller, must outlive the handle; the library writes to it.
 *   mk_init    DEVICE [B][Hkv][init_len][d] in `dtype`: the paper's MK (rows beyond
 *              init_len do not exist yet).  NULL allowed iff init_len == 0.
 *   mv_init    DEVICE, same shape: the paper's MV_0.  NULL with init_len > 0 means
 *              zeros (one of the two initialisations Method, "Model Structure" allows).
 * The import is enqueued on cuda_stream.  On success *out receives the handle.
 */
bct_status_t bct_cache_create(const bct_params_t *params, void *workspace, size_t bytes,
                              const void *mk_init, const void *mv_init, void *cuda_stream,
                              bct_cache_t **out);

/*
 * One token per sequence (Method steps 2-5 for the write, softmax attention for the read).
 *   q    DEVICE [B][Hq][d]   read queries; heads h*G .. h*G+G-1 belong to kv-head h
 *   k    DEVICE [B][Hkv][d]  write queries wq_t (appended as keys during the fill phase)
 *   v    DEVICE [B][Hkv][d]  write key-value vectors wv_t
 *   out  DEVICE [B][Hq][d]   attention outputs, written by the call
 * all contiguous, in the cache's dtype (out in float with BCT_FLAG_OUT_F32).  The cache advances by one token.
 */
bct_status_t bct_decode_step(bct_cache_t *cache, const void *q, const void *k, const void *v,
                             void *out, void *cuda_stream);

/*
 * T tokens per sequence, equivalent to T successive bct_decode_step calls within
 * rounding (Algorithm 1's loop over t = 1..N; with out == NULL it is UpdateKV itself,
 * which returns only the final MV_N).
 *   q    DEVICE [B][T][Hq][d]
 *   k,v  DEVICE [B][T][Hkv][d]
 *   out  DEVICE [B][T][Hq][d] or NULL
 * May be called repeatedly; successive calls concatenate.  T >= 1.  With out == NULL and a full cache
 * the call takes the write-only route of bct_update_kv (q is then not read).
 */
bct_status_t bct_prefill_stream(bct_cache_t *cache, const void *q, const void *k, const void *v,
                                void *out, int64_t T, void *cuda_stream);

/*
 * The two calls above with a step size for each token's write (Features, "Learning Rate
 * Adaptation": the step size is adjusted for each token; the paper prints no formula, so
 * the step size is an input and scales the increment of Method step 4):
 *     MV_t = MV_{t-1} + eta_t * ww_t^T . wv_t
 *   eta  DEVICE float [B][Hkv] (decode) / [B][T][Hkv] (stream), 4-byte aligned, read by
 *        the kernels of this call only; NULL means all ones, which is the call above.
 * Tokens of the fill phase are appended as they are and ignore eta; with
 * BCT_FLAG_WRITE_THEN_READ the token's own read sees the scaled write.  write_eps is
 * compared with ww_t, not with eta_t * ww_t.  Everything else as in the calls above.
 */
bct_status_t bct_decode_step_eta(bct_cache_t *cache, const void *q, const void *k, const void *v,
                                 const float *eta, void *out, void *cuda_stream);
bct_status_t bct_prefill_stream_eta(bct_cache_t *cache, const void *q, const void *k, const void *v,
                                    const float *eta, void *out, int64_t T, void *cuda_stream);

/*
 * Algorithm 1 itself, procedure UpdateKV: the write queries and write key-value vectors of T tokens
 * go into the state, MV_N = MV_0 + sum_t eta_t ww_t^T wv_t, and nothing is read.  The same state as
 * bct_prefill_stream_eta with out == NULL (within rounding), in chunks of up to 128 tokens whose
 * write weights are formed together (Key Implementation Aspects, "Optimized for Parallelism": MK is
 * never assigned, so the tokens' write weights do not depend on one another).
 *   wq   DEVICE [B][T][Hkv][d]  write queries     wv  DEVICE [B][T][Hkv][d]  write key-value vectors
 *   eta  DEVICE float [B][T][Hkv] or NULL (all ones)
 * Needs a full cache (the paper's full-size MV_0; BCT_ERR_STATE otherwise) of the shape the chunked
 * tensor-core kernel serves: bfloat16, head_dim 128, 128..16384 slots, no BCT_FLAG_SKIP_FIRST_WRITE
 * (BCT_ERR_UNSUPPORTED otherwise: use bct_prefill_stream with out == NULL).
 */
bct_status_t bct_update_kv(bct_cache_t *cache, const void *wq, const void *wv, const float *eta, int64_t T,
                           void *cuda_stream);

/*
 * Backward of bct_update_kv (Key Implementation Aspects, "Optimized for Parallelism": token-level
 * parallel training; Algorithm 1 as the forward).  For a scalar loss L and G = dL/dMV_N, with
 * ww_t = softmax(write_scale * wq_t . MK^T) of the cache's resident MK:
 *     r_t = sum_j ww_tj G_j      d_wv_t = eta_t r_t      d_eta_t = <wv_t, r_t>
 *     ds_tj = write_scale * ww_tj * (eta_t <wv_t, G_j> - eta_t d_eta_t)
 *     d_wq_t = sum_j ds_tj MK_j      d_mk_j = sum_t ds_tj wq_t      dL/dMV_0 = G (not written: it is d_mv)
 * Slots whose write weight is below write_eps are left out of r_t and of <wv_t, G_j>, as the forward
 * leaves their increments out.  The cache is read (MK only), not modified, and need not hold the MV_0
 * of the forward call: the state does not enter the gradients.
 *   wq, wv  DEVICE bfloat16 [B][T][Hkv][d]   the forward call's inputs
 *   eta     DEVICE float [B][T][Hkv] or NULL (all ones)
 *   d_mv    DEVICE bfloat16 [B][Hkv][C][d]   G
 *   d_wq, d_wv  DEVICE float [B][T][Hkv][d], written
 *   d_mk    DEVICE float [B][Hkv][C][d], written (zeroed, then summed with atomic adds: the order of the
 *           additions, hence the last bits, may differ from run to run when T > 128), or NULL
 *   d_eta   DEVICE float [B][T][Hkv], written, or NULL
 * bfloat16 operands, fp32 accumulation.  Needs a full cache of the shape the chunked kernels serve
 * (bfloat16, head_dim 128, 128..16384 slots): BCT_ERR_STATE / BCT_ERR_UNSUPPORTED otherwise.
 */
bct_status_t bct_update_kv_backward(bct_cache_t *cache, const void *wq, const void *wv, const float *eta,
                                    const void *d_mv, int64_t T, float *d_wq, float *d_wv, float *d_mk,
                                    float *d_eta, void *cuda_stream);

/*
 * The projections in front of the layer (Algorithm 1, first two statements of the loop body:
 * wq_t = W_wq x_t and wv_t = W_wv x_t; the read query q_t = W_q x_t of the attention layer
 * likewise), for a block of tokens, as one tensor-core contraction:
 *     q = x W_q^T   [n_tokens][n_q]      k = x W_wq^T, v = x W_wv^T   [n_tokens][n_kv]
 *   x      DEVICE bfloat16 [n_tokens][d_model]      one row per token (tokens of all sequences, [B][T] order)
 *   w_q    DEVICE bfloat16 [n_q][d_model]           one row per output feature, n_q = Hq * head_dim
 *   w_wq   DEVICE bfloat16 [n_kv][d_model]          n_kv = Hkv * head_dim
 *   w_wv   DEVICE bfloat16 [n_kv][d_model]
 *   q,k,v  DEVICE bfloat16, written by the call: exactly the step arrays bct_prefill_stream reads
 * fp32 accumulation, one rounding to bfloat16.  d_model a multiple of 8, n_q and n_kv multiples of 32,
 * every pointer 16-byte aligned; sm_100 devices only (BCT_ERR_UNSUPPORTED elsewhere).  Asynchronous on
 * cuda_stream; allocates nothing.
 */
bct_status_t bct_project_qkv(int64_t n_tokens, int32_t d_model, int32_t n_q, int32_t n_kv, const void *x,
                             const void *w_q, const void *w_wq, const void *w_wv, void *q, void *k, void *v,
                             void *cuda_stream);

/*
 * One layer call on the tokens themselves: the projections above, then bct_prefill_stream_eta on
 * their results (Algorithm 1's loop body from x_t to MV_t, plus the read).  bfloat16 caches only.
 *   x        DEVICE bfloat16 [B][T][d_model]
 *   eta      DEVICE float [B][T][Hkv] or NULL (all ones)
 *   scratch  DEVICE, 256-byte aligned, at least bct_layer_scratch_bytes(cache, T) bytes: holds q, k, v
 *            between the two steps; owned by the caller, free for reuse once the stream has passed the call
 *   out      DEVICE [B][T][Hq][d] or NULL
 */
bct_status_t bct_layer_scratch_bytes(const bct_cache_t *cache, int64_t T, size_t *bytes);
bct_status_t bct_layer_forward(bct_cache_t *cache, const void *x, const void *w_q, const void *w_wq,
                               const void *w_wv, int32_t d_model, const float *eta, void *scratch,
                               size_t scratch_bytes, void *out, int64_t T, void *cuda_stream);

/*
 * A stack of layers (Method, "Model Structure": the mechanism sits in every attention layer of the
 * decoder): layer 0 reads x, layer l > 0 reads the outputs of layer l - 1 taken as its tokens,
 * [B][T][Hq * d] of layer l - 1 = [B][T][d_model] of layer l; each layer is one bct_layer_forward on its own
 * cache.  No residual path, normalisation or feed-forward block is applied between the layers: those are
 * outside this library.
 *   caches   HOST array of n_layers handles (bfloat16, the same batch, without BCT_FLAG_OUT_F32)
 *   w_q, w_wq, w_wv   HOST arrays of n_layers DEVICE pointers: layer l's weights, [Hq_l * d][d_model_l] etc.,
 *            d_model_0 = d_model, d_model_l = Hq_(l-1) * head_dim
 *   scratch  DEVICE, 256-byte aligned, at least bct_stack_scratch_bytes bytes
 *   out      DEVICE [B][T][Hq][d] of the last layer
 * BCT_ERR_CUDA after the first layers have been enqueued leaves those layers' caches advanced by T tokens.
 */
bct_status_t bct_stack_scratch_bytes(bct_cache_t *const *caches, int32_t n_layers, int64_t T, size_t *bytes);
bct_status_t bct_stack_forward(bct_cache_t *const *caches, int32_t n_layers, const void *x, int32_t d_model,
                               const void *const *w_q, const void *const *w_wq, const void *const *w_wv,
                               void *scratch, size_t scratch_bytes, void *out, int64_t T, void *cuda_stream);

/*
 * Linear attention with a decay for each head: the update rule of the bounded cache with the key itself as the
 * address.  Where UpdateKV adds softmax(wq_t . MK^T)^T . wv_t to a state of C slots, here a state of head_dim
 * rows takes k_t^T . v_t and forgets at a rate of its own:
 *     S_t = exp(log_decay[h]) * S_(t-1) + k_t^T v_t        o_g = scale * q_g . S_t      (the token sees its own write)
 * per (sequence, kv-head), G = n_q_heads / n_kv_heads query heads reading each state.  The calls keep no handle:
 * the state is the caller's, DEVICE float [B][Hkv][d][d], the key's features in its rows, the value's in its
 * columns.
 *   log_decay  DEVICE float [Hkv], 4-byte aligned: the logarithm of the decay, <= 0; 0 never forgets, minus infinity
 *              keeps only the token itself.  A constant of the head: the backward forms no gradient for it.
 * Roundings.  BCT_F32, and the step in either type: fp32 throughout, one rounding to `dtype`.  Prompts and their
 * backward in BCT_BF16 run on the tensor cores: the products of pairs (q_t . k_s and their like, weighted with the
 * decay) and the state where it enters a product are each rounded to bfloat16 once, sums are fp32, and `out` and the
 * gradients are rounded once; the float states (state_out, d_state_in) are fp32 sums of unrounded products, off by less
 * than 1e-6 of them (root mean square) for every decay and length.
 * Range.  BCT_F32 and the step have fp32's.  Prompts and their backward in BCT_BF16 carry the results of a token, until
 * the last product, as multiples of exp(log_decay)^n or 2^-64, whichever is larger, n <= 128 being the token's distance
 * from the end of the chunk before it (in reverse, from the start of the one behind it).  Under a strong decay the
 * products of pairs and the results without `scale` therefore have to stay below 2^63, 9e18 (beyond, infinities), and a
 * state whose share has decayed below 2^-64 is still seen with 2^-64.  d_state / scale has to be in fp32's range.
 * No atomics: the same call gives the same bits.  A NaN or an infinity in a token that counts may also reach the
 * results of up to 127 tokens before it (of those after it, in the backward), as 0 * infinity; one in a padding row
 * reaches nothing.
 * No output may overlap an input or another output, except where stated (BCT_ERR_INVALID_ARG).
 */
typedef struct bct_linear_params {
    int32_t batch;      /* B  >= 1 sequences */
    int32_t n_q_heads;  /* Hq in 1..65536, a multiple of n_kv_heads */
    int32_t n_kv_heads; /* Hkv >= 1, B * Hkv <= 2^20 */
    int32_t head_dim;   /* d in {64, 128}, of keys and values alike */
    int32_t dtype;      /* BCT_F32 or BCT_BF16: q, k, v, out and their gradients; states are float */
    float scale;        /* <= 0 selects 1/sqrt(head_dim) */
} bct_linear_params_t;

/* Bytes of scratch that bct_linear_forward (backward = 0), bct_linear_backward (backward = 1) or the latter with
 * d_state_in NULL (backward = 2) needs for T tokens: long calls of few heads are split over the tokens, and the states
 * between the parts live there, with 1, G > 1 and BCT_BF16 also what each query head adds to d_state_in.  0 for many
 * calls.  Depends on the arguments only. */
bct_status_t bct_linear_scratch_bytes(const bct_linear_params_t *params, int64_t T, int32_t backward, size_t *bytes);

/*
 * One token per sequence.
 *   q, out  DEVICE [B][Hq][d]     k, v  DEVICE [B][Hkv][d]
 *   state, state_out   the state before and after; state_out may be `state` itself (exactly) or a buffer of its own
 */
bct_status_t bct_linear_step(const bct_linear_params_t *params, const void *q, const void *k, const void *v,
                             const float *log_decay, const float *state, float *state_out, void *out,
                             void *cuda_stream);

/*
 * T tokens per sequence, equal to T bct_linear_step calls within rounding, in chunks whose products are formed
 * together.
 *   q, out     DEVICE [B][T][Hq][d]      k, v  DEVICE [B][T][Hkv][d]
 *   lens       DEVICE int32 [B] or NULL (all T): tokens of each sequence, 0..T (clamped); the rows behind them are
 *              padding, which is not read into any result, and `out` is zero there
 *   state      the state before the first token, or NULL (zeros)
 *   state_out  the state after each sequence's last token, or NULL; may be `state` itself (exactly)
 *   scratch    DEVICE, 256-byte aligned, bct_linear_scratch_bytes(params, T, 0); NULL where that is 0.  In use until
 *              the stream has passed the call: calls that may overlap need a scratch each
 */
bct_status_t bct_linear_forward(const bct_linear_params_t *params, int64_t T, const void *q, const void *k,
                                const void *v, const float *log_decay, const int32_t *lens, const float *state,
                                float *state_out, void *out, void *scratch, size_t scratch_bytes, void *cuda_stream);

/*
 * Backward of bct_linear_forward, from its inputs alone.  With do_t = dL/do_t (summing over the G heads of a group):
 *     d_q_t = scale * S_t do_t                          S_t forward in time, from `state`
 *     d_k_t = R_t v_t,  d_v_t = R_t^T k_t               R_t = exp(log_decay) R_(t+1) + scale * q_t^T do_t
 *     d_state_in = exp(log_decay) * R_1
 * where R_(len) + .. starts from d_state, the gradient of the state after the last token.
 *   d_out      DEVICE [B][T][Hq][d]      q, k, v, lens, state   the forward call's (state NULL: zeros)
 *   d_state    DEVICE float [B][Hkv][d][d], or NULL (zeros)
 *   d_q        DEVICE [B][T][Hq][d]      d_k, d_v  DEVICE [B][T][Hkv][d], in `dtype`; zero in padding rows
 *   d_state_in DEVICE float [B][Hkv][d][d], or NULL: with G > 1 in BCT_BF16 it costs a pass of its own over q and d_out
 *   scratch    as above, bct_linear_scratch_bytes(params, T, 1), or (params, T, 2) where d_state_in is NULL
 */
bct_status_t bct_linear_backward(const bct_linear_params_t *params, int64_t T, const void *d_out, const void *q,
                                 const void *k, const void *v, const float *log_decay, const int32_t *lens,
                                 const float *state, const float *d_state, void *d_q, void *d_k, void *d_v,
                                 float *d_state_in, void *scratch, size_t scratch_bytes, void *cuda_stream);

/*
 * Norms of queries and keys for each head, and the rotation by the token's position in the same pass: what stands
 * between bct_project_qkv and an attention step that knows positions.  For every head vector x of q and k
 *     y = x / sqrt(mean(x^2) + eps) * w        out = y with its first rot_dim features turned in pairs:
 *     (y_a, y_b) -> (y_a cos p f - y_b sin p f, y_a sin p f + y_b cos p f),   p the token's position, f = freq[i]
 * with the pairs (i, i + rot_dim/2), or (2i, 2i + 1) with BCT_ROTATE_INTERLEAVED, i < rot_dim/2.
 *   q, q_out   DEVICE [n_tokens][Hq][d]       k, k_out  DEVICE [n_tokens][Hkv][d], in `dtype`; q_out may be q itself
 *              and k_out k itself (exactly), any other overlap is refused
 *   w_q, w_k   DEVICE [d] in `dtype`, or NULL (ones)
 *   positions  DEVICE int64 [n_tokens]        freq  DEVICE double [rot_dim/2], radians per position; the angle is
 *              formed in double.  Both may be NULL with rot_dim = 0 (norm only)
 *   rot_dim    0..head_dim, a multiple of 16 (BCT_ERR_UNSUPPORTED otherwise);  head_dim in {64, 128}
 *   eps        >= 0.  mean(x^2) is formed in fp32, so |x| has to stay below 1e18, and above 1e-18 where eps is 0; a
 *              vector of zeros with eps = 0 is 0 / 0
 */
#define BCT_ROTATE_INTERLEAVED 1u
bct_status_t bct_norm_rotate(int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                             const void *q, const void *k, const void *w_q, const void *w_k, float eps,
                             const int64_t *positions, const double *freq, int32_t rot_dim, uint32_t flags, void *q_out,
                             void *k_out, void *cuda_stream);

/*
 * Backward of bct_norm_rotate: d_q, d_k (in `dtype`; d_q may be d_q_out itself and d_k d_k_out itself) and the weights'
 * gradients d_w_q, d_w_k (DEVICE float [d], summed over tokens and heads in a fixed order), each of which may be NULL.
 *   q, k      the forward call's inputs, before the norm
 *   scratch   DEVICE, 256-byte aligned, bct_norm_rotate_scratch_bytes bytes: the blocks' shares of d_w; not used, and may
 *             be NULL, when both d_w_q and d_w_k are NULL.  Calls that may overlap need a scratch each
 */
bct_status_t bct_norm_rotate_scratch_bytes(int64_t n_tokens, int32_t head_dim, size_t *bytes);
bct_status_t bct_norm_rotate_backward(int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                      int32_t dtype, const void *d_q_out, const void *d_k_out, const void *q,
                                      const void *k, const void *w_q, const void *w_k, float eps,
                                      const int64_t *positions, const double *freq, int32_t rot_dim, uint32_t flags,
                                      void *d_q, void *d_k, float *d_w_q, float *d_w_k, void *scratch,
                                      size_t scratch_bytes, void *cuda_stream);

/*
 * A cache of predefined capacity held in 8 bits, which throws out the slots that attention has used least: the other way
 * to keep a bounded cache than the update rule above, which rewrites its values.  The calls keep no handle: the cache is
 * the caller's memory, described by a struct of sizes and DEVICE pointers (16-byte aligned, contiguous, no two
 * overlapping).  A zeroed `state` is an empty cache; the other planes need no initial values.
 *
 * Codes.  The key of slot j is k[j] * k_scale[j / 32], its value v[j] * v_scale[j / 32] (fp32).  A block of 32 slots that holds
 * nothing takes the scale amax / 127 (rounded to fp32; at least 2^-126) of what is written into it, amax being its largest
 * magnitude.  A block that holds something keeps its scale s while amax <= 127.5 s; otherwise s is multiplied by the
 * smallest power of two with which that holds, and the codes it keeps are divided by it.  Codes are rounded to the nearest,
 * ties to the even one, and limited to -127..127.  So a value is off by half a step when it is written, and by less than
 * one step of its block's scale at any time (a slot that an eviction moves is rounded once more, as a new one).  A NaN or an
 * infinity makes its block's scale a NaN, and every output that sees the block, until the block is written anew; in a key, also
 * the weights that the rows which see it give.
 */
#define BCT_QCACHE_BLOCK 32
typedef struct bct_qcache {
    int32_t batch;      /* B  >= 1 sequences */
    int32_t n_kv_heads; /* Hkv >= 1, B * Hkv <= 2^20 */
    int32_t head_dim;   /* d in {64, 128} */
    int32_t capacity;   /* C in 1..2^24 slots */
    int8_t *k, *v;      /* [B][Hkv][C][d] */
    float *k_scale, *v_scale; /* [B][Hkv][ceil(C / 32)] */
    float *weight;      /* [B][Hkv][C]: what attention has given the slot so far */
    int32_t *position;  /* [B][Hkv][C]: the number of the slot's token in its sequence, from 0 */
    int32_t *state;     /* [3][B]: slots held (0..C, of every head of the sequence alike), tokens seen (below 2^31), a word
                           of the library's own that is zero between calls */
} bct_qcache_t;

/*
 * Append T tokens per sequence behind the slots held, with weight 0 and the positions that follow the tokens seen.
 *   k, v   DEVICE [B][T][Hkv][d] in `dtype` (BCT_F32 or BCT_BF16)
 *   lens   DEVICE int32 [B] or NULL (all T): valid tokens of each sequence, 0..T (clamped); the others are padding, which
 *          is not read
 * Tokens that find no slot free are dropped, and neither held nor seen: make room first (bct_qcache_evict).
 */
bct_status_t bct_qcache_append(const bct_qcache_t *cache, int64_t T, int32_t dtype, const void *k, const void *v,
                               const int32_t *lens, void *cuda_stream);

/*
 * Softmax attention of the last T tokens appended to each sequence over what its cache holds: token i of n sees the first
 * held - n + i + 1 slots (so the call goes behind the append of these tokens, before an eviction moves slots).
 *     s = scale q . k_j        p = softmax_j(s), or softmax_j(cap tanh(s / cap)) with cap = score_cap > 0
 *     out = sum_j p_j v_j      weight_j += p_j, summed over the tokens and the query heads, if `accumulate`
 *   q, out  DEVICE [B][T][Hq][d] in `dtype`; heads h*G .. h*G+G-1 read kv-head h, G = Hq / Hkv; Hq in 1..65536
 *   lens    as above: n of each sequence.  Rows behind them are not read, add nothing, and their `out` is zero; so is that of
 *           a row that sees no slot
 * A NaN in a query makes its row's `out` NaN and, as p_j is, with `accumulate` the weight of every slot that the row sees, which then
 * counts as more than any number (below); an infinity may.  Other rows, and slots that only others see, are as without it.
 *   scale   <= 0 selects 1/sqrt(head_dim).  scale log2(e), score_cap log2(e) and scale / score_cap are within fp32's range
 *   scratch DEVICE, 256-byte aligned, bct_qcache_attend_scratch_bytes bytes.  In use until the stream has passed the call:
 *           calls that may overlap need a scratch each
 * Roundings.  fp32 sums and softmax.  BCT_BF16: exact products of queries and codes, probabilities rounded to 11 bits where
 * they multiply values, one rounding of `out`.  BCT_F32: queries and probabilities rounded to 22 bits or more.  In any case a
 * term p_j v_j is off by up to 2^-39 of v_j, p_j = 1 being the row's largest.  BCT_BF16 calls with T * G > 32 multiply p_j by ratios
 * of v_scales, in fp32 powers of two (2^-19 of p_j; 2^-17 where a ratio is below 2^-21): there a term is off by up to 2^-31 of 127 s,
 * s the largest v_scale of the 128 slots (from a multiple of 128 on) that j is among, seen by the row or not, or, if that is more,
 * by 2^-92 of 127 times the largest v_scale in front of them.  The weights are fp32 sums.  No atomics: the same call gives the
 * same bits.
 * Range.  `out` is that precise while the blocks' largest values are 0 or at least 2^-90, and at most 2^112 divided by the number of
 * slots seen (the sums hold 2^15 times the probabilities); scores, in powers of two, have to be within fp32's range.
 */
bct_status_t bct_qcache_attend_scratch_bytes(const bct_qcache_t *cache, int64_t T, int32_t n_q_heads, int32_t dtype,
                                             int32_t accumulate, size_t *bytes);
bct_status_t bct_qcache_attend(const bct_qcache_t *cache, int64_t T, int32_t n_q_heads, int32_t dtype, const void *q,
                               const int32_t *lens, float scale, float score_cap, int32_t accumulate, void *out,
                               void *scratch, size_t scratch_bytes, void *cuda_stream);

/*
 * Evict from every cache that holds more than `keep` slots all but `keep`, head by head: those of the least weight go, of
 * equal weights the lower slots first, but none of the last `recent` tokens (position >= tokens seen - recent).  The slots
 * that stay behind the new end move, in their order, into the places before it that have become free, in theirs; no other
 * slot moves.  A NaN counts as more weight than any number.
 *   keep    0..capacity          recent  0..keep
 *   scratch DEVICE, 256-byte aligned, bct_qcache_evict_scratch_bytes bytes (0, and NULL, with keep = capacity); as above
 */
bct_status_t bct_qcache_evict_scratch_bytes(const bct_qcache_t *cache, int32_t keep, size_t *bytes);
bct_status_t bct_qcache_evict(const bct_qcache_t *cache, int32_t keep, int32_t recent, void *scratch, size_t scratch_bytes,
                              void *cuda_stream);

/*
 * Host-buffer forms of bct_decode_step and bct_prefill_stream: the same shapes, but q, k, v and out are
 * HOST pointers.  The inputs are copied into the workspace's staging area (two sets, used
 * alternately, on a copy stream the handle owns, so that one call's copies overlap the
 * previous call's kernel), the step runs on cuda_stream after them, and out is copied back
 * on cuda_stream; the call returns without synchronising, so out is valid once cuda_stream
 * has drained, and q, k, v must stay unchanged until then.  T must not exceed the
 * max_stream given at create.
 */
bct_status_t bct_decode_step_host(bct_cache_t *cache, const void *q, const void *k, const void *v,
                                  void *out, void *cuda_stream);
bct_status_t bct_prefill_stream_host(bct_cache_t *cache, const void *q, const void *k,
                                     const void *v, void *out, int64_t T, void *cuda_stream);

/*
 * bct_prefill_stream_host for callers that cannot allocate device memory.  (The paper has
 * no counterpart: this is plumbing of this library, not a step of the method.)
 *
 * bct_prefill_stream_host stages q, k, v and out in the workspace, in an area whose size the
 * caller fixed with max_stream before allocating the workspace.  Some callers can never
 * enlarge it afterwards because they cannot call cudaMalloc at all: code that runs inside a
 * memory pool frozen at start-up (a latency-bound serving loop), a plug-in that owns only
 * the arena its host application handed it, a process whose other libraries have taken the
 * rest of the device.  This call uses a staging area built into the library instead: one
 * file-scope device array of BCT_STATIC_STAGE_BYTES that every GPU holds from the moment
 * the library is loaded until the process exits.  It allocates and frees nothing.
 *
 *   q, k, v, out  HOST pointers, shapes and meaning as in bct_prefill_stream_host;
 *                 out must not be NULL.
 *   T             tokens per sequence; the rounded-up sizes of q, k, v and out for T tokens
 *                 must fit BCT_STATIC_STAGE_BYTES together, else BCT_ERR_INVALID_ARG and
 *                 nothing is enqueued (bct_last_error() gives the sizes).  max_stream does
 *                 not limit T here.
 * The cache's device must be the current device.  The first call on each device looks up
 * the array's device address (cudaGetSymbolAddress); make that first call outside any
 * stream capture.  The array is shared by every cache and every call on that device and
 * keeps the previous call's bytes; this call overwrites every byte it later reads, so
 * nothing has to be cleared, but two calls whose work overlaps on the GPU (different
 * streams without ordering, or different threads) race on it: order them on one stream.
 * Results are those of bct_prefill_stream_host.
 */
#define BCT_STATIC_STAGE_BYTES (8u << 20)
bct_status_t bct_prefill_stream_host_static(bct_cache_t *cache, const void *q, const void *k,
                                            const void *v, void *out, int64_t T,
                                            void *cuda_stream);

/* Resident slots (0..C) after the work enqueued so far. Host bookkeeping; no sync. */
bct_status_t bct_cache_len(const bct_cache_t *cache, int32_t *len);

/*
 * Copy the state out in the canonical layout (Method step 5, the store of the updated
 * sequence, made visible): k_out DEVICE [B][Hkv][C][d] in the cache dtype, v_out DEVICE
 * [B][Hkv][C][d] in v_dtype (BCT_F32 gives the bfloat16 value plus its residual,
 * exactly; BCT_BF16 the rounded value; BCT_BF16_PAIR both planes bit for bit).  Rows
 * >= len are written as zeros.  Either pointer may be NULL to skip that plane.
 */
bct_status_t bct_cache_export(bct_cache_t *cache, void *k_out, void *v_out, int32_t v_dtype,
                              void *cuda_stream);

/*
 * Replace the state: k_in DEVICE [B][Hkv][len][d] in the cache dtype, v_in DEVICE
 * [B][Hkv][len][d] in v_dtype (NULL = zeros), 0 <= len <= C.  Counters of tokens seen
 * are kept.  export followed by import into a fresh cache resumes bit-exactly with
 * v_dtype BCT_BF16_PAIR (bfloat16 cache) or BCT_F32 (float cache); a bfloat16 cache
 * re-imported from BCT_F32 holds the same values but may split a few of them
 * differently between the value and residual planes.
 */
bct_status_t bct_cache_import(bct_cache_t *cache, const void *k_in, const void *v_in,
                              int32_t v_dtype, int32_t len, void *cuda_stream);

/*
 * Synchronise cuda_stream and report the device-side status word: BCT_OK, or
 * BCT_ERR_TIMEOUT if a bounded wait inside a kernel gave up (the affected step's
 * results are then undefined; the context stays usable).  The only call that blocks.
 */
bct_status_t bct_cache_status(bct_cache_t *cache, void *cuda_stream);

/* Set the device-side status word back to BCT_OK (enqueued on cuda_stream, no synchronisation):
 * after a reported BCT_ERR_TIMEOUT the cache can be re-imported and used again. */
bct_status_t bct_cache_status_clear(bct_cache_t *cache, void *cuda_stream);

/*
 * Rows of MV that the kernels of this cache have stored back so far (Method step 5: the store of the
 * updated sequence): decode steps count the slots whose write weight reached write_eps (every slot
 * with BCT_FLAG_DENSE_WRITE), the chunked stream kernel rebuilds whole tiles and counts every slot
 * of every chunk; appended fill-phase slots are not counted.  Synchronises cuda_stream like
 * bct_cache_status.  The fraction w = rows / (units * full-phase tokens * capacity) is the share of
 * MV the update rule rewrites per token, the term w*C*d*s of the bytes a decode step must move.
 *   rows  HOST, receives the count (64 bits).
 */
bct_status_t bct_cache_rows_rewritten(bct_cache_t *cache, void *cuda_stream, uint64_t *rows);

/*
 * Self-test of the bounded device-side waits (no step of the method): launches one thread block on
 * cuda_stream that waits, with a limit of about a thousand polls, on a barrier in its shared memory
 * that nothing ever arrives on; the wait gives up, the block records BCT_ERR_TIMEOUT with site code
 * 99 in the cache's status word and returns normally.  Nothing faults, hangs or traps, and the cache's
 * planes are not touched.  bct_cache_status then reports BCT_ERR_TIMEOUT until
 * bct_cache_status_clear.  Asynchronous.
 */
bct_status_t bct_selftest_timeout(bct_cache_t *cache, void *cuda_stream);

/* *yes = 1 if this cache's decode steps run on the tensor-core kernel (tcgen05 + TMA tensor
 * copies: bfloat16, head_dim 128, G <= 15, 128 <= C <= 65536, no PRECISE_READ / CUDA_CORES
 * flag), 0 if on the CUDA-core kernel.  Both compute the same step (Algorithm 1 + read). */
bct_status_t bct_cache_tensor_path(const bct_cache_t *cache, int32_t *yes);

/* Number of kernels this handle has launched so far (host counter). */
bct_status_t bct_cache_launches(const bct_cache_t *cache, int64_t *launches);

/* Free the host-side handle (NULL is accepted).  Never touches the workspace, never
 * synchronises: the caller drains the stream before reusing the workspace. */
bct_status_t bct_cache_destroy(bct_cache_t *cache);

#ifdef __cplusplus
}
#endif
#endif /* BCT_H_ */
