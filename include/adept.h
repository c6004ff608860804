/*
 * adept.h -- C ABI of the GB300 (sm_103a) library for ADEPT's token-level
 * early-exit forward pass (arXiv 2601.03700).
 *
 * Notation follows the paper's problem statement (Sec. 3): N layers, indexed
 * i = 1..N (1-based everywhere in this API), tokens j, hidden size D_h
 * (d_model), query/key/value size D_q (heads x head_dim), exit layer i*.
 *
 * Conventions shared by every call:
 *  - Pointers prefixed d_ are DEVICE pointers owned by the caller; they must stay
 *    valid until the work queued on `stream` has finished.  Pointers prefixed
 *    h_ are host pointers read before the call returns.
 *  - `stream` is a cudaStream_t (NULL = legacy default stream).  Every call that
 *    takes a stream only enqueues work on it and returns; results are valid once
 *    the stream has been synchronised.
 *  - The library owns its copy of the weights, the paged KV cache and its
 *    workspaces (allocated by adept_model_load, released by adept_free).
 *  - Errors are returned as adept_status; nothing is thrown across the ABI.
 *    Argument errors are detected on the host before anything is enqueued.
 *    Device-side input errors (a forced exit layer or token id out of range)
 *    set a device error word that adept_check_device_status reports.
 *    adept_last_error returns a message for the last failing call.
 *  - A model is not thread-safe: calls on one model must be serialised.
 */
#ifndef ADEPT_H
#define ADEPT_H

#include <stdint.h>

#if defined(__GNUC__)
#define ADEPT_API __attribute__((visibility("default")))
#else
#define ADEPT_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  ADEPT_OK = 0,
  ADEPT_ERR_INVALID_ARG = 1,   /* bad argument; nothing was enqueued */
  ADEPT_ERR_OOM = 2,           /* device allocation failed */
  ADEPT_ERR_CAPACITY = 3,      /* batch / sequence / KV-block capacity exceeded */
  ADEPT_ERR_CUDA = 4,          /* a CUDA runtime or driver call failed */
  ADEPT_ERR_TIMEOUT = 5,       /* a bounded device-side wait gave up */
  ADEPT_ERR_DEVICE_INPUT = 6   /* device-side validation of an input failed */
} adept_status;

enum { ADEPT_FAMILY_LLAMA = 0,   /* RMSNorm pre-norm, RoPE, SwiGLU, untied head */
       ADEPT_FAMILY_GPT2 = 1,    /* LayerNorm pre-norm, learned positions, tanh-GELU, biases, tied head */
       ADEPT_FAMILY_BERT = 2 };  /* post-LN encoder, bidirectional, pooler + classifier */

enum { ADEPT_DTYPE_F32 = 0, ADEPT_DTYPE_BF16 = 1 };
enum { ADEPT_KV_F32 = 0, ADEPT_KV_BF16 = 1, ADEPT_KV_E4M3 = 2 };   /* element types of a K/V cache (adept_kv_cache) */

typedef struct {
  int family;          /* ADEPT_FAMILY_* */
  int n_layers;        /* N */
  int d_model;         /* D_h */
  int n_heads;
  int n_kv_heads;      /* 0 -> n_heads */
  int head_dim;        /* D_q = n_heads * head_dim; must be even, <= 128 */
  int d_ffn;
  int vocab;
  int max_pos;         /* learned-position table size (GPT-2 / BERT) */
  int n_classes;       /* encoder classifier outputs */
  int dtype;           /* ADEPT_DTYPE_*: storage and GEMM-input precision; accumulation is fp32 */
  float norm_eps;
  float rope_theta;
  float hsm_eps;       /* eps of the three RMS normalisations inside the HSM */
  int hsm_m1;          /* HSM FC1 / FC3 output width (Table S1: 4 D_h) */
  int hsm_m2;          /* HSM FC2 output width (Table S1: 8 D_h) */
  int kv_block_tokens; /* positions per KV-cache block (16) */
  int max_batch;       /* sequences */
  int max_seq;         /* positions per sequence (prompt + generated) */
  int kv_pool_blocks;  /* 0 -> max_batch * ceil(max_seq / kv_block_tokens) */
  int max_pass_tokens; /* rows of the per-pass workspaces; 0 -> max_batch * max_seq */
  uint64_t block_shuffle_seed; /* 0: KV blocks handed out in order; else a seeded permutation */
  int max_src;         /* > 0 (GPT-2 family only): an encoder-decoder decoder whose layers
                          cross-attend to up to max_src encoder states per sequence
                          (adept_set_cross_source); 0: no cross-attention */
  int kv_type;         /* 0: the cache holds the model's type; ADEPT_KV_E4M3 (bf16 decoders, blocks of 16):
                          8-bit floats with an exponent per position and head, about half the memory of a
                          bf16 cache and half of what attention reads of it.  Held besides, in bf16: two layers'
                          caches (staging of new entries, and what the attention of longer chunks widens entries
                          into) and a block per sequence and layer (the steps' staging).  Not for the
                          cross-attention's source cache */
} adept_config;

/* One named weight tensor.  `data` may be a host or a device pointer (it is read
 * with cudaMemcpyDefault); its element type is the model dtype; `numel` must equal
 * the element count of the named shape.  Names (0-based layer slot l = paper layer
 * l+1; matrices are [out, in] row-major):
 *   tok_emb [V,D]; pos_emb [max_pos,D] (GPT-2/BERT); type_emb [D], emb_ln.g/.b [D] (BERT)
 *   layers.l.attn_norm.g/.b, layers.l.ffn_norm.g/.b [D]   (.b not for LLAMA)
 *   layers.l.wq [D_q,D], wk [D_kv,D], wv [D_kv,D], wo [D,D_q]; bq bk bv bo (not LLAMA)
 *   LLAMA: layers.l.w_gate [F,D], w_up [F,D], w_down [D,F]
 *   GPT2/BERT: layers.l.w_fc [F,D], b_fc [F], w_proj [D,F], b_proj [D]
 *   LLAMA: final_norm.g [D], lm_head [V,D]; GPT2: final_norm.g/.b [D] (head tied to tok_emb)
 *   BERT: pool.w [D,D], pool.b [D], cls.w [C,D], cls.b [C]
 *   max_src > 0 (cross-attention sublayer, pre-LN, between self-attention and the FFN):
 *     layers.l.cross_norm.g/.b [D], cwq [D_q,D], cwk [D_kv,D], cwv [D_kv,D], cwo [D,D_q],
 *     cbq cbk cbv cbo
 *   HSM (App. B Table S1): hsm.g0 [D], hsm.conv_w [3,3], hsm.conv_b [1],
 *     hsm.fc1_w [m1,D], hsm.fc1_b, hsm.fc2_w [m2,m1], hsm.fc2_b, hsm.fc3_w [m1,m2],
 *     hsm.fc3_b, hsm.g1 [m1], hsm.fc4_w [D,m1], hsm.fc4_b [D], hsm.g2 [D]      */
typedef struct {
  const char* name;
  const void* data;
  int64_t numel;
} adept_tensor;

typedef struct {
  const adept_tensor* tensors;
  int n_tensors;
} adept_tensor_table;

typedef struct adept_model adept_model;  /* opaque, library-owned */

/* Load a model: validate `cfg`, allocate device memory, copy and repack the weights
 * (norm gains and LN shifts are folded into the following projection), allocate
 * the paged KV pool.  Synchronises `stream` before returning.
 * Errors: INVALID_ARG (bad config, missing or mis-sized tensor), OOM, CUDA. */
ADEPT_API adept_status adept_model_load(const adept_config* cfg, const adept_tensor_table* weights,
                              void* stream, adept_model** out);

/* Prompt pass (prefill) of `batch` sequences of `prompt_len` tokens each; resets
 * sequences 0..batch-1 and reserves KV blocks for their whole max_seq.
 * Per layer i (App. I): the still-active tokens run layer i; for 2 <= i <= N-1 each
 * active token tests <s_hat_i, I_hat> >= delta (Sec. 4.1), or, where
 * d_forced_exit[j] != 0, exits exactly at that layer; exiting tokens are mapped by
 * the HSM (Sec. 4.2) and their K/V for every skipped layer r > i* are produced
 * from s~_N (Sec. 4.3) before layer r's attention.
 *   d_tokens        [batch*prompt_len] int32 token ids, sequence-major
 *   delta           exit threshold (+inf: never exit)
 *   d_forced_exit   [batch*prompt_len] int32, 0 = use delta, else i* in [2, N]; or NULL
 *   d_exit_layer_out[batch*prompt_len] int32 i* per token (N = full depth); or NULL
 *   d_logits_out    decoder: [batch, vocab] fp32 logits of each sequence's last token;
 *                   encoder: [batch, n_classes] classifier logits of position 0; or NULL
 *   d_next_token_out[batch] int32 greedy argmax of the logits (lowest index on ties); or NULL
 *   d_sim_out       [batch*prompt_len, N] fp32 cosine at each tested layer, NaN elsewhere; or NULL
 * Errors: INVALID_ARG, CAPACITY (batch > max_batch, prompt_len > max_seq). */
ADEPT_API adept_status adept_prefill(adept_model* m, int batch, int prompt_len, const int32_t* d_tokens,
                           float delta, const int32_t* d_forced_exit, int32_t* d_exit_layer_out,
                           float* d_logits_out, int32_t* d_next_token_out, float* d_sim_out,
                           void* stream);

/* One generation step (App. I, generation phase): token b of sequence b is appended
 * at that sequence's next position and exits independently of the others.  Same
 * per-token outputs as adept_prefill with batch rows.  Decoder families only.
 * Errors: INVALID_ARG, CAPACITY (a sequence is full). */
ADEPT_API adept_status adept_decode_step(adept_model* m, int batch, const int32_t* d_tokens, float delta,
                               const int32_t* d_forced_exit, int32_t* d_exit_layer_out,
                               float* d_logits_out, int32_t* d_next_token_out, float* d_sim_out,
                               void* stream);

/* The next chunk of each of sequences 0..batch-1, appended behind what the sequence holds: a
 * conversation's next turn, a piece of a long prompt, proposed tokens to check, or, after
 * adept_seq_reserve with lengths 0, prompts of different lengths.  h_lens[b] >= 0 new tokens of sequence
 * b (at least one token in all); d_tokens, d_forced_exit, d_exit_layer_out and d_sim_out hold the
 * sum of h_lens rows, sequence-major; the rest as in adept_prefill (of which it is the continuation:
 * a prompt in one call or in pieces gives the same states, exits and cache up to rounding).
 * d_logits_out, d_next_token_out: row b is sequence b's last new token; rows of sequences without new
 * tokens are not written.  Decoder families only; not with ADEPT_OPT_ALL_AT_ONCE.
 * The first call allocates its workspace.  The lengths come from the host: the call cannot be captured
 * into a graph (nor adept_prefill of a model with an 8-bit cache).
 * Errors: INVALID_ARG (NULL pointers, a negative length, no token, a sequence not reserved, a stream in
 * capture), CAPACITY
 * (batch > max_batch, a sequence beyond max_seq, more tokens than the pass workspace), OOM. */
ADEPT_API adept_status adept_extend(adept_model* m, int batch, const int32_t* h_lens, const int32_t* d_tokens, float delta,
                          const int32_t* d_forced_exit, int32_t* d_exit_layer_out, float* d_logits_out,
                          int32_t* d_next_token_out, float* d_sim_out, void* stream);

/* adept_extend, and the chunks verified: h_lens[b] tokens of sequence b, the last accepted one and then drafts (of its own earlier
 * exits, another model, a look-up), against this pass's logits.  d_logits_out [sum of h_lens][vocab] fp32 (not NULL) receives those
 * of every token; d_draft, d_temperature, d_u, d_accepted_out, d_next_token_out and d_logprob_out are those of adept_verify_drafts, whose
 * d_start are the chunks' (a sequence without tokens: 0, -1).  The sequences hold their whole chunks afterwards: adept_seq_trim takes away what
 * was not accepted (of 1 + d drafts' tokens, 1 + accepted stay).
 * Drafts of the model's own: generation steps with a threshold that lets tokens leave early, then adept_seq_trim back to where
 * they began, and this call over the same tokens at the threshold that is to hold (+infinity: full depth), which writes their K/V anew.
 * The first call allocates its workspace.  Errors: as adept_extend, and INVALID_ARG for what adept_verify_drafts refuses; a sequence that
 * the verification leaves out flags DEVICE_INPUT. */
ADEPT_API adept_status adept_extend_verify(adept_model* m, int batch, const int32_t* h_lens, const int32_t* d_tokens, float delta,
                                 const int32_t* d_forced_exit, int draft_dtype, const void* d_draft, int64_t ld_draft,
                                 const float* d_temperature, const float* d_u, int32_t* d_exit_layer_out, float* d_logits_out,
                                 int32_t* d_accepted_out, int32_t* d_next_token_out, float* d_logprob_out, float* d_sim_out,
                                 void* stream);

/* Cuts sequences 0..batch-1 back to their first h_lens[b] positions (at most what they hold; their blocks stay reserved), for what is
 * enqueued on `stream` after it.  Not in a captured stream.  Errors: INVALID_ARG, CAPACITY (batch > max_batch), CUDA. */
ADEPT_API adept_status adept_seq_trim(adept_model* m, int batch, const int32_t* h_lens, void* stream);

/* Threshold calibration (Sec. 4.1: delta is set to meet the computation budget; Sec. 5.1):
 * bisection on delta in [lo, hi] over prompt passes of the calibration batch d_tokens
 * [batch, prompt_len] (threshold exits, no forced exits) until the batch's reduction in
 * computation RDC = 1 - sum(exit layer) / (batch prompt_len N) is within tol of target_rdc,
 * or max_iter passes have run.  A pass whose RDC is above the target raises the
 * threshold (lo = delta), otherwise it lowers it (hi = delta).
 *   delta_out, rdc_out, iters_out: host pointers (the last pass's delta and RDC, passes run)
 * Synchronous: waits for each pass on `stream`.  Like adept_prefill it resets sequences
 * 0..batch-1.  Errors: INVALID_ARG (target outside [0, 1), tol < 0, max_iter < 1,
 * lo >= hi, NULL pointers), and those of adept_prefill. */
ADEPT_API adept_status adept_calibrate_threshold(adept_model* m, int batch, int prompt_len, const int32_t* d_tokens,
                                       float target_rdc, float tol, int max_iter, float lo, float hi,
                                       float* delta_out, float* rdc_out, int* iters_out, void* stream);

/* Decoupled skipped-layer KV fill (Eq. 6, the decoupling of Sec. 4; Eq. 9, KV
 * generation in Sec. 4.3): for every token j and every layer r = i*_j+1..N, writes layer r's
 * K = RoPE(W_K^r norm_r(s~_j) + b_K^r) and V = W_V^r norm_r(s~_j) + b_V^r into the
 * KV cache at (d_seq[j], d_pos[j]); all (token, layer) pairs in one grouped launch.
 *   d_h_mapped  [n_tokens, D] mapped states s~_N in the model dtype
 *   d_exit_layer[n_tokens] int32 i* in [1, N] (N: nothing to fill)
 *   d_seq, d_pos[n_tokens] int32 sequence and position; their KV blocks must have been
 *               reserved (adept_prefill or adept_seq_reserve)
 * Errors: INVALID_ARG, CAPACITY (n_tokens above the fill workspace limit, 1<<20). */
ADEPT_API adept_status adept_skip_kv_fill(adept_model* m, int n_tokens, const void* d_h_mapped,
                                const int32_t* d_exit_layer, const int32_t* d_seq,
                                const int32_t* d_pos, void* stream);

/* Allocation-free variant of adept_skip_kv_fill.  The paper has no counterpart: this is
 * an interface for callers that cannot allocate device memory -- code recording a CUDA
 * graph (allocation and the synchronisation of cudaFree cannot be captured), serving
 * loops under a fixed memory budget or their own allocator, and latency-critical paths
 * that must not synchronise the device.  adept_skip_kv_fill grows a per-model workspace
 * with cudaMalloc when a call brings more tokens than before; this call keeps the same
 * working set in a fixed file-scope device array of ADEPT_NOALLOC_SCRATCH_BYTES bytes
 * (16 MiB, held by every GPU that loads the library until the process exits) and calls
 * no cudaMalloc, cudaFree or other allocating routine.  Same arguments and results as
 * adept_skip_kv_fill; bf16 models only, without an 8-bit cache.
 *  - Limit: n_tokens * (d_model * 2 + 4) bytes plus about 3 KiB must fit the array
 *    (about 2000 tokens at d_model 4096, 10900 at d_model 768); larger calls return
 *    ADEPT_ERR_CAPACITY with the limit in adept_last_error and enqueue nothing.
 *  - The first call on a device looks up the array's device address (with that device
 *    current); make that first call before any stream capture.
 *  - Every call shares the array and it keeps the last call's contents (each call clears
 *    the counters it needs zeroed).  Calls that overlap on the GPU -- on different streams
 *    or for different models on one device -- race on it: serialise them.
 *  - On the host the call keeps its launch description on the calling thread's stack and
 *    in thread-local storage: host threads that drive different models (on different
 *    devices, or one after the other on the GPU of one device) do not share host state.
 *    The calling thread's programmatic-dependent-launch setting is restored on return. */
#define ADEPT_NOALLOC_SCRATCH_BYTES ((size_t)16 << 20)
ADEPT_API adept_status adept_skip_kv_fill_noalloc(adept_model* m, int n_tokens, const void* d_h_mapped,
                                                  const int32_t* d_exit_layer, const int32_t* d_seq,
                                                  const int32_t* d_pos, void* stream);

/* Release everything the model owns (synchronises the device first).  NULL is a no-op. */
ADEPT_API void adept_free(adept_model* m);

/* Encoder-decoder models (Sec. 5.2, the OFA setting: an early-exiting encoder whose final
 * states feed a decoder that exits token by token too).  For a decoder loaded with
 * max_src > 0: set the source of every layer's cross-attention for sequences 0..n_seq-1.
 * d_states: fp32 [sum_b h_src_len[b]][d_model], device, in sequence order -- the encoder's
 * final states (s_N of tokens that ran to full depth, s~_N of exited ones; for an encoder
 * pass of n_seq x P tokens, the rows adept_read_final_states returns, with h_src_len[b] = P).
 * h_src_len[b] in [1, max_src].  Computes each decoder layer's source K/V (its cross K/V
 * projection of the states, rounded to bf16 for bf16 models) into the model's source cache;
 * later prompt passes and generation steps of these sequences cross-attend over all
 * h_src_len[b] source positions (not causal).  The states may be released once `stream` has
 * passed the call.  Errors: INVALID_ARG (no cross-attention, n_seq or a length out of range,
 * NULL pointer), CUDA. */
ADEPT_API adept_status adept_set_cross_source(adept_model* m, int n_seq, const int32_t* h_src_len,
                                              const float* d_states, void* stream);

/* ---- helpers (not part of the method; used by tests and the benchmark) ---- */

/* Message of the last failing call on `m`; with m NULL, of the calling thread's last failed load or
 * call on an adept_kv_cache. */
ADEPT_API const char* adept_last_error(const adept_model* m);
ADEPT_API const char* adept_status_string(adept_status s);

/* Reset sequences 0..batch-1 to lengths h_lens[b] and reserve their KV blocks for
 * max_seq positions (no compute; the cached values are left undefined). */
ADEPT_API adept_status adept_seq_reserve(adept_model* m, int batch, const int32_t* h_lens);

/* Copy K and V of `n_pos` positions starting at pos0 of sequence `seq` at layer
 * `layer` (1-based) out of the paged cache into d_k_out / d_v_out, each
 * [n_pos, n_kv_heads, head_dim] in the model dtype (what an 8-bit cache holds: exactly). */
ADEPT_API adept_status adept_read_kv(adept_model* m, int layer, int seq, int pos0, int n_pos,
                           void* d_k_out, void* d_v_out, void* stream);

/* Copy the final states of the last prefill/decode pass ([rows, D] fp32: s~_N of
 * exited tokens, s_N of the rest) into d_out; rows = tokens of that pass. */
ADEPT_API adept_status adept_read_final_states(adept_model* m, float* d_out, int rows, void* stream);

/* Synchronise `stream`, then read and clear the device error word.
 * Returns DEVICE_INPUT if a kernel flagged an invalid input, TIMEOUT if a bounded
 * wait gave up, CUDA on an asynchronous CUDA error, else OK. */
ADEPT_API adept_status adept_check_device_status(adept_model* m, void* stream);

/* Options (ADEPT_OPT_*).  HSM_IDENTITY=1 replaces the HSM by s~ = s_i* (test switch).
 * PROFILE=1 records CUDA events around the GEMM, fill and attention launches so that
 * adept_profile_read can report launch counts and device time per kernel class
 * (generation steps then run as direct launches).  GEMM_SIMT=1 routes GEMMs to the
 * SIMT kernels (cross-check).  DECODE_GRAPH (default 1): from its second call with a
 * given batch size, adept_decode_step replays a CUDA graph of the step captured once;
 * 0 launches every kernel directly.  DECODE_GEMM (default 1): GEMMs of few rows of bf16 models
 * (generation steps, short prompts, output heads, the mapper's products, small fills) run on the
 * weight-streaming kernels: up to 8 rows on the generation-step kernels, with the input
 * standardisation fused in (products of 128 MB of weights and more, and 9 to 128 rows: on the
 * weight-streaming tcgen05 kernel, after a separate standardisation launch); 0 routes them to the
 * tiled tcgen05 kernel.  DECODE_STREAM (default 1): those
 * weight-streaming GEMMs that are wide (at least 8192 outputs, or a grouped fill) and large
 * enough to stream (at least 8 MB of weights), and whose rows fit in shared memory, run on the
 * stream-K kernel (equal shares of the weight stream per SM, split tiles finished by the last
 * CTA to arrive); 0 keeps every one of them on the cluster K-split kernel.  DECODE_TILED (default 1): bf16 decoders keep a tile-contiguous copy of every streamed
 * weight (layer projections, LM head, the mapper's FC weights; made at load, refreshed after
 * each mapper training step; it doubles the weights' device memory) from which the weight-
 * streaming kernels fetch each 32-row x 256-k unit with one contiguous bulk copy; 0 makes them
 * read the row-major weights through tensor maps instead.  EXIT_METRIC (App. H.3): 0 (default) the global similarity of Sec. 4.1,
 * cos(s_i, sum_{d<i} s_hat_d); 1 the local similarity cos(s_i, s_{i-1}); 2 both (a token leaves
 * when both reach delta; the reported similarity is their minimum).  ALL_AT_ONCE (App. H.2):
 * 1 makes every token of a prompt take the exit decision of its sequence's last prompt token,
 * so a sequence leaves at once (generation steps are unaffected: one token per sequence).
 * Default 0.  STOP_ENTIRELY (bf16 encoders; Sec. 4.3 on downstream tasks): 1 stops an exited
 * token's computation entirely — no K/V of deeper layers, and deeper layers' attention sees
 * only the tokens still active there; its mapped state still feeds the classifier.  Default 0.
 * SPAN_TIMER (instrumentation, default 0): 1 makes the weight-streaming GEMM launches (the
 * stream-K and the cluster K-split kernel: generation steps, output heads of short passes,
 * fills of a few tokens) record their span on the device timer, from the first CTA past the
 * grid-dependency wait to the end of the last CTA, summed per kernel class by a small kernel at
 * the end of each pass (read with adept_span_read; a pass records its first 1024 such launches).
 * Launches keep programmatic dependent launch and graph replay (graphs are captured again),
 * so spans are taken in the step as it runs; consecutive launches' spans do not overlap.
 * ATTN_TC (default 1): the prompt-pass attention of bf16 models (self- and cross-attention,
 * head_dim 64 or 128) runs on the tcgen05 kernel (S and O accumulated in tensor memory, P
 * rounded to bf16); 0 keeps the mma.sync kernel (which the encoder's stop-entirely variant
 * always uses).  FUSED_EXIT (default 1): in generation steps of at most 4 sequences whose QKV
 * product runs on the stream-K kernel (decoders without cross-attention, global exit
 * similarity), the exit step of layer i (test, inertia update, compaction) is taken by layer
 * i+1's QKV launch: every CTA reduces the layer's rows and takes the same decisions, so the
 * separate exit kernel and its launch leave the step; 0 launches the exit kernel after every
 * layer. */
enum { ADEPT_OPT_HSM_IDENTITY = 1, ADEPT_OPT_PROFILE = 2, ADEPT_OPT_GEMM_SIMT = 3, ADEPT_OPT_DECODE_GRAPH = 4,
       ADEPT_OPT_DECODE_GEMM = 5, ADEPT_OPT_EXIT_METRIC = 7, ADEPT_OPT_ALL_AT_ONCE = 8,
       ADEPT_OPT_STOP_ENTIRELY = 9, ADEPT_OPT_DECODE_STREAM = 10, ADEPT_OPT_DECODE_TILED = 11,
       ADEPT_OPT_SPAN_TIMER = 12, ADEPT_OPT_ATTN_TC = 13, ADEPT_OPT_FUSED_EXIT = 14 };
ADEPT_API adept_status adept_set_option(adept_model* m, int option, int value);

/* Kernel classes reported by adept_profile_read: the GEMMs of prompt passes (layer
 * projections, HSM, head, and the per-layer skipped-layer fills co-launched with
 * layer i's QKV), the GEMMs of generation steps, the grouped skipped-layer fill
 * launches (end of a generation step and adept_skip_kv_fill), attention, and the GEMMs
 * of HSM training steps. */
enum { ADEPT_PROF_GEMM_PREFILL = 0, ADEPT_PROF_KV_FILL = 1, ADEPT_PROF_ATTENTION = 2,
       ADEPT_PROF_GEMM_DECODE = 3, ADEPT_PROF_GEMM_TRAIN = 4, ADEPT_PROF_NCLASS = 5 };
/* Synchronise, then return the number of recorded launches of kernel class `cls` and
 * their total device time in ms (CUDA events on the launching stream); resets the
 * record.  flops / bytes are reserved (returned as 0). */
ADEPT_API adept_status adept_profile_read(adept_model* m, int cls, int64_t* launches, double* total_ms,
                                double* flops, double* bytes);
/* Synchronise, then return the launches of class `cls` recorded by the span timer and their
 * summed spans in ms; resets the class total.  Zeros when the timer was never on. */
ADEPT_API adept_status adept_span_read(adept_model* m, int cls, int64_t* launches, double* total_ms);

/* ---- HSM training (Sec. 4.2; Sec. 4.3; Sec. 5.1 "Training"; App. D) -------------------
 * The Hidden State Mapper is trained with the base model frozen.  Decoders: its mapped state
 * s~ of an example (s_i, s_{i-1}, I) goes through the frozen final norm and LM head, and the
 * mean cross-entropy against the example's target token (the next input token) is minimised
 * (adept_hsm_train_step).  Encoders: a similarity loss against the original final hidden
 * states plus the frozen classifier's cross-entropy on the labelled rows
 * (adept_hsm_train_step_cls).  Both with AdamW (decoupled weight decay, bias-corrected
 * moments).
 *
 * Parameters, in this order (Table S1): 0 g0 [D], 1 conv_w [3][3], 2 conv_b [1], 3 fc1_w
 * [m1][D], 4 fc1_b [m1], 5 fc2_w [m2][m1], 6 fc2_b [m2], 7 fc3_w [m1][m2], 8 fc3_b [m1], 9 g1
 * [m1], 10 fc4_w [D][m1], 11 fc4_b [D], 12 g2 [D].  The library keeps fp32 master copies and
 * the two AdamW moments of each; the products run on the model dtype's GEMMs (bf16 models:
 * bf16 operands, fp32 accumulation), everything else in fp32.  After every step the model's
 * own HSM weights (used by adept_prefill / adept_decode_step) hold the updated values. */
typedef struct {
  float lr, beta1, beta2, eps, weight_decay;
} adept_adamw;

/* Starts HSM training: master parameters from the model's current HSM weights, zero moments,
 * step count 0, and device workspaces for up to max_rows examples per step (a second call
 * frees the previous ones and starts over).  Synchronous on `stream`.
 * Errors: INVALID_ARG (max_rows < 1, an encoder whose n_classes is outside [1, 64], a bf16
 * model whose D, m1 or m2 is not a multiple of 8), OOM. */
ADEPT_API adept_status adept_hsm_train_init(adept_model* m, int max_rows, void* stream);

/* One training step on n examples, enqueued on `stream`: forward (Table S1) with the
 * activations kept, frozen head, cross-entropy, backward, AdamW with step number t = (steps
 * so far) + 1, write-back of the model's HSM weights.
 *   d_s_i, d_s_prev, d_inertia  [n, D] fp32 device rows: s_i, s_{i-1} and I of each example
 *   d_target                    [n] int32 device token ids in [0, vocab) (a bad id flags
 *                               DEVICE_INPUT at adept_check_device_status; its row adds
 *                               nothing to the loss or the gradients)
 *   hp                          host pointer to the hyperparameters
 *   d_loss_out                  device float: the mean loss before the update (NULL: not written)
 * Errors: INVALID_ARG (no adept_hsm_train_init, an encoder model, n outside [1, max_rows],
 * NULL pointers, lr < 0, beta outside [0, 1), eps <= 0, weight_decay < 0). */
ADEPT_API adept_status adept_hsm_train_step(adept_model* m, int n, const float* d_s_i, const float* d_s_prev,
                                  const float* d_inertia, const int32_t* d_target, const adept_adamw* hp,
                                  float* d_loss_out, void* stream);

/* One training step of an encoder's HSM for classification (Sec. 4.3), enqueued on `stream`:
 * with no next token to predict, the loss is the similarity loss against the original final
 * hidden states, mean over the n examples of 1 - cos(s~, s_N) (cos = 0 where a norm is 0),
 * plus cls_weight times the frozen pooler + classifier's softmax cross-entropy (for two
 * classes, the binary cross-entropy) on the first n_cls examples, the labelled [CLS] rows,
 * averaged over them.  Then backward, AdamW and the weight write-back as adept_hsm_train_step.
 *   d_s_i, d_s_prev, d_inertia  [n, D] fp32 device rows as in adept_hsm_train_step
 *   d_s_final                   [n, D] fp32 device rows: the original final hidden states
 *   n_cls, d_label              labelled rows 0..n_cls-1 (0 <= n_cls <= n) and their int32 class
 *                               ids in [0, n_classes) on the device (NULL allowed when n_cls = 0;
 *                               a bad id flags DEVICE_INPUT at adept_check_device_status and its
 *                               row adds no task loss or gradient)
 *   cls_weight                  weight of the task loss (>= 0; the paper adds the two: 1)
 *   hp, d_loss_out              as in adept_hsm_train_step
 * Errors: INVALID_ARG (no adept_hsm_train_init, a decoder model, n or n_cls out of range, NULL
 * pointers, cls_weight < 0 or not finite, AdamW hyperparameters as above). */
ADEPT_API adept_status adept_hsm_train_step_cls(adept_model* m, int n, const float* d_s_i, const float* d_s_prev,
                                      const float* d_inertia, const float* d_s_final, int n_cls,
                                      const int32_t* d_label, float cls_weight, const adept_adamw* hp,
                                      float* d_loss_out, void* stream);

/* Copies one parameter's fp32 training values to device memory d_out (count = its element
 * count, adept_hsm_param_numel): what = ADEPT_HSM_PARAMS (master values), ADEPT_HSM_GRADS
 * (gradients of the last step), ADEPT_HSM_MOMENT1 / ADEPT_HSM_MOMENT2 (AdamW moments).
 * Enqueued on `stream`.  Errors: INVALID_ARG (no training state, bad what / param / count). */
enum { ADEPT_HSM_PARAMS = 0, ADEPT_HSM_GRADS = 1, ADEPT_HSM_MOMENT1 = 2, ADEPT_HSM_MOMENT2 = 3 };
ADEPT_API adept_status adept_hsm_train_read(adept_model* m, int what, int param, float* d_out, int64_t count,
                                  void* stream);
/* Element count of HSM parameter `param` (0..12), or -1. */
ADEPT_API int64_t adept_hsm_param_numel(const adept_model* m, int param);

/* ---- operators on a caller-owned paged K/V cache ---------------------------------------
 * The cache of one layer (or of anything that keys and values are kept of), in the layout of the
 * models' own: K and V as [n_blocks][n_kv_heads][block_tokens][head_dim], position p of sequence b
 * in block d_block_table[b][p / block_tokens], slot p % block_tokens.  kv_type:
 *   ADEPT_KV_F32, ADEPT_KV_BF16   plain elements
 *   ADEPT_KV_E4M3                 one byte an element and one exponent byte per (position, head) in
 *     d_k_exp / d_v_exp [n_blocks][n_kv_heads][block_tokens]: value = e4m3 * 2^(byte - 127).  Written
 *     from x: with a = max |x| over the head's finite elements, a = m 2^E, m in [1/2, 1), the
 *     exponent is e = E - 9, E - 8 where m > 7/8 (so that a 2^-e <= 448), at least -126, and 0 for
 *     a = 0; an element is e4m3(x 2^-e), rounded once, to nearest even.  NaN stays NaN; an infinity
 *     is stored as NaN.  What is read back is exact in fp32, and in bf16 above its subnormals (only
 *     an element that rounded up to 2^128 reads back as infinity).
 * The buffers are the caller's, on the current device; d_k, d_v and the exponents start on 16 bytes.  The calls
 * allocate nothing, hold no state between calls and (but for the check) can be captured into a graph; calls on one
 * cache are ordered by their streams as any other work on shared buffers is.
 * d_err (may be NULL): a device word that kernels set where an input read on the device is out of
 * range (zero it first); adept_kv_check reports and clears it. */
typedef struct {
  int kv_type;              /* ADEPT_KV_* */
  int n_blocks;
  int n_kv_heads;
  int head_dim;             /* 32, 64 or 128 */
  int block_tokens;
  int n_seq;                /* rows of the block table */
  int max_blocks_per_seq;   /* its columns; at most 2^30 positions a row, and 2^20 elements a position */
  void* d_k;
  void* d_v;
  uint8_t* d_k_exp;         /* ADEPT_KV_E4M3 only */
  uint8_t* d_v_exp;
  const int32_t* d_block_table;
  uint32_t* d_err;
} adept_kv_cache;

/* Writes n_rows rows of K and of V (row r: n_kv_heads * head_dim elements of ADEPT_DTYPE_* dtype at
 * d_k + r * ld_k, so that rows may lie inside a wider product) to position d_pos[r] of sequence
 * d_seq[r], in the cache's type.  d_seq[r] < 0: the row is left out.  A sequence, position or block
 * out of range flags DEVICE_INPUT and leaves the row out.  Each (sequence, position) at most once
 * a call: of two rows with the same one the entry may mix both.
 * Errors: INVALID_ARG (bad cache, n_rows < 0, NULL or misaligned pointers, a stride below a row), CUDA. */
ADEPT_API adept_status adept_kv_append(const adept_kv_cache* c, int n_rows, int dtype, const void* d_k, int64_t ld_k,
                             const void* d_v, int64_t ld_v, const int32_t* d_seq, const int32_t* d_pos, void* stream);
/* The other way: the entries at (d_seq[r], d_pos[r]) into rows of ADEPT_DTYPE_* dtype (a row with
 * d_seq[r] < 0, or out of range, is not written; an entry may be asked for more than once). */
ADEPT_API adept_status adept_kv_gather(const adept_kv_cache* c, int n_rows, int dtype, void* d_k, int64_t ld_k, void* d_v,
                             int64_t ld_v, const int32_t* d_seq, const int32_t* d_pos, void* stream);

/* Causal attention of a chunk of new tokens whose K and V are in the cache already.  Sequence b
 * (row b of the block table) brings the rows d_q_start[b] .. d_q_start[b + 1] - 1 of Q: its last
 * positions, up to d_kv_len[b] - 1.  The row at position p attends positions 0 .. p: query head h
 * with KV head h / (n_heads / n_kv_heads), scores q.k / sqrt(head_dim).  A sequence may bring no row
 * (it is not read), one (a generation step) or thousands; a row at a position below 0 gives zeros.
 * What is behind a row's position (the chunk's later tokens, unwritten slots) does not enter it,
 * whatever it holds; a NaN or infinite V entry that a row does attend makes that output NaN or
 * infinite.
 *   d_q, d_out   [n_rows][ld] (n_heads * head_dim elements a row): bf16, or fp32 for an fp32 cache;
 *                they must not overlap.  Rows that no sequence holds are not written.
 *   d_q_start [n_seq + 1], d_kv_len [n_seq]   int32, read on the device
 *   d_row_pos [n_rows] or NULL   int32, read on the device: the rows' own positions, ascending within a
 *                sequence (else that sequence's rows hold anything), each below its d_kv_len (rows of
 *                tokens that are still active where others have left); NULL: the last positions
 *   max_q_len, max_kv_len   bounds on a sequence's rows and positions; a sequence beyond them, or with
 *                rows outside 0 .. n_rows, flags DEVICE_INPUT and is left out, as is a key whose block
 *                is out of range (a row of such keys alone, or of scores that are all -infinity, gives zeros)
 *   d_ws         adept_chunk_attention_workspace bytes on 16 bytes (NULL where that is 0), of any
 *                contents; calls that may overlap on the GPU need one each
 * Sums run in fp32 over weights of up to 2^8, and scores are fp32: V elements above 2^100 may overflow the sums, products
 * of Q and K beyond fp32's range make scores infinite or NaN, and elements of an 8-bit row whose largest is below 2^-100
 * may lose bits.
 * For the same lengths a call's results are the same bits every time.
 * Errors: INVALID_ARG (bad cache, n_heads no multiple of n_kv_heads or above 2^15, max_kv_len above the table, a
 * stride below a row, NULL or misaligned pointers, a workspace too small), CAPACITY (n_rows *
 * n_heads or n_seq * n_heads above 2^30, or more than 2^31 tiles of 128 rows and 128 keys), CUDA. */
ADEPT_API adept_status adept_chunk_attention(const adept_kv_cache* c, int n_heads, int n_rows, const void* d_q, int64_t ld_q,
                                   const int32_t* d_q_start, const int32_t* d_kv_len, const int32_t* d_row_pos,
                                   int max_q_len, int max_kv_len, void* d_out, int64_t ld_out, void* d_ws, int64_t ws_bytes, void* stream);
/* Bytes of d_ws that such a call needs, or -1 (bad arguments); a call of smaller bounds or fewer sequences
 * on the same pool needs no more.  For longer chunks over an 8-bit cache they hold K and V in bf16, for as many
 * blocks as the pool has or as n_seq sequences of max_kv_len positions take, whichever are fewer. */
ADEPT_API int64_t adept_chunk_attention_workspace(const adept_kv_cache* c, int n_heads, int n_rows, int max_q_len,
                                        int max_kv_len);
/* Synchronise `stream`, then read and clear the cache's error word: DEVICE_INPUT, TIMEOUT or OK.  What calls on
 * other streams set meanwhile is reported now or by the next check.
 * Errors: INVALID_ARG (no error word, a stream in capture), CUDA. */
ADEPT_API adept_status adept_kv_check(const adept_kv_cache* c, void* stream);

/* ---- pages behind the sequences of a paged K/V cache -------------------------------------
 * The block table of an adept_kv_cache, or of several (the layers of a model share one table), with a count per block: d_ref[i] =
 * rows of the table that hold block i, plus what the program itself adds to keep a block (a prefix that no row holds at the
 * moment); 0: free.  Rows may share blocks.  The table starts as all -1 with counts 0, or as the program sets both.
 * The calls decide on the device, from the tables and lengths there, in row and block order: the same tables give the same
 * result every time.  They allocate nothing, hold no state between calls and can be captured into a graph; calls on the
 * same pages are ordered by their streams.  A row's entry that is neither -1 nor a block, a block that is held but
 * counted as free, and lengths or rows out of range flag DEVICE_INPUT in d_err (adept_error_check) where a call meets them (below: which
 * entries it checks); such an entry counts as -1, a row with such a length or source stays as it is.
 *   d_ws   adept_kv_pages_workspace bytes on 16 bytes, of any contents; calls that may overlap on the GPU need one each
 * Errors of all: INVALID_ARG (bad pages, NULL or misaligned pointers, a workspace too small), CUDA. */
typedef struct {
  int n_blocks;
  int block_tokens;
  int n_seq;                /* rows of the block table */
  int max_blocks_per_seq;   /* its columns; at most 2^30 positions a row */
  int32_t* d_block_table;
  int32_t* d_ref;           /* [n_blocks], on 16 bytes */
  uint32_t* d_err;          /* or NULL */
} adept_kv_pages;
ADEPT_API int64_t adept_kv_pages_workspace(const adept_kv_pages* p);

/* Every row at once: row b becomes the first d_length[b] positions of what row d_source[b] held before the call (their blocks
 * shared, counted once more), the rest of the row -1; blocks that nobody holds any more are free.  d_source[b] = b with the row's
 * length: unchanged; a shorter length: cut back (drafts that were not accepted); d_source[b] < 0, or no positions (a length of 0 or
 * less): dropped; another row: a fork, or beams reordered.  Both [n_seq] int32.  Checked are the entries that a row takes from another,
 * which are -1 where they are flagged, and those that it gives up, whose block's count then stays as it is. */
ADEPT_API adept_status adept_kv_fork(const adept_kv_pages* p, const int32_t* d_source, const int32_t* d_length, void* d_ws, int64_t ws_bytes,
                           void* stream);

/* Makes positions d_length[b] .. d_new_length[b] - 1 of every row b writable: entries without a block get the free block of the
 * lowest number (rows in order, a row's entries in order), and an entry whose block other rows hold too gets one of its own.
 * Where such a block also holds positions below d_length[b], its contents have to follow: d_copy_src[b], d_copy_dst[b] name the
 * blocks (-1: none), to be copied by adept_kv_copy_blocks before anything is written.  Of several rows that share that block and
 * all grow, while nobody else holds it, the last keeps it.
 * Rows are served in order while blocks last: row b if what the rows up to it ask for is there (a row that asks for no block
 * always, unless it would keep a shared one that an earlier row did not get away from).  d_got[b] = d_new_length[b] where row b was served or holds what it
 * needs, else d_length[b], and nothing of the row has changed.  d_new_length[b] <= d_length[b]: nothing is asked for.
 * All [n_seq] int32; d_got may be d_length or d_new_length, else nothing overlaps.  A block that the call frees is given by the next.
 * Checked are the entries that a row asks to write; one whose block is counted as free is -1 from then on, whether the row is served or not.
 * CAPACITY: more than 4096 rows. */
ADEPT_API adept_status adept_kv_reserve(const adept_kv_pages* p, const int32_t* d_length, const int32_t* d_new_length, int32_t* d_got,
                              int32_t* d_copy_src, int32_t* d_copy_dst, void* d_ws, int64_t ws_bytes, void* stream);

/* Moves the blocks in use to the front: with U of them in use (*d_used), the k-th in use past the first U goes to the k-th
 * free one among those (both in ascending order), in the table and in the counts.  d_copy_src[k], d_copy_dst[k] ([n_blocks / 2]
 * int32 each) name the moves, for adept_kv_copy_blocks, and for the program where it holds blocks itself; entries behind the last are -1.  Sources and targets are
 * disjoint.  Checked are all entries; one that is flagged stays in the table, unless another block has come to the number that it names: then it is -1. */
ADEPT_API adept_status adept_kv_compact(const adept_kv_pages* p, int32_t* d_used, int32_t* d_copy_src, int32_t* d_copy_dst, void* d_ws,
                              int64_t ws_bytes, void* stream);

/* Block d_dst[i] = block d_src[i], K and V (and exponents), in each of n_caches caches (an array of structs: the layers; of one
 * type and size) for i < n_pairs; a pair with a negative number is left out, one out of range flags DEVICE_INPUT in the first cache's
 * word.  Targets are distinct, and none is also a source (else it holds anything of either). */
ADEPT_API adept_status adept_kv_copy_blocks(const adept_kv_cache* caches, int n_caches, int n_pairs, const int32_t* d_src, const int32_t* d_dst,
                                  void* stream);

/* ---- drafted tokens against the target's logits ------------------------------------------
 * Sequence b's chunk is rows d_start[b] .. d_start[b + 1] - 1 (n_rows in all): d_tokens[r] is the chunk's token (its first the last
 * one that was accepted, the others drafts, as a pass over the chunk takes them), row r of d_target the target's logits behind
 * it.  With p_r = softmax(target_r / T), q_r = softmax(draft_r / T) (without d_draft: 1 at the draft itself) and x the draft
 * d_tokens[r + 1], the drafts are accepted in order while log u_r + log q_r(x) < log p_r(x).  At the first that is not, the next
 * token is drawn from w = max(p_r - q_r, 0) (from p_r where the sum of that is below 2^-20); behind the last draft, from
 * w = p_r: the least i with w_0 + .. + w_i > (u + 2^-25) sum w, u the number of the sequence's last row.  With u uniform the tokens are
 * distributed as the target's own.  T = 0 (greedy): drafts are accepted while they are the target's best token (the
 * lowest of equals), and the next token is that; d_draft and d_u are not looked at.
 *   d_target, d_draft   [n_rows][ld] ADEPT_DTYPE_* logits, -infinity allowed (a masked token); d_draft (may be NULL): row r is what
 *                       d_tokens[r + 1] was drawn from, a sequence's last row may hold anything
 *   d_start       [n_seq + 1] int32, ascending; a sequence may have no row (0 accepted, next token -1)
 *   d_temperature [n_seq] fp32, 0 or 2^-10 .. 2^10; NULL: 1
 *   d_u           [n_rows] fp32 in [0, 1) (not NULL, also where every sequence is greedy)
 *   d_accepted, d_next  [n_seq] int32: drafts accepted, the next token
 *   d_logprob     [n_rows] fp32 or NULL: log p_r of each accepted draft (at its r), and of the next token at the row that it was drawn
 *                 from (greedy: at T = 1); other rows are not written
 *   d_err         error word or NULL
 * Whatever the rows behind the deciding one hold does not enter.  A sequence whose rows are out of range, or which meets a row of a sequence
 * before it, a token or number out of range, logits with NaN or +infinity, or with nothing above -infinity, gets -1, -1 and flags DEVICE_INPUT.
 * Which draft is accepted follows from sums of weights that are off by 2^-36 at most (2^-40 as a rule), whatever the logits' type, and so does
 * a token drawn from p_r.  max(p_r - q_r, 0) has the errors of both: where it sums to s (1 to 2^-20), the sums that it is drawn by are off by
 * 2^-33 / s at most (2^-40 / s as a rule).  The log probabilities are off by some 10^-6.  The same call gives the same bits.
 *   d_ws          adept_verify_workspace(n_rows) bytes on 16 bytes; calls that may overlap on the GPU need one each.  No
 *                 smaller call needs more.
 * The results overlap neither what is read nor each other.
 * Errors: INVALID_ARG (a size, type, stride or pointer), CAPACITY (above 2^24 rows or 2^16 sequences), CUDA. */
ADEPT_API adept_status adept_verify_drafts(int n_seq, int n_rows, int vocab, int target_dtype, const void* d_target, int64_t ld_target,
                                 int draft_dtype, const void* d_draft, int64_t ld_draft, const int32_t* d_tokens,
                                 const int32_t* d_start, const float* d_temperature, const float* d_u, int32_t* d_accepted,
                                 int32_t* d_next, float* d_logprob, uint32_t* d_err, void* d_ws, int64_t ws_bytes, void* stream);
ADEPT_API int64_t adept_verify_workspace(int n_rows);

/* adept_kv_check for an error word by itself. */
ADEPT_API adept_status adept_error_check(uint32_t* d_err, void* stream);

/* ---- failure injection (tests of the error paths; no GPU fault is involved) ------------
 * adept_set_wait_limit: limit, in SM cycles, of the kernels' bounded waits on pipeline
 * progress (a ring slot being filled or released, an accumulator becoming ready) in the
 * tensor-core, weight-streaming and stream-K GEMMs; 0 restores the default (4e9 cycles, about
 * 2 s).  A wait that runs out sets the device error word, its CTA stops, lets the copies it
 * has in flight land (those waits, and the waits of cross-CTA reductions, keep their own long
 * limits), frees its tensor memory and exits, and adept_check_device_status then returns
 * ADEPT_ERR_TIMEOUT; the outputs of that call are undefined and the model stays usable.
 * Applies to every model of the process on the current device.  Errors: INVALID_ARG
 * (cycles < 0), CUDA.
 * adept_set_alloc_fail_after: after n more device allocations by the library (making the graph of
 * a generation step counts as one), every further allocation fails as if the device were out of
 * memory (n < 0: off, the default); calls that need memory then return ADEPT_ERR_OOM with
 * everything they allocated released, and can be made again. */
ADEPT_API adept_status adept_set_wait_limit(int64_t cycles);
ADEPT_API void adept_set_alloc_fail_after(int64_t n);

/* Number of kernel launches the library enqueued since the last call (then reset). */
ADEPT_API int64_t adept_launch_count(adept_model* m);

#ifdef __cplusplus
}
#endif
#endif /* ADEPT_H */
