/*
 * aio.h -- C ABI of the batch-1 decode step on MI355X (gfx950).
 *
 * The operation.  A-IO (arXiv 2604.09752) routes requests between a 1B probe
 * and a 7B backbone because batch-1 autoregressive decoding is bound by HBM
 * bandwidth: every generated token fetches the full weight set (Section 2.1,
 * "The Memory-Bound Dilemma"; Section 3.1, about 14 GB per token for the 7B
 * and 2 GB for the 1B).  This library is that decode step for a dense
 * decoder-only transformer -- pre-norm RMSNorm, rotate-half RoPE,
 * grouped-query attention, SwiGLU FFN, untied LM head, no biases -- in
 * hand-written HIP kernels.  It also provides the two variants the paper
 * toggles per request (Section 3.3 "Strategy Routing", Section 4.2): W8A16
 * storage-only quantization (int8 weights, fp16 per-output-channel scales,
 * dequantised inside the matrix-vector kernels) and the one-forward
 * verification of prompt-lookup drafts.
 *
 * Conventions.
 *  - Every pointer named *_dev is a device pointer on the current HIP device;
 *    the caller allocates and owns it (weights, KV cache, workspace, logits,
 *    token buffers).  The library only borrows them, never frees them, and
 *    keeps using the weight, KV and workspace pointers until aio_model_free.
 *  - The library owns only the model handle, a RoPE cos/sin table and any
 *    captured graph; aio_model_free releases exactly those.
 *  - Weight matrices are row-major [out][in] (y = W x).  bf16 is stored as
 *    uint16 bit patterns, fp16 scales likewise.
 *  - Device pointers must be 16-byte aligned (the workspace 256-byte
 *    aligned); d_model and ffn_dim must be multiples of 64.
 *  - All calls are asynchronous on the stream given at load time: a return of
 *    AIO_OK means the work is enqueued.  Results are valid after a stream
 *    synchronisation; device faults surface there.
 *  - Every argument is checked on the host before anything is enqueued; a
 *    rejected call enqueues nothing and changes nothing.  No call aborts or
 *    exits the process and no C++ exception crosses this interface.
 *  - A handle is not thread-safe; distinct handles are independent (a 1B and a
 *    7B model can be resident together, as in the paper's Section 3.1).
 *  - Decode state is (KV cache contents, position), owned by the caller.  Rows
 *    of the cache beyond the current position are never read, so rolling back
 *    after a rejected draft is just calling again at the earlier position.
 */
#ifndef AIO_H
#define AIO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------- errors */
enum {
  AIO_OK = 0,
  AIO_EINVAL = -1,       /* null or misaligned pointer, inconsistent config */
  AIO_ERANGE = -2,       /* token or position out of range, k out of range  */
  AIO_EUNSUPPORTED = -3, /* shape or device this build does not handle      */
  AIO_EHIP = -4,         /* a HIP runtime or launch error; see aio_last_hip_error */
  AIO_ENOMEM = -5,       /* the library's own small allocations failed      */
  AIO_EDEVICE = -6       /* a bounded wait inside a kernel gave up
                            (aio_device_status); the handle's results from
                            then on are invalid: free it and load again */
};

/* Weight storage formats. */
enum {
  AIO_WFMT_BF16 = 0, /* every projection and the LM head in bf16            */
  AIO_WFMT_INT8 = 1  /* W8A16: int8 [out][in] + fp16 scale [out], symmetric,
                        no zero point, W[n,k] = q[n,k] * s[n]; embedding and
                        norm gains stay bf16                                 */
};

/* Largest number of rows (the current token plus drafts) one aio_verify call
 * scores. */
#define AIO_MAX_VERIFY_ROWS 10

typedef struct aio_config {
  int32_t n_layers;   /* L                                                  */
  int32_t d_model;    /* d, multiple of 64                                  */
  int32_t n_heads;    /* H query heads                                      */
  int32_t n_kv_heads; /* Hkv key/value heads, H % Hkv == 0                  */
  int32_t head_dim;   /* hd, 64 or 128                                      */
  int32_t ffn_dim;    /* F, multiple of 64                                  */
  int32_t vocab;      /* V                                                  */
  int32_t max_ctx;    /* positions the KV cache holds                       */
  int32_t max_verify; /* rows per aio_verify call, 1..AIO_MAX_VERIFY_ROWS   */
  int32_t wfmt;       /* AIO_WFMT_BF16 or AIO_WFMT_INT8                     */
  float rms_eps;      /* RMSNorm epsilon (inside the square root)           */
  float rope_base;    /* RoPE base; theta_i = base^(-2i/hd)                 */
} aio_config;

/* Per-layer weights (device pointers).  Norm gains are bf16 [d].  With
 * AIO_WFMT_BF16 the projections are bf16 and the s_* scales must be NULL; with
 * AIO_WFMT_INT8 they are int8 and every s_* is an fp16 [out] array. */
typedef struct aio_layer_weights {
  const void* attn_norm; /* [d]                  */
  const void* ffn_norm;  /* [d]                  */
  const void* wq;        /* [H*hd][d]            */
  const void* wk;        /* [Hkv*hd][d]          */
  const void* wv;        /* [Hkv*hd][d]          */
  const void* wo;        /* [d][H*hd]            */
  const void* w_gate;    /* [F][d]               */
  const void* w_up;      /* [F][d]               */
  const void* w_down;    /* [d][F]               */
  const void *sq, *sk, *sv, *so, *s_gate, *s_up, *s_down;
} aio_layer_weights;

typedef struct aio_weights {
  const void* embed;               /* bf16 [V][d]                             */
  const void* final_norm;          /* bf16 [d]                                */
  const void* lm_head;             /* bf16 or int8 [V][d] (untied)            */
  const void* s_lm_head;           /* fp16 [V] for int8, else NULL            */
  const aio_layer_weights* layers; /* HOST array of n_layers entries; copied   */
} aio_weights;

typedef struct aio_model aio_model;

/* ----------------------------------------------------------- pure host calls */

/* Bytes of the KV cache: bf16 [n_layers][2 (K, V)][n_kv_heads][max_ctx][head_dim].
 * Returns 0 for an invalid config. */
size_t aio_kv_bytes(const aio_config* cfg);

/* Bytes of device workspace the model needs (activations, split-KV partials,
 * a small state block).  Returns 0 for an invalid config. */
size_t aio_workspace_bytes(const aio_config* cfg);

/* AIO_OK, or the error aio_model_load would return for this config. */
int aio_check_config(const aio_config* cfg);

/* Checks of one call's scalar arguments against a config, exactly as the entry
 * points make them (AIO_OK, AIO_EINVAL or AIO_ERANGE). */
int aio_check_decode(const aio_config* cfg, int32_t token, int32_t pos);
int aio_check_verify(const aio_config* cfg, int32_t token, const int32_t* drafts, int32_t k,
                     int32_t pos);

const char* aio_strerror(int code);

/* The last hipError_t this library saw on the calling thread (0 if none). */
int aio_last_hip_error(void);

/* ---------------------------------------------------------- model lifecycle */

/* Binds a model to caller-owned device memory.  One handle is one resident
 * model; the paper keeps its 1B probe and 7B backbone resident together in
 * full precision and switches between them per request (Section 3.1,
 * "System Architecture and Bandwidth Conservation"; Section 5.3), which here
 * is two handles.
 *  cfg, w      host structs; copied.
 *  kv_dev      aio_kv_bytes(cfg) bytes; positions the caller has not written
 *              are never read before a decode or verify call writes them.
 *  ws_dev      aio_workspace_bytes(cfg) bytes, used only by this handle; what
 *              it holds does not matter.
 *  hip_stream  hipStream_t every later call enqueues on (NULL = default stream).
 *  out         receives the handle.
 * Allocates and fills the RoPE table (fp32 cos/sin of angles computed in
 * double on the host), so it synchronises once.  Fails with AIO_EUNSUPPORTED
 * on a device that is not gfx950. */
int aio_model_load(const aio_config* cfg, const aio_weights* w, void* kv_dev, void* ws_dev,
                   void* hip_stream, aio_model** out);

void aio_model_free(aio_model* m);

/* ------------------------------------------------------------- the hot path */

/* One decode step (Section 2.1, Section 3.1): consume `token` at position
 * `pos` (0-based; the cache must hold positions 0..pos-1), write its K and V
 * at `pos` in every layer, attend over positions [0, pos], and write fp32
 * logits [vocab] to logits_dev.
 * AIO_ERANGE: token not in [0, vocab) or pos not in [0, max_ctx). */
int aio_decode_step(aio_model* m, int32_t token, int32_t pos, float* logits_dev);

/* Prompt-lookup verification in one forward (Section 3.3, Section 4.2): rows
 * are [token, drafts[0..k-1]] (drafts is a HOST array) at positions
 * pos..pos+k.  Writes K/V of all k+1 rows; row i of logits_dev (fp32
 * [k+1][vocab]) equals the logits of aio_decode_step on row i's token after
 * rows 0..i-1, i.e. row i attends over positions [0, pos+i].
 * AIO_ERANGE: k < 0, k+1 > max_verify, pos < 0, pos+k >= max_ctx, or a token
 * outside [0, vocab). */
int aio_verify(aio_model* m, int32_t token, const int32_t* drafts, int32_t k, int32_t pos,
               float* logits_dev);

/* Greedy argmax of `rows` rows of `n` fp32 values each (row-major), one
 * int32 index per row into out_dev: the next token of greedy decoding, and
 * for a verify forward the per-row ids that prompt-lookup acceptance
 * compares with the drafts (Section 3.3, Strategy Routing; Section 4.2, PLD
 * Configuration).  The lowest index wins ties; NaN ranks above +Inf (the
 * first NaN wins), as torch.argmax orders them.  logits_dev and out_dev
 * 4-byte aligned.  AIO_ERANGE: rows outside [1, 65535] or n outside
 * [1, 2^30]. */
int aio_argmax(aio_model* m, const float* logits_dev, int32_t rows, int32_t n, int32_t* out_dev);

/* Device-resident greedy decoding for timing: consume `token` at `pos`, then
 * feed each step's argmax as the next token, for n_steps steps, with no host
 * round trip inside the loop (the persistent step kernel reads the token and
 * position from device state and advances them; the per-operation path
 * replays a captured HIP graph unless AIO_GRAPH is "0").  tokens_dev (int32 [n_steps]) receives the
 * argmax of every step; logits_dev (fp32 [vocab]) holds the last step's
 * logits.  AIO_ERANGE if pos + n_steps > max_ctx. */
int aio_decode_greedy(aio_model* m, int32_t token, int32_t pos, int32_t n_steps,
                      int32_t* tokens_dev, float* logits_dev);

/* Profiling: one aio_decode_step with a HIP event recorded on the model's
 * stream before the first kernel and after every kernel, then a wait for the
 * last event.  kernel_ms (host, max_kernels floats) receives each kernel's
 * event-to-event time in launch order -- one entry for the persistent step
 * kernel, else per layer: qkv, attention, split merge, o-projection,
 * gate/up, down; then the LM head -- and *n_kernels the count written.
 * Synchronises; not for the timed loop. */
int aio_profile_step(aio_model* m, int32_t token, int32_t pos, float* logits_dev,
                     float* kernel_ms, int32_t max_kernels, int32_t* n_kernels);

/* 1 if this handle runs each decode step as the single persistent kernel
 * (the default where the shape allows it and AIO_MEGA is not "0"), else 0
 * (a sequence of per-operation kernels). */
int aio_uses_step_kernel(const aio_model* m);

/* Phase timing of one decode step of the persistent kernel: the same work as
 * aio_decode_step, with workgroup 0 recording the device clock as it
 * publishes the outputs of each phase.  phase_us (host, max_phases doubles)
 * receives the time between consecutive phases' outputs, i.e. per layer:
 * attention, O projection, gate/up, down, next layer's QKV; *n_phases the
 * count written.  Synchronises.  AIO_EUNSUPPORTED when the handle does not
 * use that kernel. */
int aio_trace_step(aio_model* m, int32_t token, int32_t pos, float* logits_dev, double* phase_us,
                   int32_t max_phases, int32_t* n_phases);

/* Per-workgroup timing of one step of the persistent kernel, device clock
 * (100 MHz).  Phase k = 5 l + 1 .. 5 l + 5 of layer l is QKV, attention, O,
 * gate/up, down.  arrive[k][b] receives the time workgroup b published its
 * outputs of phase k, leave[k][b] the time it had the inputs of phase k + 1
 * (entry 0 unused).  With max_entries >= 4 (5 L + 1) x blocks, arrive also
 * carries, after its first (5 L + 1) x blocks entries, [phase][workgroup][2]
 * the start and end of each workgroup's weight loop (attention: the end of
 * its splits and of its merge).  n_barriers and n_blocks receive the
 * dimensions (5 L + 1 and blocks).  Allocates a device buffer and
 * synchronises; a profiling aid.  AIO_EUNSUPPORTED when the handle does not
 * use that kernel. */
int aio_trace_barriers(aio_model* m, int32_t token, int32_t pos, float* logits_dev,
                       uint64_t* arrive, uint64_t* leave, int32_t max_entries,
                       int32_t* n_barriers, int32_t* n_blocks);

/* Calibrates the persistent kernel's split of the gate/up rows over its
 * workgroups: runs `rounds` decode steps of `token` at `pos` (so it writes
 * that cache row, like aio_decode_step) with every workgroup timing its
 * gate/up loops, and after each moves every workgroup's share of rows
 * halfway towards its measured streaming rate (CUs and XCDs stream at
 * slightly different rates, steadily; an even split waits for the slowest).
 * The split stays with the handle for all later steps; results are
 * unchanged up to fp32 rounding order, which does not depend on the split.
 * Synchronises.  AIO_ERANGE: rounds outside [1, 64] or a bad token or pos;
 * AIO_EUNSUPPORTED when the handle does not use the persistent kernel. */
int aio_tune_step(aio_model* m, int32_t token, int32_t pos, float* logits_dev, int32_t rounds);

/* Synchronises the model's stream and reports the device-side status word:
 * 0, or 1 if a bounded wait for another workgroup's data (in the persistent
 * kernel or in a prefill product) gave up.  The word is sticky: once set, the results of
 * that step and of every later call on the handle are invalid (free the
 * handle and load again).  Synchronises. */
int aio_device_status(aio_model* m, int32_t* status);

/* ------------------------------------------ prompt-lookup decoding (host) */

/* Prompt-lookup drafts: the draft source of PLD, which Section 3.3
 * ("Dynamic Policy Routing and Execution", Strategy Routing) enables per
 * request and Section 4.2 ("Models and Baselines", PLD Configuration)
 * configures by an n-gram window and a look-ahead length.  Pure host
 * function, no device work.  For n from min(ngram_max, n_hist - 1) down to
 * ngram_min, looks for the last n tokens of hist[0..n_hist) earlier in hist;
 * the earliest earlier occurrence that is followed by at least one token
 * wins, and the up to k tokens that follow it are the drafts.  drafts (host,
 * k int32) receives them and *n_drafts their count (0 when no n-gram
 * recurs).
 * AIO_EINVAL: a null pointer.  AIO_ERANGE: n_hist < 0, k < 0, ngram_min < 1
 * or ngram_max < ngram_min. */
int aio_pld_match(const int32_t* hist, int32_t n_hist, int32_t ngram_max, int32_t ngram_min,
                  int32_t k, int32_t* drafts, int32_t* n_drafts);

typedef struct aio_pld_stats {
  int32_t forwards; /* model forwards: verify calls plus single decode steps */
  int32_t verifies; /* forwards that scored drafts                          */
  int32_t drafted;  /* draft tokens scored                                  */
  int32_t accepted; /* draft tokens accepted                                */
} aio_pld_stats;

/* Greedy generation with prompt-lookup decoding (Section 3.3, Strategy
 * Routing; Section 4.2, PLD Configuration).  history (host, pos int32) holds
 * the tokens at positions 0..pos-1, whose K/V the cache already holds;
 * `token` is consumed at pos.  Each round drafts up to k tokens with
 * aio_pld_match over everything consumed so far plus `token` (never more
 * drafts than tokens still wanted, nor past the end of the cache), scores
 * [token, drafts] in one aio_verify (or one aio_decode_step when nothing
 * matches), takes each row's greedy argmax on the device, and accepts the
 * longest prefix of drafts in which every draft equals the argmax of the row
 * before it.  The argmax of the row after the last accepted draft is the
 * next token, consumed by the next round at pos + accepted + 1 (cache rows
 * written past that are overwritten later, never read).  out (host, n_new
 * int32) receives the generated tokens; they are the tokens plain greedy
 * decoding produces from the same state, whatever the acceptance.
 * logits_dev (fp32 [k+1][vocab], 16-byte aligned) and argmax_dev (int32
 * [k+1]) are scratch.  stats may be NULL.  Synchronises the model's stream
 * once per round and returns when all n_new tokens are generated, or with
 * AIO_EDEVICE as soon as a round finds the device status word set.
 * AIO_ERANGE: token outside [0, vocab), pos < 0, n_new < 1,
 * pos + n_new > max_ctx, k < 0, k + 1 > max_verify, ngram_min < 1 or
 * ngram_max < ngram_min.  AIO_EINVAL: a null pointer or a history token
 * outside [0, vocab). */
int aio_pld_generate(aio_model* m, const int32_t* history, int32_t pos, int32_t token,
                     int32_t n_new, int32_t ngram_max, int32_t ngram_min, int32_t k,
                     float* logits_dev, int32_t* argmax_dev, int32_t* out, aio_pld_stats* stats);

/* -------------------------------------------- the probe's front end (host) */

/* The probe's single forward over its templated request (Section 3.2,
 * "Probe-Based Request-Level Intent Sensing"; its cost is the "1B
 * Single-Token Prefill" of Section 5.3): consumes tokens[0..n) (host) at
 * positions pos .. pos+n-1 in prompt-length matrix products (up to 2048
 * rows per pass over the weights) with causal attention, writes every
 * token's K/V in every layer, and writes the logits after the last token,
 * fp32 [vocab], to logits_dev (16-byte aligned).  The result equals n
 * aio_decode_step calls up to rounding.  A single token is one decode step
 * (the kernels of aio_decode_step), and a prompt of 2 to max_verify tokens
 * goes through the verify forward (the kernels of aio_verify); neither takes
 * scratch beyond the workspace.  The scratch
 * (4 (1 + 2 d + H hd + max(d, H hd) + F) + d / 16 bytes per row, for up to
 * 2048 rows) is allocated by the library on the first call that needs more
 * and kept until
 * aio_model_free, so such a call synchronises once.  Asynchronous
 * otherwise, like aio_verify.
 * AIO_ERANGE: n < 1, pos < 0, pos + n > max_ctx or a token outside
 * [0, vocab); AIO_EINVAL: a null pointer; AIO_ENOMEM: the scratch could not
 * be allocated. */
int aio_prefill(aio_model* m, const int32_t* tokens, int32_t n, int32_t pos, float* logits_dev);

/* Bytes of the device array aio_prefill_noalloc takes its scratch from. */
#define AIO_PREFILL_NOALLOC_SCRATCH_BYTES (32u << 20)

/* aio_prefill for callers that cannot allocate device memory (code under
 * HIP graph capture, serving loops, harnesses that forbid allocation): the
 * same operation and kernels, with the scratch taken from a fixed array of
 * AIO_PREFILL_NOALLOC_SCRATCH_BYTES in the library's device memory instead
 * of library-allocated memory.  It calls no hipMalloc, hipFree or other
 * allocating routine.  The prompt goes through in passes of at most
 * aio_prefill_noalloc_rows(cfg) rows (the array divided by the scratch of
 * one row: 4 (1 + 2 d + H hd + max(d, H hd) + F) + d / 16 bytes, at most 2048),
 * so any n works; results equal aio_prefill's up to rounding (bit-identical
 * where both take the prompt in one pass; a prompt of at most max_verify
 * tokens takes aio_prefill's verify route and needs none of the array).
 * Every GPU holds one such array
 * for the whole process, shared by all calls on that GPU: calls that
 * overlap on one GPU (handles on different streams) race and must be
 * serialised by the caller.  Nothing in the array needs to start at zero:
 * each call writes every region before reading it.  Asynchronous like
 * aio_verify; the tokens are copied from host memory on the model's stream.
 * Errors as aio_prefill, and AIO_EUNSUPPORTED when a prompt of more than
 * max_verify tokens meets a config whose one row's scratch exceeds the
 * array (aio_prefill_noalloc_rows(cfg) == 0). */
int aio_prefill_noalloc(aio_model* m, const int32_t* tokens, int32_t n, int32_t pos,
                        float* logits_dev);

/* Rows aio_prefill_noalloc takes per pass for this config (0 for an
 * invalid config or when one row's scratch exceeds the array). */
int aio_prefill_noalloc_rows(const aio_config* cfg);

/* The probe's routing decision (Section 3.2 and Section 3.3, "Dynamic
 * Policy Routing and Execution"), pure host: the categories' scores are the
 * probe's logits of the n_categories label tokens (host array).  The
 * category is their argmax (lowest index on ties) and H(X) the Shannon
 * entropy, in nats, of their softmax.  The request goes to the small model
 * (return 1) when the category is `code_category`, ctx_len <= ctx_limit and
 * H(X) <= tau; otherwise to the large one (return 0).  *entropy and
 * *category receive H(X) and the category when not NULL.  Negative error
 * code (AIO_EINVAL: null logits; AIO_ERANGE: n_categories < 1 or
 * code_category outside [0, n_categories)) on bad arguments. */
int aio_probe_route(const float* category_logits, int32_t n_categories, int32_t code_category,
                    int32_t ctx_len, int32_t ctx_limit, float tau, float* entropy,
                    int32_t* category);

/* The probe's category scores on the device (Section 3.2): reads the
 * logits of the n_labels label tokens label_ids[0 .. n_labels) (host array
 * of vocabulary indices) from logits_dev (one fp32 row, e.g. what
 * aio_prefill wrote) and writes out_dev[0] = H(X), the Shannon entropy in
 * nats of their softmax, and out_dev[1] = the category (argmax, lowest index
 * on ties) as a float; the same values aio_probe_route computes on the host
 * from the same logits.  Enqueued on the model's stream; only the two floats
 * need to cross to the host for the routing decision (Section 3.3).
 * Returns AIO_EINVAL on null or misaligned pointers, AIO_ERANGE when
 * n_labels is outside [1, AIO_MAX_CATEGORIES] or a label id outside
 * [0, vocab). */
#define AIO_MAX_CATEGORIES 64
int aio_category_entropy(aio_model* m, const float* logits_dev, const int32_t* label_ids,
                         int32_t n_labels, float* out_dev);

/* ------------------------------------- draft-model speculative decoding */

typedef struct aio_spec_stats {
  int32_t rounds;      /* target forwards (verify calls plus single decode steps) */
  int32_t drafted;     /* draft tokens scored by the target                       */
  int32_t accepted;    /* draft tokens accepted                                   */
  int32_t draft_steps; /* decode steps of the draft model                         */
} aio_spec_stats;

/* Greedy generation with a draft model (Section 4.2, the DraftModel
 * baseline: the 1B model drafts for the 7B).  `target` and `draft` are two
 * resident models with the same vocabulary whose caches both hold the
 * sequence at positions 0..pos-1; `token` is consumed at pos.  Each round
 * the draft decodes up to k tokens greedily from the current token, the
 * target scores [token, drafts] in one aio_verify (one aio_decode_step when
 * no draft is wanted), and the longest prefix of drafts in which every draft
 * equals the target's argmax of the row before it is accepted; the target's
 * argmax after it is the next token.  When every draft is accepted the
 * draft model also consumes the last draft, so both caches hold the
 * sequence; rows past the accepted prefix are overwritten later, never
 * read.  out (host, n_new int32) receives the generated tokens, which equal
 * those of plain greedy decoding of the target.  target_logits_dev (fp32
 * [k+1][vocab]), draft_logits_dev (fp32 [vocab]), argmax_dev (int32 [k+1])
 * and draft_tokens_dev (int32 [k]) are scratch, each 16-byte aligned (the
 * int32 buffers 4-byte aligned); stats may be NULL.  Synchronises both
 * models' streams twice per round; returns AIO_EDEVICE as soon as either
 * model's device status word is found set.
 * AIO_EINVAL: a null handle or buffer, or vocabularies that differ.
 * AIO_ERANGE: token outside [0, vocab), pos < 0, n_new < 1, pos + n_new
 * beyond either cache, k < 0 or k + 1 > the target's max_verify. */
int aio_spec_generate(aio_model* target, aio_model* draft, int32_t pos, int32_t token,
                      int32_t n_new, int32_t k, float* target_logits_dev,
                      float* draft_logits_dev, int32_t* argmax_dev, int32_t* draft_tokens_dev,
                      int32_t* out, aio_spec_stats* stats);

/* --------------------------------------- several sequences in one pool */

/* The models above serve one sequence per handle.  A router (Section 3.1)
 * holds many requests, most of them behind shared templates (Section 3.2).
 * The operators below keep the keys and values of several sequences in one
 * pool of pages, attend over them, and score what a model answered.  They
 * take no handle but the hipStream_t they enqueue on (NULL = the default
 * stream): any layer of any model can use them, and aio_paged_forward runs a
 * whole model on them.  Device pointers belong to the current HIP device and
 * are 16-byte aligned unless stated otherwise; every scalar and every host
 * array is checked before anything is enqueued.  What lies in device memory
 * (lengths, page ids) cannot be checked on the host: the kernels bound it, so
 * no value there makes them read or write outside the buffers described.  No
 * call allocates, synchronises or keeps state, so all of them can be captured
 * into a HIP graph (which keeps the pointers and host values of the capture). */

/* Element types of rows and logits. */
enum { AIO_F32 = 0, AIO_BF16 = 1 };

/* Keys and values of one layer, bf16, in pages: slot s of kv head h of page p
 * is the head_dim elements at p page_stride + h head_stride + s head_dim. */
typedef struct aio_paged_kv {
  void* k_dev;
  void* v_dev;
  int64_t page_stride; /* elements, a multiple of 8                        */
  int64_t head_stride; /* elements, a multiple of 8                        */
  int32_t n_pages;
  int32_t page_size;   /* positions per page: a power of two, 8 .. 256      */
  int32_t n_kv_heads;
  int32_t head_dim;    /* 64 or 128                                         */
} aio_paged_kv;

/* Keys and values of one layer, bf16, of several sequences packed behind one
 * another: row t of kv head h is the head_dim elements at t row_stride +
 * h head_stride. */
typedef struct aio_packed_kv {
  const void* k_dev;
  const void* v_dev;
  int64_t row_stride;  /* elements, a multiple of 8                         */
  int64_t head_stride; /* elements, a multiple of 8                         */
  int32_t n_rows;
  int32_t n_kv_heads;
  int32_t head_dim;    /* 64 or 128                                         */
} aio_packed_kv;

/* The sequences of a call.  Sequence i has the rows cu_q[i] .. cu_q[i+1] - 1
 * (cu_q_dev NULL: row i, one new token each, n_rows == n_seqs), which are the
 * last of its keys: its keys number lens[i] in pages, cu_k[i+1] - cu_k[i]
 * packed, and row r of its q rows sees keys 0 .. keys - q + r.  In pages,
 * key j is slot j mod page_size of page table[i][j / page_size].  A page id
 * outside [0, n_pages) is a hole (an evicted page): its keys are seen by no
 * row.  Keys past max_len or past the table's width are not there either, and
 * change no row's own place.  A row that sees no key gets zeros and the
 * log-sum-exp -infinity; rows of no sequence are left as they are.  What the
 * places hold that a row does not see (infinities and NaN among it) does not
 * reach it. */
typedef struct aio_seqs {
  int32_t n_seqs;
  int32_t n_rows;            /* rows of q and out (of k and v rows to append) */
  int32_t max_len;           /* no sequence has more keys; at most 2^30       */
  const int32_t* cu_q_dev;   /* [n_seqs + 1], ascending from 0, or NULL       */
  const int32_t* lens_dev;   /* pages: [n_seqs] keys, the new rows among them */
  const int32_t* table_dev;  /* pages: [n_seqs][table_stride] page ids        */
  int32_t table_stride;      /* its width, all of it readable                 */
  const int32_t* cu_k_dev;   /* packed: [n_seqs + 1], ascending from 0        */
} aio_seqs;

/* Queries and outputs of an attention: [n_rows][n_heads][head_dim], fp32 or
 * bf16 (both the same), rows q_stride and out_stride elements apart (whole
 * numbers of 16 bytes; output rows must not overlap).  out_dev may be q_dev with
 * the same stride.  fp32 queries keep fp32 accuracy throughout (exact
 * splits into three bf16 terms, of the queries and of the softmax weights);
 * with bf16 ones the softmax weights are rounded to bf16 too.  Sums and
 * softmax statistics are fp32 in both, long ones carried in two floats (the
 * weights' sum always, the outputs of fp32 queries).  A value that is not
 * finite makes the outputs that see it not finite (infinite or NaN), however
 * little it weighs, and no others; a key that is not finite may do so to the
 * rows that see it, or weigh nothing, its value included, where a score is
 * -infinity.  Query head h reads kv head h / (n_heads / n_kv_heads). */
typedef struct aio_attn {
  const void* q_dev;
  void* out_dev;
  float* lse_dev;     /* fp32 [n_rows][n_heads], natural log, or NULL        */
  int64_t q_stride;
  int64_t out_stride;
  int32_t dtype;      /* AIO_F32 or AIO_BF16                                 */
  int32_t n_heads;    /* a multiple of n_kv_heads, at most 16 times as many  */
  float scale;        /* of the scores, > 0 (1 / sqrt(head_dim))             */
} aio_attn;

/* Bytes of workspace that an attention over these sequences takes (0: none;
 * its ws_dev may then be NULL): the partial results of a split over the keys.
 * Pure host, reads only the sizes and whether cu_q_dev and cu_k_dev are
 * NULL.  What the workspace holds does not matter, before or after; calls
 * that may overlap need one each.  Returns 0 for bad sizes, too. */
size_t aio_attn_workspace_bytes(const aio_seqs* s, int32_t n_heads, int32_t n_kv_heads,
                                int32_t head_dim);

/* Attention over paged keys and values: of one new token per sequence
 * (cu_q_dev NULL), the decode step of several requests, or of the rows of
 * several prompts, each behind what its pages hold already (a cached template,
 * an earlier turn).  The rows' own keys have to be in the pages
 * (aio_page_append).  An idle place in a padded batch has lens 0.
 * AIO_EINVAL: a null or misaligned pointer or stride, a bad shape or type, a
 * scale that is not positive and below 2.3e38, or a workspace smaller than
 * aio_attn_workspace_bytes says.  AIO_ERANGE: negative counts, cu_q_dev NULL with n_rows !=
 * n_seqs, or more work than one launch covers.  AIO_EUNSUPPORTED: a page
 * size, head dimension or number of heads per kv head not listed above. */
int aio_paged_attention(const aio_paged_kv* kv, const aio_seqs* s, const aio_attn* a,
                        void* ws_dev, size_t ws_bytes, void* hip_stream);

/* Causal attention over the rows of several prompts whose keys and values are
 * packed behind one another (cu_q_dev and cu_k_dev; lens and table are not
 * read).  A sequence may have more keys than rows (its rows are the last
 * ones); rows before its first key see nothing.  Errors as
 * aio_paged_attention. */
int aio_packed_attention(const aio_packed_kv* kv, const aio_seqs* s, const aio_attn* a,
                         void* ws_dev, size_t ws_bytes, void* hip_stream);

/* Writes the new rows' keys and values (fp32 or bf16, [n_rows][n_kv_heads]
 * [head_dim], rows row_stride and heads head_stride elements apart, both whole
 * numbers of 16 bytes) into their pages: row r of sequence i's q rows is key lens[i] - q + r.
 * fp32 is rounded to the nearest bf16, ties to even, as everywhere in a cache.
 * A row that falls before key 0, past max_len or the table's width, or into a hole
 * is not written.  Two sequences of one call must not write the same slot
 * (aio_pages_extend sees to that), nor may pages or heads of the pool, or its K
 * and V, overlap (AIO_EINVAL where two strides show it).  Errors as
 * aio_paged_attention. */
int aio_page_append(const aio_paged_kv* kv, const aio_seqs* s, const void* k_rows_dev,
                    const void* v_rows_dev, int32_t dtype, int64_t row_stride,
                    int64_t head_stride, void* hip_stream);

/* Keys and values of one layer in pages of 8-bit codes: slot s of kv head h of
 * page p is the head_dim int8 codes at byte p page_stride + h head_stride +
 * s head_dim and one unsigned byte b at p exp_page_stride + h exp_head_stride +
 * s of k_exp_dev or v_exp_dev; its elements are code 2^(b - 127), half the bytes
 * of a bf16 page.  b lies from 8 to 248; b = 255 with codes of 0 stands for a
 * row that held something not finite, and reads as NaN.  (Codes and bytes of a
 * page that lie behind one another are one copy for aio_page_copy.) */
typedef struct aio_q8_kv {
  void* k_dev;
  void* v_dev;
  void* k_exp_dev;         /* 8-byte aligned                                 */
  void* v_exp_dev;         /* 8-byte aligned                                 */
  int64_t page_stride;     /* bytes, a multiple of 16                        */
  int64_t head_stride;     /* bytes, a multiple of 16                        */
  int64_t exp_page_stride; /* bytes, a multiple of 8                         */
  int64_t exp_head_stride; /* bytes, a multiple of 8                         */
  int32_t n_pages;
  int32_t page_size;       /* positions per page: a power of two, 8 .. 256   */
  int32_t n_kv_heads;
  int32_t head_dim;        /* 64 or 128                                      */
} aio_q8_kv;

/* aio_page_append into pages of 8-bit codes.  For a head's row of K or V with
 * the largest magnitude A, b is the least from 8 to 248 for which A / 2^(b - 127),
 * rounded to the nearest integer, ties to even, is at most 127 (248 where none is),
 * and the codes are the elements over 2^(b - 127), rounded alike and held to 127: an
 * element is off by at most A / 127, or by 2^-120 where that is more.  A row with an infinity
 * or NaN gets b = 255 and codes of 0.  Which rows are written, and the errors, as
 * aio_page_append; pages, heads, K and V, codes and bytes must not overlap
 * (AIO_EINVAL). */
int aio_q8_append(const aio_q8_kv* kv, const aio_seqs* s, const void* k_rows_dev,
                  const void* v_rows_dev, int32_t dtype, int64_t row_stride,
                  int64_t head_stride, void* hip_stream);

/* aio_paged_attention over pages of 8-bit codes (an element is exactly a bf16,
 * so nothing is rounded on the way to the products; but for one new token per
 * sequence the powers of two go to the weights, which bf16 terms hold to 2^-133:
 * outputs are off by another 2^-126 n / l, of n keys and the sum l of their weights
 * over the largest, which values below 2^-100 show).  Its workspace is
 * aio_q8_workspace_bytes's.  Errors as aio_paged_attention. */
int aio_q8_attention(const aio_q8_kv* kv, const aio_seqs* s, const aio_attn* a, void* ws_dev,
                     size_t ws_bytes, void* hip_stream);

/* Bytes of workspace that an attention over 8-bit pages takes, as
 * aio_attn_workspace_bytes. */
size_t aio_q8_workspace_bytes(const aio_seqs* s, int32_t n_heads, int32_t n_kv_heads,
                              int32_t head_dim);

/* Groups of sequences that begin with the same keys (requests behind one
 * template): group g is the sequences cu_seqs[g] .. cu_seqs[g + 1] - 1, whose
 * first prefix_lens[g] keys are alike.  Sequences of no group share nothing. */
typedef struct aio_prefixes {
  int32_t n_groups;                /* at most 2^30                           */
  int32_t max_prefix;              /* more keys than that are not shared     */
                                   /* (see aio_prefix_attention)             */
  const int32_t* cu_seqs_dev;      /* [n_groups + 1], ascending              */
  const int32_t* prefix_lens_dev;  /* [n_groups]                             */
} aio_prefixes;

/* aio_paged_attention that reads a group's first keys once for all of its
 * rows instead of once for each sequence: the same results up to rounding.
 * They are read through the table of the group's first sequence, up to its
 * own length, in whole multiples of 64; the others' tables have to list pages of the
 * same contents (a fork's are the same pages).  A sequence that is not
 * to share (an idle place with lens 0, new rows that begin within the prefix)
 * computes all of its keys by itself.  max_len - max_prefix is taken for the number of
 * keys that a sequence has beyond its prefix, which are split by that: state max_prefix
 * closely where they are many (one sequence of 32768 keys on 8 kv heads behind 1024: 38
 * us with 1024, 107 with max_len, 35 without groups).  Sharing does not pay where the rows of
 * prompts fill whole tiles by themselves, nor for few shared keys.  Its workspace is
 * aio_prefix_workspace_bytes's.  Errors as aio_paged_attention; AIO_EINVAL: a null
 * or misaligned array of the groups; AIO_ERANGE: negative counts, or more groups than 2^30. */
int aio_prefix_attention(const aio_paged_kv* kv, const aio_seqs* s, const aio_prefixes* x,
                         const aio_attn* a, void* ws_dev, size_t ws_bytes, void* hip_stream);

/* The same over pages of 8-bit codes. */
int aio_q8_prefix_attention(const aio_q8_kv* kv, const aio_seqs* s, const aio_prefixes* x,
                            const aio_attn* a, void* ws_dev, size_t ws_bytes, void* hip_stream);

/* Bytes of workspace that an attention with these groups takes, as
 * aio_attn_workspace_bytes; of the groups only the two numbers are read. */
size_t aio_prefix_workspace_bytes(const aio_seqs* s, const aio_prefixes* x, int32_t n_heads,
                                  int32_t n_kv_heads, int32_t head_dim);

/* Query and key rows to be normalised and rotated: [n_rows][heads][head_dim],
 * all fp32 or all bf16, rows the strides apart (whole numbers of 16 bytes; rows
 * of outputs must not overlap). */
typedef struct aio_qk_rows {
  const void* q_dev;
  const void* k_dev;
  void* q_out_dev;
  void* k_out_dev;
  int64_t q_stride;
  int64_t k_stride;
  int64_t q_out_stride;
  int64_t k_out_stride;
  int32_t dtype;       /* AIO_F32 or AIO_BF16 */
  int32_t n_rows;
  int32_t n_heads;
  int32_t n_kv_heads;
  int32_t head_dim;    /* 64 or 128           */
} aio_qk_rows;

/* RMS norm of each head of the query and key rows, then the rotation by the
 * row's position, in one pass: y = w x / sqrt(mean x^2 + eps), and for i below
 * head_dim / 2 with t = position base^(-2i / head_dim) the pair (y_i,
 * y_(i + head_dim / 2)) turned by t.  positions_dev: int32 [n_rows], any value;
 * q_weight_dev and k_weight_dev: bf16 [head_dim], or NULL for 1.  Angles are
 * computed in 64 bits, the rest in 32, rounded once to the outputs' type.  An output
 * may take its input's place (the same pointer and stride); otherwise outputs
 * overlap nothing.  AIO_EINVAL: a null or misaligned pointer or stride, a bad
 * type, outputs that overlap, eps not positive and finite, base not above 1 and
 * finite; AIO_ERANGE: n_rows outside [0, 2^24) or heads outside [1, 2^16];
 * AIO_EUNSUPPORTED: another head dimension. */
int aio_qk_norm_rope(const aio_qk_rows* r, const int32_t* positions_dev,
                     const void* q_weight_dev, const void* k_weight_dev, float eps, float base,
                     void* hip_stream);

/* Copies pages in every plane of a pool (a plane: K or V of one layer):
 * page_bytes bytes from page src[i] to page dst[i] of each of n_planes planes,
 * which are plane_bytes apart, pages page_stride_bytes apart (all three whole
 * numbers of 16, page_stride_bytes >= page_bytes).  src and dst are host
 * arrays of n entries, read before the call returns.  AIO_ERANGE: n
 * outside [0, 2^31 - 2^16], n_planes outside [1, 2^31 - 2^16] or a page id
 * outside [0, n_pages).  AIO_EINVAL: a page that is the destination of two
 * copies or both source and destination (the copies run at once, so their
 * order would matter), planes or pages that overlap, or a null or misaligned
 * argument. */
int aio_page_copy(void* pool_dev, int32_t n_planes, int64_t plane_bytes, int32_t n_pages,
                  int64_t page_stride_bytes, int64_t page_bytes, const int32_t* src,
                  const int32_t* dst, int32_t n, void* hip_stream);

/* A whole model's paged cache: layer l's keys and values are those of `first`
 * l layer_stride elements further on. */
typedef struct aio_paged_pool {
  aio_paged_kv first;
  int64_t layer_stride; /* elements, a multiple of 8 */
  int32_t n_layers;
} aio_paged_pool;

/* The most rows of one aio_paged_forward. */
#define AIO_MAX_PAGED_ROWS 2048

/* One pass of a model over the next tokens of several sequences, whose keys
 * and values live in pages instead of the handle's own cache: decode steps,
 * prompts and continued prompts together, the layers' weights read once for all
 * of them (the products of aio_prefill, aio_page_append and aio_paged_attention
 * per layer), the LM head's once for every max_verify of the rows asked for.  Host arrays: sequence i consumes rows[i] >= 0 tokens (`tokens`
 * holds them one sequence after the other, at most AIO_MAX_PAGED_ROWS in all)
 * at positions lens[i] - rows[i] .. lens[i] - 1, and its pages are
 * table[i][0 .. table_stride); a page id below 0 is a hole, allowed before the
 * page of its first new token.  Every row attends over the sequence's keys up
 * to its own.  The logits (fp32 [n_out][vocab]) of rows out_rows[0 .. n_out) of the
 * packed tokens go to logits_dev (16-byte aligned): the last row of each
 * sequence to generate, every row to score a prompt or drafts.  Rows equal
 * those of aio_prefill or aio_decode_step on a cache of their own up to
 * rounding.  scratch_dev: aio_paged_forward_bytes bytes, 256-byte aligned, its
 * contents of no matter.  Enqueued on the model's stream; the host arrays are
 * read before the call returns (which waits for the stream's earlier work only
 * if they hold megabytes: 1 MB is copied in 0.4 ms, 4 MB are waited for).  Not for graph capture (it copies from host
 * memory): AIO_EINVAL where the stream is captured.
 * AIO_EINVAL: a null or misaligned pointer, a pool whose shape is not the
 * model's or whose layers, K and V, pages or heads overlap (where two strides
 * show it), a scratch too small, or two sequences that would write the same page.
 * AIO_ERANGE: counts (n_out up to 2^31 - 2^16), lengths (up to max_ctx and the
 * table's width), tokens, pages or out_rows out of range. */
int aio_paged_forward(aio_model* m, const aio_paged_pool* pool, int32_t n_seqs,
                      const int32_t* rows, const int32_t* lens, const int32_t* table,
                      int32_t table_stride, const int32_t* tokens, const int32_t* out_rows,
                      int32_t n_out, float* logits_dev, void* scratch_dev, size_t scratch_bytes);

/* Scratch bytes for up to n_rows rows of up to n_seqs sequences with tables
 * up to table_stride wide (0 for a bad config or sizes).  Pure host. */
size_t aio_paged_forward_bytes(const aio_config* cfg, int32_t n_seqs, int32_t n_rows,
                               int32_t table_stride);

/* Log probabilities of logit rows ([rows][n], fp32 or bf16, rows `stride`
 * elements apart, 4- or 2-byte aligned): logprob[r] = x[target[r]] - log sum_j
 * e^x[j], entropy[r] the Shannon entropy in nats of the row's softmax, and the
 * `top` largest logits' indices and log probabilities, largest first, the
 * lower index first among equals; NaN ranks above +Inf, as in aio_argmax.
 * Scores the tokens of a prompt, a verify forward's drafts, or an answer.
 * targets_dev (int32 [rows]) may be NULL with logprob_dev; a target outside
 * [0, n) has none, and its logprob is NaN.  entropy_dev may be NULL;
 * top_ids_dev (int32 [rows][top]) and top_logprobs_dev (fp32 [rows][top]) may
 * be NULL where top is 0.  -Inf logits (forbidden tokens) have probability 0;
 * a row of nothing else, or one with a NaN or +Inf, gives NaN.  ws_dev: see
 * aio_logprobs_workspace_bytes.  AIO_ERANGE: rows outside [0, 2^31 - 2^16], n
 * outside [1, 2^30], stride < n or top outside [0, min(n, AIO_MAX_TOP)];
 * AIO_EINVAL: null or misaligned pointers, a bad type or too small a workspace. */
#define AIO_MAX_TOP 32
int aio_logprobs(const void* logits_dev, int32_t dtype, int32_t rows, int32_t n, int64_t stride,
                 const int32_t* targets_dev, int32_t top, float* logprob_dev, float* entropy_dev,
                 int32_t* top_ids_dev, float* top_logprobs_dev, void* ws_dev, size_t ws_bytes,
                 void* hip_stream);

/* Bytes of workspace aio_logprobs takes (0: none), as
 * aio_attn_workspace_bytes. */
size_t aio_logprobs_workspace_bytes(int32_t rows, int32_t n, int32_t top);

/* ----------------------------------------------- page tables (pure host) */

/* Which pages of a pool each sequence holds.  Pages are counted per sequence
 * that holds them: a fork shares its parent's, and the first to write into a
 * shared, partly filled page gets a copy of it.  A handle is not thread-safe
 * and makes no device call: the caller enqueues the copies that it is told
 * (aio_page_copy), before anything that writes to the pool afterwards. */
typedef struct aio_pages aio_pages;

/* AIO_ERANGE: n_pages or max_seqs outside [1, 2^30] or a page size that
 * aio_paged_kv does not take. */
int aio_pages_create(int32_t n_pages, int32_t page_size, int32_t max_seqs, aio_pages** out);
void aio_pages_destroy(aio_pages* p);

/* A new, empty sequence; *seq receives its number, the lowest that is not in
 * use.  AIO_ENOMEM: max_seqs are open. */
int aio_pages_open(aio_pages* p, int32_t* seq);
/* Drops the sequence; pages that no other one holds are free again. */
int aio_pages_close(aio_pages* p, int32_t seq);
/* A new sequence of the same contents, which holds the same pages. */
int aio_pages_fork(aio_pages* p, int32_t seq, int32_t* child);
/* Room for n more positions.  *n_copies (0 or 1) receives how many pages have
 * to be copied first, *src and *dst which.  AIO_ENOMEM: too few free pages
 * (nothing has changed then); AIO_ERANGE: n < 0 or over 2^30 positions. */
int aio_pages_extend(aio_pages* p, int32_t seq, int32_t n, int32_t* src, int32_t* dst,
                     int32_t* n_copies);
/* Keeps the first len positions (after rejected drafts, say). */
int aio_pages_truncate(aio_pages* p, int32_t seq, int32_t len);
/* Moves the pages in use to the front of the pool: src and dst (room for
 * `room` entries each) receive the *n copies to enqueue, at once, before any
 * other use of the pool.  AIO_ERANGE: room is too small (nothing has changed;
 * *n says how many are needed). */
int aio_pages_compact(aio_pages* p, int32_t* src, int32_t* dst, int32_t room, int32_t* n);
/* The sequence's length and its row of a page table: `width` ids, -1 behind
 * the last.  row may be NULL.  AIO_ERANGE: width is too small. */
int aio_pages_row(const aio_pages* p, int32_t seq, int32_t* row, int32_t width, int32_t* len);
/* Pages that no sequence holds (AIO_EINVAL: null). */
int aio_pages_free(const aio_pages* p);

#ifdef __cplusplus
}
#endif
#endif /* AIO_H */
