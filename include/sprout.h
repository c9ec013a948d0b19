/*
 * sprout.h -- C ABI of the MI355X (gfx950) batched, ragged-length Llama-2
 * greedy decode library.
 *
 * The operation is the inference server's hot loop in Sprout (arXiv
 * 2403.12900): autoregressive generation with a KV cache, where every request
 * carries a generation-directive prefix placed before its prompt and stops at
 * its own generation limit.  Section II-A defines the loop (predict the next
 * token until EOS or a preset limit; cached keys/values of earlier tokens are
 * reused); Definition 1 and Section III-E fix the token order (directive
 * first, as a system prompt ahead of the user prompt); Section IV names the
 * served model (Llama 2).  The model is a random-init Llama-2 architecture
 * drawn on the device from a seed.
 *
 * Conventions for every entry point:
 *   - Return value: SPR_OK (0) or a negative spr_status.  No exception or
 *     longjmp crosses the ABI.  spr_last_error() gives a message for the last
 *     failure on the calling thread.
 *   - Arguments are validated against the model's state before anything is
 *     enqueued; a call that fails validation changes no state.
 *   - A HIP runtime failure (SPR_ERR_HIP) is sticky: every later call on that
 *     model returns SPR_ERR_HIP; the model must be released.
 *   - Device-side checks: a decode step fed a token id outside [0, vocab)
 *     (possible only through the caller-written device token buffer), or a
 *     logits row holding a NaN or no finite maximum, sets a flag in mapped
 *     host memory.  The first call that starts after the faulty work has
 *     completed on the device returns SPR_ERR_DEVICE_CHECK, and so does every
 *     later call: the model must be released.  (The step itself reads the
 *     clamped id, or emits token 0, so no access leaves its buffers.)
 *   - Pointers marked "host" are read (or written) during the call only.
 *     Pointers marked "device" must stay valid until the work enqueued on the
 *     model's stream has completed; device outputs are valid once the caller
 *     has synchronised that stream.
 *   - Calls on one model are not re-entrant and must come from one thread at
 *     a time.  Work is enqueued on the HIP stream given at init.
 */
#ifndef SPROUT_H_
#define SPROUT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SPR_OK = 0,
  SPR_ERR_INVALID_ARG = -1, /* malformed argument or unsupported shape */
  SPR_ERR_WORKSPACE = -2,   /* workspace missing, misaligned or too small */
  SPR_ERR_KV_FULL = -3,     /* not enough free KV-cache blocks */
  SPR_ERR_STATE = -4,       /* call does not match the slot state */
  SPR_ERR_HIP = -5,         /* HIP runtime error (sticky) */
  SPR_ERR_DEVICE_CHECK = -6 /* a device-side check of an earlier call failed (sticky) */
} spr_status;

typedef enum { SPR_F32 = 0, SPR_BF16 = 1 } spr_dtype;

/*
 * Model shape and capacity.  Llama-2 architecture (Section IV): pre-norm
 * decoder layers of RMSNorm -> attention with rotary position embedding ->
 * residual, RMSNorm -> SwiGLU MLP -> residual; untied embedding and LM head;
 * no biases.  Weights are stored in `dtype` and the KV cache in `kv_dtype`
 * (keys and values are rounded to it, nearest-even, when cached); the
 * residual stream, norms, softmax, accumulation and logits are fp32.
 *
 * Constraints: n_layers 1..255; head_dim 64 or 128; n_heads a multiple of
 * n_kv_heads with n_heads / n_kv_heads <= 16; d_model a multiple of 16;
 * d_ff, vocab >= 1; kv_block must be 16; max_slots 1..64; max_ctx >= 1;
 * kv_blocks >= 1 (the shared pool of 16-position blocks).
 */
typedef struct {
  int32_t n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ff, vocab;
  float rope_base; /* 10000 for Llama 2 */
  float rms_eps;   /* 1e-5 for Llama 2 */
  int32_t dtype;   /* spr_dtype */
  int32_t kv_block;  /* positions per KV block: 16 */
  int32_t max_slots; /* concurrent requests */
  int32_t max_ctx;   /* positions per request: prompt + generated - 1 */
  int32_t kv_blocks; /* KV blocks in the pool */
  int32_t kv_dtype;  /* spr_dtype of the KV cache; fp32 models need SPR_F32 */
} spr_config;

typedef struct spr_model spr_model; /* opaque, library-owned host state */

/* Device bytes the caller must provide for `cfg` (0 if cfg is invalid). */
size_t spr_workspace_bytes(const spr_config* cfg);

/*
 * Creates a model in the caller's device workspace and draws its weights on
 * the device.  dev_ws: device pointer, 256-byte aligned, ws_bytes >=
 * spr_workspace_bytes(cfg); owned by the caller, who keeps it alive until
 * spr_release.  The library allocates no device memory of its own.
 * hip_stream: a hipStream_t (NULL = the null stream).  Weight element (r, c)
 * of each matrix is the counter-based N(0, 0.02) draw of its row-major index
 * (SplitMix64 outputs -> Irwin-Hall sum of eight 16-bit lanes -> one fp32
 * multiply -> round to `dtype`); all RMSNorm gains are 1.  Synchronous: the
 * weights are ready when it returns.  *out receives the model.
 */
spr_status spr_init(const spr_config* cfg, uint64_t seed, void* dev_ws, size_t ws_bytes, void* hip_stream,
                    spr_model** out);

/*
 * Prefill: fills the KV cache of n new requests with their prompts and emits
 * each one's first generated token (Section II-A: the prompt populates the
 * cache; generation follows).  A request's prompt is its directive prefix
 * followed by its user prompt (Section III-E), at positions 0..seq_len-1.
 *   slots      host [n]: distinct free slot ids in [0, max_slots)
 *   tokens     host [sum(seq_lens)]: the prompts, concatenated in order
 *   seq_lens   host [n]: >= 1
 *   stop_lens  host [n]: tokens to generate, >= 1, seq_len + stop_len - 1 <= max_ctx
 *   tok        device int32 [max_slots], indexed by slot: tok[slot] receives
 *              the first generated token
 *   logits     device fp32 [n, vocab] or NULL: logits of each last prompt position
 *   retired    host int32 [n] or NULL: 1 where stop_len == 1 (the request is done)
 * KV blocks for seq_len + stop_len - 1 positions are reserved per request;
 * the call fails with SPR_ERR_KV_FULL (and reserves nothing) if the pool
 * cannot hold them all.
 */
spr_status spr_prefill(spr_model* m, int32_t n, const int32_t* slots, const int32_t* tokens,
                       const int32_t* seq_lens, const int32_t* stop_lens, int32_t* tok, float* logits,
                       int32_t* retired);

/*
 * One decode step over the active requests (Section II-A's loop, one
 * iteration for each request in the batch).  Each listed slot feeds
 * tok[slot] at position lens[k], attends to its cached positions 0..lens[k],
 * and tok[slot] is overwritten with the greedy (lowest index on ties) next
 * token.  tok may therefore be the buffer the previous step wrote
 * (free-running greedy decode without a host round trip) or hold tokens the
 * caller forced.
 *   n_active   1..max_slots
 *   slots      host [n_active]: distinct active slots
 *   lens       host [n_active]: cached positions of each slot; must equal the
 *              library's count (SPR_ERR_STATE otherwise)
 *   tok        device int32 [max_slots], indexed by slot, read then written
 *   logits     device fp32 [n_active, vocab] or NULL: row k = logits of slots[k]
 *   retired    host int32 [n_active] or NULL: 1 where this step produced the
 *              slot's stop_len-th token; that slot then accepts no more steps
 *              until spr_rewind_slot, and keeps its KV blocks until
 *              spr_free_slot
 */
spr_status spr_decode_step(spr_model* m, int32_t n_active, const int32_t* slots, const int32_t* lens, int32_t* tok,
                           float* logits, int32_t* retired);

/*
 * spr_decode_step for callers that cannot allocate device memory or touch the
 * model's workspace scratch (code under HIP graph capture, tight serving
 * loops, harnesses that forbid allocation): identical arguments, semantics
 * and results, but the step's scratch -- split partials (of attention and of
 * the projections' split-K slices), arrival counters and the LM head's
 * greedy candidates -- lives in a fixed 24 MiB array in device memory that
 * the library holds on each device it runs on until the process ends.  The call allocates nothing and makes no
 * allocating runtime call; it clears the counters it uses with a kernel
 * before the step.  Every call on one device shares that device's array:
 * calls that overlap on one device (on different streams, or from different
 * threads) race and must not be issued.  SPR_ERR_INVALID_ARG when the model
 * or batch does not fit the array (more than 128 KV heads, a vocabulary
 * above 130048, n_heads * (head_dim + 4) * 4 bytes * n_active above 16 MiB)
 * or is wider than the call takes (d_model above 32784, d_ff or (n_heads + 2
 * * n_kv_heads) * head_dim above 30840); other errors as spr_decode_step.
 */
spr_status spr_decode_step_static_scratch(spr_model* m, int32_t n_active, const int32_t* slots, const int32_t* lens,
                                          int32_t* tok, float* logits, int32_t* retired);

/*
 * Rolls a prefilled slot back to `len` cached positions with `produced`
 * tokens generated.  The prompt stays: 1 <= produced <= the tokens produced
 * so far, and len == prompt length + produced - 1 (SPR_ERR_INVALID_ARG
 * otherwise; SPR_ERR_STATE for a free slot).  Positions >= len are dropped;
 * the slot is active again if produced < its stop length.  Used to
 * regenerate from a prompt.
 */
spr_status spr_rewind_slot(spr_model* m, int32_t slot, int32_t len, int32_t produced);

/* Returns a slot's KV blocks to the pool and frees the slot. */
spr_status spr_free_slot(spr_model* m, int32_t slot);

/* Cached positions of a slot (-1 if free) and tokens produced so far. */
spr_status spr_slot_info(const spr_model* m, int32_t slot, int32_t* len, int32_t* produced, int32_t* stop_len);

/* Free KV blocks in the pool. */
int32_t spr_free_blocks(const spr_model* m);

/*
 * Reads rows [row0, row0 + nrows) of one logical weight matrix back as fp32
 * (exact values), row-major, into device memory `out` [nrows, cols].
 * tensor: 0 embedding [vocab, d], 1 Wq [H*hd, d], 2 Wk [Hkv*hd, d],
 * 3 Wv [Hkv*hd, d], 4 Wo [d, H*hd], 5 W1 gate [d_ff, d], 6 W3 up [d_ff, d],
 * 7 W2 down [d, d_ff], 8 LM head [vocab, d].  For checking the device
 * generator against an independent one.
 */
spr_status spr_export_weight_rows(spr_model* m, int32_t tensor, int32_t layer, int32_t row0, int32_t nrows,
                                  float* out);

/*
 * Measurement aid: enqueues `reps` back-to-back launches of one projection
 * kernel exactly as a decode step over n_rows rows launches it (launch r uses
 * layer r mod n_layers, so every layer's weights are streamed in turn),
 * brackets them with HIP events on the model's stream, waits, and writes the
 * mean launch duration in microseconds to *avg_us.  projection: 1 = O
 * (x += o Wo^T), 2 = gate/up with SwiGLU, 3 = down (x += h W2^T), 4 = LM head
 * with the greedy candidates.  It reads and writes only the forward pass's
 * scratch buffers (activations, residual, greedy candidates), which every
 * decode step rewrites before reading, so cached state is untouched; the QKV
 * projection, which appends to the KV cache, is refused (SPR_ERR_INVALID_ARG).
 * n_rows 1..128, reps 1..100000.  Synchronous.
 */
spr_status spr_time_projection(spr_model* m, int32_t projection, int32_t n_rows, int32_t reps, float* avg_us);

/*
 * Test aid (for tests of the greedy tie rule and of the device checks; no
 * other caller needs it): overwrites row dst of the LM-head matrix, with row
 * src when src >= 0 (a planted exact tie: both rows then give bitwise equal
 * logits), else with `fill` rounded to the weight format (a NaN fill makes
 * every later logits row hold a NaN).  The model is changed for the rest of
 * its life.  dst in [0, vocab), src < vocab, else SPR_ERR_INVALID_ARG.
 * Synchronous.
 */
spr_status spr_test_write_lm_head_row(spr_model* m, int32_t dst, int32_t src, float fill);

/*
 * Measurement aid: the HBM read ceiling of the projections' load form.
 * Streams every weight matrix a decode step reads (all layers' projections
 * and the LM head, resident in the model's workspace) once per rep with
 * 16-byte nontemporal loads, 8 in flight per thread and no arithmetic, brackets
 * the reps with HIP events on the model's stream, waits, and writes the mean
 * read rate in GB/s (1e9 bytes/s) to *gbps and the bytes read per rep to
 * *bytes.  Reads only; model state is untouched.  reps 1..1000; null outputs
 * are SPR_ERR_INVALID_ARG.  Synchronous.
 */
spr_status spr_time_read_ceiling(spr_model* m, int32_t reps, double* gbps, uint64_t* bytes);

#define SPR_MAX_LEVELS 8 /* directive levels a serving run can profile */

/* One request of a serving run (host memory, read during the call). */
typedef struct {
  const int32_t* tokens; /* prompt: directive prefix followed by the user prompt */
  int32_t n_tokens;      /* >= 1 */
  int32_t stop_len;      /* generation limit, >= 1; n_tokens + stop_len - 1 <= max_ctx */
  int32_t arrival;       /* first scheduler iteration it may be admitted in (0 = at once) */
  int32_t level;         /* directive level (Definition 1), 0..SPR_MAX_LEVELS-1; profiling tag only */
} spr_request;

typedef struct {
  int64_t iterations;    /* scheduler iterations run */
  int64_t decode_steps;  /* decode steps launched */
  int64_t prefill_calls; /* batched prefills launched */
  int64_t decode_tokens; /* decode rows launched (tokens past an EOS included) */
  int32_t max_batch;     /* largest decode batch */
  double mean_batch;     /* mean decode batch */
  double device_seconds; /* device time from the call's first work to its last iteration */
  /* Per directive level, the profiles Eq. 2 consumes (p: processing time per
     request).  Each iteration's device time is shared equally by the
     requests it served; a request's time is the sum of its shares. */
  int32_t level_requests[SPR_MAX_LEVELS]; /* requests of the level */
  double level_tokens[SPR_MAX_LEVELS];    /* mean generated tokens (lengths) per request */
  double level_seconds[SPR_MAX_LEVELS];   /* p: mean device seconds per request */
} spr_serve_stats;

/*
 * Serves n requests with continuous (iteration-level) batching: the
 * scheduling of the inference servers the paper deploys on (Section IV:
 * vLLM's paged KV cache; related work: Orca's iteration-level batching),
 * here over the decode step above.  Every iteration
 *   1. admits waiting requests, first come first served, whose arrival
 *      iteration has come, into free slots while fewer than max_active
 *      requests are in flight and the KV pool can reserve their blocks (a
 *      request that does not fit yet holds back the ones behind it);
 *   2. prefills the admitted requests together (first tokens);
 *   3. runs one decode step over every request still generating;
 *   4. retires requests that reached their stop length, freeing their slots
 *      and KV blocks for the next iteration;
 *   5. retires requests whose previous-iteration token was eos_id (Section
 *      II-A: generation ends at EOS or at the preset limit).  The tokens are
 *      read back one iteration late, so the host never waits for the
 *      iteration it has just enqueued; such a request runs one more decode
 *      row (two if EOS was its prefill token), whose token is discarded.
 * Iterations with nothing in flight skip to the next arrival.  Outputs are
 * the greedy tokens each request would get served alone.
 *   max_active 1..max_slots
 *   eos_id     token id that ends a request, or negative for none
 *   tok        device int32 [max_slots]: scratch token buffer, indexed by slot
 *   out        device int32 [sum of stop_len]: request i's tokens at offset
 *              stop_len[0] + ... + stop_len[i-1]; entries past its length
 *              are unspecified
 *   lengths    host int32 [n] or NULL: tokens generated per request, up to
 *              and including the first EOS, else stop_len
 *   stats      host, or NULL
 * Needs every slot free on entry (SPR_ERR_STATE otherwise) and leaves them
 * free.  A malformed request, or one that max_ctx or the KV pool could never
 * hold, fails with SPR_ERR_INVALID_ARG before any work is enqueued.
 * Synchronous: out is complete when it returns.  Uses a few HIP events and,
 * with an EOS id, 16 * max_slots bytes of pinned host memory for the call.
 */
spr_status spr_serve(spr_model* m, int32_t n, const spr_request* reqs, int32_t max_active, int32_t eos_id,
                     int32_t* tok, int32_t* out, int32_t* lengths, spr_serve_stats* stats);

/* ---------------------------------------------------------------------------
 * Speculative decoding: several drafted tokens of a request are run through
 * the model in one pass, the ones that the target model's distribution
 * accepts are kept, and the rest leave no trace.  The loop is Section II-A's;
 * the accepted tokens are distributed as its own (equal to them where greedy).
 *
 * A request's drafted tokens form a tree of n_nodes nodes.  Node 0, the root,
 * is the request's last token (not yet cached); node j > 0 is a drafted token
 * that continues node parents[j] < j.  Node j's keys and values sit at cache
 * position len + j while the tree is open, whatever its depth; its rotary
 * position is len + depth(j).  Calls take the nodes of all requests as token
 * rows, request after request.
 *
 * The three operators (spr_tree_attention, spr_tree_verify, spr_tree_keep)
 * run on caller-owned tensors through an operator handle; spr_tree_step runs
 * them inside a whole model pass.
 * ------------------------------------------------------------------------ */

#define SPR_MAX_TREE_REQUESTS 64 /* requests of one call */
#define SPR_MAX_TREE_NODES 64    /* nodes of one request's tree */
#define SPR_MAX_TREE_ROWS 128    /* nodes of one call, over all requests */

/*
 * A paged KV cache.  Block b of layer l holds 16 positions of every KV head:
 * n_kv_heads tiles of 16 * head_dim elements from element
 * ((l * n_blocks + b) * n_kv_heads) * 16 * head_dim of k and of v.  Position t
 * of request i is position t % 16 of block block_table[slots[i]][t / 16].
 * With P = 16 / element size, element (t, d) of a tile (position t < 16,
 * dimension d) is at
 *   keys:   ((d / 4P) * 64 + (d % 4P) / P * 16 + t) * P + d % P
 *   values: fp32  (((d / 16) * 4 + t / 4) * 16 + d % 16) * 4 + t % 4
 *           bf16  ((((d / 32) * 4 + t / 4) * 16 + d % 16) * 2 + (d / 16) % 2) * 4 + t % 4
 * (keys as the matrix unit's operand of K q^T, values of V^T p).
 * Constraints: head_dim 64 or 128; n_kv_heads 1..512; n_layers, n_blocks,
 * n_slots, max_blocks >= 1; k and v 16-byte aligned.  A block id outside
 * [0, n_blocks) that a call meets in the table is read as block 0 and fails
 * the handle's next call (SPR_ERR_DEVICE_CHECK); spr_tree_keep then moves
 * nothing for that request.
 */
typedef struct {
  void* k; /* device */
  void* v; /* device */
  int32_t kv_dtype; /* spr_dtype */
  int32_t n_layers, n_blocks, n_kv_heads, head_dim;
  const int32_t* block_table; /* device [n_slots][max_blocks] */
  int32_t n_slots, max_blocks;
} spr_kv_view;

/*
 * The drafted trees of one call (host memory, read during the call).
 *   n        1..SPR_MAX_TREE_REQUESTS
 *   slots    [n]: distinct rows of the block table
 *   lens     [n]: cached positions before the tree, 0..2^30
 *   n_nodes  [n]: 1..SPR_MAX_TREE_NODES each, at most SPR_MAX_TREE_ROWS in all
 *   parents  [sum(n_nodes)]: -1 for each root (its first entry), else in
 *            [0, j) for node j
 * spr_tree_verify does not read slots and lens, which may then be NULL.
 */
typedef struct {
  int32_t n;
  const int32_t *slots, *lens, *n_nodes, *parents;
} spr_tree_batch;

typedef struct spr_tree_ops spr_tree_ops; /* opaque, library-owned host state */

/* Device bytes the caller must provide to spr_tree_ops_init. */
size_t spr_tree_ops_workspace_bytes(void);

/*
 * Creates an operator handle on the current device, in the caller's device
 * workspace (256-byte aligned, kept alive until the release) and on the given
 * HIP stream.  The library allocates no device memory of its own.  The
 * conventions at the top of this file hold, with the handle in the model's
 * place: status codes, sticky HIP errors, device checks (a block id or a
 * drafted token out of range, a logits row with a NaN or no finite maximum,
 * a malformed path), and one thread at a time.  Operators enqueue kernels
 * only and may be captured into a graph; a captured call keeps the host
 * arguments it was given.  Calls of one handle share its workspace: run its
 * graphs and its eager calls one after the other, and give concurrent streams
 * a handle each.  Calls may come while another device is current.  Release a
 * handle when its work, and its graphs' last replay, have completed.
 */
spr_status spr_tree_ops_init(void* dev_ws, size_t ws_bytes, void* hip_stream, spr_tree_ops** out);

/*
 * Later calls enqueue on hip_stream.  The caller orders it after the work that
 * the handle's earlier calls put on another stream.
 */
spr_status spr_tree_ops_set_stream(spr_tree_ops* ops, void* hip_stream);

/* Releases the host state.  The workspace is the caller's to free afterwards. */
spr_status spr_tree_ops_release(spr_tree_ops* ops);

/*
 * Attention of drafted trees over the cache, for layer `layer` of the view:
 * row r = (request i, node j) and head h attend to positions 0..lens[i]-1 and
 * to positions lens[i] + a for a = j and every ancestor a of j,
 *   out[r][h] = softmax(q[r][h] . K^T / sqrt(head_dim)) V
 * (head h reads KV head h / (n_heads / n_kv_heads)).  The nodes' keys and
 * values are in the cache already.  One-node trees are ordinary decode
 * attention.  What lies in the cache behind a request's nodes, or at nodes
 * that a row does not see, does not reach its output, whatever it holds (a row
 * that sees an infinite key or value may get NaN where the formula gives it no
 * weight or an infinity: operands enter the products in parts).
 *   n_heads    a multiple of n_kv_heads, n_heads / n_kv_heads <= 16
 *   io_dtype   of q and out; scores, sums and products are held in fp32, the
 *              probabilities of bf16 outputs over a bf16 cache to 2^-16
 *   q          device [rows] x [n_heads * head_dim], row r at q + r * q_stride
 *              elements; out likewise.  16-byte aligned, strides a multiple of
 *              16 bytes and >= n_heads * head_dim.  out must not overlap q.
 * SPR_ERR_INVALID_ARG also where lens[i] + n_nodes[i] exceeds max_blocks * 16.
 */
spr_status spr_tree_attention(spr_tree_ops* ops, const spr_kv_view* kv, int32_t layer, const spr_tree_batch* batch,
                              int32_t n_heads, int32_t io_dtype, const void* q, int64_t q_stride, void* out,
                              int64_t out_stride);

/*
 * Verification of drafted tokens against the target's distribution, from the
 * caller's random numbers (speculative sampling).  logits row r = (request i,
 * node u) are the target's logits after node u; p = softmax(logits / T), T the
 * request's temperature.  From the root on, the children x_1, x_2, ... of the
 * node reached are tried in node order, with r_0 = p:
 *   child x_k is accepted, and becomes the node reached, if
 *     accept[its row] * q(x_k) < r_{k-1}(x_k);
 *   else r_k = max(r_{k-1} - q, 0) / sum.
 * q is the node's row of draft_probs (the distribution its children were drawn
 * from; entries that are negative or NaN count as 0) or, with draft_probs
 * NULL, a point mass at x_k.  Where no child is left, the next token is the
 * lowest t whose cumulative weight sum_{s <= t} r(s) exceeds
 * sample[i] * sum r (the last t of positive weight if none does), and the walk
 * ends; a node all of whose r is gone (possible only where draft_probs do not
 * sum to 1) draws from p.  T = 0 is greedy: a child is accepted if it is the
 * row's argmax (lowest index on ties), and the argmax is the next token.
 * Probabilities and their sums are held in fp64.
 *   vocab         1..1048576
 *   dtype         of logits and draft_probs; row r at r * stride elements
 *   tokens        device int32 [rows]: the drafted tokens (roots' are not read);
 *                 one outside [0, vocab) is never accepted and fails the
 *                 handle's next call
 *   temperature   host [n], >= 0 and finite, or NULL: 1
 *   accept        device fp32 [rows]: uniform in [0, 1) (roots' are not read)
 *   sample        device fp32 [n]: uniform in [0, 1)
 *   emitted       device int32 [rows]: request i's accepted tokens and the next
 *                 token, from its root's row on, -1 behind them
 *   path          device int32 [rows]: the nodes walked, 0 first, likewise
 *   count         device int32 [n]: tokens emitted = nodes walked (accepted + 1);
 *                 0 (and -1 in every entry) where the walk met a logits row
 *                 with a NaN or no finite maximum
 */
spr_status spr_tree_verify(spr_tree_ops* ops, const spr_tree_batch* batch, int32_t vocab, int32_t dtype,
                           const int32_t* tokens, const void* logits, int64_t logits_stride, const void* draft_probs,
                           int64_t draft_stride, const float* temperature, const float* accept, const float* sample,
                           int32_t* emitted, int32_t* path, int32_t* count);

/*
 * Closes trees in the cache: in every layer, the keys and values of node
 * path[root row of i + k] move to position lens[i] + k for k < count[i].
 * Positions from lens[i] + count[i] on are left as they were or hold what
 * rejected nodes left there.  Per request, nodes 0 <= path[0] < path[1] < ...
 * < n_nodes[i] and count[i] <= n_nodes[i]; one that breaks this is left as it
 * is and fails the handle's next call.  count[i] < 1 moves nothing.  The blocks
 * that hold a request's nodes are its alone (cached ones may be shared).
 *   path    device int32 [rows], count device int32 [n]: as spr_tree_verify
 *           writes them
 */
spr_status spr_tree_keep(spr_tree_ops* ops, const spr_kv_view* kv, const spr_tree_batch* batch, const int32_t* path,
                         const int32_t* count);

/*
 * The model's own cache as a view (keys, values and block table in its
 * workspace; slots are its slot ids), for the operators above or for reading.
 */
spr_status spr_model_kv_view(spr_model* m, spr_kv_view* out);

/*
 * One decode step over drafted trees: every node runs through the model in
 * one pass (spr_tree_attention in each layer), spr_tree_verify picks each
 * request's path, and spr_tree_keep closes the trees in all layers.  With
 * one-node trees and temperature 0 it is a decode step.
 *   batch         slots: distinct active slots; lens: as in spr_decode_step.
 *                 The tree takes positions of the slot's reserved blocks:
 *                 lens[i] + n_nodes[i] must not exceed 16 * their number
 *                 (SPR_ERR_KV_FULL), and a tree has at most as many levels as
 *                 the slot still has tokens to generate (SPR_ERR_INVALID_ARG).
 *   tok           device int32 [max_slots], indexed by slot: the roots' tokens
 *                 are read from it, and each request's last emitted token is
 *                 written to it, so tree steps and decode steps alternate
 *                 freely
 *   tokens        device int32 [rows]: the drafted tokens (roots' are not read)
 *   draft_probs   device fp32 [rows, vocab] or NULL
 *   temperature, accept, sample, emitted: as in spr_tree_verify (accept and
 *                 sample may be NULL where every temperature is 0)
 *   logits        device fp32 [rows, vocab]: each node's logits
 *   count         host int32 [n]: tokens emitted, 1..levels of the tree
 *   retired       host int32 [n] or NULL: 1 where the slot reached its stop_len
 * Each slot advances by count[i] positions and tokens; spr_rewind_slot drops
 * them again.  Synchronous: the counts are the host's.  A drafted token
 * outside [0, vocab) or a bad logits row on the way fails this call
 * (SPR_ERR_DEVICE_CHECK), not the next.
 */
spr_status spr_tree_step(spr_model* m, const spr_tree_batch* batch, int32_t* tok, const int32_t* tokens,
                         const float* draft_probs, const float* temperature, const float* accept, const float* sample,
                         float* logits, int32_t* emitted, int32_t* count, int32_t* retired);

/* ---------------------------------------------------------------------------
 * A paged KV cache held in 4 bits (Section II-A's cached keys and values at a
 * quarter of bf16's bytes), and what a serving loop does with it: rotary
 * positions, appending a step's keys and values, reading them back, attention
 * over the cache, and the sharing and moving of its blocks.
 *
 * Stored values: 32 consecutive dimensions of one position and head share a
 * scale 2^s, s in -120..125, and each is a 4-bit code (sign, two exponent bits,
 * one mantissa bit) for +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} times that scale.  s is
 * the smallest with max|x| <= 7 * 2^s (so that no element is off by more than
 * half a step; from 7 * 2^125 on elements are cut to 6 * 2^125); an element is rounded to
 * the nearest value, of two as near the one whose code is even.  A group that
 * holds an infinity or a NaN is stored as NaN, all 32 of it.
 *
 * The operators run on caller-owned tensors through an operator handle of
 * their own, under the conventions of spr_tree_ops_init.
 * ------------------------------------------------------------------------ */

#define SPR_MAX_CACHE_REQUESTS 128  /* requests (or forks) of one call */
#define SPR_MAX_CACHE_ROWS 1048576  /* token rows of one call */

/*
 * Block b of layer l holds 16 positions of every KV head: n_kv_heads tiles of
 * 17 * head_dim bytes from byte ((l * n_blocks + b) * n_kv_heads) * 17 *
 * head_dim of data.  With P = head_dim / 32, position t < 16 and dimension d
 * of a tile:
 *   key codes    byte (d / 32 * 16 + t) * 16 + d % 32 / 2, low nibble for even d
 *   value codes  byte 8 * head_dim + ((t / 4 * 16 + d % 16) * P + d / 32) * 4 + t % 4,
 *                low nibble for d % 32 < 16
 *   key scales   byte 16 * head_dim + d / 32 * 16 + t: s + 127, or 255 for NaN
 *   value scales byte 16.5 * head_dim + (t / 4 * P + d / 32) * 4 + t % 4, likewise
 * (keys as the matrix unit's operand of K q^T, values of V^T p).  Constraints
 * and block ids outside the pool: as for spr_kv_view; data is 16-byte aligned.
 * Positions that a call attends to or reads hold what spr_cache_append wrote
 * (other scale bytes are not told apart from 2^(byte - 127)).
 */
typedef struct {
  void* data; /* device */
  int32_t n_layers, n_blocks, n_kv_heads, head_dim;
  const int32_t* block_table; /* device [n_slots][max_blocks] */
  int32_t n_slots, max_blocks;
} spr_kv4_view;

/*
 * The requests of one call (host memory, read during the call): request i's
 * rows are positions lens[i] .. lens[i] + rows[i] - 1 of its slot, and the
 * token rows of a call's tensors are those of all requests, one after the other.
 *   n      1..SPR_MAX_CACHE_REQUESTS
 *   slots  [n]: distinct rows of the block table
 *   lens   [n]: positions before the rows, 0..2^30
 *   rows   [n]: >= 1 each, at most SPR_MAX_CACHE_ROWS in all
 * lens[i] + rows[i] must not exceed max_blocks * 16.
 */
typedef struct {
  int32_t n;
  const int32_t *slots, *lens, *rows;
} spr_cache_batch;

/*
 * Rotary positions: pair k of a head's first dims dimensions is turned by
 * position * 2 pi * turns[k] and scaled by amplitude; the dimensions behind
 * them stay as they are.  Filled in by spr_rotary_init.
 */
typedef struct {
  int32_t dims;  /* even, 2..128 */
  int32_t pairs; /* pair k is dimensions 0: (k, k + dims / 2), 1: (2k, 2k + 1) */
  double amplitude;
  double turns[64];
} spr_rotary;

/*
 * Frequencies w_k = base^(-2k / dims).  For contexts longer than the
 * `original` positions a model was made for (factor > 1), a frequency that
 * turns t = original * w / (2 pi) times over those is taken as
 *   w (keep + (1 - keep) / factor),  keep = clamp((t - low) / (high - low), 0, 1):
 * quick ones as they are, slow ones divided by the factor.  factor 1 does not
 * read original, low and high.  Host only, enqueues nothing.
 *   base > 0; factor >= 1; original > 0; high > low; amplitude finite
 */
spr_status spr_rotary_init(int32_t dims, int32_t pairs, double base, double factor, double original, double low,
                           double high, double amplitude, spr_rotary* out);

typedef struct spr_cache_ops spr_cache_ops; /* opaque, library-owned host state */

/*
 * Workspace, creation, stream and release of a handle: as for spr_tree_ops.
 * Its device checks: a block id out of range, a fork's fresh block that another
 * of its forks copies from.
 */
size_t spr_cache_ops_workspace_bytes(void);
spr_status spr_cache_ops_init(void* dev_ws, size_t ws_bytes, void* hip_stream, spr_cache_ops** out);
spr_status spr_cache_ops_set_stream(spr_cache_ops* ops, void* hip_stream);
spr_status spr_cache_ops_release(spr_cache_ops* ops);

/*
 * Rotary positions of queries (or of anything in heads): row r and head h of
 * out are x's turned at positions[r], each element rounded once (angles,
 * sines and products are held in 64 bits).
 *   rows       1..SPR_MAX_CACHE_ROWS; n_heads 1..8192; head_dim 64 or 128, >= rotary->dims
 *   rotary     host, read during the call
 *   dtype      of x and out
 *   positions  device int32 [rows], of any sign
 *   x, out     device [rows] x [n_heads * head_dim], row r at r * stride
 *              elements; 16-byte aligned, strides a multiple of 16 bytes and >=
 *              n_heads * head_dim.  out may be x itself, else they must not overlap
 */
spr_status spr_cache_rotary(spr_cache_ops* ops, const spr_rotary* rotary, int32_t rows, int32_t n_heads, int32_t head_dim,
                            int32_t dtype, const int32_t* positions, const void* x, int64_t x_stride, void* out,
                            int64_t out_stride);

/*
 * Writes the keys and values of the batch's rows to layer `layer` of the
 * cache, keys turned at their cache positions first (rotary NULL: as they
 * are).  Nothing but the rows' own positions is written; a row whose block id
 * lies outside the pool is not.  The blocks that rows go to are their
 * request's alone (earlier ones may be shared).
 *   dtype  of k and v: device [rows] x [n_kv_heads * head_dim], strides in elements,
 *          aligned as in spr_cache_rotary
 */
spr_status spr_cache_append(spr_cache_ops* ops, const spr_kv4_view* kv, int32_t layer, const spr_cache_batch* batch,
                            const spr_rotary* rotary, int32_t dtype, const void* k, int64_t k_stride, const void* v,
                            int64_t v_stride);

/*
 * The other way: the values that the cache holds at the batch's rows, into k
 * and v (exact in either dtype).  k and v must not overlap.
 */
spr_status spr_cache_read(spr_cache_ops* ops, const spr_kv4_view* kv, int32_t layer, const spr_cache_batch* batch,
                          int32_t dtype, void* k, int64_t k_stride, void* v, int64_t v_stride);

/*
 * Attention of the batch's rows over layer `layer`: row j of request i and
 * head h attend to positions 0 .. lens[i] + j, the row's own the last of them
 * (its keys and values are in the cache already),
 *   out[r][h] = softmax(q[r][h] . K^T / sqrt(head_dim)) V
 * (head h reads KV head h / (n_heads / n_kv_heads)).  One row a request is a
 * decode step, more a prompt's chunk or drafted tokens in a line.  What lies
 * in the cache behind a row's last position does not reach its output,
 * whatever it holds.
 *   n_heads  a multiple of n_kv_heads, n_heads / n_kv_heads <= 16
 *   dtype    of q and out; scores and sums are held in fp32.  Probabilities enter
 *            their product with the values to 2^-11 of themselves for bf16
 *            outputs and to 2^-22 for fp32 ones, small ones to 2^-32 and 2^-36
 *            of the row's largest.  The sums are up to 2^8 times their values:
 *            values beyond 2^120 over the number of positions may overflow
 *   q, out   device [rows] x [n_heads * head_dim], aligned as in
 *            spr_cache_rotary.  out must not overlap q.
 */
spr_status spr_cache_attention(spr_cache_ops* ops, const spr_kv4_view* kv, int32_t layer, const spr_cache_batch* batch,
                               int32_t n_heads, int32_t dtype, const void* q, int64_t q_stride, void* out,
                               int64_t out_stride);

/*
 * The blocks of any paged cache as bytes: block b of layer l is block_bytes
 * bytes from byte (l * n_blocks + b) * block_bytes of k, and of v where that
 * is not NULL (a 4-bit cache has one pool: data as k).  block_bytes is a
 * multiple of 16, the pools are 16-byte aligned.  Views of a model's own cache
 * are not for spr_cache_fork and spr_cache_move: its slots own its blocks.
 * A launch has fewer than 2^24 work-groups, and calls that would need more are
 * refused: a fork one for each of the n table rows and, for every block it
 * copies (once for all its forks), one for each started 4 KiB in each layer of
 * k and v; a move one for each started 1024 table entries and, for up to 384 of
 * its blocks (more take further launches), one for each started 16 KiB likewise.
 */
typedef struct {
  void* k; /* device */
  void* v; /* device or NULL */
  int64_t block_bytes;
  int32_t n_layers, n_blocks;
  int32_t* block_table; /* device [n_slots][max_blocks] */
  int32_t n_slots, max_blocks;
} spr_pages;

/*
 * Forks requests: slot target[i] continues the first lens[i] positions of slot
 * source[i].  Its table row gets the source's full blocks (lens[i] / 16 of
 * them, shared from now on) and, where positions are left, block fresh[i] with
 * a copy of the source's next block in every layer; entries behind stay.
 *   n       1..SPR_MAX_CACHE_REQUESTS
 *   source, target  host [n]: slots; targets distinct, and none of them a source
 *   lens    host [n]: 0 .. max_blocks * 16
 *   fresh   host [n]: distinct free blocks (not read where lens[i] % 16 == 0)
 * A source entry outside the pool, or one that is a fresh block of the call,
 * is not copied to the target's row, nor is its block, and fails the handle's
 * next call.  No fork writes to a block that another of the call copies from;
 * a fresh block that is one of the sources' full blocks is written all the
 * same (that fresh blocks are free is the caller's to see to).
 */
spr_status spr_cache_fork(spr_cache_ops* ops, const spr_pages* pages, int32_t n, const int32_t* source,
                          const int32_t* target, const int32_t* lens, const int32_t* fresh);

/*
 * Moves block src[i] to dst[i] in every layer, and every table entry that is
 * src[i] to dst[i] (compaction, say).  What src[i] holds stays there.
 *   n         1..n_blocks
 *   src, dst  host [n]: blocks of the pool, distinct, and no dst is a src (what
 *             dst[i] holds is lost: that it is free is the caller's to see to)
 */
spr_status spr_cache_move(spr_cache_ops* ops, const spr_pages* pages, int32_t n, const int32_t* src, const int32_t* dst);

/* Releases the host state.  The workspace is the caller's to free afterwards. */
spr_status spr_release(spr_model* m);

/* Message for the last failure on the calling thread ("" if none). */
const char* spr_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* SPROUT_H_ */
