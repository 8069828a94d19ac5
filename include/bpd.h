/*
 * bpd.h -- C ABI of the blockwise-parallel-decoding library for NVIDIA B200 (sm_100a).
 *
 * The library runs the merged score-and-propose iteration of blockwise parallel
 * decoding (Stern, Shazeer, Uszkoreit 2018, Sections 3, 4 and 6) on one GPU:
 * a KV-cached Transformer decoder pass over the k proposed positions, the k
 * proposal heads at every position, a fused top-1 over the vocabulary, the
 * longest-prefix verification and the cache commit.
 *
 * Conventions
 *  - Every function returns BPD_OK (0) or a negative bpd_status.  Nothing throws,
 *    aborts or exits.  bpd_last_error() returns a thread-local message for the
 *    last failing call on this thread.
 *  - "host" pointers are ordinary CPU memory, "device" pointers are CUDA global
 *    memory of the current device.  The caller owns every buffer it passes and
 *    keeps it alive as long as the model / session that was given it.
 *  - The library allocates no device memory.  Weights live in a caller-provided
 *    device buffer (bpd_load_weights), all per-session state (encoder memory,
 *    paged KV cache, activations, reduction workspace) in another one
 *    (bpd_session_create); bpd_query_sizes tells how large they must be.
 *  - `cuda_stream` arguments are a cudaStream_t passed as void*; all work of a
 *    model / session is issued on the stream given at creation.
 *  - Token ids are int32.  Decoder input u_0 is id 0 (start); positions count
 *    from 0.  eos_id = -1 selects fixed-length termination (Section 2: language
 *    tasks stop at an end-of-sequence token, image tasks after a fixed number of
 *    steps).
 *  - Argmax ties go to the lowest id.
 */
#ifndef BPD_H_
#define BPD_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  BPD_OK = 0,
  BPD_E_INVALID = -1,     /* null pointer or argument out of range              */
  BPD_E_SHAPE = -2,       /* sizes inconsistent with the model / session         */
  BPD_E_FORMAT = -3,      /* malformed weight blob                               */
  BPD_E_NOMEM = -4,       /* a caller-provided buffer is too small               */
  BPD_E_STATE = -5,       /* call out of order (e.g. decode before encode)       */
  BPD_E_CUDA = -6,        /* a CUDA runtime call failed; message has the detail  */
  BPD_E_TIMEOUT = -7,     /* a bounded device-side wait expired                  */
  BPD_E_UNSUPPORTED = -8  /* valid request this build does not implement         */
} bpd_status;

typedef struct bpd_model bpd_model;     /* opaque: parsed config + device weight pointers  */
typedef struct bpd_session bpd_session; /* opaque: B rows of decode state in device memory */

/* Acceptance criteria for the Verify substep (the accept_mode argument).
 * Whatever the criterion, the token that is kept is the proposal (Section 3,
 * Accept).  BPD_ACCEPT_MIN_BLOCK(l) may be OR-ed in: at least l proposals are
 * taken per iteration regardless of the criterion (Section 5.3). */
enum {
  BPD_ACCEPT_EXACT = 0     /* Section 3: proposal == argmax p_1; the output equals greedy decoding */
};
#define BPD_ACCEPT_TOPN(n)       ((1 << 8) | ((n) & 0xff))    /* Section 5.1: proposal among the n best of p_1, 1 <= n <= 255 */
#define BPD_ACCEPT_DISTANCE(eps) ((2 << 8) | ((eps) & 0xff))  /* Section 5.2: |proposal - argmax p_1| <= eps (intensities)  */
#define BPD_ACCEPT_MIN_BLOCK(l)  (((l) & 0xff) << 16)         /* Section 5.3: 1 <= l <= k                                   */

#define BPD_MAX_K 16       /* largest block size / number of proposal heads */

/* Decode statistics.  "iterations" are score-and-propose passes (the priming
 * pass is not one); "invocations" = iterations + priming passes, the paper's
 * model-invocation count (Section 4: m/k + 1 in the best case).  Mean accepted
 * block size = tokens / iterations, summed over rows. */
typedef struct {
  int64_t tokens;                  /* tokens emitted, all rows                          */
  int64_t iterations;              /* passes of the slowest row                         */
  int64_t invocations;             /* model passes launched                             */
  int64_t row_iterations;          /* sum over rows of iterations that row took part in */
  int64_t khat_hist[BPD_MAX_K + 1];/* khat_hist[c] = (row, iteration) pairs accepting c */
  double  device_ms;               /* CUDA-event time of the decode loop                */
} bpd_stats;

/* Result of one bpd_iteration call.  Host arrays are filled when non-NULL
 * (the call then synchronises); device dumps are written when non-NULL. */
typedef struct {
  int32_t* khat;         /* host [B]       accepted block size (0 for finished rows)             */
  int32_t* accepted;     /* host [B,k]     accepted tokens, -1 beyond khat                       */
  int32_t* table;        /* host [B,k,k]   table[b][r][i] = argmax of head i+1 at block position r */
  int32_t* next_block;   /* host [B,k]     proposals for the next iteration (row khat of table)  */
  int32_t* block;        /* host [B,k]     the proposals this iteration scored                   */
  float*   logits_dev;   /* device [B,k,k,V] fp32 logits of every head at every position, or NULL */
  float*   hidden_dev;   /* device [B,k,d]   fp32 decoder outputs (after the final norm), or NULL  */
  float*   layers_dev;   /* device [n_dec,B,k,d] fp32 residual stream after every decoder layer
                            (before the final norm), or NULL; for parity debugging             */
} bpd_iter_out;

/* Execution strategies a session may use.  They change how the passes are
 * scheduled on the GPU, never what is computed: every combination decodes the
 * same tokens (sums are split differently, so hidden states agree to fp32
 * rounding).  Each field: -1 = the library's choice for this model and batch,
 * 0 = off, 1 = on where the shapes allow it.  Initialise with
 * bpd_session_options_init and change what you need. */
typedef struct {
  int32_t struct_bytes;       /* sizeof(bpd_session_options), set by bpd_session_options_init              */
  int32_t tensor_cores;       /* bf16 models: tcgen05 / TMA projection kernels (0: CUDA-core kernels)       */
  int32_t cuda_graphs;        /* replay each pass as a CUDA graph (needs a non-default stream)              */
  int32_t dependent_launch;   /* programmatic dependent launch between the kernels of a pass               */
  int32_t lazy_heads;         /* two-stage heads: p_1 at all k positions, all heads only at the accepted
                                 one (default: on when batch * k_model >= 64)                              */
  int32_t fold_layer_norms;   /* layer norms folded into the projections after them (decoder, and encoder;
                                 default in the encoder: up to batch * max_src = 768)                      */
  int32_t cluster_layers;     /* decoder layers as three cluster launches each (<= 16 rows per pass)        */
  int32_t persistent_layers;  /* all decoder layers of a pass in one persistent TMA-fed kernel (<= 16 rows
                                 per pass, d_model 256 / 512 / 1024; takes precedence over cluster_layers).
                                 Default: on for sessions of at most 256 positions whose encoder rows fit
                                 the staging tile, and for one sequence of any length where a CTA has an
                                 SM to itself (measured faster there), while no other live session of
                                 the device has it, off elsewhere; 1 asks for it wherever it runs.
                                 Several sequences (also more than 16 rows) run as groups side by side
                                 where the device holds n_heads * 8 CTAs for each group.  See
                                 bpd_session_create_opt for what it needs                                  */
  int32_t stage_encoder_rows; /* encoder keys / values staged in shared memory for cross-attention          */
  int32_t l2_stream_hints;    /* weights read once per pass are loaded "evict first"                        */
} bpd_session_options;

/* ---- set-up ------------------------------------------------------------- */

/* Sizes of the two device buffers the caller must provide.
 * blob: host, the weight container (self-describing header, then tensors).
 * weight_bytes / session_bytes: host outputs, either may be NULL. */
int bpd_query_sizes(const void* blob, size_t blob_bytes, int batch, int max_src, int max_tgt,
                    size_t* weight_bytes, size_t* session_bytes);

/* session_bytes for an already loaded model (same value bpd_query_sizes gives). */
int bpd_session_bytes(const bpd_model* model, int batch, int max_src, int max_tgt, size_t* session_bytes);

/* Which form the session's decoder layers take: 0 = one kernel per projection, 1 = three cluster launches per
 * layer, 2 = one persistent kernel per pass.  The options of bpd_session_create_opt are requests: a shape or a
 * device that a form does not take falls back to the next one, and this call tells.  Negative on a null handle. */
int bpd_session_layer_path(const bpd_session* s);

/* Copy the blob's tensors into dev_weight_buf (device, 256-byte aligned,
 * >= weight_bytes) and return a model handle.  The blob may be freed after the
 * call returns (the call synchronises the stream). */
int bpd_load_weights(const void* blob, size_t blob_bytes, void* dev_weight_buf, size_t dev_bytes,
                     void* cuda_stream, bpd_model** out);

/* Lay a session of `batch` rows out in dev_session_buf (device, 256-byte
 * aligned, >= session_bytes for these arguments).  max_src bounds the source
 * length, max_tgt the number of decoded tokens per row. */
int bpd_session_create(const bpd_model* model, int batch, int max_src, int max_tgt,
                       void* dev_session_buf, size_t dev_bytes, void* cuda_stream, bpd_session** out);

/* The same with explicit options (NULL = all defaults).  A session that runs
 * its decoder layers in the persistent kernel (persistent_layers; see
 * bpd_session_layer_path) occupies most of the GPU with CTAs that wait for
 * one another: passes of two such sessions must not overlap on one GPU (keep
 * them on one stream, or finish one decode before starting another); if they
 * do, their bounded waits expire after about a second and the calls return
 * BPD_E_TIMEOUT.  Left to the library (the default), at most one live session
 * per device gets the persistent kernel -- a session created while another
 * holds it runs the cluster launches, which may overlap with anything -- so
 * only sessions that ask for it with persistent_layers = 1 can meet this. */
void bpd_session_options_init(bpd_session_options* options);
int bpd_session_create_opt(const bpd_model* model, int batch, int max_src, int max_tgt,
                           void* dev_session_buf, size_t dev_bytes, void* cuda_stream,
                           const bpd_session_options* options, bpd_session** out);

int bpd_session_destroy(bpd_session* s);
int bpd_model_destroy(bpd_model* m);
const char* bpd_last_error(void);

/* ---- the decoding path (Sections 2-4) ------------------------------------ */

/* Run the encoder over the source rows, fill the cross-attention keys/values
 * of every decoder layer, and reset all rows to "nothing decoded".
 * src_ids: host [batch, max_src] (row b valid in [0, src_len[b]), rest ignored);
 * src_len: host [batch], 1 <= src_len[b] <= max_src. */
int bpd_encode(bpd_session* s, const int32_t* src_ids, const int32_t* src_len);

/* Greedy decoding (Section 2): one decoder pass per token, head p_1 only.
 * out_ids: host [batch, max_new] or NULL; out_len: host [batch] or NULL.  When
 * out_ids is NULL the call only enqueues the work and results stay on the
 * device (bpd_fetch_output reads them).  stats may be NULL. */
int bpd_decode_greedy(bpd_session* s, int max_new, int32_t eos_id,
                      int32_t* out_ids, int32_t* out_len, bpd_stats* stats);

/* Blockwise parallel decoding with the combined model (Sections 3 and 4): a
 * priming pass, then merged verify+predict iterations until every row has
 * max_new tokens or has accepted eos_id.  1 <= k <= k_model uses the first k
 * heads.  Output arguments as for bpd_decode_greedy. */
int bpd_decode_blockwise(bpd_session* s, int k, int accept_mode, int max_new, int32_t eos_id,
                         int32_t* out_ids, int32_t* out_len, bpd_stats* stats);

/* Blockwise parallel decoding in its two-call form (Section 3: predict,
 * verify, accept), kept for comparison with the merged form of Section 4:
 * every iteration is a Verify invocation (p_1 alone at the k block positions,
 * followed by acceptance and the cache commit) and a Predict invocation (all
 * k heads at the last accepted token, whose position is recomputed).  The
 * ids and accepted block sizes are those of bpd_decode_blockwise; the number
 * of model invocations is 2 per iteration instead of 1 per iteration + 1
 * (stats->invocations), which is why the merged form is the product path.
 * Arguments, outputs, forced plans and error behaviour as for
 * bpd_decode_blockwise. */
int bpd_decode_blockwise_twocall(bpd_session* s, int k, int accept_mode, int max_new, int32_t eos_id,
                                 int32_t* out_ids, int32_t* out_len, bpd_stats* stats);

/* One merged score-and-propose iteration (Section 4) on the session's current
 * state; on a freshly encoded session the priming pass runs first.
 * forced_tail: host [batch, k-1] replacing proposals 2..k of every row, or
 * NULL.  Proposal 1 is never replaced: it is p_1's own argmax (Section 3, the
 * remark that khat >= 1).  max_new / eos_id bound acceptance as in the decode
 * calls.  out may be NULL (no synchronisation then). */
int bpd_iteration(bpd_session* s, int k, int accept_mode, int max_new, int32_t eos_id,
                  const int32_t* forced_tail, bpd_iter_out* out);

/* Controlled acceptance: install (plan != NULL) or clear (NULL) a table of
 * forced proposal tails, host [batch, plan_len, k-1]: an iteration of row b
 * that starts with j tokens accepted (j < plan_len) replaces its proposals
 * 2..k by plan[b][j][:].  Stays in force for bpd_decode_blockwise and
 * bpd_iteration (when that is given no forced_tail) until cleared or until
 * the next bpd_encode.  Needs plan_len <= max_tgt and k <= k_model. */
int bpd_set_forced_plan(bpd_session* s, const int32_t* plan, int plan_len, int k);

/* Forget everything decoded (rows back to "nothing decoded") but keep the
 * encoder memory and any forced plan: the state bpd_encode leaves, without
 * running the encoder again.  Asynchronous. */
int bpd_rewind(bpd_session* s);

/* Copy the tokens decoded so far to the host (synchronises).
 * out_ids: host [batch, max_new]; out_len: host [batch] (either may be NULL). */
int bpd_fetch_output(bpd_session* s, int max_new, int32_t* out_ids, int32_t* out_len, bpd_stats* stats);

/* ---- instrumentation ------------------------------------------------------ */

/* Number of CUDA kernels this library has launched in this process so far. */
long long bpd_kernel_launches(void);

/* Per-phase device timing of the decoder pass.  bpd_profile(s, 1) clears the
 * record and makes every following pass bracket four phases with CUDA events on
 * the session's stream; bpd_profile(s, 0) stops.  bpd_profile_read returns how
 * many times `phase` ran and the summed device time.  Phases: 0 = embedding,
 * decoder layers and final norm; 1 = head hidden layer; 2 = head output layers
 * (+ residual); 3 = vocabulary projection with top-1; for bf16 models also the
 * individual kernels inside phase 0: 4 = embedding, 5 = layer norms, 6 = QKV
 * projection, 7 = self-attention, 8 = output projection, 9 = cross-attention
 * query projection, 10 = cross-attention, 11 = cross-attention output
 * projection, 12 / 13 = feed-forward layers 1 / 2, 14 = verify and commit. */
int bpd_profile(bpd_session* s, int enable);
int bpd_profile_read(bpd_session* s, int phase, int64_t* launches, double* total_ms);

/* Self test of the bounded device-side waits: launches one CTA that waits on a
 * barrier nothing ever arrives on, then one that waits for tagged words nobody
 * writes (the two kinds of wait the kernels have), each with a limit of about
 * limit_us microseconds.  The waits give up, the kernels record their error words
 * and return normally (without waiting again where more waits follow), and the
 * call reports BPD_E_TIMEOUT -- the status a real
 * decode call returns if one of its kernels' waits ever expires.  BPD_OK or
 * BPD_E_CUDA would mean that a wait did not expire the way it should.
 * dev_word: device int32 used as the error word.  Synchronises the stream. */
int bpd_debug_wait_timeout(int32_t* dev_word, int limit_us, void* cuda_stream);

/* ---- single operators (used by tests and profiling) ----------------------- */

/* Top-1 of a vocabulary projection without materialising logits (Section 4's
 * "k separate softmaxes per position", of which only the argmax is needed):
 * out_idx[r] = argmin-id argmax_v sum_c x[r][c] * w[v][c].
 * x: device [rows, d]; w: device [vocab, d]; both of `dtype` (0 = float32,
 * 1 = bfloat16), row-major.  scratch: device workspace of at least
 * bpd_op_vocab_argmax_scratch_bytes(rows, d, vocab, dtype) bytes.
 * out_idx: device int32 [rows]; out_val: device float [rows] or NULL. */
size_t bpd_op_vocab_argmax_scratch_bytes(int rows, int d, int vocab, int dtype);
int bpd_op_vocab_argmax(const void* x, const void* w, int rows, int d, int vocab, int dtype,
                        void* scratch, size_t scratch_bytes, int32_t* out_idx, float* out_val,
                        void* cuda_stream);

/* The same top-1 for callers that cannot hand over a workspace and must not
 * trigger a device allocation: code running under a framework that has already
 * claimed the whole GPU for its own pool, a serving loop that cannot afford the
 * device-wide synchronisation an allocation may cause, or a plug-in callback
 * that is only allowed to enqueue work.  (The paper has no counterpart; this is
 * a deployment convenience.)  The cross-CTA reduction workspace is a fixed
 * 33 KiB array inside the library image, resident on every GPU that loads the
 * library until the process exits.  Limits: rows <= 256, vocab <= 65536
 * (beyond them the call returns BPD_E_NOMEM) and d <= 1024, a multiple of 8
 * (BPD_E_SHAPE, as for bpd_op_vocab_argmax); a refused call leaves the outputs
 * untouched.  Arguments as bpd_op_vocab_argmax, minus the scratch.
 * The call performs no cudaMalloc/cudaFree and uses no allocating library.
 * The first call on each device is a set-up call: it looks the array's device
 * address up (with that device current), and, as with any kernel, the CUDA
 * driver loads the kernel's code when a data type is first launched (memory of
 * the driver's own: about 2 MiB in a fresh process) -- make one call per device
 * and data type at start-up, outside any stream capture; from then on the
 * device's free memory stays exactly as it is across calls.  All calls
 * share the one array: the call clears the arrival counters it needs, but two
 * calls whose kernels may overlap on the GPU (different streams, or different
 * host threads) race on it -- keep them on one stream or serialise them. */
int bpd_op_vocab_argmax_noalloc(const void* x, const void* w, int rows, int d, int vocab, int dtype,
                                int32_t* out_idx, float* out_val, void* cuda_stream);

/* y[r][n] = act(sum_c x[r][c] * w[n][c] + bias[n]); the projection used by every
 * layer.  x: device [rows, in_f] `dtype`; w: device [out_f, in_f] `dtype`; bias:
 * device [out_f] `dtype` or NULL; y: device [rows, out_f] float32; relu != 0
 * applies max(0, .).  scratch as above (bpd_op_linear_scratch_bytes). */
size_t bpd_op_linear_scratch_bytes(int rows, int in_f, int out_f, int dtype);
int bpd_op_linear(const void* x, const void* w, const void* bias, int rows, int in_f, int out_f,
                  int dtype, int relu, void* scratch, size_t scratch_bytes, float* y,
                  void* cuda_stream);

/* ---- operators on a paged cache --------------------------------------------
 *
 * For programs that keep caches of their own and draft more than a block: trees
 * of proposals (Section 4's heads rank several candidates each), caches bounded
 * by a budget, and caches so long that a step reads a part of them.  The cache
 * has the layout of the decoding path: pages of 64 positions, one pool per
 * layer, one page table for all layers.
 *
 * All of these calls only enqueue work on cuda_stream: they may be captured into
 * a graph (after one call of the kind outside of any capture, which loads the
 * kernels), and keep nothing between calls.  A scratch belongs to one call until
 * that call's kernels are done (calls on one stream may share one if they are
 * enqueued one after the other); a scratch_bytes call answers 0 where none is
 * needed, and for arguments that the call itself refuses.  Kernels trust no value in a device array: a
 * length outside [0, capacity] is clamped to it, a node count to [0, nodes], a
 * parent that does not lie before its node is taken as -1, and a page outside
 * [0, n_pages) is no page: its positions count as masked and are not written.
 * Two table entries of different rows may name the same page as long as no call
 * writes a position of it.  capacity = pages_per_row * 64.  Limits (BPD_E_SHAPE
 * beyond them): kv_heads <= 1024, heads <= 4096, batch and layers <= 65535,
 * n_pages <= 2^24, pages_per_row <= 2^20; other head widths are
 * BPD_E_UNSUPPORTED.  A refused call leaves everything as it was.
 *
 * Outputs overlap no input.  What a row does not see -- positions behind a
 * length, other nodes -- may hold anything; what it sees counts as it is.  A key
 * with infinite elements whose score is -inf weighs 0; an infinite or NaN value
 * leaves no finite output in its column.  Scores, softmax sums and outputs before
 * their division are held in 32 bits: values above 2^100 may leave that range.
 * Launches are planned by pages_per_row, not by the lengths on the device: a
 * table much wider than its rows are long costs short calls 2 to 6 us. */
typedef struct {
  void* k_pool;               /* device [layers][n_pages][64][kv_heads][head_dim] of dtype, 16-byte aligned */
  void* v_pool;               /* the same for the values; may be NULL where a call only reads keys      */
  const int32_t* page_table;  /* device [batch][pages_per_row]: page of the row's positions 64 p .. 64 p + 63 */
  int32_t layers;             /* attention and weights calls look at one layer: pass its pools           */
  int32_t n_pages;
  int32_t pages_per_row;
  int32_t batch;
  int32_t kv_heads;
  int32_t head_dim;           /* 16, 32, 64 or 128 */
  int32_t dtype;              /* 0 = float32, 1 = bfloat16; queries, drafted keys and outputs have it too */
} bpd_cache;

/* Attention of drafted nodes over the cache and their own tree:
 *   out[b][t] = sum_s softmax_s(scale * q . k_s) v_s,  s in positions [0, lens[b]) and node t's line
 * where the line of node t is t itself, parents[b][t], and so on up to a node
 * whose parent is -1 (the last cached token).  parents[b][t] < t; a chain is
 * parents = t - 1, a single token nodes = 1 and parents = -1.  Queries may have
 * more heads than the cache: heads is a multiple of kv_heads, and head i reads
 * key head i / (heads / kv_heads).
 * q: device [batch * nodes] rows of [heads][head_dim], q_stride elements apart;
 * k_new, v_new: device [batch * nodes] rows of [kv_heads][head_dim], kv_stride
 * elements apart (slices of one fused projection will do; rows begin on 16-byte
 * boundaries).  They are not written to the cache: bpd_op_tree_commit does that
 * for the accepted ones.  n_nodes: device [batch] or NULL: row b has the first
 * n_nodes[b] nodes; behind them the outputs are 0 and lse is -inf.  1 <= nodes
 * <= 256, scale > 0.  out: device [batch][nodes][heads][head_dim] of dtype.  lse: device
 * float [batch][nodes][heads] or NULL: log of the softmax's sum. */
size_t bpd_op_tree_attention_scratch_bytes(const bpd_cache* cache, int nodes, int heads);
int bpd_op_tree_attention(const bpd_cache* cache, const void* q, const void* k_new, const void* v_new, int nodes, int heads,
                          int64_t q_stride, int64_t kv_stride, const int32_t* lens, const int32_t* parents,
                          const int32_t* n_nodes, float scale, void* scratch, size_t scratch_bytes, void* out, float* lse,
                          void* cuda_stream);

/* Verify and commit for trees (Section 3's Verify and Accept with several
 * candidates per position).  From the last cached token on, the walk goes to the
 * lowest child whose token is the base model's prediction (last_top1[b] for the
 * first step, top1[b][node] after), until there is none, the cache is full, or
 * a token equal to eos_id (>= 0) has been taken.  The path's keys and values go
 * to positions lens[b], lens[b] + 1, ... of every layer.
 * k_new, v_new: device [layers][batch][nodes] rows, kv_stride elements apart.
 * tokens, top1, parents: device [batch][nodes].  Outputs, device int32:
 * out_lens [batch], out_accepted [batch], out_path [batch][nodes] (the nodes
 * taken, -1 behind them), out_next [batch]: the prediction after the last node
 * taken, i.e. what the next step passes as last_top1 (keep two arrays and swap
 * them).  No output may overlap an input: every CTA of a sequence walks its tree
 * (BPD_E_INVALID).  A row whose length is negative takes no node; out_lens is
 * the clamped length. */
int bpd_op_tree_commit(const bpd_cache* cache, const void* k_new, const void* v_new, int nodes, int64_t kv_stride,
                       const int32_t* lens, const int32_t* parents, const int32_t* tokens, const int32_t* top1,
                       const int32_t* last_top1, const int32_t* n_nodes, int32_t eos_id, int32_t* out_lens,
                       int32_t* out_accepted, int32_t* out_path, int32_t* out_next, void* cuda_stream);

/* Attention weight that the accepted nodes gave to every cached position, added
 * up: for node path[b][i], i < accepted[b], which sits at position lens[b] + i by
 * now (lens as before the commit), and positions s <= lens[b] + i,
 *   weights[b][h][s] += sum over the heads of key head h of exp(scale * q . k_s - lse).
 * Entries of this commit (s >= lens[b]) start from 0, and positions[b][h][s] is
 * set to seen[b] + s - lens[b], where seen[b] is the number of tokens committed
 * before, evicted ones included.  Everything else is left as it was.
 * q, lse: as given to and returned by the attention.  weights: device float
 * [batch][kv_heads][capacity]; positions: device int32 of the same shape. */
int bpd_op_cache_weights(const bpd_cache* cache, const void* q, int nodes, int heads, int64_t q_stride, const float* lse,
                         const int32_t* path, const int32_t* accepted, const int32_t* lens, const int32_t* seen, float scale,
                         float* weights, int32_t* positions, void* cuda_stream);

/* Eviction: of every list (layer, row, key head) longer than budget, budget
 * entries stay -- those with positions >= seen[b] - recent (the last `recent`
 * tokens), then the largest weights (equal ones: the lower slot; NaN counts as
 * the smallest).  Survivors keep their slots below budget; the holes there, in
 * ascending order, take the survivors above, in ascending order: keys, values,
 * weights and positions move together (an entry without a page: its weight and
 * position alone), what lies at slots >= budget is left as it was.  Slots are then in no order, which attention does not mind and
 * `positions` records.  1 <= budget, 0 <= recent <= budget.
 * weights, positions: device [layers][batch][kv_heads][capacity].  out_lens:
 * device [batch]: min(lens, budget); may not overlap lens, seen or the page
 * table (BPD_E_INVALID). */
size_t bpd_op_cache_evict_scratch_bytes(const bpd_cache* cache, int budget);
int bpd_op_cache_evict(const bpd_cache* cache, const int32_t* lens, const int32_t* seen, int budget, int recent,
                       float* weights, int32_t* positions, void* scratch, size_t scratch_bytes, int32_t* out_lens,
                       void* cuda_stream);

/* Means of the keys of the pages that became full between lens_from[b] and
 * lens[b] (both device [batch]): means[l][b][p][h][:], device float
 * [layers][batch][pages_per_row][kv_heads][head_dim].  Sums are in 64 bits and
 * rounded once.  Other entries are left as they were. */
int bpd_op_page_means(const bpd_cache* cache, const int32_t* lens_from, const int32_t* lens, float* means, void* cuda_stream);

/* bpd_op_tree_attention over a part of the cache: every node and key head sees
 * the `select` full pages whose mean key scores highest against the sum of its
 * group's queries (scores in 64 bits; equal ones: the lower page; NaN counts as
 * the smallest), the positions behind the last full page, and the node's line.
 * means: device float [batch][pages_per_row][kv_heads][head_dim] of this layer.
 * 1 <= select <= pages_per_row.  pages: device int32 [batch][nodes][kv_heads]
 * [select] or NULL: the selected pages (indices into the row's table), ascending,
 * -1 behind the last. */
size_t bpd_op_page_attention_scratch_bytes(const bpd_cache* cache, int nodes, int heads, int select);
int bpd_op_page_attention(const bpd_cache* cache, const float* means, const void* q, const void* k_new, const void* v_new,
                          int nodes, int heads, int64_t q_stride, int64_t kv_stride, const int32_t* lens, const int32_t* parents,
                          const int32_t* n_nodes, int select, float scale, void* scratch, size_t scratch_bytes, void* out,
                          float* lse, int32_t* pages, void* cuda_stream);

/* What the operators on a paged cache cannot report as they only enqueue work:
 * whether a bounded wait inside one of their kernels has expired on the current
 * device since this was last asked (BPD_E_TIMEOUT; never seen outside of broken
 * hardware or a debugger).  Synchronises the stream. */
int bpd_op_status(void* cuda_stream);

/* Self test of the above, as bpd_debug_wait_timeout: enqueues one CTA that waits
 * as those kernels do, on a barrier nothing ever arrives on, with a limit of about
 * limit_us microseconds (1..2000000).  The wait gives up, and the next
 * bpd_op_status reports it, once. */
int bpd_debug_op_wait_timeout(int limit_us, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* BPD_H_ */
