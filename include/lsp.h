/*
 * lsp.h -- C ABI of the fixed-cost drafting round (LongSpark, arxiv 2609.37029).
 *
 * One drafting round (Sec. 2.4 "Inference", Fig. 2):
 *   1. lsp_view_update: fold the target verification pass's newly accepted rows
 *      into the fixed-size context interface -- the global summary (Eq.
 *      global-summary maintained by the merge of App. A.2, Eq. summary-update),
 *      the recent KV window and the boundary hidden states (Sec. 2.2).
 *   2. lsp_draft: the block-diffusion drafter forward over [block; window;
 *      summary] (Sec. 2.3, Eq. draft-context, App. A.1), the frozen final norm
 *      and LM head (base logits z^(0)), then lsp_sample's correction+sampling.
 *   3. lsp_sample: the low-rank Markov correction (Eq. markov) and sequential
 *      sampling of the B proposals (Eq. proposal-factorization).
 *
 * Conventions shared by every call:
 *   - Every call returns an int status: LSP_OK (0) or a negative LSP_ERR_*.
 *     Argument and shape errors are detected on the host before any launch and
 *     nothing is enqueued then.  No exception or abort crosses the ABI.
 *   - All device work is enqueued on the caller's stream (lsp_stream_t is a
 *     cudaStream_t; NULL means the legacy default stream) and returns without
 *     synchronising, except where a call says otherwise.
 *   - Pointers documented as "device" must be device (or managed) memory owned
 *     by the caller, valid until the enqueued work completes.  The library owns
 *     only what lsp_state_create allocates.
 *   - Element type of every tensor argument documented as "dtype" is the
 *     config's dtype: LSP_DTYPE_BF16 (bfloat16) or LSP_DTYPE_F32 (float).
 *   - Errors a kernel detects (a token id out of range, accepted_len beyond the
 *     row capacity, a bounded wait that timed out) set bits of a device error
 *     word (LSP_DEV_*) read by lsp_get_error; kernels never trap.
 *   - Layouts are dense and row-major; linear weights are [out][in] with `in`
 *     contiguous (y = W x).
 *   - Concurrency: the device work of one state (its interface, workspace and
 *     synchronisation words) must be ordered -- one stream, or streams the
 *     caller synchronises; calls on different states, and lsp_linear calls
 *     with different workspaces, may overlap from any threads and streams.
 *     The one process-wide buffer is lsp_sample_noalloc's scratch (below).
 *   - No environment variable changes what the library computes or how.
 */
#ifndef LSP_H
#define LSP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LSP_MAX_DRAFT_LAYERS 16

/* status codes */
#define LSP_OK 0
#define LSP_ERR_ARG (-1)          /* null pointer / invalid scalar argument */
#define LSP_ERR_SHAPE (-2)        /* config or size outside what the kernels support */
#define LSP_ERR_CUDA (-3)         /* a CUDA runtime or driver call failed */
#define LSP_ERR_TIMEOUT (-4)      /* a device wait gave up (see lsp_get_error) */
#define LSP_ERR_STATE (-5)        /* state not initialised or device error pending */
#define LSP_ERR_NOMEM (-6)        /* device allocation failed in lsp_state_create */
#define LSP_ERR_UNSUPPORTED (-7)  /* no sm_103a device / feature unavailable */

/* device error word bits (lsp_get_error) */
#define LSP_DEV_TIMEOUT 1u        /* a bounded mbarrier/flag wait expired */
#define LSP_DEV_BAD_TOKEN 2u      /* a token id outside [-1, V) (slot 0: outside [0, V)) */
#define LSP_DEV_BAD_DELTA 4u      /* accepted_len outside [0, row capacity] (lsp_verify_probs: n_draft outside [0, B]) */
#define LSP_DEV_BAD_SEQ 8u        /* a cache entry a call cannot use: sequence or page index, length, row range */
#define LSP_DEV_NO_PAGE 16u       /* lsp_pages_reserve: not enough free pages */

#define LSP_DTYPE_BF16 0
#define LSP_DTYPE_F32 1
#define LSP_DTYPE_Q4 2            /* lsp_kv_cache only: a cache held in 4 bits */

/* lsp_config.flags.  LSP_NO_BOUNDARY: the "w/o boundary state" variant of the
 * ablation (Sec. 3.4, Fig. 5): the state keeps no boundary hidden state, the
 * boundary fusion is not run and the input slots are E[u_i] + P_i alone.  The
 * other two variants are shapes: w/o global summary is R = 0, w/o recent KV
 * window is W = 0. */
#define LSP_NO_BOUNDARY 1u

typedef void* lsp_stream_t;       /* cudaStream_t */
typedef struct lsp_state lsp_state; /* opaque, library-owned */

/*
 * Shapes of one drafter + target pairing.
 *   C   concurrency: requests processed together (state rows)
 *   B   draft block slots = proposals per round (Sec. 2.3)
 *   L   tapped target layers (the set of Sec. 2.2; App. B.1 uses 5)
 *   D   drafter layers (App. B.1: 5)
 *   H   hidden size; nq / nkv query / key-value heads of head dim d (the
 *       target's, since draft queries score target window keys)
 *   F   drafter MLP width; V vocabulary; rc rank of the Markov correction
 *   W   recent window rows per tapped layer (App. B.1: 256)
 *   R   summary queries per tapped layer and query head (App. B.1: 16)
 *   layer_map[j]  tapped-layer index draft layer j reads its window and summary
 *       from (Sec. 2.3 pairs draft layer j with tapped layer l(j)); a value < 0
 *       selects floor(j * L / D)
 *   rope_theta  rotary base of the drafter's block queries/keys; rms_eps RMSNorm eps
 *   flags  0 or LSP_NO_BOUNDARY
 * Supported: dtype BF16 with d == 128, B <= 16, nq % nkv == 0, nq/nkv <= 8;
 * dtype F32 with d <= 128 even; H, nq*d, nkv*d, F multiples of 64; C*B <= 512;
 * W >= 0 and R >= 0 (0 removes the window / the summary from the context).
 */
typedef struct lsp_config {
  int C, B, L, D, H, nq, nkv, d, F, V, W, R, rc;
  int dtype;
  int layer_map[LSP_MAX_DRAFT_LAYERS];
  float rope_theta;
  float rms_eps;
  unsigned flags;
} lsp_config;

/*
 * New target rows of one verification pass (Sec. 2.1, 2.4): for request b,
 * tapped layer l and new row j < accepted_len[b]:
 *   k[b][l][j][0..nkv)[0..d)   key rows as cached by the target (rotary applied)
 *   v[b][l][j][0..nkv)[0..d)   value rows
 *   h[b][l][j][0..H)           hidden state at that row (only row accepted_len-1 is read)
 * All three are device pointers of dtype with row capacity `rows` per (b, l);
 * h may be null (and is not read) with LSP_NO_BOUNDARY.
 * h_rows: rows of h per (b, l).  0 (the default when the struct is zeroed) or
 * `rows`: the layout above.  1: h[b][l][0..H) holds only the boundary row --
 * the hidden state at row accepted_len[b]-1 (for lsp_prefill: at row t-1) --
 * which is all the interface reads (Sec. 2.2), so a caller that stages the
 * rows from host memory copies C*L*H elements instead of C*L*rows*H.  Any
 * other value is LSP_ERR_ARG.
 */
typedef struct lsp_target_feats {
  const void* k;
  const void* v;
  const void* h;
  int rows;
  int h_rows;
} lsp_target_feats;

/* One Qwen3-style draft layer (App. B.1); device pointers of dtype. */
typedef struct lsp_layer_weights {
  const void* in_norm;    /* [H] */
  const void* wq;         /* [nq*d][H] */
  const void* wk;         /* [nkv*d][H] */
  const void* wv;         /* [nkv*d][H] */
  const void* q_norm;     /* [d] per-head RMSNorm of block queries */
  const void* k_norm;     /* [d] per-head RMSNorm of block keys */
  const void* wo;         /* [H][nq*d] */
  const void* post_norm;  /* [H] */
  const void* w_gate;     /* [F][H] */
  const void* w_up;       /* [F][H] */
  const void* w_down;     /* [H][F] */
} lsp_layer_weights;

/* Drafter weights (device pointers of dtype). The target's embedding, final
 * norm and LM head are reused frozen (Sec. 2.3, App. B.1). */
typedef struct lsp_weights {
  const void* embed;       /* [V][H] target token embedding */
  const void* final_norm;  /* [H] target final RMSNorm weight */
  const void* lm_head;     /* [V][H] target vocabulary head */
  const void* fuse;        /* [H][L*H] boundary fusion: c_t = fuse . [h^l1;...;h^lL] (Sec. 2.2);
                              may be null with LSP_NO_BOUNDARY */
  const void* pos;         /* [B][H] within-block positional encodings (Sec. 2.3) */
  const void* mask_emb;    /* [H] mask-token embedding of slots 1..B-1 */
  const void* Ec;          /* [V][rc] correction embedding E_c (Eq. markov) */
  const void* Wc;          /* [V][rc] correction output map W_c (Eq. markov) */
  lsp_layer_weights layer[LSP_MAX_DRAFT_LAYERS];
} lsp_weights;

/*
 * Sampling of the proposals (Eq. proposal-factorization).  temperature == 0:
 * greedy, y_i = argmax_v z_i[v].  temperature > 0: Gumbel-max,
 * y_i = argmax_v (z_i[v] / T + g) (z / T taken in fp32 as z * fl(1/T), exact at T = 1),
 * g = -log(-log u), u = ((x >> 9) + 0.5) * 2^-23,
 * x = word (v & 3) of Philox4x32-10 with key (seed lo32, seed hi32) and counter
 * (v >> 2, i, b, round).  Ties go to the lowest vocabulary index.
 */
typedef struct lsp_sample_params {
  float temperature;
  uint32_t round;
  uint64_t seed;
} lsp_sample_params;

/* Human-readable name of a status code (static string). */
const char* lsp_status_string(int status);

/* Bytes of the persistent per-state interface for `cfg` (window, summary
 * (m, eta), boundary h, counters), all C requests: a function of the shapes
 * only, never of the prefix length (Sec. 2.4 "Fixed-cost complexity").
 * Returns 0 for an invalid config. Host-only; needs no GPU. */
size_t lsp_state_bytes(const lsp_config* cfg);

/* Validate `cfg` on the host. LSP_OK or LSP_ERR_SHAPE / LSP_ERR_ARG. Needs no GPU. */
int lsp_config_check(const lsp_config* cfg);

/* Allocate a state on the current device: the interface (lsp_state_bytes) and
 * a fixed workspace for the drafter's activations, logits and sampler
 * partials.  Synchronous; the only call that allocates device memory.  The
 * state starts uninitialised (call lsp_state_init). */
int lsp_state_create(const lsp_config* cfg, lsp_state** out);

/* Free everything lsp_state_create allocated (synchronises the device first).
 * NULL is ignored. */
void lsp_state_destroy(lsp_state* st);

/* Reset the interface to the empty prefix -- m = 0, eta = -inf, empty window,
 * zero boundary, t = 0, device error word cleared -- and copy the summary
 * queries G (device, dtype, [L][nq][R][d]; Sec. 2.2, App. B.2 "Summary
 * queries", held fixed during inference) into the state.  The summary over a
 * prefix is then built by lsp_view_update calls over its rows in chunks of any
 * size (the merge of App. A.2 makes the chunking exact); this is the one-time
 * O(t) prefill the paper attributes to target prefill (Fig. 3). */
int lsp_state_init(lsp_state* st, const void* G, lsp_stream_t stream);

/* Fold accepted_len[b] new target rows of request b (device int32 [C], each in
 * [0, feats->rows]; 0 leaves request b untouched) into the interface:
 *  - summary: for every tapped layer l, query head h and summary query r,
 *    the attention statistics of g_r over the new keys of KV head h/(nq/nkv)
 *    are merged into (eta, m) by Eq. summary-update;
 *  - window: the new K/V rows enter the ring of the last W rows (row p of the
 *    prefix lives in slot p mod W);
 *  - boundary: h of the last new row replaces the boundary state;
 *  - t += accepted_len[b].
 * Reads only the new rows, never the prefix (Sec. 2.4). */
int lsp_view_update(lsp_state* st, const lsp_target_feats* feats,
                    const int32_t* accepted_len, lsp_stream_t stream);

/* One drafter forward for all C requests (Sec. 2.3, App. A.1) followed by the
 * sampler of lsp_sample.
 *   block_tokens  device int32 [C][B]: slot 0 = committed token a (also y_0 of
 *                 the Markov correction); slots >= 1: -1 for the mask embedding
 *                 or a token id to embed
 *   w             weights (host struct of device pointers)
 *   sp            sampling parameters (host struct)
 *   out_tokens    device int32 [C][B]: proposals y_1..y_B
 *   out_logits    device float [C][B][V] corrected logits z_i (the verification
 *                 distributions q_i = softmax(z_i)), or NULL to skip writing them
 * Rotary positions of slot i are t + i (t = rows folded so far).  Uses only
 * the state's fixed workspace; allocates nothing. */
int lsp_draft(lsp_state* st, const int32_t* block_tokens, const lsp_weights* w,
              const lsp_sample_params* sp, int32_t* out_tokens, float* out_logits,
              lsp_stream_t stream);

/* Correction + sampling alone (Eq. markov, Eq. proposal-factorization) on given
 * base logits, with the state's config (C, B, V, rc, dtype) and workspace:
 *   base_logits  device float [C][B][V] (z^(0); not modified)
 *   prev_token   device int32 [C]: y_0 = a of each request
 *   Ec, Wc       device dtype [V][rc]
 *   out_tokens   device int32 [C][B]; out_logits device float [C][B][V] or NULL
 * For i = 1..B in order: z_i = z_i^(0) + W_c E_c[y_{i-1}], y_i drawn per sp. */
int lsp_sample(lsp_state* st, const float* base_logits, const int32_t* prev_token,
               const void* Ec, const void* Wc, const lsp_sample_params* sp,
               int32_t* out_tokens, float* out_logits, lsp_stream_t stream);

/* Correction + sampling without a state and without any device allocation,
 * for callers that cannot allocate device memory where they sample (a loop
 * running under another framework's caching allocator that already reserved
 * the device, or code that must not create an lsp_state).  The paper has no
 * counterpart: this is a deployment variant of lsp_sample.
 *   Same computation and tensor arguments as lsp_sample; the shapes are passed
 *   explicitly (1 <= C <= 64, B >= 1, V and rc multiples of 16, rc <= 256) and
 *   dtype is LSP_DTYPE_BF16 or LSP_DTYPE_F32 for Ec / Wc.
 *   dev_error: optional device uint32 that receives LSP_DEV_* bits (OR-ed in;
 *   NULL skips error reporting).
 * Scratch: a fixed 512 KiB __device__ array inside the library, held by every
 * GPU that loads it until the process exits.  A call needs
 *   align256(16 * nblk * C) + align256(2048 * B + 4 * B) bytes of it,
 * with nblk = min(2 * SMs, 512) and align256(x) = x rounded up to 256, and
 * returns LSP_ERR_SHAPE beyond 512 KiB (on 152 SMs: C = 16 fits B <= 217,
 * C = 64 fits B <= 103).  The first successful call on a device looks up the
 * array's device address and the SM count (a failed lookup is retried by the
 * next call); make that first call before any stream capture on the device.
 * Every call shares the array: calls that overlap on the GPU (other streams
 * or threads) race, so the caller must serialise them.  The step counters are
 * cleared on the caller's stream before each launch.  Allocates nothing and
 * calls no allocating CUDA or library routine. */
int lsp_sample_noalloc(const float* base_logits, const int32_t* prev_token, const void* Ec,
                       const void* Wc, int dtype, int C, int B, int V, int rc,
                       const lsp_sample_params* sp, int32_t* out_tokens, float* out_logits,
                       uint32_t* dev_error, lsp_stream_t stream);

/* Prefill (Sec. 2.2, Eq. global-summary, App. A.2; Fig. 3: the summary is
 * initialised over the full prefix during target prefill): replace request
 * b's interface by the one its whole prefix of t = f->rows rows defines --
 * summary (eta, m) = attention of the R summary queries of every tapped layer
 * and query head over all t rows, window ring = the last min(t, W) rows
 * (prefix row p in slot p mod W), boundary = hidden state of row t-1, and t.
 *   f->k, f->v: device dtype [L][t][nkv][d] (request b only); f->h: device
 *   dtype [L][t][H]; borrowed for the call's duration on `stream`.
 * Equivalent to folding the t rows into an empty request with
 * lsp_view_update, but split over the whole GPU (segments of the prefix
 * merged in order with Eq. summary-update; deterministic).  Needs an
 * initialised state (G); bf16 storage with d = 128, 0 <= R <= 16, nq/nkv <= 8 (else
 * LSP_ERR_UNSUPPORTED: use lsp_view_update).  Other requests are untouched. */
int lsp_prefill(lsp_state* st, int b, const lsp_target_feats* f, lsp_stream_t stream);

/* Target-side verification of the drafted blocks (Sec. 2.1, Eq. acceptance,
 * Eq. residual): for each request the candidates y_1..y_B are tested in order,
 * y_i accepted with probability min(1, p_i(y_i) / q_i(y_i)); at the first
 * rejected position i a correction token is drawn from [p_i - q_i]_+; if all B
 * are accepted a bonus token is drawn from p_{B+1}.  p_i = softmax(target
 * logits_i / T), q_i = softmax(draft logits_i / T); T = 0 is greedy (accept
 * y_i iff y_i = argmax p_i, emit argmax p_{r+1}; ties to the lowest index).
 *   target_logits: device float [C][B+1][V] (position B: p(. | s, y_1..y_B));
 *   draft_logits: device float [C][B][V] (lsp_draft's out_logits);
 *   draft_tokens: device int32 [C][B] (lsp_draft's out_tokens);
 *   sp: the round's sampling parameters (the ones lsp_draft used);
 *   accepted_len: device int32 [C] = r in [0, B]; next_token: device int32 [C].
 *   16-byte aligned logits.  The round then advances each request by r + 1
 *   tokens (the next round's accepted_len is r + 1 and its committed token is
 *   next_token).
 * Randomness: Philox4x32-10 with key `seed`; acceptance uniform of position i =
 * word 0 of counter (0, 2^30 + i, b, round), u = ((x >> 9) + 1/2) 2^-23,
 * accepted iff u q_i(y_i) < p_i(y_i); the draw at position i is Gumbel-max with
 * the words of counters (v >> 2, 2^31 + i, b, round).  Drafted tokens outside
 * [0, V) set LSP_DEV_BAD_TOKEN.  Asynchronous on `stream`. */
int lsp_verify(lsp_state* st, const float* target_logits, const float* draft_logits,
               const int32_t* draft_tokens, const lsp_sample_params* sp, int32_t* accepted_len,
               int32_t* next_token, lsp_stream_t stream);

/* Dense projection Y = X W^T with the drafter's tensor-core GEMM (the kernel
 * every projection of lsp_draft uses), for checking it on its own.
 *   X device dtype [M][K]; W device dtype [N][K]; Y device float [M][N].
 *   M <= 512; K * element size a multiple of 16 bytes.
 *   splits: split-K factor (1..16, at most the number of K blocks).  With
 *   splits > 1 the kernel writes fp32 partial sums to `workspace` (device, at
 *   least lsp_linear_workspace_bytes(M, N, splits) bytes) and a second kernel
 *   sums them in split order into Y; with splits == 1 Y is written directly
 *   and `workspace` may be NULL. */
size_t lsp_linear_workspace_bytes(int M, int N, int splits);

/* Diagnostic, host only (needs no GPU): the launch plan the drafter's
 * projection GEMM takes for M token rows, N output features and reduction
 * length K on a device with num_sms SMs.
 *   swiglu = 0: a projection whose fp32 split-K partials a consumer sums
 *   (the q/k/v, o, down and boundary-fusion projections); swiglu = 1: the
 *   fused gate/up projection with N = F (gate and up each [F][K]).
 *   *splits: split-K factor; *tok_groups: CTAs per weight tile, each over
 *   *tokens_per_group consecutive token rows (a multiple of 16).
 * LSP_ERR_ARG for null outputs, M outside [1, 512], N, K or num_sms < 1 or
 * an unknown dtype. */
int lsp_gemm_plan_info(int dtype, int M, int N, int K, int swiglu, int num_sms, int* splits,
                       int* tok_groups, int* tokens_per_group);
int lsp_linear(const void* X, const void* W, float* Y, int M, int N, int K, int dtype,
               int splits, void* workspace, size_t workspace_bytes, lsp_stream_t stream);

/* Raw Philox4x32-10 words of the sampler stream, for checking the generator:
 * out[n] (device uint32) = word (v & 3) of block (v >> 2) with v = n, counter
 * (v >> 2, i, b, round) and key (seed lo32, seed hi32); n < count. */
int lsp_philox_words(uint64_t seed, uint32_t round, uint32_t b, uint32_t i,
                     uint32_t* out, int count, lsp_stream_t stream);

/* Stage timing hook (observability; no effect on results).  With n_events > 0,
 * lsp_view_update and lsp_draft record the caller's CUDA events (cudaEvent_t
 * handles, created by the caller with timing enabled, owned by the caller) at
 * stage boundaries on the call's stream: stage k runs between events[k] and
 * events[k+1].  Stages of one round, in order (lsp_stage_count / lsp_stage_name):
 *   0 view_update, 1 fuse, 2 combine, then per draft layer j: qkv, attention,
 *   o_proj, post_norm, gate_up, down, next_norm, then lm_head and sampler
 *   (with LSP_NO_BOUNDARY the fuse stage is empty).
 * n_events must be 0 (off) or lsp_stage_count(st) + 1.  Event records are
 * capturable, so a captured round carries them as graph nodes. */
int lsp_stage_count(lsp_state* st);
/* Number of kernel launches one round (lsp_view_update + lsp_draft) issues
 * for this state's config on the current device (the sampler is one launch
 * or B + 1 depending on the shape); 0 for a null state. */
int lsp_round_launches(lsp_state* st);
const char* lsp_stage_name(lsp_state* st, int k);
int lsp_set_stage_events(lsp_state* st, void* const* events, int n_events);

/* Read (and clear, if clear != 0) the state's device error word into
 * *dev_error (LSP_DEV_* bits).  Synchronises `stream`.  Returns LSP_OK,
 * or LSP_ERR_TIMEOUT / LSP_ERR_STATE when bits are set. */
int lsp_get_error(lsp_state* st, uint32_t* dev_error, int clear, lsp_stream_t stream);

/* Copy the interface (exactly lsp_state_bytes(cfg) bytes, including t) to /
 * from a host buffer, so a state can be checkpointed or built elsewhere.
 * Synchronous on `stream`. Layout (all per state, dense, in this order):
 *   win_k dtype [C][L][nkv][W][d], win_v dtype [C][L][nkv][W][d],
 *   m float [C][L][nq][R][d], eta float [C][L][nq][R], h dtype [C][L][H],
 *   t int64 [C]. */
int lsp_state_export(lsp_state* st, void* host_buf, size_t bytes, lsp_stream_t stream);
int lsp_state_import(lsp_state* st, const void* host_buf, size_t bytes, lsp_stream_t stream);

/* ---------------------------------------------------------------- target side of a round
 *
 * The round's other half runs in the target: its candidate rows (the committed
 * token and the drafted block) are appended to the target's key/value cache,
 * attend over it, and the proposals are accepted or rejected (Sec. 2.1).  The
 * calls below are its operators over a paged cache that the caller owns.  They
 * need no lsp_state, allocate nothing, and follow the conventions above; a
 * condition that only the device can see sets bits of the optional device word
 * `dev_error` (OR-ed in; NULL: not reported) and the entry concerned is left
 * as it was.  A round, for sequences that share a prompt:
 *   lsp_pages_fork     branches hold the prompt's pages (no data is copied)
 *   lsp_pages_reserve  room for the new rows of each sequence; a page that is
 *                      only partly filled and shared is copied first
 *   per target layer:  lsp_pages_write, lsp_prefix_attention
 *   lsp_verify_probs   (or lsp_verify) accepts r of the drafted tokens
 *   lsp_logprobs       what a server answers beside them: log probabilities,
 *                      entropies, the likeliest alternatives
 *   lsp_pages_trim     gives back the rejected rows' pages
 * A cache held in 4 bits takes lsp_pages_write_q4 and lsp_prefix_attention_q4
 * instead of the two calls per layer.  lsp_pages_read gives the rows of any cache
 * back in the layout that lsp_prefill and lsp_view_update take.
 */

/*
 * A paged key/value cache; every pointer is device memory of the caller.
 *   k, v   element (layer, page, head, slot, dim) at
 *          layer*s_layer + page*s_page + head*s_head + slot*s_slot + dim
 *          (strides in elements, the same for k and v, any order; each a
 *          positive multiple of 16 bytes; k and v 16-byte aligned)
 *   table  [seqs][max_pages]: the page of tokens [i*page, (i+1)*page) of a
 *          sequence, -1 past its last page
 *   len    [seqs] tokens of each sequence
 *   refs   [pages] how many sequences hold each page; 0 = free
 * An empty cache has table = -1, len = 0, refs = 0.  A sequence whose len is
 * outside [0, max_pages * page] counts as one outside the cache: every call
 * leaves an entry with it as it was (LSP_DEV_BAD_SEQ).  So do lsp_pages_fork,
 * trim and reserve where a page they would let go of, hand on or grow is none of
 * the pool.
 * Supported: page 16, 32, 64, 128 or 256; d 64 or 128; dtype BF16, F32 or Q4;
 * pages <= 2^20; seqs * max_pages <= 2^30; max_pages * page <= 2^30.
 *
 * dtype Q4: keys and values in 4 bits, 4.5 with their scales.  Each 32 dims of a
 * token's head are a group: with a = max |x| of its values, s, its scale, is the
 * least number of five significant bits with 7 s >= a (below 2^-126: the least
 * multiple of 2^-130; 0 if a = 0), and x is held as the whole number c in -7..7
 * nearest x / s, ties to even.  It stands for c s: of eight significant bits, so
 * bfloat16 has it exactly (where it passes bfloat16's largest number: infinity).
 * A group with a value that is not finite is held as NaN throughout.
 * The slots of a (layer, page, head) lie in one block of page * d * 9/16 bytes:
 * codes c + 8 [page][d/2 bytes], then scales [page][d/32] in bfloat16.  Element
 * 8 w + 2 k + h (k < 4, h < 2) of a group is at bits 16 h + 4 k of its 32-bit word
 * w.  Strides are in bytes, multiples of 16, s_slot = d * 9/16 (of s_layer, s_page
 * and s_head in any order, each at least the block).  lsp_pages_fork, reserve, trim
 * and compact take such a cache as any other; lsp_pages_write and
 * lsp_prefix_attention refuse it (LSP_ERR_ARG).
 */
typedef struct lsp_kv_cache {
  void* k;
  void* v;
  int32_t* table;
  int32_t* len;
  int32_t* refs;
  int64_t s_layer, s_page, s_head, s_slot;
  int layers, pages, page, nkv, d, dtype, seqs, max_pages;
} lsp_kv_cache;

/* Bytes of device workspace that lsp_pages_reserve and lsp_pages_compact need
 * for this cache (0 for one that is not supported).  Host only. */
size_t lsp_pages_workspace_bytes(const lsp_kv_cache* cache);

/* Sequence dst[i] becomes another holder of src[i]'s pages, and as long (i < n
 * <= 1024; device int32).  What dst[i] held is let go first.  A pair with an
 * index outside [0, seqs), a dst listed before or a dst listed as a src sets
 * LSP_DEV_BAD_SEQ and is skipped.  One launch; no key or value is copied. */
int lsp_pages_fork(const lsp_kv_cache* cache, const int32_t* src, const int32_t* dst, int n,
                   uint32_t* dev_error, lsp_stream_t stream);

/* Make room for add[i] more tokens of sequence seqs[i] (i < n <= 1024; device
 * int32): its len grows by add[i] and its table by the pages this takes.  If
 * its last page is partly filled and other sequences hold it too, it gets its
 * own copy first (the filled slots, every layer); of several such entries of
 * one call the last holder keeps the page.  Pages are handed out in list order,
 * an entry's copy first, each the lowest free one.  An entry with an index
 * outside [0, seqs), listed before, add < 0 or too long for max_pages is
 * skipped (LSP_DEV_BAD_SEQ).  If the free pages do not suffice
 * (LSP_DEV_NO_PAGE), the first entry that does not fit and all after it are
 * left as they were.  workspace: lsp_pages_workspace_bytes, 16-byte aligned,
 * not initialised, not shared with a call that may overlap. */
int lsp_pages_reserve(const lsp_kv_cache* cache, const int32_t* seqs, const int32_t* add, int n,
                      void* workspace, size_t workspace_bytes, uint32_t* dev_error,
                      lsp_stream_t stream);

/* Store the keys and values of new rows in one layer: rows [start[i],
 * start[i+1]) (device int32 [n+1]) become the last start[i+1] - start[i]
 * tokens of sequence seqs[i].  k_new, v_new: device dtype, row r at r *
 * row_stride elements, [nkv][d] dense within (row_stride and the pointers
 * multiples of 16 bytes); total: rows in all.  Rows of an entry whose sequence,
 * range or page is outside the cache are dropped (LSP_DEV_BAD_SEQ). */
int lsp_pages_write(const lsp_kv_cache* cache, int layer, const int32_t* seqs, const int32_t* start,
                    int n, const void* k_new, const void* v_new, int64_t row_stride, int total,
                    uint32_t* dev_error, lsp_stream_t stream);

/* lsp_pages_write into a cache of dtype Q4: the rows are quantised as they are
 * stored.  k_new, v_new: device, `dtype` BF16 or F32, else as there.  (Of rows
 * that one call stores in the same slot, a sequence listed twice, nothing is
 * promised, in either call.) */
int lsp_pages_write_q4(const lsp_kv_cache* cache, int layer, const int32_t* seqs, const int32_t* start,
                       int n, const void* k_new, const void* v_new, int dtype, int64_t row_stride,
                       int total, uint32_t* dev_error, lsp_stream_t stream);

/* Read keys and values of one layer back into dense rows: the last start[i+1] -
 * start[i] tokens of sequence seqs[i] become rows [start[i], start[i+1]) (device
 * int32 [n+1]).  k_out, v_out: device, `dtype` -- the cache's, or BF16 or F32 for
 * a cache of dtype Q4, both exact -- row r at r * row_stride elements, [nkv][d]
 * dense within (row_stride and the pointers multiples of 16 bytes); total: rows in
 * all.  Rows of no entry, and of an entry whose sequence or range is outside the
 * cache (LSP_DEV_BAD_SEQ), are left as they were; tokens of a page outside the
 * pool are zero (LSP_DEV_BAD_SEQ).  The cache is only read. */
int lsp_pages_read(const lsp_kv_cache* cache, int layer, const int32_t* seqs, const int32_t* start,
                   int n, void* k_out, void* v_out, int dtype, int64_t row_stride, int total,
                   uint32_t* dev_error, lsp_stream_t stream);

/* Cut sequence seqs[i] down to its first new_len[i] tokens (i < n <= 1024;
 * device int32; 0 frees it, more than it has changes nothing): the pages past
 * them lose a holder.  An index outside [0, seqs), one listed before or a
 * negative length is skipped (LSP_DEV_BAD_SEQ). */
int lsp_pages_trim(const lsp_kv_cache* cache, const int32_t* seqs, const int32_t* new_len, int n,
                   uint32_t* dev_error, lsp_stream_t stream);

/* Move the live pages (refs > 0) to the front of the pool, every layer: with
 * `live` of them, the k-th live page at an index >= live goes to the k-th free
 * index < live; table and refs follow, whatever a sequence's length.  A table
 * entry that names a free page stays.  live: device int32, receives the count,
 * or NULL.  workspace as for lsp_pages_reserve. */
int lsp_pages_compact(const lsp_kv_cache* cache, int32_t* live, void* workspace,
                      size_t workspace_bytes, lsp_stream_t stream);

/* Bytes of device workspace of lsp_prefix_attention for n sequences and
 * total rows (0 for what it does not support).  The greatest over the calls a
 * program makes is enough for all.  Host only, but it asks the current device
 * for its size. */
size_t lsp_prefix_attention_workspace_bytes(const lsp_kv_cache* cache, int nq, int n, int total);

/* Causal attention of the batch's newest rows over their sequences in one
 * layer of the cache, the pages that all of them share read once for the batch.
 *   q       device dtype, row t at t * q_stride elements, [nq][d] within
 *           (q_stride and q multiples of 16 bytes); nq / nkv a whole number <= 64
 *   seqs    device int32 [n], n <= 1024: the batch's sequences
 *   start   device int32 [n+1]: rows [start[i], start[i+1]) of q, c of them, are
 *           the last c tokens of sequence seqs[i] (already in the cache)
 *   total   rows of q in all
 *   shared_len  the first shared_len tokens of every listed sequence are in the
 *           same pages (as lsp_pages_fork leaves them); 0: nothing is shared.
 *           Only whole pages of it before every row's position are read for
 *           all, from the table of the first sequence that has rows.
 *   scale   > 0, of the scores (d^-1/2 as a rule)
 *   out     device dtype [total][nq][d]; 16-byte aligned
 *   lse     device float [total][nq] or NULL: log sum exp of the scaled scores
 * A row at position t sees tokens 0..t:  out = softmax(scale q K^T) V.  A row
 * with no token to see (a sequence shorter than its rows) gives 0 and lse
 * -inf, and so does one of no sequence, or of one outside the cache
 * (LSP_DEV_BAD_SEQ); table entries outside the pool read as zero keys and values
 * (LSP_DEV_BAD_SEQ).  What lies in unused slots of a page is never seen,
 * whatever its bits; the keys and values of a sequence's own tokens are taken
 * to be finite (a NaN in a key makes out and lse NaN in the rows that see it, one
 * in a row's query in that row; one in a value reaches rows of the call that do
 * not see it yet).  bf16: scores and sums in fp32, weights rounded to bf16 for
 * the product with V; f32: fp32 throughout. */
int lsp_prefix_attention(const lsp_kv_cache* cache, int layer, const void* q, int64_t q_stride,
                         int nq, const int32_t* seqs, const int32_t* start, int n, int total,
                         int shared_len, float scale, void* out, float* lse, void* workspace,
                         size_t workspace_bytes, uint32_t* dev_error, lsp_stream_t stream);

/* The same for lsp_prefix_attention_q4 with rows of `dtype`. */
size_t lsp_prefix_attention_q4_workspace_bytes(const lsp_kv_cache* cache, int dtype, int nq, int n,
                                               int total);

/* lsp_prefix_attention over a cache of dtype Q4, whose keys and values enter as
 * the numbers they stand for: the same rows, shared pages and results, for q and
 * out of `dtype` BF16 or F32.  (One past bfloat16's largest number enters as
 * infinity or as itself.)  A group that is NaN makes NaN, in the rows that see it
 * and no others, of out and lse if it is a key's, of its dims of out if it is a
 * value's, whatever its weight.  Nothing is unpacked to memory.  bf16: scores and
 * sums in fp32, weights rounded to bf16 for the product with V.  f32: q and the
 * weights enter the tensor cores as sums of three bf16 numbers each (24 bits), the
 * products are exact and summed in fp32.  scale up to 2^120.  workspace: at least
 * lsp_prefix_attention_q4_workspace_bytes, 256-byte aligned, not initialised. */
int lsp_prefix_attention_q4(const lsp_kv_cache* cache, int layer, const void* q, int dtype,
                            int64_t q_stride, int nq, const int32_t* seqs, const int32_t* start, int n,
                            int total, int shared_len, float scale, void* out, float* lse,
                            void* workspace, size_t workspace_bytes, uint32_t* dev_error,
                            lsp_stream_t stream);

/* Acceptance of drafted tokens (Eq. acceptance, Eq. residual) from
 * probabilities and random numbers that the caller gives: lsp_verify for
 * programs that shape their distributions (top-k, top-p, ...) or draw their
 * randomness elsewhere.
 *   target_probs  device dtype, row (b, i) of [C][B+1] at (b (B+1) + i) ld_target
 *           elements, V within: p_{i+1}; need not be normalised
 *   draft_probs  the same for [C][B] with ld_draft: q_{i+1}; NULL: the drafts were
 *           not drawn (each q a point mass on its token)
 *   draft_tokens  device int32 [C][B];  n_draft: device int32 [C], how many of
 *           them count, in [0, B] (else clamped, LSP_DEV_BAD_DELTA); NULL: all
 *   u       device float [C][B], uniforms of the acceptance tests
 *   e       device float [C][V], Exp(1) variates of the draw
 * y_i is accepted iff u_i q_i(y_i) < p_i(y_i), in order, in fp32; with r accepted,
 * next_token = argmax_v w_v / e_v over w_v > 0, w = [p_{r+1} - q_{r+1}]_+ if y_{r+1}
 * was rejected (p_{r+1} where that is 0 throughout), w = p_{r+1} if none was left;
 * ties go to the lowest index, -1 if no w_v > 0.  A drafted token outside [0, V)
 * is rejected (LSP_DEV_BAD_TOKEN).
 *   accepted_len, next_token  device int32 [C]
 *   out_tokens  device int32 [C][B+1] or NULL: the accepted tokens, next_token, -1
 * C >= 1, B in [0, 1024], V in [1, 2^30], ld >= V.  One launch. */
int lsp_verify_probs(const void* target_probs, const void* draft_probs, int dtype,
                     const int32_t* draft_tokens, const int32_t* n_draft, const float* u,
                     const float* e, int C, int B, int V, int64_t ld_target, int64_t ld_draft,
                     int32_t* accepted_len, int32_t* next_token, int32_t* out_tokens,
                     uint32_t* dev_error, lsp_stream_t stream);

/* Log probabilities of given tokens (what lsp_verify_probs leaves in out_tokens,
 * or any others), with the entropy and the likeliest alternatives of each row of
 * logits.  With x_v = z_v / T and lse = log sum_v exp(x_v), per row:
 *   logprob = x_token - lse,  entropy = lse - sum_v exp(x_v - lse) x_v  (nats; a
 *   term of x_v = -inf is 0),  and the k largest z_v in order, ties to the lowest
 *   index: top = their v, top_logprob = x_v - lse.
 *   logits  device dtype BF16 or F32, row r at r * ld elements, V within, no
 *           alignment beyond the type's
 *   tokens  device int32 [rows]; -1: no token, the row is not read and gives
 *           logprob -inf, entropy 0, top -1 and top_logprob -inf.  One outside
 *           [-1, V) is taken as -1 (LSP_DEV_BAD_TOKEN)
 *   logprob, entropy  device float [rows];  entropy may be NULL
 *   top     device int32 [rows][k], top_logprob device float [rows][k]; either may
 *           be NULL, and both are not written with k = 0
 * A row whose largest logit is not finite (all -inf, a +inf) or that has a NaN has
 * no distribution: NaN in logprob, entropy and top_logprob, -1 in top.  (In other
 * rows tokens of -inf follow the finite ones, with top_logprob -inf.)
 * T in [2^-100, 2^100]; rows in [0, 2^27], V in [1, 2^26], ld >= V, k in
 * [0, min(V, 32)].  One launch; each row is read once, and what may hold its k
 * largest logits once more (k times where more than a thousand that belong there
 * crowd into a few places of a row).  In fp32; the same call gives the same bits.
 * How many rows there are, and a row's address modulo 16 bytes, decide how it is
 * split: its sums may differ in their last bits, the tokens never. */
int lsp_logprobs(const void* logits, int dtype, const int32_t* tokens, int rows, int V, int64_t ld,
                 float temperature, int k, float* logprob, float* entropy, int32_t* top,
                 float* top_logprob, uint32_t* dev_error, lsp_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* LSP_H */
