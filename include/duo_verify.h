/*
 * duo_verify.h -- C ABI of the MI355X (gfx950) target-side verification step of DuoDecoding
 * (arxiv 2503.00784).
 *
 * One call scores n draft sequences of k tokens with the target model in a single forward
 * pass (Alg. 1, right column: p <- M_p(x); Sec. 1: all candidates are scored by one pass of the
 * target), the sequences being independent branches of a shared prefix (Sec. 3.2,
 * Fig. 2), then verifies them by speculative sampling (Alg. 2, Sec. 3.3) and commits the
 * accepted tokens' keys and values to the cache.  The draft model, the draft budget and the
 * CPU/GPU scheduling of Alg. 1 are host work and not part of this library: draft tokens,
 * draft distributions and the uniform random numbers of Alg. 2 are inputs.
 *
 * Conventions
 *   - Every pointer below is a DEVICE pointer unless it is marked HOST.  The library never
 *     allocates, frees or keeps caller memory; scratch space is the caller's `workspace`.
 *   - All work is enqueued on `hip_stream` (a hipStream_t cast to void*; NULL = default
 *     stream) without host synchronisation.  Arguments are validated on the host before
 *     anything is enqueued; a negative return code means nothing was enqueued.
 *   - 16-bit values (weights, gains, embedding, KV cache) are passed as uint16_t bit patterns.  The library is
 *     built twice from the same sources with the same entry points: libduo_verify.so takes them as bf16
 *     (wherever this header says bf16), libduo_verify_fp16.so as IEEE fp16, the precision the paper ran its
 *     target model in (Sec. 4.1).  A process may load both.  Matrices compute y = x W^T, are 16-byte
 *     aligned, and have an input dimension that is a multiple of 32.
 *   - A call with the same inputs and the same `host_prefix_len` is repeatable: cache slots
 *     below the prefix length are only read, slots at and above it are scratch.
 */
#ifndef DUO_VERIFY_H
#define DUO_VERIFY_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DUO_OK               0
#define DUO_ERR_NULL        -1  /* a required pointer is NULL */
#define DUO_ERR_SHAPE       -2  /* unsupported model geometry or n, k out of range */
#define DUO_ERR_CAPACITY    -3  /* prefix + rows of this call exceed max_seq */
#define DUO_ERR_ALIGN       -4  /* a pointer is not 16-byte aligned */
#define DUO_ERR_WORKSPACE   -5  /* workspace smaller than duo_workspace_bytes() */
#define DUO_ERR_TOKEN_RANGE -6  /* root_token >= vocab */
#define DUO_ERR_HIP         -7  /* a HIP call failed; see duo_last_hip_error() */
#define DUO_ERR_ARG         -8  /* temperature < 0 or NaN, unknown select_mode, ... */
#define DUO_ERR_SCRATCH     -9  /* duo_spec_sample_noalloc: vocabulary above DUO_NOALLOC_MAX_VOCAB, or top_p asked for */

/* Most rows one call can score: n*k (+1 with a root token). */
#define DUO_MAX_ROWS 80
#define DUO_MAX_PREFILL_ROWS 1024 /* rows of one duo_prefill_chunk call */

/* Bits of the device-side status word (duo_result.status), set by kernels that cannot be
 * checked on the host without a synchronisation.  A call whose status word is not clean FAILED ON THE DEVICE and
 * commits nothing: *cache.prefix_len and every cache slot below it are left exactly as they were (on a prefix
 * mismatch the pass writes no keys or values at all; slots at and above the device's prefix length are scratch in any
 * case), root_logits is not replaced by duo_prefill_chunk, and the commit record reads
 * {-1, 0, -1, unchanged prefix length}.  accept_len / next_token / logits_out then hold no usable result. */
#define DUO_STATUS_TOKEN_CLAMPED   1  /* a draft token id was outside [0, vocab) and was clamped */
#define DUO_STATUS_PREFIX_MISMATCH 2  /* *cache.prefix_len differed from call.host_prefix_len */

#define DUO_SELECT_INDEPENDENT_LONGEST 0
#define DUO_SELECT_PAPER_SEQUENTIAL    1

/* Geometry of the Llama-shaped target (the architecture of the paper's targets, Sec. 4.1
 * "Models").  head_dim is 64 or 128; d_model is a multiple of 64 (at most 8192), n_q_heads*head_dim and d_ff
 * are multiples of 32; n_q_heads is a multiple of n_kv_heads; max_seq is a multiple of 32. */
typedef struct duo_model_config {
    int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ff, vocab, max_seq;
    float   rope_theta; /* rotary base; pair (d, d + head_dim/2) turns by pos * theta^(-2d/head_dim) */
    float   rms_eps;
} duo_model_config;

/*
 * Parameters, bf16.  Every matrix the step streams is held in the library's STREAMING LAYOUT, made
 * once at load time by the duo_pack_* calls below from ordinary row-major [out][in] matrices: bands
 * of 16 output rows, cut into 16 x 32 tiles of 1 KiB that are contiguous and ordered the way one MFMA
 * operand sits in a wavefront's registers, so that a wave reads its band as one linear stream.  The
 * embedding table is gathered, not streamed, and stays row-major.  The seven per-layer tables are
 * HOST arrays of n_layers DEVICE pointers.
 */
typedef struct duo_weights {
    const uint16_t *embed;                    /* row-major [vocab][d_model] */
    const uint16_t *const *wqkv;              /* duo_pack_qkv of wq [n_q_heads*head_dim][d_model] and
                                                 wk, wv [n_kv_heads*head_dim][d_model] */
    const uint16_t *const *wo;                /* duo_pack_matrix of [d_model][n_q_heads*head_dim] */
    const uint16_t *const *w_gate_up;         /* duo_pack_gate_up of w_gate, w_up [d_ff][d_model] */
    const uint16_t *const *w_down;            /* duo_pack_matrix of [d_model][d_ff] */
    const uint16_t *const *g_attn, *const *g_ffn; /* RMSNorm gains [d_model] */
    const uint16_t *g_final;                  /* [d_model] */
    const uint16_t *lm_head;                  /* duo_pack_matrix of [vocab][d_model] */
} duo_weights;

/*
 * Repacking into the streaming layout (device to device, enqueued on the stream, done once per
 * model).  src matrices are row-major bf16, 16-byte aligned, K a multiple of 32.  dst needs
 * duo_packed_elems(N, K) uint16 elements: N is rounded up to a multiple of 32 rows, missing rows are
 * zero.  duo_pack_qkv needs duo_packed_elems((n_q_heads + 2*n_kv_heads)*head_dim, d_model) and orders
 * the rows so that every band holds eight channels of a head next to their eight rotary partners;
 * duo_pack_gate_up needs duo_packed_elems(2*d_ff, d_model) and interleaves gate and up bands.
 */
size_t duo_packed_elems(int N, int K);
int duo_pack_matrix(const uint16_t *src, int N, int K, uint16_t *dst, void *hip_stream);
int duo_pack_qkv(const duo_model_config *cfg, const uint16_t *wq, const uint16_t *wk, const uint16_t *wv,
                 uint16_t *dst, void *hip_stream);
int duo_pack_gate_up(const duo_model_config *cfg, const uint16_t *w_gate, const uint16_t *w_up, uint16_t *dst,
                     void *hip_stream);
/* Activation rows [rows][K] (row-major) -> operand layout for duo_skinny_gemm; dst needs
 * ((rows + 15) / 16) * 16 * K elements. */
int duo_pack_activations(const uint16_t *src, int rows, int K, uint16_t *dst, void *hip_stream);

/* KV cache, bf16, caller-owned: k and v each hold n_layers * n_kv_heads planes of max_seq * head_dim
 * elements (plane index layer * n_kv_heads + kv_head).  Inside a plane both are stored as the 1 KiB tiles the
 * attention kernels feed to the matrix cores, 32 slots at a time, so that a wavefront fetches a tile with one
 * fully coalesced load.  Keys are stored after the rotary embedding.  With D = head_dim, block B = slot / 32
 * and w = slot % 32, the element (slot, channel d) of a plane is at
 *   K: ((((B*2 + t) * (D/32) + d/32) * 64 + ((d%32)/8) * 16 + 4*(w/8) + w%4) * 8 + d%8,  t = (w%8)/4
 *   V: (((B * (D/16) + d/16) * 64 + (w/8) * 16 + d%16) * 8 + w%8
 * (V is in effect transposed: a lane's eight consecutive elements are eight consecutive slots of one channel).
 * duo_k_cache_offset / duo_v_cache_offset evaluate these on the host.  Slots [0, *prefix_len) hold the shared
 * prefix. */
size_t duo_k_cache_offset(int head_dim, int slot, int channel);
size_t duo_v_cache_offset(int head_dim, int slot, int channel);

typedef struct duo_kv_cache {
    uint16_t *k;
    uint16_t *v;
    int32_t  *prefix_len;   /* device scalar P; advanced by the commit */
    float    *root_logits;  /* fp32 [vocab]: target logits after the last prefix token (from
                               prefill); read when root_token < 0, may be NULL otherwise */
} duo_kv_cache;

typedef struct duo_call {
    int32_t n, k;            /* n sequences of k draft tokens, n*k + (root?1:0) <= DUO_MAX_ROWS */
    float   temperature;     /* p = softmax(logits / temperature), > 0; exactly 0 = the greedy limit of Alg. 2: p is
                                one-hot at the largest logit (lowest id among equal logits), so a draft token is
                                accepted iff it is that id and every correction / bonus token is that id; the
                                uniforms are still read but cannot change the outcome */
    int32_t select_mode;     /* DUO_SELECT_* */
    int32_t root_token;      /* >= 0: the token emitted by the previous step, scored as one shared
                                row in front of every sequence (its logits judge the first draft
                                tokens); < 0: cache.root_logits judges them */
    int32_t host_prefix_len; /* P as the host knows it; sizes the launch and is checked on device */
    float   top_p;           /* 0 < top_p < 1 (and temperature > 0): every target distribution is first restricted to its
                                nucleus, the most probable tokens in order of decreasing probability (equal ones by
                                ascending id) up to and including the one with which their mass reaches top_p, and
                                renormalised; Alg. 2 then runs on the restricted distributions.  Any other value
                                (0 included): no restriction.  The draft distributions are taken as given. */
} duo_call;

/* Outputs (device).  Alg. 2 returns the new prefix length, the new prefix and the unverified
 * suffix; here: per-sequence accepted lengths, the correction / bonus token, and the commit. */
typedef struct duo_result {
    int32_t *accept_len; /* [n]  leading accepted draft tokens of each sequence; in paper mode 0 for
                                 sequences rejected before the selected one, -1 for those after it */
    int32_t *next_token; /* [n]  correction token (residual sample at the first rejection) or bonus
                                 token (all k accepted); paper mode: only the selected entry, else -1 */
    int32_t *commit;     /* [4]  {selected sequence or -1, commit_len, commit_token, new prefix length} */
    int32_t *status;     /* [1]  DUO_STATUS_* bits, 0 when clean */
    float   *logits_out; /* optional fp32 [rows][vocab] (rows = (root?1:0) + n*k), may be NULL */
} duo_result;

/* Bytes of device scratch a call of up to `max_rows` rows needs: duo_verify takes at most DUO_MAX_ROWS rows,
 * duo_prefill_chunk at most DUO_MAX_PREFILL_ROWS.  Not monotonic across DUO_MAX_ROWS (a pass of more rows keeps the
 * logits of its last row only): a caller that makes both kinds of call allocates the larger of
 * duo_workspace_bytes(DUO_MAX_ROWS) and duo_workspace_bytes(its largest prefill chunk). */
int duo_workspace_bytes(const duo_model_config *cfg, int max_rows, size_t *bytes);

/*
 * The whole step.  Rows: the root token (if any) at position P and cache slot P, draft token
 * (i, j) at position P + R + j and slot P + R + i*k + j (R = 1 with a root token).  Row (i, j)
 * attends to the prefix, the root and (i, j' <= j).  logits of row (i, j) score the token after
 * draft (i, j): draft (i, 0) is judged by the root distribution, draft (i, j >= 1) by row
 * (i, j-1), the bonus token is drawn from row (i, k-1).
 *
 * Speculative sampling (Alg. 2; accept iff u * q(t) < p(t), i.e. with probability
 * min(1, p/q); on rejection sample norm(max(0, p - q)) by inverse CDF over ascending ids):
 *   INDEPENDENT_LONGEST  every sequence is verified on its own, token by token, as one sequence is in plain
 *                        speculative sampling (Sec. 3.3); the longest (lowest index on ties) is committed.
 *   PAPER_SEQUENTIAL     first tokens are tested in order against the root distribution, which
 *                        is replaced by its normalised residual after each rejection (Alg. 2,
 *                        multi-sequence block); the first accepted sequence is verified to its
 *                        end; if none is accepted a token is drawn from the final residual.
 * uniforms[i][j] (j < k) tests draft (i, j); uniforms[i][k] drives the correction / bonus sample
 * (paper mode, none accepted: uniforms[n-1][k]).
 *
 * Commit: keys/values of the selected sequence's first commit_len tokens are moved to slots
 * P + R + 0.., *prefix_len becomes P + R + commit_len.  The emitted token is not in the cache;
 * pass it as root_token to the next call.
 *
 * draft_tokens int32 [n][k]; draft_probs fp32 [n][k][vocab] (full draft distributions, needed
 * for residuals); uniforms fp32 [n][k+1] in [0, 1).
 */
int duo_verify(const duo_model_config *cfg, const duo_weights *w, duo_kv_cache *cache,
               const int32_t *draft_tokens, const float *draft_probs, const float *uniforms,
               const duo_call *call, duo_result *out,
               void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Scores m <= DUO_MAX_PREFILL_ROWS tokens (device int32) as a continuation of the cached prefix with a
 * plain causal mask, appends their keys/values, advances *prefix_len by m and stores the last
 * row's logits in cache->root_logits: the target pass of Alg. 1 applied to prompt tokens (the target model's
 * share of the time to first token, Sec. 4.1).  Up to DUO_MAX_ROWS rows run through the verify pass's
 * weight-streaming kernels; more rows through projection kernels that stage both operands in LDS, and only
 * the last row's logits are computed.  `workspace` needs duo_workspace_bytes(cfg, m) bytes.
 */
int duo_prefill_chunk(const duo_model_config *cfg, const duo_weights *w, duo_kv_cache *cache,
                      const int32_t *tokens, int m, int host_prefix_len, int32_t *status,
                      void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Speculative sampling alone (the second half of duo_verify) on logits the caller supplies:
 * logits fp32 [R + n*k][vocab] with row stride `vocab`.  Does not touch any KV cache; writes
 * accept_len, next_token and commit as duo_verify does (new prefix length = host_prefix_len +
 * R + commit_len).  `workspace` needs duo_sample_workspace_bytes(vocab, n, k) bytes.
 */
int duo_sample_workspace_bytes(int vocab, int n, int k, size_t *bytes);
int duo_spec_sample(const float *logits, const float *root_logits, int vocab,
                    const int32_t *draft_tokens, const float *draft_probs, const float *uniforms,
                    const duo_call *call, duo_result *out,
                    void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * duo_spec_sample for callers that cannot allocate or pass a workspace (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc): the same sampling kernels, with their scratch (softmax statistics, accept
 * flags, one running distribution) in a static device array of DUO_NOALLOC_SCRATCH_BYTES inside the library, which
 * every device the library runs on holds until the process ends.  Same arguments and results as duo_spec_sample
 * without the workspace.  Limits: vocab <= DUO_NOALLOC_MAX_VOCAB and no nucleus restriction (0 < top_p < 1 at a
 * positive temperature), else DUO_ERR_SCRATCH and nothing is enqueued.  Calls no hipMalloc / hipFree and no
 * allocating routine.  The first call on a device (with that device current, as for every call) asks the runtime
 * for the address of that device's copy of the array; make it outside a stream capture.  All calls on one device
 * share the array: calls that overlap on one device (different streams) race, calls on one stream do not.  Nothing
 * in the array needs clearing between calls: every entry a call reads it has written first.
 */
#define DUO_NOALLOC_MAX_VOCAB 131072
#define DUO_NOALLOC_SCRATCH_BYTES (20480 + 131072 * 8 + 512)
int duo_spec_sample_noalloc(const float *logits, const float *root_logits, int vocab,
                            const int32_t *draft_tokens, const float *draft_probs, const float *uniforms,
                            const duo_call *call, duo_result *out, void *hip_stream);

/*
 * Alg. 2 in the form the paper lists it, for one round of the pipelined loop of Alg. 1: the pass
 * scores the l tokens that the previous round appended without verifying them (the unverified
 * suffix), then
 *   - verifies them in order (accept token m iff u_m * q_m(t) < p_m(t)); at the first rejection the
 *     token is replaced by a draw from norm(max(0, p_m - q_m)) and everything after it is dropped;
 *   - if all l were accepted, judges ONLY THE FIRST TOKEN of each of s new draft sequences, in index
 *     order, against the target distribution after the last scored token, replacing that
 *     distribution by its normalised residual after every rejection; the first accepted sequence is
 *     taken whole (its first token verified, the rest becoming the next round's unverified suffix);
 *   - if none is accepted, draws one token from the final residual.
 * Inputs (device): unverified_tokens int32 [l]; unverified_probs fp32 [l][vocab] (the draft
 * distributions they were drawn from); uniforms fp32 [l + 1]: u_0 .. u_{l-1} and the uniform of the
 * final draw; first_tokens int32 [s], first_probs fp32 [s][vocab], uniforms_first fp32 [s] (s may be
 * 0: then the pointers may be NULL and the last case applies).  call->n must be 1, call->k = l,
 * call->select_mode must hold a valid value and is otherwise ignored, root_token / host_prefix_len as in
 * duo_verify; s <= DUO_MAX_ROWS.
 * l = 0 is the round after a rejection (Alg. 2 then leaves no unverified suffix) and the first round after the
 * prompt: unverified_tokens / unverified_probs may be NULL, uniforms holds the one uniform of the final draw, and
 * the new sequences are judged by the distribution after the root token (the pass scores that one row), or, with
 * root_token < 0, by cache.root_logits without any forward pass.
 * Outputs: out->accept_len[0] = number of accepted suffix tokens a (0..l); out->commit =
 * {index of the accepted new sequence or -1, a, emitted token or -1 when a sequence was accepted,
 * new prefix length P + R + a}; out->next_token[0] = the emitted token or -1.  The keys/values of
 * the accepted suffix tokens stay where the pass wrote them (slots P + R ..) and *prefix_len becomes
 * P + R + a.  An accepted sequence is not in the cache yet: the next round passes its first token as
 * root_token and the rest as the unverified suffix.
 */
int duo_verify_deferred(const duo_model_config *cfg, const duo_weights *w, duo_kv_cache *cache,
                        const int32_t *unverified_tokens, const float *unverified_probs, const float *uniforms,
                        const int32_t *first_tokens, const float *first_probs, const float *uniforms_first,
                        int s, const duo_call *call, duo_result *out,
                        void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * The sampling half of duo_verify_deferred on logits the caller supplies (fp32 [R + l][vocab], row
 * stride vocab; root_logits judge the first suffix token when call->root_token < 0).  No KV cache is
 * touched; `workspace` needs duo_sample_workspace_bytes(vocab, 1, l) bytes.
 */
int duo_deferred_sample(const float *logits, const float *root_logits, int vocab,
                        const int32_t *unverified_tokens, const float *unverified_probs, const float *uniforms,
                        const int32_t *first_tokens, const float *first_probs, const float *uniforms_first,
                        int s, const duo_call *call, duo_result *out,
                        void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * ---- Many requests on a paged cache.
 *
 * duo_verify serves one request whose cache is one plane of max_seq slots.  A server holds many requests of very
 * different lengths: their keys and values lie in PAGES of a common pool, and a step of all of them is
 *
 *   duo_page_plan -> for every layer (duo_page_append -> duo_page_attention) -> sampling -> duo_page_commit
 *
 * with the projections in between as the caller makes them.  A request has `cached` tokens in the cache and brings new
 * rows: `trunk` tokens in a row (the token emitted last, a prompt or a part of one), then n branches of k draft tokens,
 * each a continuation of the trunk (n * k = 0: none).  Its new rows are consecutive rows of the step's matrices, trunk
 * first, then branch after branch; row t lies in the request's logical slot cached + t and has the rotary position
 * cached + t in the trunk, cached + trunk + j for token j of a branch.  A row sees the request's cached slots, the trunk up
 * to itself and the tokens of its own branch up to itself.  trunk = n * k = 0 is a request that sits this step out.
 *
 * Logical slot s of request r is slot s % page_slots of page block_table[r][s / page_slots].  Inside a page the planes
 * [n_kv_heads][page_slots * head_dim] hold the tiles described at duo_kv_cache (duo_k_cache_offset / duo_v_cache_offset
 * with the slot in the page).
 *
 * What the lengths ask for is decided on the device from the arrays of duo_page_batch: calls are sized by the batch's
 * maxima alone, so a captured graph of a step serves steps of other lengths.  What only the device can see is reported in
 * batch.status (DUO_PAGE_* bits, cleared by duo_page_plan):
 *   a plan that fails (NO_PAGES, BAD_REQUEST) changes no table, takes no page, sets every slot and position to -1, and the
 *   calls behind it do nothing, until a plan succeeds;
 *   a page id outside the pool (BAD_PAGE) is not followed: its keys and values are not written, and reads take page 0
 *   instead (the request's output is then of no use);
 *   a workspace that holds no plan of this batch and geometry (NO_PLAN): the call does nothing;
 *   a commit record that names no branch of its request (BAD_RECORD): nothing of that request is committed.
 */
#define DUO_PAGE_NO_PAGES    4  /* fewer free pages than the step needs */
#define DUO_PAGE_BAD_REQUEST 8  /* a length or count of the batch or the tables is negative or beyond its maximum */
#define DUO_PAGE_BAD_PAGE   16
#define DUO_PAGE_NO_PLAN    32
#define DUO_PAGE_BAD_RECORD 64

#define DUO_PAGE_MAX_REQUESTS 4096
#define DUO_PAGE_MAX_ROWS     262144   /* rows of a step */
#define DUO_PAGE_MAX_SLOTS    8388608  /* slots of a request: max_pages * page_slots */

typedef struct duo_page_cache {
    uint16_t *k, *v;         /* [n_layers][n_pages][n_kv_heads][page_slots * head_dim] each, 16-byte aligned */
    int32_t n_pages;         /* n_pages * page_slots < 2^31 */
    int32_t page_slots;      /* 32, 64, 128, ... 1024 */
    int32_t max_pages;       /* columns of the block table: the most pages of a request */
} duo_page_cache;

/* Who holds which page.  A caller starts with held = 0 everywhere and free_pages = all page ids in any order. */
typedef struct duo_page_tables {
    int32_t *block_table;    /* [n_requests][max_pages]; columns from held[r] on are neither read nor written */
    int32_t *held;           /* [n_requests] pages of the request */
    int32_t *free_pages;     /* [n_pages] a stack; what a plan finds behind *free_count is not read, and written only up to the new count */
    int32_t *free_count;     /* [1] */
} duo_page_tables;

typedef struct duo_page_batch {
    const int32_t *cached, *trunk, *n, *k;  /* [n_requests] */
    int32_t *row_start;      /* [n_requests + 1] by duo_page_plan: first row of every request, then the rows in all */
    int32_t *position;       /* [max_rows] by duo_page_plan: rotary position of a row, -1 behind the last row */
    int32_t *slot;           /* [max_rows] by duo_page_plan: page * page_slots + slot in the page, -1 behind the last row */
    int32_t *status;         /* [1] */
    int32_t n_requests;      /* rows of the block table, at most DUO_PAGE_MAX_REQUESTS */
    int32_t max_rows;        /* rows of the step's matrices, at most DUO_PAGE_MAX_ROWS */
    int32_t max_new;         /* the most new rows of a request, at most max_rows */
} duo_page_batch;

/* Bytes of workspace of the calls below for this geometry (the fields of batch that count are n_requests, max_rows and
 * max_new; the pointers of cache and batch are not looked at).  duo_page_plan leaves the step's schedule in it, which duo_page_attention
 * and duo_page_commit read, and attention keeps partial results there: one workspace per step in flight, and the calls on it one after
 * another.  How the keys are split over workgroups, and with it the order of the sums, follows from the lengths of all requests of the
 * step, from the batch's maxima and from max_pages * page_slots; equal steps give equal bits. */
int duo_page_workspace_bytes(const duo_model_config *cfg, const duo_page_cache *cache, const duo_page_batch *batch, size_t *bytes);

/*
 * Plans a step: every request gets exactly the ceil((cached + new rows) / page_slots) pages it needs.  Requests that hold
 * more (rejected branches, a request that has ended: cached = trunk = n * k = 0) release their last columns.  With F free
 * pages the released ones (requests in order, columns ascending) are pushed behind them; missing pages are popped from
 * that stack in the order in which requests and columns ask for them.  Writes row_start, position, slot and status of the batch and
 * the schedule in the workspace.  `to` may be `from` (in place); otherwise the two share no memory, and `from` is left as it is.
 * Of tables with more rows than n_requests the rows behind are left alone, in `to` as well.
 * A request may hold fewer pages than its cached tokens take, one whose keys and values are to be brought back from elsewhere for instance: it is
 * given pages for those columns too and status stays 0.  What lies in them is the caller's to write in front of the step's attention, which until
 * then reads what the pages' last owner left there; a caller that brings nothing back has to hold held * page_slots >= cached.
 */
int duo_page_plan(const duo_model_config *cfg, const duo_page_cache *cache, const duo_page_tables *from, const duo_page_tables *to,
                  const duo_page_batch *batch, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Rotates queries and keys of max_rows rows to their positions and writes keys and values into the pages of `layer`: q
 * [max_rows][n_q_heads * head_dim], k and v [max_rows][n_kv_heads * head_dim], each with its own distance between rows in elements (a
 * multiple of 8; so they can be column ranges of one projection's output).  q_out as q; it is q or shares no element with it, and none with
 * k or v (else DUO_ERR_ARG; column ranges of one matrix, the same distance between rows, are told apart, other matrices by the ranges of their
 * addresses).  Rows whose slot is -1 are left out, in q_out too; the slots of the others differ.  Only position, slot, status and max_rows of the
 * batch are read.  The rotation is computed in fp32 from angles reduced in double precision, and rounded once.
 */
int duo_page_append(const duo_model_config *cfg, const duo_page_cache *cache, const duo_page_batch *batch, int layer,
                    const uint16_t *q, int64_t q_stride, const uint16_t *k, int64_t k_stride, const uint16_t *v, int64_t v_stride,
                    uint16_t *q_out, int64_t q_out_stride, void *hip_stream);

/*
 * out = softmax(scale q K^T) V of every row of the planned step over what it sees (grouped heads: query head h reads kv
 * head h / (n_q_heads / n_kv_heads)).  q and out as above; out shares no element with q (else DUO_ERR_ARG); rows of out behind the step's last
 * row are left as they are.  scale > 0, or 0 for 1 / sqrt(head_dim).  Scores, maxima, sums and outputs are fp32; softmax weights
 * enter the second product in the 16-bit type, as pairs (hi + lo) for requests of at most 64 rows * heads of a group,
 * once rounded beyond; the output is rounded once.  Weights that the type does not hold become zero, next to a row's largest of 1: below 2^-126
 * in bf16; below 2^-32 in fp16, where weights of less than 2^-21 are off by up to that.  What a row does not see does not touch it, infinities
 * and NaN included; an infinite value or NaN that it sees reaches its channel however small the weight is (down to fp32's least).
 * The fp32 sums are divided at the end: values whose sum under weights of up to 2^8 is beyond fp32 (bf16 values of 2^100 and more) may give infinity.
 */
int duo_page_attention(const duo_model_config *cfg, const duo_page_cache *cache, const int32_t *block_table, const duo_page_batch *batch,
                       int layer, const uint16_t *q, int64_t q_stride, uint16_t *out, int64_t out_stride, float scale,
                       void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Commits the planned step.  records int32 [n_requests][4] are commit records as duo_spec_sample writes them: {accepted
 * branch or -1, its accepted tokens a, emitted token, ...}.  In every layer the keys and values of the branch's first a tokens
 * move to the slots behind the trunk, and cached_out[r] = cached + trunk + a.  Branch -1: a = 0, the trunk alone is
 * committed.  Branch and token both -1 (a sampling call that failed on the device), or a record that names no branch:
 * cached_out[r] = cached.  Requests without branches commit their trunk whatever the record holds.  cached_out may be
 * batch.cached.  Pages that are no longer needed are released by the next plan.
 */
int duo_page_commit(const duo_model_config *cfg, const duo_page_cache *cache, const int32_t *block_table, const duo_page_batch *batch,
                    const int32_t *records, int32_t *cached_out, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * ---- Matrices in 8-bit floating point.
 *
 * A verify step of few rows is the stream of its matrices; held in e4m3 (4 exponent bits, 3 mantissa bits, magnitudes up to
 * 448) they are half as many bytes.  Every block of 128 rows x 128 columns has a scale, a power of two 2^e: the smallest that
 * brings the block's largest finite magnitude to 448 or below, e kept within [-110, 120].  A stored value is e4m3(v / 2^e),
 * rounded to nearest even; infinities and NaN are stored as NaN.  (bf16 magnitudes from 1.9375 * 2^127 on round to 2^128, which is infinite in
 * fp32 and as a factor of a product.)
 *
 * duo_scaled_pack makes such a matrix, once, from row-major [N][K] in 16 bits (16-byte aligned, K a multiple of 32):
 * duo_scaled_bytes(N, K) bytes (0 for sizes that are not taken), 16-byte aligned.  With NB = ceil(N / 128) and KB =
 * ceil(K / 128), value (n, k) is byte ((n / 16) * KB + k / 128) * 2048 + ((k % 128) / 64) * 1024 + ((k % 64) / 16) * 256 +
 * (n % 16) * 16 + k % 16, and the scale of block (n / 128, k / 128) is byte NB * KB * 16384 + (n / 128) * KB + k / 128, as e + 127;
 * rows and columns that fill up the last blocks are zero.
 */
#define DUO_SCALED_MAX_N      1048576
#define DUO_SCALED_MAX_K      65536
#define DUO_SCALED_MAX_ROWS   262144
#define DUO_SCALED_DIRECT_ROWS 16  /* up to which a product needs no workspace */
#define DUO_SCALED_MAX_STRIDE 2147483647 /* elements from row to row */
size_t duo_scaled_bytes(int N, int K);
int duo_scaled_pack(const uint16_t *src, int N, int K, void *dst, void *hip_stream);

/*
 * y[m][n] = sum over k of x'[m][k] * w[n][k], w from duo_scaled_pack.  x' is x brought to e4m3 on the way, by the same rule
 * with a scale for every 128 consecutive values of a row (a row with an infinity or NaN becomes NaN, the others are not touched).
 * x [rows][K] in 16 bits, x_stride elements from row to row (a multiple of 8, at least K).  y [rows][N] in 16 bits, or in fp32
 * where y_fp32 is 1, y_stride elements from row to row (a multiple of 8, of 4 in fp32; at least N).  x, w and y are 16-byte aligned; y
 * shares no memory with x or w (else DUO_ERR_ARG; told by the ranges of their addresses).  What lies between the rows of y is left as it is.
 * Products are exact and sums are fp32, rounded once, except: 16-bit outputs of more than DUO_MAX_ROWS rows go through the 8-bit
 * matrix instruction, which cuts eight consecutive products to units of 2^-13 of the largest one's power of two before it adds them up in
 * fp32: at most 2^-10 of the largest product of each eight, a 64th of what the rounding of its factors to e4m3 may take from it.
 * `workspace` needs duo_scaled_workspace_bytes(rows, N, K) bytes (0 up to DUO_SCALED_DIRECT_ROWS rows: it may then be NULL).
 */
int duo_scaled_workspace_bytes(int rows, int N, int K, size_t *bytes);
int duo_scaled_gemm(const uint16_t *x, int64_t x_stride, const void *w, void *y, int64_t y_stride, int y_fp32, int rows, int N, int K,
                    void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * ---- A layer of experts for the rows of a verify step (at most DUO_MAX_ROWS).
 *
 *   l = x R^T;  S = the top_k experts with the largest l;  g = softmax(l), over all experts or (renormalise = 1) over S;
 *   y = sum over e in S of g_e * (silu(x G_e^T) * (x U_e^T)) D_e^T
 *
 * R [n_experts][d_model] row-major in 16 bits; G_e, U_e [d_ff][d_model] and D_e [d_model][d_ff] in 16 bits or (scaled = 1) in
 * the 8-bit blocks above; the rows themselves are never brought to 8 bits.  l is formed in 64 bits: equal logits are taken in ascending
 * order of the experts, NaN counts as minus infinity.  Sums are fp32; silu(..) * (..) * g_e enters the last product as a pair of bf16 values (16
 * bits of mantissa, fp32's range); y is rounded once.
 *
 * duo_moe_pack puts one expert (row-major matrices in 16 bits, 16-byte aligned) at its place among the n_experts *
 * duo_moe_expert_bytes(cfg) bytes of `experts` (16-byte aligned): its gate, up and down matrices one behind the other, as duo_pack_matrix or
 * duo_scaled_pack make them.
 */
#define DUO_MOE_MAX_EXPERTS 512
#define DUO_MOE_MAX_TOP     16
#define DUO_MOE_MAX_STRIDE  8388608 /* elements from row to row */
typedef struct duo_moe_config {
    int32_t d_model;     /* a multiple of 64, at most 8192 */
    int32_t d_ff;        /* a multiple of 32, at most DUO_SCALED_MAX_K */
    int32_t n_experts;   /* at most DUO_MOE_MAX_EXPERTS */
    int32_t top_k;       /* at most n_experts and DUO_MOE_MAX_TOP */
    int32_t scaled;      /* 1: the experts' matrices are held in 8 bits */
    int32_t renormalise; /* 1: the shares of a row's experts add up to one */
} duo_moe_config;
size_t duo_moe_expert_bytes(const duo_moe_config *cfg);
int duo_moe_pack(const duo_moe_config *cfg, const uint16_t *w_gate, const uint16_t *w_up, const uint16_t *w_down, int expert,
                 void *experts, void *hip_stream);

/*
 * The layer.  x and y [rows][d_model] in 16 bits, each with its own distance between rows in elements (a multiple of 8, at least
 * d_model), 16-byte aligned; y may be x, or overlap it: x is not read any more when y is written.  position int32 [rows] (optional): rows
 * with a negative entry are neither read nor written, in any output; duo_page_plan marks the rows behind a step's last one like this.
 * chosen int32 [rows][top_k] and share fp32 [rows][top_k] (optional) receive S, by descending l, and g.  `workspace` needs
 * duo_moe_workspace_bytes(cfg, rows) bytes; nothing in it needs clearing, and it serves one call at a time.
 */
int duo_moe_workspace_bytes(const duo_moe_config *cfg, int rows, size_t *bytes);
int duo_moe_layer(const duo_moe_config *cfg, const uint16_t *router, const void *experts, const uint16_t *x, int64_t x_stride, int rows,
                  const int32_t *position, uint16_t *y, int64_t y_stride, int32_t *chosen, float *share, void *workspace,
                  size_t workspace_bytes, void *hip_stream);

/*
 * One skinny weight-streaming product, the building block of the target pass:
 * y[m][n] = sum_k x[m][k] * w[n][k]; x from duo_pack_activations (rows <= DUO_MAX_ROWS), w from
 * duo_pack_matrix (N x K, K % 32 == 0), y fp32 [rows][N] row-major.
 */
int duo_skinny_gemm(const uint16_t *x_packed, const uint16_t *w_packed, float *y, int rows, int N, int K,
                    void *hip_stream);

/*
 * The projection kernel of the many-row (prefill) pass on its own, for tests and kernel benchmarks.  The
 * activations are bf16 pairs a = hi + lo: x_packed comes from duo_pack_activations over 2*PR rows, PR = rows
 * rounded up to a multiple of 16, rows [0, rows) holding the hi parts and rows [PR, PR + rows) the lo parts
 * (all other rows zero).  y[m][n] = sum_k (hi + lo)[m][k] * w[n][k], fp32 [rows][N] row-major; w from
 * duo_pack_matrix; rows <= DUO_MAX_PREFILL_ROWS, K % 32 == 0.  Device pointers.
 */
int duo_block_gemm(const uint16_t *x_packed, const uint16_t *w_packed, float *y, int rows, int N, int K,
                   void *hip_stream);

/*
 * Measurement aid: reads `bytes` (rounded down to a multiple of 16) of device memory once with 16-byte loads (ordinary
 * ones, or with nontemporal != 0 loads that carry the non-temporal hint, as the projection kernels' weight loads do),
 * min(sink_len, 2048) workgroups of 256 lanes, and xors what it read into sink[0 .. min(sink_len, 2048)) (device,
 * uint32, caller-initialised).  Timed over a buffer much larger than the caches it gives the read bandwidth a
 * weight-streaming kernel can reach on the device at hand, next to which the projection kernels' rates are read.
 */
int duo_stream_read_probe(const void *src, size_t bytes, uint32_t *sink, int sink_len, int nontemporal, void *hip_stream);

/*
 * Per-kernel timing for the roofline report (the per-iteration time breakdown of Sec. 4.4
 * "Profiling", at kernel granularity).  While enabled, every kernel that duo_verify /
 * duo_prefill_chunk, the duo_page_* calls, duo_scaled_gemm and duo_moe_layer launch carries a start and a stop HIP event that take the dispatch's own begin and
 * end timestamps; duo_profile_read waits for them, adds each kernel's duration to its class, returns
 * the sums (milliseconds) and launch counts accumulated since the last read, and resets them.
 * Enabling allocates a pool of events, and at most 8192 launches are recorded between two reads (a 64-row step is
 * about 260); duo_profile_dropped returns how many launches since the last read (or enable) found the pool
 * empty and went untimed -- call it before duo_profile_read, which resets it.  A call made while profiling is
 * not allocation-free or capturable.  Not thread-safe.
 * ms and launches are HOST arrays: of DUO_PROF_CLASSES entries for duo_profile_read, which reports the classes below that and leaves out what was
 * launched under the others; of `classes` entries (1 or more, else DUO_ERR_ARG) for duo_profile_read_classes, which reports as many, DUO_PROF_ALL_CLASSES
 * being all there are (entries behind them receive zero).  Classes that are added later raise DUO_PROF_ALL_CLASSES alone: a program that was built
 * before them hands over arrays as long as they have to be.  Either call resets the sums of all classes.
 */
#define DUO_PROF_SETUP     0  /* rotary table, embedding gather + first RMSNorm, input checks, root statistics; duo_page_plan */
#define DUO_PROF_QKV       1  /* fused QKV projection + rotary + KV scatter */
#define DUO_PROF_ATTN      2  /* masked attention over prefix + drafts (chunk partials); duo_page_attention */
#define DUO_PROF_ATTN_COMB 3  /* merge of the chunk partials (long contexts only), of the key ranges in duo_page_attention */
#define DUO_PROF_OPROJ     4  /* O projection + residual */
#define DUO_PROF_RESID_REDUCE 5 /* sum of the K-split O/down partial results + residual (more than 16 rows; from 9 rows on where d_ff >= 8192); prompt chunks of more than 80 rows: also the row sums of squares behind an unsplit one */
#define DUO_PROF_GATEUP    6  /* gate/up projection + SwiGLU */
#define DUO_PROF_DOWN      7  /* down projection + residual */
#define DUO_PROF_LMHEAD    8  /* LM head */
#define DUO_PROF_SAMPLE    9  /* softmax statistics, accept tests, correction/bonus sampling */
#define DUO_PROF_COMMIT    10 /* sequence selection + KV commit; duo_page_commit */
#define DUO_PROF_QKV_FINISH 11 /* 49 rows and more: sum of the K-split Q/K/V partial results + rotary + KV scatter; duo_page_append */
#define DUO_PROF_CLASSES    12 /* entries of duo_profile_read */
#define DUO_PROF_SCALED     12 /* duo_scaled_gemm */
#define DUO_PROF_MOE_ROUTER 13 /* duo_moe_layer: logits, choice of experts */
#define DUO_PROF_MOE_GATEUP 14 /* duo_moe_layer: gate/up products + SwiGLU */
#define DUO_PROF_MOE_DOWN   15 /* duo_moe_layer: down product, sum over a row's experts */
#define DUO_PROF_ALL_CLASSES 16
int duo_profile_enable(int enable);
int duo_profile_read(double *ms, int32_t *launches);
int duo_profile_read_classes(double *ms, int32_t *launches, int classes);
int duo_profile_dropped(void);
/* Name, with template arguments as a kernel trace prints them, of the projection kernel most recently launched under
 * class `cls` while the timer was enabled ("" if none, or if that class's kernels are not named); HOST string, valid until
 * the next profiled launch of the class.  It lets a timing be matched with profiler counter summaries of that kernel. */
const char *duo_profile_kernel_name(int cls);

const char *duo_status_string(int code);
const char *duo_last_hip_error(void);

#ifdef __cplusplus
}
#endif
#endif /* DUO_VERIFY_H */
