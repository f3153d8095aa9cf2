/*
 * lda_mi355x.h -- C ABI of the MI355X (gfx950) LightLDA sweep library.
 *
 * The library runs the data-parallel hot path of LightLDA (arXiv 1412.1576):
 * the O(1) cycle Metropolis-Hastings sweep over all tokens of a corpus
 * (Sec. 4.2-4.3, Eq. 6-13), the per-word alias tables it draws from
 * (Sec. 4.2, Fig. 2), and the rebuild of the count tables n_kd, n_kw, n_k
 * (Sec. 3, text after Eq. 1).  Every step runs in hand-written HIP kernels on
 * one GPU; the host side only marshals arguments.
 *
 * Semantics fixed by this library (the paper leaves them open):
 *   - Snapshot sweeps: every token of a sweep reads the assignment z and all
 *     counts as of the start of the sweep (the limit of the paper's immutable
 *     model slice with delayed updates, Sec. 6 "Multi-thread Efficiency").
 *     A token's own contribution is removed at its snapshot topic.
 *   - One MH step is one proposal plus one accept test; step j of a token is a
 *     word-proposal for even j and a doc-proposal for odd j (Eq. 13).
 *   - Randomness is Philox4x32-10 with key = seed and counter
 *     (token id low, token id high, sweep index, step index), so results do not
 *     depend on launch geometry.  Every accept test has the outcome that its
 *     products have in fp64, separately rounded (most are decided in fp32 with a
 *     margin that no rounding crosses).
 *
 * Conventions
 *   - All pointers in the signatures are HOST pointers unless stated otherwise (the operators on
 *     rows, and lda_doc_topics, take device pointers).
 *     The library copies what it needs; the caller keeps ownership of its buffers
 *     and may free them as soon as a call returns.
 *   - Token order at the boundary is the caller's CSR (document-major) order:
 *     token g is word_ids[g]; document d owns g in [doc_offsets[d], doc_offsets[d+1]).
 *   - Return value 0 (LDA_OK) on success, a negative LDA_ERR_* otherwise; no call
 *     throws.  lda_last_error() returns a message for the last failure.
 *   - lda_build_alias, lda_sweep and lda_rebuild_counts enqueue work on the
 *     context's HIP stream and return; accessors and lda_loglik synchronise.
 *     (lda_build_alias may run part of its kernels on a second stream of the
 *     library's own, of default priority, forked from and joined to the context's
 *     stream by events: work queued after the call still sees every table.  With
 *     stream_block_tokens the copies of the blocks run on two more such streams;
 *     lda_sync waits for them too.)
 *   - A context is not thread-safe.  Calls must follow the state machine
 *       COUNTS_VALID --lda_build_alias--> ALIAS_VALID --lda_sweep--> SWEPT
 *       SWEPT --lda_rebuild_counts--> COUNTS_VALID
 *     and return LDA_ERR_STATE otherwise.
 */
#ifndef LDA_MI355X_H
#define LDA_MI355X_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LDA_OK 0
#define LDA_ERR_ARG (-1)         /* bad pointer, size, id out of range, alpha/beta <= 0, ... */
#define LDA_ERR_STATE (-2)       /* call out of order */
#define LDA_ERR_OOM (-3)         /* host or device allocation failed */
#define LDA_ERR_HIP (-4)         /* a HIP runtime call or kernel launch failed */
#define LDA_ERR_UNSUPPORTED (-5) /* valid request outside what this build supports */

typedef struct lda_ctx lda_ctx; /* opaque; owns all device memory of one corpus */

/* Options for lda_init.  A zeroed struct (or a NULL pointer) selects the defaults. */
typedef struct lda_options {
    void* hip_stream;              /* hipStream_t all work is enqueued on; NULL: the null stream */
    /* Device allocator of the caller (e.g. a framework's caching allocator); both NULL: hipMalloc
       and hipFree.  When set, every device buffer of the context -- at lda_init and the ones
       that later calls grow or create on first use -- comes from dev_alloc(bytes, alloc_user),
       which returns device memory aligned to 256 bytes or NULL (reported as LDA_ERR_OOM), and
       goes back through dev_free(ptr, alloc_user), at lda_destroy at the latest, and only when
       no work queued on the context's stream uses it any more.  The callbacks run on the thread
       that calls the library; setting only one is LDA_ERR_ARG.
       rocprim's temporary storage is requested through them as well. */
    void* (*dev_alloc)(size_t bytes, void* alloc_user);
    void (*dev_free)(void* ptr, void* alloc_user);
    void* alloc_user;
    int32_t dense_rows;            /* hybrid store (Sec. 5): word ids [0, dense_rows) keep a dense n_kw
                                      row, the others a sorted (topic, count) list plus a hash row;
                                      0: every row dense; -1: no dense row */
    int32_t dense_alias_min_count; /* words with corpus frequency >= this draw from a dense K-bin
                                      table, the others from the sparsified mixture (Sec. 4.2);
                                      0: every word uses the dense table.  A word that draws from a
                                      dense table must have a dense row (LDA_ERR_ARG otherwise). */
    int32_t proposal_mode;         /* 0: cycle word,doc,word,... (Eq. 13); 1: word only; 2: doc only */
    int32_t sweep_chunk_tokens;    /* tuning: tokens per sweep workgroup tile; 0: default */
    int32_t sweep_block_threads;   /* tuning: threads per sweep workgroup; 0: default */
    int32_t rebuild_tile_tokens;   /* tuning: tokens per count-rebuild tile; 0: default */
    int32_t time_sweep_passes;     /* 1: lda_sweep records HIP events around its two passes on the
                                      context's stream (read them with lda_sweep_pass_ms) */
    int32_t record_bucket_tokens;  /* tuning: the per-token records the two passes of a sweep
                                      exchange are ordered by buckets of this many consecutive
                                      tokens (a power of two), inside a bucket by word; 0: default
                                      (2^22 when every n_kw row is dense and the corpus has at
                                      least 2^28 tokens, else one bucket);
                                      -1: one bucket (plain word order).  Words of at least
                                      max(256, N / 2^16) tokens keep word order either way */
    int32_t doc_refresh;           /* 1: lda_sweep refreshes the doc side after every token (Sec. 4.2,
                                      footnote 4): the tokens of a document are visited in order
                                      and each sees, in n_kd and in the doc-proposal's draw, the
                                      topics its predecessors of the same sweep were just given;
                                      the word side stays at the snapshot (Sec. 6).  All-dense
                                      store with dense tables, documents of at most 4096 tokens,
                                      at most 4 steps (LDA_ERR_UNSUPPORTED otherwise).  0: every
                                      token reads the snapshot (the default, and the fast path) */
    int32_t stream_block_tokens;   /* > 0: streamed data blocks (Sec. 3; Sec. 6, Fig. 7).  The model
                                      stays on the device; the per-token arrays move to pinned
                                      host memory when lda_init is done and every lda_sweep brings
                                      them in block by block -- runs of whole documents of about
                                      this many tokens, the next block loading while the current
                                      one is swept -- and takes the new topics back.  4 bytes per
                                      token stay resident (the word-major copy of z that the count
                                      rebuild reads).  Results are those of the resident run, bit
                                      for bit.  lda_init itself still holds the whole corpus on
                                      the device once.  Not with doc_refresh (LDA_ERR_ARG), not
                                      with documents longer than a sweep tile, not
                                      lda_update_counts (LDA_ERR_UNSUPPORTED).  0: resident */
    int32_t reserved[5];           /* must be zero */
} lda_options;

/*
 * lda_init -- take a corpus and set up the sampler state (problem statement: Sec. 3).
 *   D            number of documents (>= 1); empty documents are legal
 *   V, K         vocabulary size and number of topics (>= 1); K <= 2^20 - 2; dense rows and
 *                dense tables are limited to 10^10 and 4 * 10^9 entries (LDA_ERR_UNSUPPORTED)
 *   doc_offsets  [D+1] host, doc_offsets[0] = 0, non-decreasing, N = doc_offsets[D] in [1, 2^31 - 2^20 - 1]
 *   word_ids     [N] host, each in [0, V)
 *   alpha, beta  symmetric Dirichlet parameters (> 0) of Eq. (1)
 *   seed         Philox key
 * Copies the corpus to the device, builds the word-major token order and the
 * document tiling, draws the initial assignment z[g] = floor(x0 * K / 2^32) from
 * the Philox counter (g, 0xFFFFFFFF, 0) and counts n_kw, n_k.  On success
 * *out is a new context in state COUNTS_VALID with sweep index 0.
 */
int lda_init(lda_ctx** out, int64_t D, int32_t V, int32_t K, const int64_t* doc_offsets,
             const int32_t* word_ids, double alpha, double beta, uint64_t seed,
             const lda_options* opt);

/*
 * lda_build_alias -- word-proposal tables of Eq. (6) for every word, from the
 * current counts: per bin a split point and an alias (Sec. 4.2, Fig. 2), plus the
 * bin capacity of the table.  Words of the dense form get one table over all K
 * topics; words of the mixture form (Sec. 4.2, the sparsified table) one table
 * over their non-zero topics, and all of them share one table over
 * beta/(n_k + V beta).  In the all-dense store the table of a word with few tokens may be held as
 * its topics with running sums, from which a draw computes the bin it hits; sweeps that run as one
 * kernel and lda_get_alias_row make such words' bins when they need them.  This takes 20 bytes per token
 * of these words from lda_init on; where that finds no room, or a sweep later finds none for its
 * records beside it, every word has its bins.
 * COUNTS_VALID -> ALIAS_VALID.
 */
int lda_build_alias(lda_ctx* ctx);

/*
 * lda_sweep -- one sweep: for every token mh_steps (>= 1) Metropolis-Hastings
 * steps alternating the word-proposal (Eq. 6-8) and the doc-proposal
 * (Eq. 9-12) against the conditional of Eq. (4), all reads from the snapshot.
 * Uses the context's sweep index as Philox counter word 2 and increments it.
 * The longest chain asked for decides how much the context holds for the records its passes
 * exchange, from the first such sweep until lda_destroy: 20 bytes per token for 2 steps, 40 for 4,
 * 72 or 80 for 5 to 8 (K > 65536: 24, 48, and 80 or 96); LDA_ERR_OOM if there is no room.  Chains
 * of 5 to 8 steps use records only where they gain (many tokens of the mixture form, or of long
 * documents) and run as one kernel without them otherwise, as longer chains always do; so they do,
 * more slowly, where there is no room or the records would have to be allocated while the stream is
 * being captured.  A context that was refused the memory once does not ask for as much again.
 * ALIAS_VALID -> SWEPT (the counts no longer match z).
 */
int lda_sweep(lda_ctx* ctx, int32_t mh_steps);

/*
 * lda_sweep_pass_ms -- device time of the last sweep's two passes, from the HIP events
 * recorded with the option time_sweep_passes: *word_pass_ms covers the word pass (every
 * kernel that evaluates the word side of the chains, Eq. 6-8, in word-major order),
 * *doc_pass_ms the one kernel that runs the accept tests over the document tiles.
 * Waits for the events.  LDA_ERR_STATE if the option is off, no sweep has run, or the
 * last sweep had more than 4 steps or ran as one fused kernel (word-only or doc-only chains of
 * several steps, tiles of more than 4 tokens per thread).
 */
int lda_sweep_pass_ms(lda_ctx* ctx, float* word_pass_ms, float* doc_pass_ms);

/*
 * lda_rebuild_counts -- recount n_kw (per-word histogram of the word-major
 * token segments: dense rows, and for words without a dense row the sorted
 * (topic, count) list and hash row of Sec. 5) and n_k from the current
 * assignment; the per-document counts n_kd are formed inside the sweep from the
 * document's assignments.  SWEPT (or any state) -> COUNTS_VALID.
 */
int lda_rebuild_counts(lda_ctx* ctx);

/*
 * lda_update_counts -- the counts after a sweep by the paper's own rule (Sec. 3, text after
 * Eq. 1; applied late as in Sec. 6, "Multi-thread Efficiency"): for every token the last
 * lda_sweep moved from topic a to topic b, n_kw[w][a] and n_k[a] lose one, n_kw[w][b] and
 * n_k[b] gain one.  Same tables as lda_rebuild_counts, bit for bit, and cheaper when few tokens
 * move (late in training).  Where the recount can be the cheaper form, a sample of the tokens taken
 * on the device, without the host waiting, decides which of the two makes the tables; that costs
 * some 10 to 40 us when few tokens move.  Needs the state SWEPT reached by lda_sweep
 * (not by lda_set_z: LDA_ERR_STATE) and the all-dense store with dense tables for every word
 * (LDA_ERR_UNSUPPORTED otherwise: lists and hash rows are only made by the recount).
 * SWEPT -> COUNTS_VALID.
 */
int lda_update_counts(lda_ctx* ctx);

/*
 * lda_loglik -- log p(w, z | alpha, beta) of the collapsed model, the metric of
 * Sec. 7 ("doc-likelihood" + "word-likelihood"); fp64.  Needs valid counts.
 * doc_part / word_part may be NULL.  Synchronises.
 */
int lda_loglik(lda_ctx* ctx, double* total, double* doc_part, double* word_part);

/*
 * lda_loglik_noalloc -- lda_loglik for callers that cannot allocate: code under HIP graph
 * capture around it, tight serving loops, harnesses that forbid hipMalloc.  Same arguments,
 * same kernels, same summation order and therefore the same value as lda_loglik; the
 * per-block partial sums go to a static device array of the library (2^20 doubles = 8 MB,
 * held by every GPU the library runs on until the process ends) instead of the context's
 * own buffer, and the host side stages them through the stack.  The call makes no device or
 * host allocation.  The context's device must be the current device.
 *   - LDA_ERR_UNSUPPORTED when the context needs more partial sums than the array holds
 *     (one per document tile: more than 2^20 tiles, or long documents); use lda_loglik then.
 *   - All contexts on one GPU share the array: two calls that overlap on one GPU (two
 *     host threads, two streams) race on it and must be serialised by the caller.  Nothing in
 *     the array needs to be zero on entry; every element that is read was written by the
 *     same call.
 */
int lda_loglik_noalloc(lda_ctx* ctx, double* total, double* doc_part, double* word_part);

/* ---- accessors (parity checks, checkpoint / warm start of Sec. 6); all synchronise ---- */
int64_t lda_num_tokens(const lda_ctx* ctx);
/* The device of the context: the current one at lda_init.  -1 for NULL.  (Does not synchronise.) */
int lda_device(const lda_ctx* ctx);
int64_t lda_sweep_index(const lda_ctx* ctx);
/* z [N] in CSR token order. */
int lda_get_z(lda_ctx* ctx, int32_t* z);
/* Replace the assignment (each z[g] in [0,K)) and the next sweep index (< 2^32-1); -> SWEPT. */
int lda_set_z(lda_ctx* ctx, const int32_t* z, int64_t next_sweep_index);
/* nk [K]; needs valid counts. */
int lda_get_nk(lda_ctx* ctx, int32_t* nk);
/* Dense copy of row w of the word-topic table, row [K]; needs valid counts. */
int lda_get_nkw_row(lda_ctx* ctx, int32_t w, int32_t* row);
/* Dense copy of row d of the doc-topic table as the sweep kernel forms it, row [K]. */
int lda_get_ndk_row(lda_ctx* ctx, int64_t d, int32_t* row);
/* Dense-form table of word w: split [K], alias [K], *cap = bin capacity; needs ALIAS_VALID. */
int lda_get_alias_row(lda_ctx* ctx, int32_t w, uint32_t* split, uint32_t* alias, uint32_t* cap);

/* Mixture-form tables (Sec. 4.2, the sparsified word-proposal); need ALIAS_VALID.
 * lda_get_sparse_table: the table of word w over its non-zero topics.  *n = number of entries;
 * when *n <= cap_entries the entries are written: topics[i] ascending, split[i], and
 * alias_topic[i] = the topic bin i falls through to.  *cap = bin capacity, *mass = integer mass
 * QS_w of the sparse term.  LDA_ERR_ARG if the word draws from a dense table.
 * lda_get_beta_table: the table over beta/(n_k + V beta) shared by all words, split [K],
 * alias [K] (topic indices), its capacity and integer mass QB. */
int lda_get_sparse_table(lda_ctx* ctx, int32_t w, int32_t cap_entries, int32_t* n, int32_t* topics,
                         uint32_t* split, int32_t* alias_topic, uint32_t* cap, uint64_t* mass);
int lda_get_beta_table(lda_ctx* ctx, uint32_t* split, uint32_t* alias, uint32_t* cap,
                       uint64_t* mass);

/* ---- operators on rows (beside the sampler; no context) ------------------------------------
 * Teacher rows out of topic counts, the distillation loss that trains a student on them, the
 * verification of tokens that a draft proposed; a classifying head (norm of hidden rows, product with the classes'
 * weights in 8 bits) and the log probabilities that are read off its logits.  All pointers inside the structs and all outputs
 * are DEVICE pointers; the structs themselves are read on the host during the call.  The calls
 * enqueue on hip_stream (NULL: the null stream) and return; they allocate nothing, wait for
 * nothing and can be captured into a graph.  The current device must be the one that holds the
 * memory and the stream.  Strides count elements; inside a row elements are adjacent.  Inputs may
 * be read by several calls at once; two calls that may overlap in time need workspaces of their
 * own.  Outputs must not overlap inputs.  Errors are those of the other entry points, the message
 * is that of lda_last_error(NULL) on the calling thread. */
#define LDA_F32 0
#define LDA_F16 1
#define LDA_BF16 2
#define LDA_I32 0
#define LDA_I64 1

/*
 * Distillation from a teacher's top logits.  Row i of the student has one logit S_v for each of
 * `classes` classes (topics, words); row i of the teacher has `slots` slots, an id and a logit t_j each.
 * A slot whose id lies outside [0, classes) is empty; ids may come in any order and more than once
 * (their masses add up in P_v; the loss has the term p_j log p_j of each, which the student does not change, so
 * that it is less than that of one slot of their mass by T^2 sum p_j log(P_v / p_j)).  With T = temperature:
 *   q = softmax(S / T), where q_v = 0 for S_v = -infinity;
 *   log_norm == NULL: p_j = softmax over the row's slots of t_j / T, r = 0;
 *   otherwise:        p_j = exp(t_j / T - log_norm), and the mass that is left, if any, is spread
 *                     evenly over the classes that no slot names: r = max(0, 1 - sum p_j) / their number
 *                     (a teacher known by its largest masses and a floor, as theta_dk is of n_kd);
 *   loss = T^2 ( sum_j p_j (log p_j - log q_id_j) + sum over classes without a slot of r (log r - log q_v) )
 *   d loss / d S_v = T (M q_v - P_v),  P_v = the p_j of v's slots, or r;  M = sum P_v.
 * A term of mass 0 is 0, and a slot of logit -infinity has no mass, whatever the norm.  A row without any
 * mass has loss 0 and gradient 0, whatever S holds.  Mass on a class of q_v = 0 makes the loss +infinity; the
 * gradient is the formula's.  NaN or +infinity in S, or in the logit of a slot that is not empty, or masses
 * whose sum 64 bits do not hold, make the row's loss and gradient NaN.
 * The softmax is summed in 32 bits; the teacher's masses are summed in 64 and rounded to 32 each, and the loss is
 * put together in 64.
 */
typedef struct lda_distill_rows {
    int64_t rows;            /* >= 0 */
    int32_t classes;         /* >= 1 */
    int32_t slots;           /* 0 .. 1024 (more: LDA_ERR_UNSUPPORTED) */
    const void* logits;      /* [rows][classes], rows logits_stride apart */
    int64_t logits_stride;
    const void* ids;         /* [rows][slots] */
    int64_t ids_stride;
    const void* teacher;     /* [rows][slots] */
    int64_t teacher_stride;
    const float* log_norm;   /* [rows] or NULL */
    const float* weight;     /* weight of row i at weight[i * weight_stride]; NULL: 1.  The gradient's factor.
                                Rows of weight 0 are left out: gradient 0 (lda_distill_step: and
                                loss 0), and their logits are not looked at.  Not used by lda_distill_loss */
    int64_t weight_stride;   /* 0: one weight for every row */
    int32_t logits_type;     /* LDA_F32, LDA_F16, LDA_BF16 */
    int32_t ids_type;        /* LDA_I32, LDA_I64 */
    int32_t teacher_type;    /* as logits_type */
    float temperature;       /* 1/1024 .. 1024 */
    void* workspace;         /* at least lda_distill_workspace() bytes, aligned to 16; what it holds is of
                                no use after the call's work */
    int64_t workspace_bytes;
    void* hip_stream;
    int32_t reserved[4];     /* must be zero */
} lda_distill_rows;

/* Bytes of workspace that a call on these rows needs (may be 0), or a negative LDA_ERR_*. */
int64_t lda_distill_workspace(const lda_distill_rows* rows);
/* loss [rows]; stats, aligned to 16 bytes: 8 floats a row for lda_distill_grad (the row's softmax
 * and teacher in short), or NULL. */
int lda_distill_loss(const lda_distill_rows* rows, float* loss, float* stats);
/* The gradient of sum_i weight_i loss_i, [rows][classes] in the logits' type, rows grad_stride
 * apart; what lies between rows is left as it was.  stats: of lda_distill_loss on the same rows. */
int lda_distill_grad(const lda_distill_rows* rows, const float* stats, void* grad, int64_t grad_stride);
/* Both in one call, for a program that knows the weights beforehand: the logits are read once from
 * memory where they fit the registers. */
int lda_distill_step(const lda_distill_rows* rows, float* loss, void* grad, int64_t grad_stride);

/*
 * Verification of drafted tokens.  Sequence b has n_b = lengths[b] drafted tokens x_i (all `steps` of
 * them if lengths is NULL; lengths are clamped to [0, steps]), drawn from the rows q_i of `draft`, and n_b + 1 rows
 * p_i of `target`.  Draft i is accepted if accept_u[b][i] * q_i(x_i) < p_i(x_i) and all before it are; a
 * token outside [0, classes) is not.  accepted[b] = a, the number of accepted drafts, and out[b] is
 * x_0 .. x_{a-1}, then one drawn token, then -1 up to steps + 1 entries.  The token is drawn from masses
 * m_v:  a = n_b: p_a(v);  else max(0, p_a(v) - q_a(v)), or p_a(v) if none of these is positive.
 * It is the first v with m_v > 0 and m_0 + .. + m_v > draw_u[b] * (sum of all), the last v with m_v > 0
 * if there is none such, -1 if no m_v is positive.  Products and sums are 64-bit.  Masses need not
 * sum to 1; a NaN has no mass.  The result is that of these random numbers, and distributed
 * as draws from the target are.  steps = 0: plain draws (draft, tokens, accept_u are not looked at).
 */
typedef struct lda_draft_rows {
    int64_t sequences;       /* >= 0 */
    int32_t steps;           /* 0 .. 4096 */
    int32_t classes;         /* >= 1 */
    const void* target;      /* [sequences][steps + 1][classes] */
    int64_t target_sequence_stride, target_row_stride;
    const void* draft;       /* [sequences][steps][classes] */
    int64_t draft_sequence_stride, draft_row_stride;
    const void* tokens;      /* [sequences][steps] */
    int64_t tokens_stride;
    const int32_t* lengths;  /* [sequences] or NULL */
    const float* accept_u;   /* [sequences][steps] */
    int64_t accept_u_stride;
    const float* draw_u;     /* [sequences] */
    int32_t probs_type;      /* of target and draft: LDA_F32, LDA_F16, LDA_BF16 */
    int32_t tokens_type;     /* of tokens and out: LDA_I32, LDA_I64 */
    void* workspace;         /* at least lda_verify_workspace() bytes, aligned to 16 */
    int64_t workspace_bytes;
    void* hip_stream;
    int32_t reserved[4];     /* must be zero */
} lda_draft_rows;

int64_t lda_verify_workspace(const lda_draft_rows* rows);
/* accepted [sequences]; out [sequences][steps + 1], rows out_stride apart */
int lda_verify_drafts(const lda_draft_rows* rows, int32_t* accepted, void* out, int64_t out_stride);

/*
 * Top topics of documents: for each, the `slots` topics that most of its tokens have, the most
 * frequent first, ties to the lower topic, with logits log(n + alpha), n the number of
 * tokens; slots without a topic get id -1 and logit -infinity.  log_norm = log(L + K alpha), L the
 * tokens counted: with these three lda_distill_loss learns the document's whole
 * theta_dk = (n_dk + alpha) / (L + K alpha), at temperature 1, when slots holds all of its topics.  Logits and log_norm have
 * 32 bits, so that a slot's mass is off by up to 2^-23 log_norm of itself, and the mass of all classes without a slot,
 * which is what the slots leave of 1, by as much of 1: of documents whose rest, about K alpha / L, is not far
 * above 10^-6 (10^5 tokens and more with a small alpha) the loss learns the slots, and the floor's size at most.
 */
typedef struct lda_topic_rows {
    int64_t rows;            /* rows of output, >= 0 */
    const int32_t* docs;     /* [rows] the document of each row, or NULL: row i is document i.  A document
                                outside [0, documents) is empty */
    int64_t documents;       /* >= 0; with docs == NULL at least rows */
    const void* offsets;     /* [documents + 1] document d is z[offsets[d]] .. z[offsets[d + 1] - 1] */
    int32_t offsets_type;    /* LDA_I32, LDA_I64 */
    int32_t K;               /* 1 .. 2^20 - 2; a z outside [0, K) is not counted */
    const int32_t* z;        /* [tokens] */
    int64_t tokens;          /* offsets are clamped to [0, tokens]; a document of more than 2^31 - 1 tokens
                                is cut there */
    int32_t slots;           /* 1 .. 1024 (more: LDA_ERR_UNSUPPORTED) */
    int32_t reserved_word;   /* must be zero */
    double alpha;            /* > 0 */
    void* workspace;         /* NULL, or aligned to 16: with lda_topics_workspace() bytes documents of many tokens
                                are shared by several workgroups; with less, fewer of them are, with
                                the same results */
    int64_t workspace_bytes;
    void* hip_stream;
    int32_t reserved[4];     /* must be zero */
} lda_topic_rows;

int64_t lda_topics_workspace(const lda_topic_rows* rows);

/* ids [rows][slots], logits [rows][slots], log_norm [rows] or NULL */
int lda_top_topics(const lda_topic_rows* rows, int32_t* ids, float* logits, float* log_norm);
/* The same from the context's current assignment, its K and alpha, on its stream; docs and the outputs are
 * device pointers, and the context's device has to be the current one.  Any state.  A captured call reads, when it
 * is replayed, what the last sweep or lda_set_z before it on the stream has left.  With stream_block_tokens:
 * LDA_ERR_UNSUPPORTED (z is in host memory). */
int lda_doc_topics(lda_ctx* ctx, int64_t rows, const int32_t* docs, int32_t slots, int32_t* ids,
                   float* logits, float* log_norm);

/*
 * Root-mean-square norm of rows with the residual's addition.  With x [rows][width], r the residual of the
 * same shape (none: 0) and w the weight [width] (none: 1):
 *   h = x + r, rounded to the sum's type;  n = h / sqrt(mean over the row of h^2 + eps);  y = n w
 * y is the norm of the sum as it is written.  A row of zeros with eps = 0 has n = 0.
 * To 8 bits: scale = max |y| / Q of the row, Q = 127 (LDA_INT8) or 448 (LDA_E4M3, the largest such number), and
 * out = y / scale, rounded to the nearest number of the type, ties to even, so that out * scale stands for y.  A row
 * whose max |y| is below 2^-100 has scale 0 and out 0, one with a NaN or an infinity in y has scale NaN and out 0.
 * Gradient, from y' of y and h' of the sum (NULL: 0), with u = y' w:
 *   x' = r' = h' + (u - n mean over the row of u n) / sqrt(mean of h^2 + eps);  w' = sum over the rows of y' n
 * Sums are 32-bit, over rows of more than 16384 numbers 64-bit but for 8 numbers each; squares that leave 32 bits are scaled.
 */
#define LDA_INT8 0
#define LDA_E4M3 1
typedef struct lda_norm_rows {
    int64_t rows;            /* >= 0 */
    int32_t width;           /* 1 .. 2^30 (more: LDA_ERR_UNSUPPORTED) */
    int32_t x_type;          /* of x, y and their gradients: LDA_F32, LDA_F16, LDA_BF16 */
    const void* x;           /* [rows][width], rows x_stride apart */
    int64_t x_stride;
    const void* residual;    /* [rows][width] or NULL */
    int64_t residual_stride;
    const void* weight;      /* [width] or NULL */
    int32_t weight_type;     /* of the weight and its gradient: x_type or LDA_F32 */
    int32_t sum_type;        /* of the residual, the sum and their gradients: x_type or LDA_F32 */
    float eps;               /* >= 0 */
    int32_t reserved_word;   /* must be zero */
    void* hip_stream;
    int32_t reserved[4];     /* must be zero */
} lda_norm_rows;

typedef struct lda_norm_gradients {
    const void* y_grad;      /* [rows][width] */
    int64_t y_grad_stride;
    const void* sum_grad;    /* [rows][width] or NULL */
    int64_t sum_grad_stride;
    const void* sum;         /* lda_norm's; not used without a residual */
    int64_t sum_stride;
    const float* stats;      /* lda_norm's */
    void* x_grad;            /* [rows][width] or NULL */
    int64_t x_grad_stride;
    void* residual_grad;     /* [rows][width] or NULL; with x_type = sum_type it is x_grad once more */
    int64_t residual_grad_stride;
    void* weight_grad;       /* [width] or NULL */
    void* workspace;         /* with weight_grad: at least lda_norm_grad_workspace() bytes, aligned to 16 */
    int64_t workspace_bytes;
    int32_t reserved[4];     /* must be zero */
} lda_norm_gradients;

/* y [rows][width]; with a residual sum [rows][width] (otherwise it is not looked at); stats, aligned to 8 bytes:
 * 2 floats a row for lda_norm_grad, or NULL. */
int lda_norm(const lda_norm_rows* rows, void* y, int64_t y_stride, void* sum, int64_t sum_stride, float* stats);
/* out [rows][width], a byte an element, scale [rows]; sum as above */
int lda_norm_bytes(const lda_norm_rows* rows, int32_t levels, void* out, int64_t out_stride, float* scale, void* sum,
                   int64_t sum_stride);
int64_t lda_norm_grad_workspace(const lda_norm_rows* rows);
/* Of the residual only that there is one is looked at. */
int lda_norm_grad(const lda_norm_rows* rows, const lda_norm_gradients* gradients);

/*
 * Product of rows of 8-bit integers a [rows][width] with the classes' weights b [classes][width], a scale for each
 * row of both:
 *   out_ij = (float(sum over k of a_ik b_jk) a_scale_i) b_scale_j, rounded to out's type.
 * The sum is exact.  Every integer may take all 256 values.
 */
typedef struct lda_product_rows {
    int64_t rows;            /* 0 .. 2^31, rows * classes up to 2^40 (more: LDA_ERR_UNSUPPORTED) */
    int32_t classes;         /* >= 1 */
    int32_t width;           /* 0 .. 131071: the sum has to fit 32 bits (more: LDA_ERR_UNSUPPORTED) */
    const void* a;           /* [rows][width], rows a_stride apart */
    int64_t a_stride;
    const float* a_scale;    /* [rows] */
    const void* b;           /* [classes][width], rows b_stride apart */
    int64_t b_stride;
    const float* b_scale;    /* [classes] */
    int32_t out_type;        /* LDA_F32, LDA_F16, LDA_BF16 */
    int32_t reserved_word;   /* must be zero */
    void* workspace;         /* at least lda_product_workspace() bytes, aligned to 16 */
    int64_t workspace_bytes;
    void* hip_stream;
    int32_t reserved[4];     /* must be zero */
} lda_product_rows;

/* Bytes of workspace that the call needs (may be 0), or a negative LDA_ERR_*. */
int64_t lda_product_workspace(const lda_product_rows* rows);
/* out [rows][classes], rows out_stride apart; what lies between rows is left as it was.  Of more than 128 rows a side
 * is copied into the workspace first, unless its pointer, its stride (below 2^22) and the width are multiples of 16. */
int lda_product(const lda_product_rows* rows, void* out, int64_t out_stride);

/*
 * Log probabilities of given tokens, entropy and top alternatives of rows of logits S [rows][classes], with T =
 * temperature and the probabilities p = softmax(S / T), where p_v = 0 for S_v = -infinity:
 *   log_prob = log p_t of the row's token t, 0 where t lies outside [0, classes);
 *   entropy = - sum of p_v log p_v over the classes with p_v > 0;
 *   ids, top: the `top` classes of the largest S_v > -infinity and their log p_v, the largest first, equal ones by class
 *   (0 and -0 are equal); slots without a class have id -1 and -infinity;
 *   gradient of sum of a log_prob + b entropy over the rows:
 *   d / d S_v = (a ([v = t] - p_v) - b p_v (log p_v + entropy)) / T,  a taken as 0 where there is no token.
 * With temperature 1, ids and top are a teacher for lda_distill_loss, with log_norm 0.
 * A row without any S_v > -infinity has log_prob -infinity, entropy 0, empty slots and gradient 0.  One with a NaN or
 * +infinity has NaN for log_prob (0 without a token), entropy, top and gradient, and ids -1.  A row with a = b = 0 has gradient
 * 0 whatever S holds, and is not looked at.  Sums are 32-bit.
 */
typedef struct lda_log_prob_rows {
    int64_t rows;            /* >= 0 */
    int32_t classes;         /* >= 1 */
    int32_t top;             /* 0 .. 256 (more: LDA_ERR_UNSUPPORTED) */
    const void* logits;      /* [rows][classes], rows logits_stride apart */
    int64_t logits_stride;
    const void* tokens;      /* token of row i at tokens[i * tokens_stride] */
    int64_t tokens_stride;
    int32_t logits_type;     /* LDA_F32, LDA_F16, LDA_BF16 */
    int32_t tokens_type;     /* LDA_I32, LDA_I64 */
    float temperature;       /* 1/1024 .. 1024 */
    int32_t reserved_word;   /* must be zero */
    void* workspace;         /* at least lda_log_probs_workspace() bytes, aligned to 16 */
    int64_t workspace_bytes;
    void* hip_stream;
    int32_t reserved[4];     /* must be zero */
} lda_log_prob_rows;

/* Bytes of workspace that lda_log_probs needs (may be 0), or a negative LDA_ERR_*. */
int64_t lda_log_probs_workspace(const lda_log_prob_rows* rows);
/* log_prob [rows]; entropy [rows] or NULL; ids and top [rows][top], not looked at with top = 0; stats, aligned to 16
 * bytes: 4 floats a row for lda_log_probs_grad, or NULL. */
int lda_log_probs(const lda_log_prob_rows* rows, float* log_prob, float* entropy, int32_t* ids, float* top, float* stats);
/* a of row i at log_prob_grad[i * log_prob_grad_stride], NULL: 0; b alike.  grad [rows][classes] in the logits'
 * type, rows grad_stride apart; what lies between rows is left as it was.  stats: of lda_log_probs on the same rows. */
int lda_log_probs_grad(const lda_log_prob_rows* rows, const float* stats, const float* log_prob_grad,
                       int64_t log_prob_grad_stride, const float* entropy_grad, int64_t entropy_grad_stride, void* grad,
                       int64_t grad_stride);

/* Wait for all work enqueued by this context. */
int lda_sync(lda_ctx* ctx);
/* Message of the last error of this context (ctx == NULL: of the last failed call on this thread,
 * lda_init and the operators on rows among them).  The string is owned by the library and valid until the next call. */
const char* lda_last_error(const lda_ctx* ctx);
/* Free the context and all its device memory.  NULL is allowed. */
void lda_destroy(lda_ctx* ctx);

#ifdef __cplusplus
}
#endif
#endif /* LDA_MI355X_H */
