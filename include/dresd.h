/*
 * dresd.h -- C ABI of the MI355X (gfx950) dense-retrieval library.
 *
 * The library implements the drafting step of DReSD (Dense Retrieval for
 * Speculative Decoding): the datastore is a key -> value map whose keys are
 * L2-normalised token embeddings and whose values are the next L tokens that
 * followed each key (Section 3.5).  A query embedding, itself L2-normalised
 * (Section 3.4, Eq. 2), retrieves the value of the most similar key under
 * cosine similarity (Section 3.5, Eq. 3).  Keys and queries have unit norm, so
 * the cosine is the inner product and the library computes the raw inner
 * product without dividing by the norms.  Batch verification consumes several
 * drafts per decode step (Section 3.6), so the argmax of Eq. 3 is returned as
 * the k best keys.  The search is exact (every key is scored), not the
 * approximate search the paper used.
 *
 * Conventions shared by every call:
 *  - Pointers marked "device" are HIP device pointers on the current device.
 *    Pointers marked "host" are ordinary host memory.
 *  - dresd_stream is a hipStream_t (NULL = the null stream).  Work is enqueued
 *    on it and the call returns; results are valid once the stream has
 *    completed, except where a call says it synchronises.
 *  - Every argument is validated before any work is enqueued: on an error
 *    return nothing has been written to any output.
 *  - No C++ exception crosses this interface.  A failing call returns a status
 *    code and sets a thread-local message readable with dresd_last_error().
 *  - Inputs must be finite.  Keys and queries are expected to be
 *    L2-normalised; the library does not renormalise.
 */
#ifndef DRESD_H
#define DRESD_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Streams and graphs.  Every search, transform and draft call only enqueues
 * kernels on the given stream once a first call of the same shapes has sized
 * the workspaces it uses (that first call may allocate and synchronise).
 * After such a warm-up call these calls can be captured in a HIP graph:
 * they issue no allocation, no synchronisation and no memset while running.
 * A call that would have to grow a workspace while its stream is being
 * captured fails with DRESD_EUNSUPPORTED instead.  A workspace that a later,
 * larger call outgrows is never freed before its owner is (the index for
 * search workspaces, the process for the sums of transforms and k-means
 * updates, one per device and stream), so a graph captured earlier stays
 * valid after such a call.  (Buffers that only uncaptured calls use are freed
 * when outgrown and by dresd_release_cached.)
 *
 * Allocation-failure test hook: with DRESD_FAIL_ALLOC_AT=n in the
 * environment, the n-th device allocation the library makes (counted from
 * when the variable last took a new value) fails as out of memory.
 */
typedef struct dresd_index dresd_index; /* opaque, library-owned */
typedef struct dresd_ivf dresd_ivf;     /* opaque: partitioned index */
typedef void *dresd_stream;             /* a hipStream_t */

/* Storage type of the keys.  Queries are always fp32; scores are fp32.
 * DRESD_F8 (e4m3, no infinities, largest value 448) is a storage type of
 * paged caches alone (dresd_kv_cache). */
typedef enum { DRESD_F32 = 0, DRESD_F16 = 1, DRESD_BF16 = 2, DRESD_F8 = 3 } dresd_dtype;

typedef enum {
  DRESD_OK = 0,
  DRESD_EINVAL = 1,      /* an argument is out of its documented range     */
  DRESD_ENOMEM = 2,      /* a device allocation failed (nothing leaked)    */
  DRESD_EDEVICE = 3,     /* a HIP call failed; message in dresd_last_error */
  DRESD_EUNSUPPORTED = 4 /* valid request the library cannot serve        */
} dresd_status;

/* Largest k a search may ask for. */
#define DRESD_K_MAX 1024
/* Largest datastore: row indices are carried in 32 bits inside the kernels. */
#define DRESD_N_MAX 4294967040LL
/* Most partitions of a partitioned index. */
#define DRESD_PARTS_MAX (1 << 24)

/*
 * Build an index over N keys (Section 3.5: keys are token embeddings, values
 * the next L tokens; building the datastore is a one-time cost, Section 5.6).
 *
 *   embeddings    device, [N, d] row-major, element type `dtype`
 *                 (f32, IEEE binary16, or bfloat16), each row L2-normalised.
 *   continuations device, [N, L] row-major int32 token ids (opaque; copied
 *                 bit for bit, including any padding id).
 *   N, d, L       1 <= N <= DRESD_N_MAX, 1 <= d <= 16384, 1 <= L <= 4096.
 *   dtype         a dresd_dtype value.
 *   stream        stream used for the copies.
 *   out           host; receives the new index.
 *
 * Ownership: both arrays are copied into library-owned device memory (keys
 * re-laid out for the scan).  The call synchronises `stream` before it
 * returns, so the caller may free or reuse its arrays immediately.  The index
 * lives on the device that was current during this call.
 * Errors: EINVAL (null pointer, size out of range, unknown dtype), ENOMEM,
 * EDEVICE.  On error *out is left unchanged and nothing is allocated.
 */
dresd_status dresd_index_create(const void *embeddings,
                                const int32_t *continuations, int64_t N,
                                int32_t d, int32_t L, int32_t dtype,
                                dresd_stream stream, dresd_index **out);

/*
 * Exact top-k retrieval for a batch of B queries (Eq. 3 taken as the k best
 * keys; the drafts of Section 3.6 are their continuations).
 *
 *   ix        index from dresd_index_create.
 *   queries   device, [B, d] fp32 row-major, each row L2-normalised.
 *   B         B >= 0; B == 0 is a no-op returning DRESD_OK.
 *   k         1 <= k <= min(N, DRESD_K_MAX).
 *   idx       device, [B, k] int64: row indices of the k best keys.
 *   score     device, [B, k] fp32: their inner products with the query.
 *   tokens    device, [B, k, L] int32: continuations of those rows, gathered
 *             bit for bit; may be NULL to skip the gather.
 *   stream    stream the search runs on.
 *
 * Order: rank r holds the r-th largest score; equal scores are ordered by
 * ascending row index.  Scores are accumulated in fp32.  For 16-bit keys and
 * B <= 4 the query enters the matrix cores as three 16-bit parts that sum to
 * it exactly (scores within fp32 summation error of the exact inner
 * product); larger bf16 batches take two parts (their sum within 2^-17
 * relative of the query: score error below 8e-6) and larger f16 batches the
 * query rounded once to f16 (score error below 5e-4); both are inside the
 * 2e-3 parity bound for 16-bit keys.
 * Determinism: identical inputs give bitwise identical outputs.
 * Ownership: outputs are caller-owned and must stay alive until `stream`
 * completes.  The index owns a workspace per stream it is searched on, which
 * grows on first use with a new batch shape (that growth allocates and
 * synchronises; outgrown workspaces are kept until the index is destroyed):
 * searches on different streams may overlap on the device, searches on one
 * stream are ordered by it.  The calls themselves are not thread-safe: calls
 * on one index from several host threads must be serialised by the caller.
 * Errors: EINVAL (null index/queries/idx/score, k out of range, B < 0),
 * ENOMEM (workspace growth failed; no output written), EUNSUPPORTED (the
 * workspace would have to grow during stream capture), EDEVICE.  Small
 * datastores list whole tiles, in a workspace of up to about 256 MiB; where
 * that cannot be had, the scan with the shorter lists runs instead.
 */
dresd_status dresd_search(dresd_index *ix, const float *queries, int32_t B,
                          int32_t k, int64_t *idx, float *score,
                          int32_t *tokens, dresd_stream stream);

/*
 * Next-token-filtered retrieval (Section 3.5, with Section 3.1): the token
 * x_{t+1} that the LLM produced with the query embedding removes every draft
 * that does not start with it.  Read as filter-then-select: for query b only
 * rows whose continuation starts with next_tok[b] (continuations[i][0] ==
 * next_tok[b]) compete, and the k best of them are returned exactly as by
 * dresd_search.  When fewer than k rows match, the ranks past them hold
 * idx -1, score -inf and zero tokens.
 *
 *   next_tok  device, [B] int32: the next token of each query.
 *   Other arguments, order, determinism, ownership and errors as for
 *   dresd_search (EINVAL also for a null next_tok when B > 0).  The first
 *   token of every row is kept by the index (4 bytes per row, built by
 *   dresd_index_create), so a filtered scan reads 64 more bytes per 16 rows.
 */
dresd_status dresd_search_filtered(dresd_index *ix, const float *queries,
                                   const int32_t *next_tok, int32_t B, int32_t k,
                                   int64_t *idx, float *score, int32_t *tokens,
                                   dresd_stream stream);

/*
 * Allocation-free search, for callers that cannot allocate device memory:
 * code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  The same search as dresd_search (same kernels, bitwise the same
 * outputs; a batch of 1,024-dim keys whose tiled-contraction lists would
 * not fit the scratch runs the shared-key scan instead, and one whose lists
 * of whole tiles would not fit the single-tile scan), with its workspace
 * in a fixed library scratch of
 * DRESD_SCRATCH_BYTES that every device the library runs on holds until the
 * process ends, instead of the index's growable workspace.  It allocates no
 * device or host memory and never synchronises; the caller still passes the
 * queries and the outputs.
 *
 *   Arguments, order, determinism and errors as for dresd_search, and
 *   EINVAL when the search needs more workspace than DRESD_SCRATCH_BYTES
 *   even so (dresd_search_plan's workspace_bytes, the need of dresd_search,
 *   is an upper bound; e.g. one query up to k = 1024, or 64 queries at
 *   k = 32, fit).  Profiling (dresd_profile_*)
 *   does not time these calls.
 * Every call on one device shares that device's scratch, which keeps the
 * last call's contents (each search writes every scratch byte it reads
 * before reading it, so nothing needs clearing): calls that overlap on one
 * device -- on different streams, or with different indexes -- race, and
 * must be serialised by the caller (e.g. issued on one stream).
 */
#define DRESD_SCRATCH_BYTES (64LL << 20)
dresd_status dresd_search_noalloc(dresd_index *ix, const float *queries, int32_t B,
                                  int32_t k, int64_t *idx, float *score,
                                  int32_t *tokens, dresd_stream stream);

/* Describe an index.  Any output pointer (host) may be NULL.
 * Errors: EINVAL when ix is NULL. */
dresd_status dresd_index_info(const dresd_index *ix, int64_t *N, int32_t *d,
                              int32_t *L, int32_t *dtype);

/* Free an index and its workspace (synchronises its device).  NULL is
 * ignored.  Blocks of at least 64 MiB that held its keys, values, first tokens
 * or (partitioned) slot tables, or the memory that grouped the rows of a build,
 * are kept for the next index that is created, together at most 1/128 of the
 * device's memory: the oldest go back to the driver first, and all of a
 * device's go back when an allocation of the library on it fails and they
 * would make room for it, or by dresd_release_cached.  Larger blocks and
 * everything smaller go back at once. */
void dresd_index_destroy(dresd_index *ix);

/* Give back to the driver the device memory that the library holds for later
 * calls and that neither an index nor a captured graph uses: the blocks kept
 * by dresd_index_destroy and dresd_ivf_destroy, and the operands and sorting
 * buffers of uncaptured transforms (at most 512 MiB per device and stream),
 * k-means assignments and updates (256 MiB each), on every device.  For programs whose
 * other allocators need the memory.  Synchronises the devices concerned; may be
 * called from any thread, but not while a stream is being captured.  Later
 * calls allocate again what they need.
 * Errors: EDEVICE, ENOMEM (the host's). */
dresd_status dresd_release_cached(void);

/* Message for the last failing call on this thread ("" if none).  The
 * pointer stays valid until the next call on this thread. */
const char *dresd_last_error(void);

/*
 * Measurement support.  When enabled, every search ties HIP events to its
 * kernels' own dispatches (hipExtLaunchKernel): the begin and end of the main
 * scan kernel (the full pass over the keys), and the begin of the search's
 * first kernel and the end of its last, so that profiling adds no packets
 * between kernels.  dresd_profile_read synchronises those events and
 * returns the summed device milliseconds and the number of searches since
 * the last read, then clears them.  Outputs are host pointers (NULL allowed).
 * Errors: EINVAL when ix is NULL; EDEVICE.
 */
dresd_status dresd_profile_enable(dresd_index *ix, int32_t on);
dresd_status dresd_profile_read(dresd_index *ix, double *scan_ms,
                                double *search_ms, int64_t *searches);

/*
 * Measurement support: the achievable HBM read bandwidth of the device with
 * the scans' access pattern (every wave streams one contiguous range in
 * 1 KiB wave loads, 16 nontemporal loads in flight), the ceiling against
 * which a scan's bandwidth is judged beside the spec sheet's figure.
 *
 *   buf         device, `bytes` readable bytes (contents do not matter;
 *               only read).
 *   bytes       a multiple of 1024, at least 1 MiB (use far more than the
 *               last-level caches, e.g. several GiB).
 *   reps        1 <= reps <= 1000 timed read passes, after one untimed pass.
 *   workgroups  workgroups of 4 waves (0: four per compute unit).
 *   ms          host; mean device milliseconds per pass (HIP events).
 * Synchronises `stream`.  Allocates nothing on the device.
 * Errors: EINVAL (null pointer, sizes out of range), EDEVICE.
 */
dresd_status dresd_bw_probe(const void *buf, int64_t bytes, int32_t reps, int32_t workgroups,
                            double *ms, dresd_stream stream);

/*
 * Query-side transform of Algorithm 1 steps 4-6, for decode-step queries (or,
 * once, for the datastore rows that become keys):
 *   z   = (x - mean) / sqrt(var + eps_z)        z-score normalisation, Eq. 1
 *   v   = z W                                   first l principal components,
 *                                               Section 3.3
 *   y   = v / max(||v||_2, eps_n)               L2 normalisation, Eq. 2
 *
 *   x       device, [M, D] fp32 row-major (e.g. last hidden states).
 *   M       0 <= M < 2^31; M == 0 is a no-op.
 *   D       1 <= D <= 2^20.
 *   mean    device, [D] fp32: E[V] of the datastore sample.
 *   var     device, [D] fp32: Var[V] of the datastore sample (>= 0).
 *   eps_z   finite, >= 0 (the paper's eps of Eq. 1; 1e-5 is a common choice).
 *   W       device, [D, l] fp32 row-major: the principal components W_l.
 *   l       1 <= l <= 16384.
 *   eps_n   finite, >= 0 (the eps of Eq. 2; 1e-12 is a common choice).
 *   y       device, [M, l] fp32 row-major output (ready for dresd_search).
 *   stream  stream the transform runs on (asynchronous).
 * Arithmetic: fp32, the projection on the fp32 matrix cores, or for large
 * batches (at least 512 rows and about 2^30 multiply-adds) on the 16-bit ones
 * with z and W in three bf16 parts each that sum to them (error no larger; a
 * workspace of 6 D l bytes, at most 256 MiB, and as much again at most for
 * partial sums, kept for later calls; in fp32
 * without it and inside a capture, whose graph may replay on any stream); batches with
 * few output tiles split D across workgroups and add the partial sums in a
 * fixed order, so results are deterministic.  Ownership: all buffers are
 * caller-owned and must stay alive until `stream` completes; the partial sums
 * use a library buffer per (device, stream) that is allocated (synchronously)
 * on the first call on that stream that needs a larger one and kept, like
 * every buffer it outgrows, until the process ends: calls on different
 * streams may overlap, calls on one stream are ordered by it, also when several
 * host threads make them.  A graph captured from a call that splits D uses that
 * stream's buffer: it must not replay beside calls on the stream, or beside
 * another such graph.
 * Errors: EINVAL (null pointer with M > 0, sizes or eps out of range),
 * ENOMEM, EUNSUPPORTED (the buffer would have to grow during stream
 * capture), EDEVICE.
 */
dresd_status dresd_transform(const float *x, int64_t M, int32_t D, const float *mean,
                             const float *var, float eps_z, const float *W, int32_t l,
                             float eps_n, float *y, dresd_stream stream);

/*
 * Draft assembly for batch verification (Section 3.6): the retrieved
 * continuations become the rows of an EOS-padded draft matrix.  For each
 * query, in rank order: a draft is the first `length` tokens of a
 * continuation with every token after its first EOS replaced by EOS; drafts
 * that start with EOS (nothing to propose, e.g. the padding ranks of
 * dresd_search_filtered) and repeats of an earlier draft are dropped; the
 * first r remaining drafts fill the rows, and rows past them are all EOS.
 *
 *   tokens  device, [B, k, L] int32 (as written by dresd_search).
 *   B >= 0 (0 is a no-op); 1 <= k <= DRESD_K_MAX; 1 <= L <= 4096;
 *   1 <= r <= k drafts; 1 <= length <= L tokens per draft; eos: the EOS id.
 *   drafts  device, [B, r, length] int32 output.
 *   count   device, [B] int32 output: drafts kept per query (<= r).
 *   stream  stream it runs on (asynchronous).
 * Deterministic; allocates nothing; buffers are caller-owned.
 * Errors: EINVAL (null pointer with B > 0, sizes out of range), EDEVICE.
 */
dresd_status dresd_pack_drafts(const int32_t *tokens, int32_t B, int32_t k, int32_t L,
                               int32_t r, int32_t length, int32_t eos, int32_t *drafts,
                               int32_t *count, dresd_stream stream);

/*
 * Batch verification (Section 3.6).  The drafts of a step go through the
 * language model in one forward beside the cached context, and the path that
 * the model's own tokens follow is accepted.  The five calls below are what
 * that forward needs around the model's weights:
 *
 *   dresd_draft_tree       drafts -> prefix tree: its tokens, parents, depths
 *                          and, for the attention, every node's ancestors
 *   dresd_kv_write         the tree's keys and values into the paged cache
 *   dresd_paged_attention  its queries over the context and their ancestors
 *   dresd_accept_drafts    the logits of its nodes -> the accepted path
 *   dresd_kv_read          (with dresd_kv_write) the accepted path's entries
 *                          out of the cache and into their final slots
 *
 * The same cache serves prompts, in chunks, and single tokens.  None of them
 * allocates, synchronises or keeps state between calls; all can be captured.
 */

/* Most nodes of a draft tree. */
#define DRESD_NODES_MAX 1024

/*
 * Prefix tree of each query's drafts.  Node 0 is next_tok[b]; draft by draft
 * in rank order, each prefix that no earlier draft has becomes a node, so a
 * parent's index is lower than its children's.  Drafts that do not start with
 * next_tok[b] cannot be accepted and are left out, and a draft ends before its
 * first EOS.  Nodes past the budget N are dropped.
 *
 *   drafts    device, [B, r, length] int32 (from dresd_pack_drafts).
 *   count     device, [B] int32: drafts per query (rows past them are not read
 *             as drafts; values outside [0, r] count as the nearer bound).
 *   next_tok  device, [B] int32.
 *   0 <= B < 2^22 (0 is a no-op); 1 <= r <= DRESD_K_MAX; 1 <= length <= 4096;
 *   1 <= N <= DRESD_NODES_MAX.  1 + r (length - 1) nodes always suffice.
 *   token     device, [B, N] int32 out: token of each node, eos past the last.
 *   parent    device, [B, N] int32 out: its parent, -1 for node 0 and past the
 *             last node.
 *   depth     device, [B, N] int32 out: its tokens after node 0 (so that the
 *             node's position is node 0's plus its depth), 0 past the last.
 *   mask      device, [B, N, W] uint64 out, W = (N + 63) / 64: bit v of row u
 *             (bit v % 64 of word v / 64) is set where v is u or an ancestor of
 *             u; 0 past the last node.  As dresd_paged_attention takes it.
 *   nodes     device, [B] int32 out: nodes of each tree, >= 1.
 * Deterministic.  Errors: EINVAL (null pointer with B > 0, sizes out of
 * range), EDEVICE.
 */
dresd_status dresd_draft_tree(const int32_t *drafts, const int32_t *count,
                              const int32_t *next_tok, int32_t B, int32_t r, int32_t length,
                              int32_t eos, int32_t N, int32_t *token, int32_t *parent,
                              int32_t *depth, uint64_t *mask, int32_t *nodes,
                              dresd_stream stream);

/*
 * A paged cache of keys and values, in the caller's memory.  Slot s is row
 * s % page_size of page s / page_size, for every head.
 *   k, v          device, [pages, heads, page_size, dim], 16-byte aligned, element
 *                 type dtype: DRESD_F16, DRESD_BF16 or DRESD_F8.
 *   k_exp, v_exp  DRESD_F8: device, [pages, heads, page_size] uint8: a row's
 *                 values are its stored ones times 2^(exp - 127); 1 <= exp <= 254 (as
 *                 dresd_kv_write stores it) where a row is read.  NULL otherwise.
 *   1 <= pages < 2^31; page_size a power of two, at most 65536;
 *   1 <= heads <= 65535; dim a multiple of 8 in [8, 256].
 */
typedef struct {
  void *k, *v;
  uint8_t *k_exp, *v_exp;
  int64_t pages;
  int32_t page_size, heads, dim, dtype;
} dresd_kv_cache;

/*
 * Write n tokens' keys and values into cache slots.
 *   k, v      device, element type dtype (DRESD_F32, DRESD_F16 or DRESD_BF16):
 *             element j of head h of token i is at i * row + h * head + j, in elements, with
 *             strides of its own for k and v (slices of a projection's output
 *             need no copy).  Pointers and strides are multiples of 16 bytes.
 *   slots     device, [n] int64: each token's slot.  A token whose slot is outside
 *             [0, pages * page_size) (-1, say) is skipped.  Two tokens of one call
 *             must not share a slot (not checked: its contents would be a mixture).
 *   n >= 0 (0 is a no-op), and n heads at most 2^29 - 32 for dim <= 64, 2^28 - 32
 *   for dim <= 128, else 2^27 - 32.
 * 16-bit caches hold the values rounded to nearest even.  DRESD_F8: a row (one
 * token of one head) is stored at the smallest power of two, not below 2^-126,
 * at which its largest magnitude is at most 448 (a zero row: 2^-9), its
 * elements rounded to nearest even (but down where 2^128 would result);
 * infinite elements are stored as NaN, as NaNs are, and do not take part in
 * the largest magnitude.  A power of two scales without rounding, so rows read
 * back in fp32 are exactly the stored ones, and those with exponents of -124 and up
 * (magnitudes past 2^-116) in bf16 too, whose smallest number is 2^-133; writing
 * such rows again stores the same values.
 * Errors: EINVAL (null pointer with n > 0, ranges, alignment, a dtype that does
 * not fit), EDEVICE.
 */
dresd_status dresd_kv_write(const dresd_kv_cache *cache, const void *k, int64_t k_row,
                            int64_t k_head, const void *v, int64_t v_row, int64_t v_head,
                            int32_t dtype, const int64_t *slots, int64_t n,
                            dresd_stream stream);

/*
 * Read cache slots back: k, v device, [n, heads, dim] out in dtype (DRESD_F32,
 * DRESD_F16 or DRESD_BF16; rounded to nearest even), 16-byte aligned; slots device, [n]
 * int64, in any order, repeats allowed.  A slot outside the cache gives zeros.
 * Errors: as dresd_kv_write.
 */
dresd_status dresd_kv_read(const dresd_kv_cache *cache, const int64_t *slots, int64_t n,
                           int32_t dtype, void *k, void *v, dresd_stream stream);

/*
 * Attention of a chunk of new tokens over a paged cache that holds their own
 * keys and values already.  Sequence b has lengths[b] tokens in the cache, the last
 * n_b of which are its chunk, and page table[b][p / page_size] holds its
 * position p.  Row t of its chunk (position lengths[b] - n_b + t) sees the
 * positions up to its own, or, with a mask, all positions before the chunk and
 * those chunk tokens j whose bit j is set in its row of the mask:
 *
 *   out = sum_p e^(s_p - lse) v_p,   s_p = scale q . k_p,   lse = log sum_p e^(s_p)
 *
 * over the visible p.  A row that sees nothing gets zeros and lse -inf.
 *
 *   q         device, dtype DRESD_F16 or DRESD_BF16 (that of a 16-bit cache): head
 *             h of row t is at t * q_row + h * q_head, in elements; pointer and
 *             strides are multiples of 16 bytes.  Rows of all chunks follow one another.
 *   q_heads   a multiple of the cache's heads: query head h reads cache head
 *             h / (q_heads / heads).
 *   starts    device, [B + 1] int32: sequence b's chunk is rows starts[b] to
 *             starts[b + 1] - 1, n_b of them, possibly none; rows before
 *             starts[0] and from starts[B] on are left as they were.  They
 *             ascend within [0, T] (not checked: where they do not, nothing outside
 *             the T rows is touched, but what they hold is not defined).
 *             Or NULL: T = B n, and every chunk has n rows.
 *   n         tokens per chunk without starts (ignored with them).
 *   T         rows of q and out, T * q_heads < 2^31; T = 0 is a no-op.
 *   table     device, [B, width] int32, width >= 1, 0 <= B heads <= 2^30: page ids.
 *             Positions past the table and pages outside [0, pages) hold nothing:
 *             they are not seen.
 *   lengths   device, [B] int32; positions from 2^31 - 256 on are not seen.
 *   mask      device, [T, words] uint64 (bits past the words are unset), or NULL.
 *   scale     finite.
 *   out       device, [T, q_heads, dim] in dtype, 16-byte aligned.
 *   lse       device, [T, q_heads] fp32 (natural logarithm), or NULL.
 *   work      device, work_bytes of workspace, 16-byte aligned: at least what
 *             dresd_paged_attention_workspace says for these arguments (which
 *             reads no device memory).  Used by this call alone until `stream`
 *             has completed it; its contents do not matter.
 * What masked positions hold does not matter, infinities and NaN included; a row that
 * sees a key that is not finite, a value past 2^88 or a score outside fp32's range
 * may become NaN throughout.
 * Scores, softmax statistics and sums are fp32; keys and queries enter the
 * matrix cores unrounded, a row's weights rounded to dtype (f16 over 8 bits: times
 * the power of two of their value; less than 2^-35 of the row's largest is lost).
 * Deterministic.
 * Errors: EINVAL (null pointer with T > 0, ranges, alignment, dtypes that do not
 * fit, too little workspace, more than some 2^24 blocks of the 16 to 128 rows of a
 * cache head that are computed together), EDEVICE.
 */
dresd_status dresd_paged_attention(const dresd_kv_cache *cache, const void *q, int64_t q_row,
                                   int64_t q_head, int32_t dtype, int32_t q_heads,
                                   const int32_t *starts, int32_t n, int32_t B, int64_t T,
                                   const int32_t *table, int32_t width, const int32_t *lengths,
                                   const uint64_t *mask, int32_t words, float scale, void *out,
                                   float *lse, void *work, int64_t work_bytes,
                                   dresd_stream stream);
dresd_status dresd_paged_attention_workspace(const dresd_kv_cache *cache, int32_t q_heads,
                                             int32_t ragged, int32_t n, int32_t B, int64_t T,
                                             int32_t width, int64_t *bytes);

/*
 * Acceptance of a draft tree by the model's own greedy tokens: from node 0,
 * with g the token of the largest logit of the present node (ties to the lower
 * token; NaN is below everything, and a row of nothing else gives token 0), go on
 * to the lowest-numbered child whose token is g, while there is one and fewer
 * than `most` nodes are accepted.
 *
 *   logits    device, dtype (DRESD_F32, DRESD_F16 or DRESD_BF16): row u of query
 *             b starts at (b N + u) * row elements, row >= V.
 *   token, parent  device, [B, N] int32, nodes device, [B] int32: the tree
 *             (dresd_draft_tree; nodes outside [0, N] count as the nearer bound).
 *   0 <= B < 2^22 (0 is a no-op); 1 <= N <= DRESD_NODES_MAX; 1 <= V <= 2^29;
 *   1 <= most <= DRESD_NODES_MAX.
 *   path      device, [B, most] int32 out: the accepted nodes, -1 past them.
 *   accepted  device, [B] int32 out: their number, >= 1 (0 for an empty tree).
 *   next_tok  device, [B] int32 out: the model's token after the last of them (-1
 *             for an empty tree).
 * Deterministic.  Errors: EINVAL (null pointer with B > 0, sizes out of range),
 * EDEVICE.
 */
dresd_status dresd_accept_drafts(const void *logits, int32_t dtype, int64_t row, int32_t V,
                                 const int32_t *token, const int32_t *parent,
                                 const int32_t *nodes, int32_t B, int32_t N, int32_t most,
                                 int32_t *path, int32_t *accepted, int32_t *next_tok,
                                 dresd_stream stream);

/*
 * Describe how the next search of this shape would run (host outputs, NULL
 * allowed): the number of passes over sampled keys before the main pass, the
 * number of waves of the main scan (of the first launch when the batch
 * takes several), the bytes of workspace it needs,
 * which scan kernel runs it: 0 = single-tile scan (batches within one
 * 16-column query tile group, queries staged in LDS), 1 = shared-key scan
 * (queries held in registers, keys staged through LDS), 2 = single-tile scan
 * serving several query groups per launch (batches whose query operands
 * exceed one workgroup's LDS; the groups share each key range through L2),
 * 3 = tiled contraction (keys of more than 1,024 dims at batches of two or
 * more query tiles, and 1,024-dim keys at batches past four query tiles: key
 * and query blocks both streamed through LDS, column by column, for panels
 * of 16 or 32 key tiles), 4 = whole-tile scan (small datastores with fp32
 * keys, or with 16-bit keys at batches of at most four queries: every key of a
 * wave's one, two or four tiles is listed for the merge), and the number of
 * launches of the main scan (each one pass over the keys for a part of the
 * batch).
 * Errors: EINVAL for the same argument errors as dresd_search.
 */
dresd_status dresd_search_plan(const dresd_index *ix, int32_t B, int32_t k,
                               int32_t *sample_passes, int32_t *scan_waves,
                               int64_t *workspace_bytes, int32_t *scan_kind,
                               int32_t *launches);

/*
 * Partitioned (approximate) search.  The paper retrieves with an approximate
 * nearest-neighbour library (Section 3.5); this is its partitioned reading,
 * an inverted file: every key belongs to one of P partitions, each with a
 * centroid, and a search scores only the keys of the nprobe partitions whose
 * centroids score highest for the query.  The result is the exact top-k over
 * those keys (same ranking, scores and tie rule as dresd_search), so it
 * differs from dresd_search only where a true top-k key lies in a partition
 * that was not probed.
 *
 * dresd_ivf_create: embeddings / continuations / N / d / L / dtype as in
 *   dresd_index_create; centroids device [P, d] fp32 (unit rows, e.g. from
 *   dresd_kmeans_*), 1 <= P <= DRESD_PARTS_MAX; assign device [N] int32, the
 *   partition of each key, in [0, P).  Keys are stored grouped by partition
 *   (each partition padded to a 16-row tile); continuations stay in row
 *   order.  Copies everything, synchronises `stream`; the caller may free its
 *   buffers afterwards.  One-time cost: the rows are grouped by a sort on the
 *   device, with 16 N bytes of temporary memory.  Errors: EINVAL (nulls, ranges, an assignment outside [0, P)),
 *   ENOMEM, EDEVICE.
 * dresd_ivf_search: like dresd_search, probing 1 <= nprobe <= min(P,
 *   DRESD_K_MAX) partitions per query (the nprobe best centroids by inner
 *   product, ties to the lower id).  Ranks past the keys of the probed
 *   partitions hold index -1, score -inf and zero tokens.  Workspaces and
 *   the probe buffer are per stream, as for dresd_search: searches on
 *   different streams may overlap on the device; calls from several host
 *   threads must be serialised by the caller.
 * dresd_ivf_search_filtered: dresd_ivf_search with the next-token filter of
 *   dresd_search_filtered (next_tok device [B] int32): among the keys of the
 *   probed partitions only those whose continuation starts with the query's
 *   next token compete; ranks past them are padded the same way.
 * dresd_ivf_search_probes: the search with caller-chosen partitions: probes
 *   device [B, S] int32, 1 <= S <= DRESD_K_MAX; entries outside [0, P) are
 *   ignored and repeats count once; next_tok: NULL, or device [B] int32 for
 *   the next-token filter.
 * dresd_ivf_create_by_token: the next-token filter of Section 3.5 (a draft
 *   that does not start with the next token is dropped) as a partitioning:
 *   partition p holds the keys whose continuation starts with the p-th
 *   smallest distinct first token (P = the number of distinct first tokens,
 *   at most DRESD_PARTS_MAX); no centroids.  Arguments as in
 *   dresd_index_create.  Copies everything and synchronises `stream`; the
 *   grouping is a device sort of the first tokens.  Errors as
 *   dresd_ivf_create.
 *   dresd_ivf_search and dresd_ivf_search_filtered reject such an index
 *   (EINVAL: no centroids); dresd_ivf_search_probes takes partition ids in
 *   ascending token order.
 * dresd_ivf_search_next_token: on an index from dresd_ivf_create_by_token,
 *   the result of dresd_search_filtered (same keys compete, same ranking and
 *   tie rule, exact top-k) computed by scanning only the query's next-token
 *   partition: next_tok device [B] int32, any value (a token no key starts
 *   with gives a fully padded row).  Its cost follows the probed partitions'
 *   sizes, so it pays when the batch's next tokens together select fewer
 *   keys than the datastore holds (small batches); the full filtered scan
 *   reads every key once for the whole batch.  Scores come from the
 *   three-part exact query split at every batch size (within the 1e-5 bound
 *   of the small-batch scans).  Errors: EINVAL (NULLs, B < 0, k out of range,
 *   an index not grouped by token), ENOMEM, EUNSUPPORTED, EDEVICE.
 * dresd_ivf_info: host outputs (NULL allowed); tiles = 16-row tiles of the
 *   partitioned layout (padding included).
 * dresd_ivf_profile_enable / _read: as dresd_profile_*, for the scan of the
 *   probed partitions and the whole search.
 */
dresd_status dresd_ivf_create(const void *embeddings, const int32_t *continuations, int64_t N,
                              int32_t d, int32_t L, int32_t dtype, const float *centroids,
                              int32_t P, const int32_t *assign, dresd_stream stream,
                              dresd_ivf **out);
void dresd_ivf_destroy(dresd_ivf *ivf);
dresd_status dresd_ivf_info(const dresd_ivf *ivf, int64_t *N, int32_t *d, int32_t *L,
                            int32_t *dtype, int32_t *P, int64_t *tiles);
dresd_status dresd_ivf_search(dresd_ivf *ivf, const float *queries, int32_t B, int32_t k,
                              int32_t nprobe, int64_t *idx, float *score, int32_t *tokens,
                              dresd_stream stream);
dresd_status dresd_ivf_search_filtered(dresd_ivf *ivf, const float *queries,
                                       const int32_t *next_tok, int32_t B, int32_t k,
                                       int32_t nprobe, int64_t *idx, float *score,
                                       int32_t *tokens, dresd_stream stream);
dresd_status dresd_ivf_search_probes(dresd_ivf *ivf, const float *queries, const int32_t *probes,
                                     int32_t S, const int32_t *next_tok, int32_t B, int32_t k,
                                     int64_t *idx, float *score, int32_t *tokens,
                                     dresd_stream stream);
dresd_status dresd_ivf_create_by_token(const void *embeddings, const int32_t *continuations,
                                       int64_t N, int32_t d, int32_t L, int32_t dtype,
                                       dresd_stream stream, dresd_ivf **out);
dresd_status dresd_ivf_search_next_token(dresd_ivf *ivf, const float *queries,
                                         const int32_t *next_tok, int32_t B, int32_t k,
                                         int64_t *idx, float *score, int32_t *tokens,
                                         dresd_stream stream);
/*
 * Spherical k-means, the partitioning of the partitioned search (the
 * centroids and assignment that dresd_ivf_create takes).  Cosine similarity
 * of unit vectors (Eq. 3) is the inner product.
 *
 * dresd_kmeans_assign: assign[i] = the centroid with the largest inner
 *   product with row i, ties to the lower id; score[i] (NULL allowed) = that
 *   inner product (fp32 accumulation of exact products).
 *   x device [n, d] row-major in dtype; 0 <= n <= DRESD_N_MAX (0: no-op);
 *   1 <= d <= 16384; centroids device [P, d] fp32, 1 <= P <= DRESD_PARTS_MAX;
 *   assign device [n] int32 out; score device [n] fp32 out.  Rows of at most
 *   256 dims are multiplied on the 16-bit matrix cores (the centroids split
 *   into three exact parts) with a workspace of about 6 P d bytes (at most
 *   256 MiB; 8 n more for small n) per (device, stream), kept for later
 *   calls; a call that cannot get one, or that is captured (its
 *   graph may replay on any stream), runs in fp32 without.
 * dresd_kmeans_update: each centroid becomes the unit vector along the sum of
 *   the rows assigned to it; a centroid with no rows (or a zero sum) is left
 *   as it is.  Sums are exact to 2^-30 per element and independent of the
 *   order of the rows (deterministic).  x as above with n < 2^31; assign
 *   device [n] int32, each in [0, P) (not checked: the caller's contract);
 *   centroids device [P, d] fp32 in/out; counts device [P] int32 out (rows per
 *   centroid, NULL allowed).  Uses a workspace of P*d*8 + P*4 bytes per
 *   (device, stream), allocated (synchronously) on first use on that stream
 *   and kept, like every buffer it outgrows, until the process ends (and, from
 *   2^24 elements to 2^24 rows, where it can be had and outside captures, 16 n
 *   more to sort them, kept for later calls): calls
 *   on different streams may overlap, calls on one stream are ordered by it,
 *   also when several host threads make them.  A graph captured from an
 *   update uses that stream's buffer of sums: it must not replay beside
 *   updates on the stream, or beside another such graph.
 * dresd_kmeans_init: the starting centroids of the iteration: P distinct
 *   rows spread evenly through the row order, centroid j = row pick(j)
 *   scaled to unit length (a zero row gives a zero centroid), with
 *   pick(j) = (o + floor(j n / P)) mod n and o = s mod n, where s is the
 *   first output of SplitMix64 (Steele, Lea and Flood, 2014) started from
 *   state `seed`.  x as above with 1 <= n; 1 <= P <= min(n,
 *   DRESD_PARTS_MAX); centroids device [P, d] fp32 out (the norm is taken in
 *   fp64 over the decoded elements, each element rounded to fp32 once).
 *   Allocates nothing.
 * All three are asynchronous on `stream`.  Errors: EINVAL (ranges, nulls),
 * ENOMEM, EDEVICE.
 */
dresd_status dresd_kmeans_assign(const void *x, int64_t n, int32_t d, int32_t dtype,
                                 const float *centroids, int32_t P, int32_t *assign,
                                 float *score, dresd_stream stream);
dresd_status dresd_kmeans_update(const void *x, int64_t n, int32_t d, int32_t dtype,
                                 const int32_t *assign, int32_t P, float *centroids,
                                 int32_t *counts, dresd_stream stream);
dresd_status dresd_kmeans_init(const void *x, int64_t n, int32_t d, int32_t dtype, int32_t P,
                               uint64_t seed, float *centroids, dresd_stream stream);

dresd_status dresd_ivf_profile_enable(dresd_ivf *ivf, int32_t on);
dresd_status dresd_ivf_profile_read(dresd_ivf *ivf, double *scan_ms, double *search_ms,
                                    int64_t *searches);

#ifdef __cplusplus
}
#endif
#endif /* DRESD_H */
