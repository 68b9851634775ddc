/*
 * libleann -- C ABI of the MI355X (gfx950) implementation of LEANN's search hot
 * path (arXiv 2506.08276): the recompute-and-score loop of best-first
 * proximity-graph search.
 *
 * Conventions that hold for every call
 *   - "dev" pointers are device (HBM) addresses on the context's GPU, "host"
 *     pointers are ordinary host memory.  All buffers are caller-owned and
 *     only borrowed for the duration of the call; the library owns the opaque
 *     handles (leann_ctx, leann_pq) and its internal workspaces.
 *   - Work is enqueued on the HIP stream given to leann_create.  Calls that
 *     write host memory or return counts synchronise that stream; the others
 *     return as soon as the work is enqueued.
 *   - Every function returns LEANN_OK (0) or a negative status; on error no
 *     output buffer has been written.  leann_last_error() gives a message for
 *     the calling thread.  Nothing is printed and nothing aborts.
 *   - Arrays are row-major.  Scores are inner-product similarities: larger is
 *     closer.  Every ranking uses the total order (score descending, id
 *     ascending).
 */
#ifndef LEANN_H
#define LEANN_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    LEANN_OK = 0,
    LEANN_EINVAL = -1,    /* bad argument value (k > ef, ratio outside (0,1], null pointer, ...) */
    LEANN_ENOMEM = -2,    /* device or host allocation failed */
    LEANN_EDEVICE = -3,   /* a HIP call failed */
    LEANN_ESHAPE = -4,    /* shape the kernels do not cover (see leann_create) or inconsistent sizes */
    LEANN_ECAPACITY = -5  /* a per-query queue outgrew its capacity */
};

enum { LEANN_F32 = 0, LEANN_BF16 = 1, LEANN_F16 = 2 };

typedef struct leann_ctx leann_ctx;
typedef struct leann_pq leann_pq;
typedef struct leann_projection leann_projection;
typedef struct leann_adapter_rows leann_adapter_rows;
typedef struct leann_attention_plan leann_attention_plan;

/* Encoder shape.  The paper fixes a BERT-style encoder of 110 M parameters with
 * 768-d output over 256-token chunks (Sec. 7 set-up); the layer equations are the
 * standard post-LN ones, see leann_embed. */
typedef struct {
    int32_t layers, hidden, heads, ffn, vocab, max_pos;
    float ln_eps;
} leann_encoder_desc;

/* Pruned proximity graph in CSR form, 4-byte neighbour ids (Sec. 5, "Space(G1)").
 * row_ptr[n+1] and col_idx[row_ptr[n]] are device pointers; entry is the fixed
 * entry point p of Algorithm 2. */
typedef struct {
    const uint64_t *row_ptr;
    const uint32_t *col_idx;
    int64_t n;
    uint32_t entry;
} leann_graph;

/* Raw chunk store as token ids: tokens[n][seq] (PAD beyond the valid length,
 * content ignored) and lengths[n] in [1, seq]; device pointers. */
typedef struct {
    const int32_t *tokens;
    const int32_t *lengths;
    int64_t n;
    int32_t seq;
} leann_chunks;

/* Optional table of stored exact embeddings (the paper's embedding cache for
 * frequently visited nodes, Sec. 3 / App. D "Relaxing Disk Constraint").
 * slot_of[n] gives the row of emb for a node, or -1 when the node must be
 * recomputed; emb[rows][d] fp32.  Device pointers.  NULL = recompute everything. */
typedef struct {
    const int32_t *slot_of;
    const float *emb;
    int64_t rows;
} leann_emb_cache;

/* Pending index updates seen by the output stage of a search (App. B "Soft
 * Deletion Strategy", "Batched Add Operation"):
 *   deleted_bits: bit (v & 31) of word (v >> 5) set = node v is soft-deleted; (n + 31) / 32
 *     words.  Deleted nodes are traversed as before (their adjacency lists stay); the exact
 *     queue is filtered by the flag before the k best active entries are returned.
 *   buffer_emb fp32[buffer_n][hidden], buffer_ids[buffer_n]: embeddings of added chunks that
 *     are not inserted into the graph yet.  Every one is scored exactly (<q, e>) and merged
 *     with the graph's result under (score descending, id ascending).
 * Device pointers, borrowed for the call; either part may be absent (NULL / 0). */
typedef struct {
    const uint32_t *deleted_bits;
    const float *buffer_emb;
    const uint32_t *buffer_ids;
    int64_t buffer_n;
} leann_updates;

/* Per-call totals over all queries of a leann_search call. */
typedef struct {
    int64_t hops;              /* exploration steps (Alg. 2: taking the best unvisited node of EQ) */
    int64_t adc_candidates;    /* neighbours scored with PQ */
    int64_t recomputed_chunks; /* exact scores taken (sum over queries, entry point included) */
    int64_t encoded_chunks;    /* chunks actually sent through the encoder (after sharing within a round) */
    int64_t encoded_tokens;    /* valid tokens of those chunks */
    int64_t flushes;           /* per-query batch flushes */
    int64_t rounds;            /* traverse -> encode -> insert rounds over the whole query set: the flushes of the query
                                * that has most of them (groups of queries that run one after the other add up) */
    int64_t cache_hits;        /* exact scores served by the stored-embedding table (part of recomputed_chunks) */
    int64_t memo_hits;         /* exact scores served by the call's embedding memo (leann_set_call_memo; part of recomputed_chunks) */
    float encoder_ms, traverse_ms, total_ms; /* device time (the GPU's own clock): total_ms from the first kernel that sets up the
                                              * queries to the last one's end, traverse_ms of it the hops, exact scores and
                                              * packing, to the end of each round's last wavefront, encoder_ms the rest */
} leann_search_stats;

/* Message of the last error on the calling thread.  ctx is accepted for symmetry with the other calls and may be
 * NULL (leann_create fails before a context exists); the string is per thread, not per context. */
const char *leann_last_error(const leann_ctx *ctx);

/*
 * Create a context holding the encoder weights.
 *   weights_dev: packed parameters on the device, dtype LEANN_F32 or LEANN_BF16
 *   (every value in that one type), in this order, linear maps stored [out][in]:
 *     tok_emb[vocab][d], pos_emb[max_pos][d], seg_emb[d], emb_ln_g[d], emb_ln_b[d],
 *     per layer: Wqkv[3d][d] (query rows, key rows, value rows), bqkv[3d], Wo[d][d], bo[d],
 *                ln1_g[d], ln1_b[d], W1[F][d], b1[F], W2[d][F], b2[d], ln2_g[d], ln2_b[d].
 *   The library keeps its own copy (matrices and embedding tables in bf16, the
 *   rest in fp32) and, if the device has memory for it, the layers' matrices a second
 *   time in another order, which small passes are faster with (layers * (8 * hidden^2 +
 *   4 * hidden * ffn) bytes; results do not depend on it; freed when leann_embed or
 *   leann_search find no memory for their workspaces); the caller may free weights_dev
 *   after the call returns.
 *   Shapes covered: hidden/heads == 64, hidden % 128 == 0, ffn % 128 == 0,
 *   sequence length <= 256; anything else is LEANN_ESHAPE.
 *   device: HIP device ordinal; hip_stream: a hipStream_t (NULL = default stream).
 */
int leann_create(leann_ctx **out, const leann_encoder_desc *desc, const void *weights_dev, int weight_dtype,
                 int device, void *hip_stream);
void leann_destroy(leann_ctx *ctx);

/*
 * Embedding recomputation (Alg. 2, the recomputation step; Sec. 3 online stage).
 * For each requested chunk: x = LN(tok_emb[id_t] + pos_emb[t] + seg_emb), t < L;
 * per layer  x = LN(x + MHA(x) Wo + bo),  x = LN(x + GELU(x W1 + b1) W2 + b2)
 * with softmax over the L valid keys only; e = mean_t x_t;  e <- e / max(|e|, 1e-12).
 * bf16 matrix products with fp32 accumulation; softmax, LayerNorm and pooling in fp32.
 *   ids_dev: int64[n_ids] chunk numbers (device), NULL = chunks 0..n_ids-1.
 *   out_emb_dev: fp32[n_ids][hidden].
 * A chunk's embedding does not depend on which other chunks share the call.
 * Errors: token id outside [0, vocab), length outside [1, seq], id outside [0, n) -> LEANN_EINVAL.
 */
int leann_embed(leann_ctx *ctx, const leann_chunks *chunks, const int64_t *ids_dev, int64_t n_ids,
                float *out_emb_dev);

/*
 * Build the PQ table of the offline stage (Sec. 3: the index keeps a small PQ table of all embeddings).
 * Splits d into m_sub contiguous sub-vectors; per subspace runs `iters` Lloyd
 * iterations with 256 centroids on min(n, 65536) rows chosen by a seeded
 * permutation (splitmix64 Fisher-Yates; the first 256 rows of it are the initial
 * centroids; an empty cluster keeps its centroid; ties go to the lowest index),
 * then encodes all n rows.  emb_dev: fp32[n][d].  d/m_sub <= 32.
 * Scratch (min(n, 65536) * (4 * d + 5 * m_sub + 8) bytes and a little) stays with the context for the next call: at most
 * 1 GiB, what is larger is freed before the call returns.  It is freed when another allocation of the context finds no
 * memory, and by leann_destroy.  Calls on one context from several threads take turns: one trains at a time.
 */
int leann_build_pq(leann_ctx *ctx, const float *emb_dev, int64_t n, int32_t d, int32_t m_sub, int32_t iters,
                   uint64_t seed, leann_pq **out);
/* The PQ table is one of the two things the index stores (Sec. 3 "Storage composition": graph + PQ codes); the
 * calls below move it between the library and the caller.
 * Copy codebook fp32[m_sub][256][d/m_sub] and codes u8[n][m_sub] to host buffers (either may be NULL). */
int leann_pq_export(leann_ctx *ctx, const leann_pq *pq, float *codebook_host, uint8_t *codes_host);
/* Make a PQ table from host copies of a codebook and codes. */
int leann_pq_import(leann_ctx *ctx, const float *codebook_host, const uint8_t *codes_host, int64_t n, int32_t d,
                    int32_t m_sub, leann_pq **out);
/* Wrap a device-resident code table without copying it: codes_dev u8[n][m_sub] stays caller-owned and must
 * outlive the handle; the codebook is copied from the host. */
int leann_pq_wrap(leann_ctx *ctx, const float *codebook_host, const uint8_t *codes_dev, int64_t n, int32_t d,
                  int32_t m_sub, leann_pq **out);
int leann_pq_info(const leann_pq *pq, int64_t *n, int32_t *d, int32_t *m_sub);
void leann_pq_free(leann_pq *pq);

/*
 * Approximate scores (Alg. 2, the step that ranks a hop's new neighbours by their PQ distance to
 * the query before they enter AQ), product quantisation's asymmetric distance: for each query a lookup table
 * lut[m][c] = -|q_m - codebook[m][c]|^2 is built (sub-vector summed in index order)
 * and out[i][j] = sum_m lut[m][codes[cand[i][j]][m]] in the fixed order m = 0..m_sub-1,
 * fp32: the negated squared distance between q and the decoded vector (larger is closer).
 *   queries_dev fp32[nq][d]; cand_ids_dev u32[nq][nc]; out_dev fp32[nq][nc].
 * Candidate ids >= n are an error (LEANN_EINVAL, reported after the kernel ran; out_dev
 * then holds -inf at those positions).
 */
int leann_adc(leann_ctx *ctx, const float *queries_dev, int64_t nq, const leann_pq *pq,
              const uint32_t *cand_ids_dev, int32_t nc, float *out_dev);

/*
 * leann_adc for callers that cannot allocate device memory: code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc.  Same kernels and same results as leann_adc; the
 * per-query lookup tables live in a fixed array inside the library (4 MiB + 256 bytes per GPU, held
 * until the process ends) instead of a grown workspace.  The call allocates nothing, records no
 * memset and does not synchronise: the work is enqueued on the context's stream.
 *   Limits: nq <= 128 and m_sub <= 32; anything larger -> LEANN_ECAPACITY, nothing enqueued.
 *   A candidate id >= n is not reported through the status (that would need a synchronisation):
 *   out_dev holds -inf at its position.
 *   All calls on one GPU share the array: calls that overlap on one GPU (different streams or
 *   contexts) race; calls on one stream are ordered and safe.
 */
int leann_adc_noalloc(leann_ctx *ctx, const float *queries_dev, int64_t nq, const leann_pq *pq,
                      const uint32_t *cand_ids_dev, int32_t nc, float *out_dev);

/*
 * Two-level search with dynamic batching (Algorithm 2, Sec. 4.1-4.2) for nq
 * independent queries, all stages on the device.
 * Per query: EQ (exact queue, size ef) starts with the entry point's exact score.
 * Each hop reads the best unvisited node u of EQ, marks it visited, ADC-scores the
 * neighbours of u that have no ADC score yet and pushes them into AQ, then moves the
 * r = ceil(rerank_ratio * number of those new neighbours) best entries of AQ (fp32
 * product; AQ holds every ADC-scored node not yet recomputed) to the pending list P.
 * When |P| >= batch, or EQ has no unvisited node, the chunks in P are re-embedded,
 * scored by inner product with the query and try-inserted into EQ in P's order
 * (insert when EQ is not full or the score beats EQ's worst entry, which is evicted).
 * The search ends when EQ has no unvisited node and P is empty; the k best of EQ
 * are returned, padded with id -1 / score -inf.
 * A query's result does not depend on nq or on the other queries of the call:
 * the encoder batches across queries, never changing a chunk's embedding.
 *   queries_dev fp32[nq][hidden]; out_ids_dev int64[nq][k]; out_scores_dev fp32[nq][k];
 *   cache: optional stored embeddings (NULL = none; a slot_of entry >= rows -> LEANN_EINVAL);
 *   stats_host: optional totals.
 * Errors: k < 1, k > ef, ef > 1024, rerank_ratio outside (0,1], batch < 1, entry >= n,
 * graph/chunk/PQ sizes that disagree -> LEANN_EINVAL / LEANN_ESHAPE; a neighbour id >= n
 * or a per-query queue overflow -> LEANN_EINVAL / LEANN_ECAPACITY after the run
 * (outputs then undefined).  Synchronises the stream before returning.  Between rounds the calling thread looks at a
 * word of pinned memory: it keeps a core busy for as long as the call takes, as a wait for a stream does by default.
 */
int leann_search(leann_ctx *ctx, const float *queries_dev, int64_t nq, const leann_graph *graph,
                 const leann_pq *pq, const leann_chunks *chunks, const leann_emb_cache *cache, int32_t ef,
                 int32_t k, float rerank_ratio, int32_t batch, int64_t *out_ids_dev, float *out_scores_dev,
                 leann_search_stats *stats_host);

/* leann_search with pending updates (see leann_updates); updates == NULL is leann_search.
 * Errors as leann_search, plus LEANN_EINVAL for a buffer with null pointers or more than
 * 2^24 rows. */
int leann_search_updates(leann_ctx *ctx, const float *queries_dev, int64_t nq, const leann_graph *graph,
                         const leann_pq *pq, const leann_chunks *chunks, const leann_emb_cache *cache,
                         const leann_updates *updates, int32_t ef, int32_t k, float rerank_ratio, int32_t batch,
                         int64_t *out_ids_dev, float *out_scores_dev, leann_search_stats *stats_host);

/*
 * Index graph construction by insertion (Algorithm 3 with the node-insertion listing of
 * the update appendix).  Nodes enter in id order.  For node v: W = best-first search
 * (Algorithm 1, exact similarities <e_v, e_x> from emb, queue length efC, start at node 0)
 * on the graph built so far; neighbours = RNG selection from W (walk by descending
 * similarity, keep x unless a kept y has <e_x, e_y> > <e_x, e_v>), at most M for nodes
 * flagged in is_hub (NULL: every node), m for the others; edges are added in both
 * directions, and a neighbour whose list exceeds M is shrunk to M with the same rule.
 * Total order (similarity descending, id ascending).
 * batch > 1: the nodes of a batch search the graph as it was before the batch (one
 * block each), then their edges are committed in id order and every node that
 * received edges is shrunk once; batch k holds min(batch, max(1, inserted / ramp)) nodes.
 * batch = 1 is the sequential listing.
 *   emb_dev fp32[n][d] (device); is_hub_dev uint8[n] or NULL (device);
 *   row_ptr_dev uint64[n + 1], col_idx_dev uint32 with room for n * M entries (device,
 *   caller-owned); n_edges_host receives the edge count.  Scratch is allocated and freed
 *   inside the call (n * (M + batch) * 4 bytes, and batch * n * 2 when n > 262144).  Synchronises the stream.
 * Errors: efC outside 1..256, M outside 1..64, m outside 1..M, batch outside 1..1024,
 * ramp < 1, n >= 2^31 -> LEANN_EINVAL.
 */
int leann_build_graph(leann_ctx *ctx, const float *emb_dev, int64_t n, int32_t d, const uint8_t *is_hub_dev,
                      int32_t efC, int32_t M, int32_t m, int32_t batch, int32_t ramp, uint64_t *row_ptr_dev,
                      uint32_t *col_idx_dev, int64_t *n_edges_host);

/* Algorithm 3's set V* of highest-degree nodes: is_hub_dev[v] = 1 for the
 * ceil(beta * n) nodes of largest out-degree in the CSR graph (ties: lower id), else 0.
 * Degrees above 4096 -> LEANN_ECAPACITY. */
int leann_top_degree(leann_ctx *ctx, const uint64_t *row_ptr_dev, int64_t n, double beta, uint8_t *is_hub_dev);

/* Tuning knobs (all optional): largest number of tokens one encoder pass holds
 * (workspace size), and the per-query capacity of the approximate queue. */
int leann_set_limits(leann_ctx *ctx, int64_t max_tokens_per_pass, int32_t aq_capacity);
/* Per-call embedding memo (off by default; an option for throughput with many queries per call): with max_rows > 0
 * a leann_search call keeps up to max_rows embeddings that its own encoder passes produced (max_rows * hidden * 4 bytes
 * of device memory plus 4 bytes per node) and serves a later request for the same chunk, by any query of the same call,
 * from there instead of encoding it again.  The memo is empty at the start of every call: nothing computed in one call
 * is reused in another, and nothing is stored with the index.  A chunk's embedding does not depend on its batch, so
 * ids, scores and every per-query count are unchanged; encoded_chunks drops and memo_hits counts the requests served.
 * A memo that fills up holds the first chunks by round, query and pending entry: the counts repeat from call to call.
 * Without it, requests for one chunk are merged only within a round.  max_rows = 0 turns it off and frees its memory. */
int leann_set_call_memo(leann_ctx *ctx, int64_t max_rows);
/* GEMM tile choice of the encoder (a tuning and test aid; results do not depend on it, every tile adds the K-slabs
 * in the same order): large_tile 256 (default) or 128 = largest block tile of the kernel for large passes (0 leaves it);
 * small_rows = passes that are expected to hold at most this many tokens may use tiles of 64x64 and smaller (default
 * 2048); with 0 every pass goes through the kernel for large passes. */
int leann_set_gemm_tiles(leann_ctx *ctx, int32_t large_tile, int32_t small_rows);

/*
 * Per-kernel device timing for the benchmark: between leann_profile_begin and leann_profile_end every kernel
 * the library launches on this context is bracketed by HIP events on the context's stream.  ms[i] / launches[i]
 * give summed duration and launch count per kernel family; tokens = valid tokens that went through the encoder,
 * so that the GEMM work is tokens * layers * 2 * (4*hidden^2 + 2*hidden*ffn) flops.  leann_profile_end
 * synchronises the stream.  TRAVERSE holds the exact scores too, which its kernel takes; SCORE_INSERT has no kernel of its own
 * and stays 0.
 */
enum {
    LEANN_PROF_GEMM_QKV = 0, LEANN_PROF_GEMM_O, LEANN_PROF_GEMM_FFN1, LEANN_PROF_GEMM_FFN2, LEANN_PROF_ATTENTION,
    LEANN_PROF_LAYERNORM, LEANN_PROF_ENC_OTHER, LEANN_PROF_TRAVERSE, LEANN_PROF_COLLECT, LEANN_PROF_SCORE_INSERT,
    LEANN_PROF_LUT, LEANN_PROF_ADC, LEANN_PROF_KINDS
};
typedef struct {
    double ms[LEANN_PROF_KINDS];
    int64_t launches[LEANN_PROF_KINDS];
    int64_t tokens;
} leann_profile;
int leann_profile_begin(leann_ctx *ctx);
int leann_profile_end(leann_ctx *ctx, leann_profile *out_host);

/*
 * Measured denominator for the encoder's roofline (benchmark hook, not on the search path): the rate this GPU
 * sustains on nothing but independent bf16 MFMA 32x32x16 instructions (8 accumulators per wave, the GEMM's wave
 * tile), `launches` launches of blocks_per_cu (1 or 2) blocks of four waves per compute unit, `iters` rounds each.
 * operand_kind: 0 zeros, 1 values near one, 2 random sign / exponent in [2^-4, 2) / mantissa.
 * tflops_host receives TFLOP/s over the timed launches (HIP events on the context's stream, after three warm-up
 * launches), ms_host (optional) the average launch duration.  Allocates and frees its buffers; synchronises.
 */
int leann_bench_mfma(leann_ctx *ctx, int32_t operand_kind, int32_t blocks_per_cu, int32_t iters, int32_t launches,
                     double *tflops_host, double *ms_host);

/*
 * Measured ceiling of the ADC scorer's access pattern (benchmark hook): 67 108 864 gathers per launch of uniformly
 * random 32-byte rows from table_dev (u8[table_rows][32], device, caller-owned), nothing else.  rows_per_s_host
 * receives rows per second over `launches` timed launches after one warm-up launch, ms_host (optional) the average
 * launch duration.  Allocates and frees 0.27 GB of ids; synchronises.
 */
int leann_bench_gather(leann_ctx *ctx, const uint8_t *table_dev, int64_t table_rows, int32_t launches,
                       double *rows_per_s_host, double *ms_host);

/*
 * Measured ceiling of the GEMM's operand feed (benchmark hook): one block of eight waves per compute unit does nothing
 * but the GEMM's operand loads (16 bytes per lane, 64-byte row pieces of 1536-byte rows, eight in flight per lane) over
 * a panel of panel_rows rows allocated inside the call: a panel of a few MB is served by the L2, a large one by memory.
 * bytes_per_s_host receives the rate over `launches` timed launches after one warm-up launch.  Synchronises.
 */
int leann_bench_l1pull(leann_ctx *ctx, int64_t panel_rows, int32_t launches, double *bytes_per_s_host, double *ms_host);

/*
 * Operators for adapting an encoder to a collection: dropout, LayerNorm with its gradient, and projections with low-rank
 * adapters.  They need a context for its device, stream and workspaces only (an encoder of no layers is enough).  What
 * holds for all of them:
 *   - Matrices are rows of unit stride, `ld` elements apart (ld >= the row's length; rows need no alignment unless a call
 *     says so).  Element offsets are 64-bit.
 *   - Everything is enqueued on the context's stream and nothing synchronises, except that a workspace which has to grow is
 *     allocated in the call; a buffer that another stream writes or reads has to be ordered with it by the caller.
 *   - The workspace stays with the context, as large as the largest call needed.  For every 16 of max_rank a projection takes 64 bytes per row and 64 n_out per adapter that has
 *     rows; its gradient 128 per row and, per adapter, 64 n_in + 32 n_out and 64 (n_in + n_out) for each of its chunks of up to 2048 rows.  It is freed when another
 *     allocation of the context finds no memory, and by leann_destroy.
 *   - Calls may be captured into a graph once a call of that size has made the workspace large enough.  The context keeps what a capture met, also when a later call needs
 *     more, until leann_destroy; handles have to live as long.  Graphs and calls of a context share a workspace: they run one after another, in the order of its stream.
 *   - Sums and statistics are fp32; every output is rounded once, to nearest.  No atomics: the bits repeat from call to call.
 *   - Zero rows are no error.  leann_profile_begin does not bracket their kernels.
 */

/* Dropout: element (row, col) of a matrix is dropped where 16 bits, a function of seed, offset, row and col, are below
 * rint(p * 65536); what stays is multiplied by 65536 / (65536 - rint(p * 65536)).  The bits are halves of the words of
 * Philox4x32-10 under the key `seed` (low word first) and the counter (col / 8, row, offset low, offset high): half
 * number col % 8, the low half of a word first.  No mask is stored: the gradient takes the same seed and offset. */
typedef struct {
    float p; /* in [0, 1] */
    uint64_t seed, offset;
} leann_dropout_desc;

/* out = dropout(x) (+ residual, NULL for none); the gradient with respect to x is the same call on the gradient of out,
 * without a residual.  Dropped infinities and NaN are 0.  x, residual and out have the type `dtype` (LEANN_F32, LEANN_BF16 or
 * LEANN_F16); out may be x or residual itself.
 * Errors: p outside [0, 1], null pointers, negative row count -> LEANN_EINVAL; ld < cols, 2^31 rows or columns -> LEANN_ESHAPE. */
int leann_dropout(leann_ctx *ctx, const void *x_dev, int64_t ldx, const void *residual_dev, int64_t ldr, int64_t rows, int64_t cols, int dtype,
                  const leann_dropout_desc *drop, void *out_dev, int64_t ldo);

/* t = dropout(x) (+ residual); out = (t - mean(t)) / sqrt(var(t) + eps) * gamma + beta over each row, biased variance.
 * drop and residual may be NULL.  For a backward pass total_dev (may be NULL) receives t rounded to dtype, mean_dev and
 * rstd_dev (both or neither; fp32[rows]) the statistics, taken before that rounding.  gamma, beta: fp32[cols].  out may be x or residual
 * itself, total may be the other one.
 * Errors: as leann_dropout; eps not positive -> LEANN_EINVAL; more than 8192 columns -> LEANN_ESHAPE. */
int leann_layernorm(leann_ctx *ctx, const void *x_dev, int64_t ldx, const void *residual_dev, int64_t ldr, int64_t rows, int32_t cols, int dtype,
                    const leann_dropout_desc *drop, const float *gamma_dev, const float *beta_dev, float eps, void *out_dev, int64_t ldo,
                    void *total_dev, int64_t ldt, float *mean_dev, float *rstd_dev);

/* Gradients of leann_layernorm from dout, the gradient of out.  total is t (x itself where there was neither dropout nor a
 * residual).  dtotal (NULL for none) is what reaches t besides, where t is used elsewhere, too (pre-LN blocks).
 *   dresidual = gradient of t, which is the residual's; dx = dropout's gradient of it (drop as in the forward call; without
 *   dropout dx is dresidual and dx_dev is not used); dgamma, dbeta: fp32[cols], the sums over the rows (written, not added to).
 * dresidual and dx may be dout or dtotal itself.  Errors: as leann_layernorm. */
int leann_layernorm_backward(leann_ctx *ctx, const void *dout_dev, int64_t ldd, const void *total_dev, int64_t ldt, int64_t rows, int32_t cols,
                             int dtype, const float *gamma_dev, const float *mean_dev, const float *rstd_dev, const void *dtotal_dev, int64_t lde,
                             const leann_dropout_desc *drop, void *dresidual_dev, int64_t ldr, void *dx_dev, int64_t ldx, float *dgamma_dev,
                             float *dbeta_dev);

/* Projections with low-rank adapters: out_t = W x_t + bias + scale_a up_a (down_a x_t), where a is the adapter of the request that
 * row t belongs to: many requests, each with its own adapter or none, in one call beside the weight that all of them share.
 * The adapters lie in two pools, down[n_adapters][max_rank][n_in] and up[n_adapters][n_out][max_rank], of which adapter a uses the
 * first rank[a] ranks; what the pools hold beyond may be anything.  Activations, W and pools have one type, LEANN_BF16 or LEANN_F16, and
 * 16-byte alignment (rows: a multiple of 8 elements apart).  What would take more than 2^24 - 1 workgroups in a launch is refused before the first one (LEANN_ESHAPE):
 * many rows with W wide or n_in below 256 (n_out, for dx) go in tiles of 64 x 64, one each; the gradients take one for 32 ranks and 32 columns of n_out of every adapter. */

/* The shared weight W[n_out][n_in] (rows without gaps) and bias fp32[n_out] (NULL for none), copied in the order that the kernels read; with_gradient: a
 * second time, transposed, for leann_adapter_project_backward's dx.  W stays as it is for the handle's life (adapters are
 * what is trained).  n_out and n_in: multiples of 8 up to 65536, else LEANN_ESHAPE.  Synchronises the stream. */
int leann_projection_create(leann_ctx *ctx, const void *w_dev, const float *bias_dev, int32_t n_out, int32_t n_in, int dtype, int with_gradient,
                            leann_projection **out);
void leann_projection_free(leann_projection *proj);

/* The rows of a batch: request i has the next rows_of_request[i] rows (0 is allowed) and adapter adapter_of_request[i], -1 for none.  rank[a] in
 * [0, max_rank] and scale[a], finite, of the n_adapters (1 to 65535) adapters; max_rank: the pools' room, a multiple of 8 from 8 to 128.  Host arrays,
 * copied.  One handle serves every projection that the batch goes through.  Synchronises the stream: some 30 us for a few dozen requests, 100 for 512 of 83 229 rows.
 * Errors: a negative row count, adapter, rank or scale outside what is said here -> LEANN_EINVAL; 2^31 - 256 rows or more, max_rank,
 * n_adapters -> LEANN_ESHAPE. */
int leann_adapter_rows_create(leann_ctx *ctx, const int32_t *rows_of_request_host, const int32_t *adapter_of_request_host, int32_t n_requests,
                              const int32_t *rank_host, const float *scale_host, int32_t n_adapters, int32_t max_rank, leann_adapter_rows **out);
void leann_adapter_rows_free(leann_adapter_rows *rows);

/* The forward pass over x[T][n_in], T the rows of the handle.  low_dev (NULL, or fp32[T][max_rank]) receives down_a x_t, which the backward pass
 * needs; zeros beyond the adapter's rank and for rows without one.  out must not overlap x (LEANN_EINVAL; their rows may lie between each other's).
 * A row's values do not depend on other rows; its bits may depend on their number and adapters, as products of different sizes add up in different orders. */
int leann_adapter_project(leann_ctx *ctx, const leann_projection *proj, const leann_adapter_rows *rows, const void *x_dev, int64_t ldx,
                          const void *down_dev, const void *up_dev, void *out_dev, int64_t ldo, float *low_dev);

/* Gradients from dout[T][n_out]: dx[T][n_in] = W^T dout + scale_a down_a^T (up_a^T dout) (NULL: not wanted; else the projection needs with_gradient), and
 * ddown[n_adapters][max_rank][n_in], dup[n_adapters][n_out][max_rank] in fp32 (both or neither; written, not added to; zeros for adapters without
 * rows and beyond their rank), which need x and the forward pass's low.  dx must not overlap dout or x (LEANN_EINVAL). */
int leann_adapter_project_backward(leann_ctx *ctx, const leann_projection *proj, const leann_adapter_rows *rows, const void *dout_dev, int64_t ldd,
                                   const void *x_dev, int64_t ldx, const float *low_dev, const void *down_dev, const void *up_dev, void *dx_dev,
                                   int64_t lddx, float *ddown_dev, float *dup_dev);

/*
 * Attention over ragged sequences.  Sequence s has the next q_rows[s] rows of q and the next k_rows[s] rows of k and v; its query i stands at position p = first[s] + i, its keys
 * at 0, 1, ...  Head h has the columns [h dim, (h + 1) dim) of q, and of k and v those of key head h / (heads / kv_heads).
 *   visible: j <= p + right and (j >= p - left or j < sinks); left or right -1: no limit to that side
 *   s_ij = scale q_i . k_j + bias[bucket_of[clamp(j - p, -distance, distance) + distance]][h]  (without buckets: no bias)
 *   lse_i = log sum over visible j of exp s_ij,  out_i = sum over visible j of exp(s_ij - lse_i) v_j;  where nothing is visible out_i is 0 and lse_i -inf
 * The scale's magnitude lies between 2^-20 and 2^20; a finite bias beyond 2^100 counts as 2^100.
 * Sums, maxima and scores are fp32; weights exp(s - max), and in gradients exp(s - lse) and the scores' gradients, are rounded to the inputs' type where they enter a product of
 * matrices.  What a query does not see does not reach it, be it infinite or NaN.  Rows and columns behind the last sequence and head are neither read nor written.
 */
typedef struct {
    int32_t heads, kv_heads, dim;     /* heads: a multiple of kv_heads, at most 1024; dim: a multiple of 8 up to 128 */
    int32_t left, right, sinks;
    int32_t buckets, distance;        /* 0, 0 without a bias; buckets up to 4096, distance up to 1024 */
    const int32_t *bucket_of_host;    /* [2 distance + 1], copied; NULL without a bias */
} leann_attention_desc;

/* The bucket of each relative position (key minus query) from -distance to distance.  Of the buckets of a direction the first half hold one distance each, the others ranges that
 * grow by equal factors up to `distance`, which belongs to the last one.  both: half of the buckets (an even number) to each direction, the upper half for keys ahead; else keys
 * ahead count as distance 0.  Any other table may be given instead.  distance above half of a direction's buckets, up to 1024, else LEANN_EINVAL. */
int leann_position_buckets(int32_t buckets, int32_t distance, int both, int32_t *bucket_of_host);

/* The sequences of a batch, one plan for the layers and directions that it goes through.  k_rows_host NULL: as q_rows (self-attention); first_host NULL: 0.  Host arrays, copied;
 * lengths of 0 are allowed.  Synchronises the stream, so not while it is captured.  Errors: negative lengths or positions, windows below -1, buckets outside the table -> LEANN_EINVAL; sizes beyond those above,
 * positions of 2^30, 2^31 - 256 rows, 2^24 workgroups of 256 -> LEANN_ESHAPE. */
int leann_attention_create(leann_ctx *ctx, const int32_t *q_rows_host, const int32_t *k_rows_host, const int32_t *first_host, int32_t n_sequences,
                           const leann_attention_desc *desc, leann_attention_plan **out);
void leann_attention_free(leann_attention_plan *plan);

/* out[Tq][heads * dim] from q[Tq][heads * dim], k and v[Tk][kv_heads * dim]: bf16 or f16, 16-byte alignment, rows a multiple of 8 elements apart and at most 2^22 (slices of one
 * projection's output are fine).  bias: fp32[buckets][heads].  lse (NULL, or fp32[heads][Tq]): what the backward pass needs.  out must not overlap q, k or v (LEANN_EINVAL).
 * Where there are few queries, their keys are split over blocks whose sums are joined: a row's bits may depend on the other sequences' lengths, not on what they hold.
 * Workspace: where keys are split (a plan with fewer blocks than two per compute unit), 32 or 128 rows of 34, 66 or 130 floats per part and head. */
int leann_attention(leann_ctx *ctx, const leann_attention_plan *plan, const void *q_dev, int64_t ldq, const void *k_dev, int64_t ldk, const void *v_dev, int64_t ldv, int dtype,
                    float scale, const float *bias_dev, void *out_dev, int64_t ldo, float *lse_dev);

/* Gradients from dout, the gradient of out, and what the forward call left in out and lse, under the same scale and bias: dq[Tq][heads * dim], dk and dv[Tk][kv_heads * dim] (the sums
 * over the heads that share a key head), dbias fp32[buckets][heads] (NULL: not wanted).  Written, not added to; dq, dk and dv may be slices of one matrix, and must not overlap
 * each other or an input (LEANN_EINVAL).  No atomics in memory: the bits repeat; a sequence's dq, dk and dv may differ in bits with the other sequences' lengths, not with what they hold.
 * A query or key that is infinite or NaN makes NaN of the gradients of the keys or queries that it meets and of no others.
 * exp(s - lse) is off by up to 2^-22 |lse| of itself; from |lse| = 2^21 on, as of a row that biases of -1e9 or fp32's lowest hide altogether, a row counts as one that sees nothing.
 * Workspace: 8 bytes per query and head; with dbias 4 (2 distance + 1) more per head and 128 queries (of every sequence), distance no more than the sequences' longest;
 * where keys have their queries split (a few that all of a long sequence see), 256 * 32, 64 or 128 floats per part and key head. */
int leann_attention_backward(leann_ctx *ctx, const leann_attention_plan *plan, const void *dout_dev, int64_t ldd, const void *q_dev, int64_t ldq, const void *k_dev, int64_t ldk,
                             const void *v_dev, int64_t ldv, const void *out_dev, int64_t ldo, const float *lse_dev, int dtype, float scale, const float *bias_dev, void *dq_dev,
                             int64_t lddq, void *dk_dev, int64_t lddk, void *dv_dev, int64_t lddv, float *dbias_dev);

/*
 * Activations kept in 8 bits between the forward and the backward pass.  Of each row's 128 columns (the last ones of a row may be fewer) a = max |x|, scale = a / 127 (fp32) and
 * code = 127 x / a to the nearest whole number, ties to even; a checkpoint stands for code * scale, off by at most half a scale.  codes: int8 rows ldc bytes apart, scales:
 * fp32[rows][ceil(cols / 128)].  128 columns with an infinity or NaN come back as NaN, all of them.  x and outputs are LEANN_F32, LEANN_BF16 or LEANN_F16; what an fp16 output cannot
 * hold becomes infinite.  Errors: as leann_dropout; 2^32 - 2^24 times 128 columns or more in all rows -> LEANN_ESHAPE.
 */
int leann_checkpoint(leann_ctx *ctx, const void *x_dev, int64_t ldx, int64_t rows, int64_t cols, int dtype, int8_t *codes_dev, int64_t ldc, float *scales_dev);
/* out = code * scale, rounded to dtype, any of the three: what a backward pass that needs x (leann_layernorm_backward, leann_adapter_project_backward, leann_attention_backward) is given. */
int leann_checkpoint_restore(leann_ctx *ctx, const int8_t *codes_dev, int64_t ldc, const float *scales_dev, int64_t rows, int64_t cols, int dtype, void *out_dev, int64_t ldo);

/* out = x Phi(x): LEANN_GELU with the normal distribution function, LEANN_GELU_TANH with (1 + tanh(sqrt(2 / pi) (x + 0.044715 x^3))) / 2 for it.  out may be x itself.
 * Phi is off by up to 1e-7, which is more and more of itself where it is small: 0.005 % at x = -3, 0.16 % at -5, 0.4 % at -6, 3 % at -12.
 * codes and scales (both or neither) receive x as a checkpoint. */
enum { LEANN_GELU = 0, LEANN_GELU_TANH = 1 };
int leann_activation(leann_ctx *ctx, const void *x_dev, int64_t ldx, int64_t rows, int64_t cols, int dtype, int kind, void *out_dev, int64_t ldo, int8_t *codes_dev, int64_t ldc,
                     float *scales_dev);
/* dx = dout times the activation's derivative at x, which is given as it was (x) or as a checkpoint (codes, scales); again (NULL for none) receives the activation of that x, which
 * the gradient of a projection behind it needs and which then need not be kept.  dx may be dout or x itself; again must not be dout, dx or x. */
int leann_activation_backward(leann_ctx *ctx, const void *dout_dev, int64_t ldd, const void *x_dev, int64_t ldx, const int8_t *codes_dev, int64_t ldc, const float *scales_dev,
                              int64_t rows, int64_t cols, int dtype, int kind, void *dx_dev, int64_t lddx, void *again_dev, int64_t lda);

#ifdef __cplusplus
}
#endif
#endif /* LEANN_H */
