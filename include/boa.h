/*
 * boa.h — C ABI of the MI355X (gfx950) filtered beam search with online
 * beamwidth adaptation ("BOA: Beamwidth Online Adaptation for
 * Filtered-ANNS on a GPU").
 *
 * Problem (Sec. II, Def. 1 and Def. 2): each base point carries a vector
 * and m numeric attributes; a query carries a vector and one inclusive
 * range [lo, hi] per attribute (Eq. 2). The answer is the k points nearest
 * to the query vector (Euclidean) among those satisfying every range.
 *
 * Method: every query is searched first at a narrow beamwidth L0; queries
 * whose result fails the confidence test (Eq. 3) are compacted on the
 * device and searched again, from scratch, at the next wider width
 * (Alg. 1); each search is the filter-aware beam search of Alg. 2 with
 * exact squared-L2 distances. BOA+ (Sec. III-A "Pipelining Multiple
 * Batches") issues the first phase as sub-batches on one stream while the
 * pooled survivors are escalated on a second stream.
 *
 * Conventions for every entry point:
 *   - Return value: BOA_OK (0) or a negative BOA_E* code; no C++ exception
 *     crosses this boundary and the library never aborts. On a non-zero
 *     return, boa_last_error() describes the failure (thread-local string).
 *   - Validation happens before any device work: on BOA_EINVAL the output
 *     buffers are untouched.
 *   - Attribute and range cells are 4 bytes: int32 for BOA_ATTR_I32
 *     columns, the IEEE bit pattern of a float32 for BOA_ATTR_F32 columns.
 *   - Distances are squared Euclidean distances in float32 (exact integers
 *     for uint8 data). float32 distances use one fixed summation order:
 *     16 partial sums, chunk c = dims 4c..4c+3 accumulated into partial
 *     c mod 16 by fused multiply-add of the float32 difference, chunks in
 *     increasing order, then the partials summed pairwise (p += p+8, +4,
 *     +2, +1).
 *   - Search ordering is lexicographic on (number of violated predicates,
 *     distance, id): the filter penalty of Alg. 2 taken larger than any
 *     distance, ties broken by id.
 *   - Not thread-safe per index: one boa_search at a time per boa_index.
 */
#ifndef BOA_H
#define BOA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct boa_index boa_index; /* opaque; owns all of its device memory */

enum {
    BOA_OK = 0,
    BOA_EINVAL = -1,       /* invalid argument */
    BOA_ENOMEM = -2,       /* host or device allocation failed */
    BOA_EHIP = -3,         /* HIP runtime error */
    BOA_EUNSUPPORTED = -4, /* valid but not supported by this build */
    BOA_EOVERFLOW = -5     /* a per-query visited table overflowed (results invalid) */
};

enum { BOA_VEC_F32 = 0, BOA_VEC_U8 = 1 };
enum { BOA_ATTR_I32 = 0, BOA_ATTR_F32 = 1 };

#define BOA_MAX_M 8          /* attributes per point */
#define BOA_MAX_R 64         /* graph out-degree */
#define BOA_MAX_L 2048       /* beamwidth */
#define BOA_MAX_PHASES 32
#define BOA_MAX_N ((int64_t)1 << 24) /* ids are packed into 24 bits */
#define BOA_MAX_BUILD_N ((int64_t)2 << 20) /* graph construction inside the library */

/*
 * Build an index from host arrays (copied into device memory; the caller
 * may free its arrays on return).
 *   vectors     host, row-major n x d; float32 (BOA_VEC_F32) or uint8 (BOA_VEC_U8).
 *               d % 4 == 0 (float32) or d % 16 == 0 (uint8); d <= 1024.
 *   attrs       host, row-major n x m 4-byte cells; 1 <= m <= BOA_MAX_M.
 *   attr_dtypes host, m entries of BOA_ATTR_I32 / BOA_ATTR_F32.
 *   adjacency   host, row-major n x R uint32 neighbour ids, padded with
 *               0xFFFFFFFF; 1 <= R <= BOA_MAX_R. A row may not hold its own
 *               id, nor any id twice.
 *               NULL: the library builds the graph (Sec. II "Graph
 *               construction"; boa_build_params): DiskANN alpha-pruning of
 *               each point's min(2R, 128) exact nearest neighbours, then of
 *               its forward and reverse neighbours; attribute-aware edges
 *               from JAG-style threshold passes (R >= 8); every row leaves
 *               one slot free, and every point is made reachable from the
 *               entry point through an in-edge from its nearest reachable
 *               candidate. Needs n <= BOA_MAX_BUILD_N (the candidates come
 *               from brute-force scans), else BOA_EUNSUPPORTED.
 *   R           the row width, 1 <= R <= BOA_MAX_R: one neighbour per lane of
 *               a 64-wide wavefront.
 *   entry       the entry point s of every search (Alg. 2), 0 <= entry < n;
 *               -1: the medoid, the point nearest (float64) to the float64
 *               centroid of the vectors, ties to the lowest id (point 0 where
 *               the vectors hold a NaN, which no distance compares with).
 *   n           1 <= n < BOA_MAX_N.
 *   out         receives the index; free it with boa_free_index.
 * Errors: BOA_EINVAL (bad sizes, null pointers, out-of-range ids in the
 * adjacency), BOA_EUNSUPPORTED, BOA_ENOMEM, BOA_EHIP.
 */
int boa_build_index_from_arrays(const void *vectors, int64_t n, int32_t d, int32_t vec_dtype,
                                const int32_t *attrs, int32_t m, const int32_t *attr_dtypes,
                                const uint32_t *adjacency, int32_t R, int64_t entry,
                                boa_index **out);

/* Graph construction parameters (used when adjacency is NULL). */
typedef struct {
    double alpha;        /* pruning slack of DiskANN's dominance rule: v is dropped
                            when a kept w has alpha * d(w, v) <= d(u, v) (Euclidean);
                            1 <= alpha <= 4; default 1.2 */
    int32_t attr_levels; /* attribute-aware passes (JAG threshold pruning, Sec. II
                            "Graph construction"), 0..4; default 4. Level l keeps, for
                            each point, R/8 alpha-pruned nearest vectors among the
                            points whose attribute distance (the largest gap of
                            per-column quantile ranks) is within the point's
                            0.1% / 1% / 5% / 20% quantile of that distance to an evenly
                            spaced sample of 4096 points. The vector-distance pass
                            keeps the rest of the row but one slot. Needs R >= 8. */
} boa_build_params;

void boa_default_build_params(boa_build_params *bp);

/* boa_build_index_from_arrays with explicit graph construction parameters
 * (bp must not be NULL). */
int boa_build_index_ex(const void *vectors, int64_t n, int32_t d, int32_t vec_dtype, const int32_t *attrs,
                       int32_t m, const int32_t *attr_dtypes, const uint32_t *adjacency, int32_t R,
                       int64_t entry, const boa_build_params *bp, boa_index **out);

/* Search parameters (Alg. 1 inputs). boa_default_params fills the defaults. */
typedef struct {
    int32_t k;              /* neighbours returned; 1 <= k <= L of the first phase */
    int32_t L0;             /* first-phase beamwidth (L_min of Alg. 1) */
    int32_t Lmax;           /* widest beamwidth; the phase at Lmax is the last */
    double alpha;           /* growth factor > 1: L <- min(ceil(alpha * L), Lmax); default 2 */
    double eps;             /* confidence threshold of Eq. 3; default 0.05 */
    double tau;             /* residual fraction: a phase runs while more than tau*nq
                               queries are active; 0 <= tau < 1; default 0 */
    int32_t fixed_L;        /* > 0: a single non-adaptive phase at this width (the
                               fixed-beamwidth baseline); overrides L0/Lmax/schedule */
    int32_t boa_plus;       /* 1: BOA+ sub-batched first phase overlapped with escalation */
    int32_t sub_batches;    /* BOA+ first-phase sub-batches; default 10 */
    int32_t lds_hash_slots; /* 0: automatic; else a power of two in [64, 16384] that forces
                               the 16-bit slots of the per-wave LDS visited table (tests
                               force spills to the HBM bitmap); at least 8 * 2^(B-15)
                               for ids of B bits */
    const int32_t *schedule; /* optional host array of explicit phase widths
                                (strictly increasing); overrides L0/Lmax/alpha */
    int32_t n_schedule;
    int32_t fused;          /* 1: run every phase in one persistent launch, each wave
                               carrying its query from width to width without waiting
                               for the other queries (identical results, since every
                               phase restarts the search; needs tau == 0). 2: split:
                               the first phase in one launch, then (after compaction
                               and a 4-byte read of the survivor count) every later
                               phase in one persistent launch over the survivors, whose
                               waves get the largest visited table that still lets all
                               survivors run at once (identical results; needs
                               tau == 0). 0: one launch per phase with device-side
                               compaction between them. Where all queries are resident
                               at once as teams (escalation_waves), 0 (with tau * nq
                               below 1) and 2 run every phase in one launch as 1 does,
                               unless lds_hash_slots forces a table. */
    int32_t warm_start;     /* 1: warm-start escalation (Sec. III-A "Redundancy
                               Avoidance"): during a phase of width L the sorted list
                               keeps up to the next phase's width, only its first L
                               entries are expanded and read by the result and Eq. 3,
                               and an escalated query continues from that list and its
                               visited set instead of restarting at the entry point.
                               The first phase is unchanged; later phases differ from a
                               restart. Runs in the fused mode only (fused = 1, so
                               tau == 0), else BOA_EUNSUPPORTED. 0: every phase restarts. */
    int32_t pq;             /* 1: traverse with product-quantised distances (Alg. 2 "PQDist",
                               the index needs boa_set_pq), then at each phase's end
                               re-rank the phase's valid worklist entries by exact
                               distance (Sec. III-B step 8); the result and Eq. 3 read
                               the re-ranked entries. k <= 128. 0: exact distances. */
    int32_t escalation_waves; /* 0 (default): a team of waves per query, with exact and with
                               product-quantised distances, in launches of as few queries
                               as are then resident at once (256 to 1,536): one owns the
                               worklist and the visited set, the others expand the nodes
                               next in order ahead of their turn (identical results);
                               1: one wave per query everywhere. */
} boa_params;

void boa_default_params(boa_params *p);

/*
 * Batched adaptive filtered search.
 *   queries   DEVICE, nq x d, same element type as the index vectors.
 *   ranges    DEVICE, nq x m x 2 cells [lo, hi] (inclusive), per-column type;
 *             an unconstrained attribute is [INT32_MIN, INT32_MAX] or [-inf, +inf].
 *   nq        >= 0 (0 is a no-op).
 *   ids       DEVICE, nq x k uint32: ids of the valid points found, nearest first;
 *             0xFFFFFFFF where fewer than k valid points were found.
 *   dists     DEVICE, nq x k float32 squared distances (+inf in padded slots).
 *   final_L   DEVICE, nq int32: beamwidth of the phase that produced the result.
 *   expansions, scored  DEVICE nq uint32 each, or NULL: per query, nodes expanded
 *             and nodes scored, summed over the phases the query ran in.
 *   stream    hipStream_t of the caller (NULL = default stream). Device buffers
 *             must be valid on it. The call returns after the results are
 *             complete (it synchronises the stream once at the end).
 * Errors: BOA_EINVAL, BOA_EUNSUPPORTED, BOA_ENOMEM, BOA_EHIP, BOA_EOVERFLOW.
 */
int boa_search(boa_index *idx, const void *queries, const int32_t *ranges, int64_t nq,
               const boa_params *p, uint32_t *ids, float *dists, int32_t *final_L,
               uint32_t *expansions, uint32_t *scored, void *stream);

/*
 * Allocation-free variant of boa_search, for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc). Same arguments, results and error codes
 * as boa_search; it calls no hipMalloc, hipFree or other allocating routine.
 *   - Its work memory (active lists, counters, confidence flags, the visited
 *     spill bitmaps) lives in one file-scope device array of
 *     BOA_NOALLOC_SCRATCH_MB MiB per GPU, held by the library until the
 *     process ends. Every call on a GPU shares that GPU's array: calls that
 *     overlap on one GPU (other streams, other threads) race and must be
 *     serialised by the caller. What must start at zero is cleared by a fill
 *     kernel at the start of each call.
 *   - nq <= BOA_NOALLOC_MAX_NQ, else BOA_EINVAL before any device work.
 *   - BOA+ (boa_plus = 1) returns BOA_EUNSUPPORTED (it needs a second
 *     stream). The other modes run; where the spill bitmaps of the planned
 *     grid (n/8 bytes per resident wave) do not fit the array, the
 *     persistent grid is made smaller (same results, less parallelism), and
 *     an index whose single block does not fit returns BOA_EUNSUPPORTED.
 *   - It keeps no statistics: boa_get_stats afterwards reports no search.
 * It synchronises `stream` before returning, like boa_search.
 */
#define BOA_NOALLOC_SCRATCH_MB 64
#define BOA_NOALLOC_MAX_NQ (1 << 18)
int boa_search_noalloc(boa_index *idx, const void *queries, const int32_t *ranges, int64_t nq,
                       const boa_params *p, uint32_t *ids, float *dists, int32_t *final_L,
                       uint32_t *expansions, uint32_t *scored, void *stream);

/* Statistics of the last boa_search on this index, one row per phase. */
typedef struct {
    int32_t L;              /* phase beamwidth */
    int32_t active;         /* queries searched in the phase */
    int32_t confident;      /* of which resolved by the confidence test */
    int32_t launches;       /* search kernels launched for the phase (BOA+: one per sub-batch;
                               a later phase whose number of queries is known on the device
                               only takes two, one for few queries and one for many, of which
                               one returns at once); where modes 0 and 2 run in one launch:
                               1 for every phase that had queries */
    int64_t expansions;     /* nodes expanded, summed over the phase's queries */
    int64_t scored;         /* nodes scored (distance + predicates) */
    double gathered_bytes;  /* algorithmic bytes the phase had to read */
    float kernel_ms;        /* device time of the launches that start at the phase: a launch
                               that covers several phases (fused, split, BOA+, and modes 0
                               and 2 where they run in one launch) counts under the first */
} boa_phase_stats;

typedef struct {
    int32_t n_phases;
    int32_t waves_per_block, blocks; /* shape of the first search launch (a team of waves per
                                        query: its waves, and a block per query) */
    int32_t lds_hash_slots;          /* its LDS visited table (0: a bitmap over all ids) */
    int64_t spilled_queries;         /* query-phases whose visited set left LDS */
    float total_ms;                  /* device time of the whole search */
    /* accumulated since boa_reset_counters: searches, search-kernel launches,
       and their summed device time (HIP events around every launch) */
    int64_t cum_searches, cum_launches;
    double cum_kernel_ms;
    boa_phase_stats phase[BOA_MAX_PHASES];
    /* accumulated like cum_*, split by the phase a launch starts at (a launch
       of all phases counts under 0, a split search's second launch under 1) */
    int64_t cum_phase_launches[BOA_MAX_PHASES];
    double cum_phase_kernel_ms[BOA_MAX_PHASES];
} boa_stats;

/* Statistics of the last search (per phase) plus the accumulated counters.
 * Copies per-query counters back from the device: call it outside timed code. */
int boa_get_stats(const boa_index *idx, boa_stats *out);

/* Zero the accumulated counters of boa_stats. */
int boa_reset_counters(boa_index *idx);

/*
 * Product-quantisation data of an index (Alg. 2 "PQDist"; Sec. III-B), copied
 * to the device (the caller may free its arrays on return).
 *   codebook  HOST, M x 16 x (d / M) float32: 16 centroids per subspace of
 *             d / M consecutive dimensions.
 *   codes     HOST, n x M / 2 bytes: byte b holds the centroid of subspace 2b
 *             in its low nibble and of subspace 2b + 1 in its high nibble.
 *   M         even, <= 256, dividing d.
 * The per-query distance table entry (m, c) is the float32 fused
 * multiply-add chain over the subspace's dimensions of (q - centroid)^2; the
 * asymmetric distance adds a point's table entries in 16 partial sums
 * (subspace m into partial m mod 16, increasing m) summed pairwise.
 * Errors: BOA_EINVAL, BOA_ENOMEM, BOA_EHIP. */
int boa_set_pq(boa_index *idx, const float *codebook, const uint8_t *codes, int32_t M);

/* The graph and entry point an index searches (e.g. the ones the library
 * built). adjacency: HOST n x R uint32, or NULL; entry: the entry point s,
 * or NULL; repaired: in-edges the library's construction added to reach
 * every point (-1 when the caller passed the adjacency), or NULL. */
int boa_get_graph(const boa_index *idx, uint32_t *adjacency, int64_t *entry, int64_t *repaired);

void boa_free_index(boa_index *idx);

const char *boa_last_error(void);

/*
 * Operators of a query tower: what turns an encoder's output into query
 * vectors, fits them to the points of an index, and serves them.
 *
 * Conventions, beside those above:
 *   - Every pointer is DEVICE memory. Matrices are row-major with the last
 *     dimension contiguous; strides are in elements, from row to row.
 *   - Calls are asynchronous on `stream`: they return once the kernels are
 *     queued, allocate nothing and can be captured into a graph. Work memory
 *     is the caller's (16-byte aligned, at least as large as the matching
 *     _workspace function says) and must not serve two calls at once.
 *   - Sums, statistics and logits are float32 whatever the element type, and
 *     results are rounded to it once; what is rounded before (the cross
 *     entropy's probabilities in bfloat16) is named below. Nothing is added in
 *     an order that depends on the schedule: the same inputs give the same bits.
 */
enum { BOA_T_F32 = 0, BOA_T_BF16 = 1, BOA_T_F16 = 2 };

#define BOA_MAX_NORM_D (1 << 20)
/*
 * Layer norm of `rows` rows of d values: y = (x - mean) * rstd * weight + bias,
 * rstd = 1 / sqrt(mean((x - mean)^2) + eps). weight and bias may be NULL (1, 0);
 * param_dtype is theirs, dtype or BOA_T_F32. y is dense (rows x d, dtype). mean
 * and rstd (float32, one per row) are what the backward pass needs, or NULL.
 * Errors: BOA_EINVAL, BOA_EHIP. */
int boa_layer_norm(const void *x, int64_t rows, int32_t d, int64_t x_stride, int32_t dtype, const void *weight,
                   const void *bias, int32_t param_dtype, float eps, void *y, float *mean, float *rstd, void *stream);

/* Work memory of boa_layer_norm_backward in bytes. */
int64_t boa_layer_norm_backward_workspace(int64_t rows, int32_t d);

/* Gradients of boa_layer_norm: dx (rows x d, dtype), dweight and dbias (d,
 * param_dtype; zeros without rows). Each may be NULL; the workspace is needed
 * for dweight or dbias only. */
int boa_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, int64_t rows, int32_t d,
                            int32_t dtype, const void *weight, int32_t param_dtype, const float *mean,
                            const float *rstd, void *dx, void *dweight, void *dbias, void *workspace,
                            int64_t workspace_bytes, void *stream);

#define BOA_MAX_XENT_D 4096
#define BOA_MAX_XENT_B (1 << 21)
enum { BOA_REDUCE_NONE = 0, BOA_REDUCE_SUM = 1, BOA_REDUCE_MEAN = 2 };
/*
 * Softmax cross entropy of B queries over V points as classes:
 *   logit[b][v] = scale * (h[b] . points[v]) + bias[v]
 *   loss[b] = log(sum_v exp(logit[b][v])) - logit[b][labels[b]]
 * The logits are formed in tiles and never stored. The gradients are sums of
 * probability times point or query: in bfloat16 each probability is rounded to
 * bfloat16 as the operand of such a product (in float32 it keeps its 24 bits).
 * The label's own entry, probability - 1, stays float32 in both and keeps its
 * digits next to 0. dbias adds unrounded probabilities.
 */
typedef struct {
    int32_t dtype;          /* of h, points, dh and dpoints: BOA_T_F32 or BOA_T_BF16 */
    int32_t d;              /* 1 .. BOA_MAX_XENT_D */
    int64_t B, V;           /* queries, 0 .. BOA_MAX_XENT_B; points, 1 .. 2^31 - 2^16 */
    const void *h;          /* B x d */
    int64_t h_stride;
    const void *points;     /* V x d */
    int64_t points_stride;
    const int64_t *labels;  /* B: the point each query belongs to. A negative label leaves its
                               query out (loss 0, gradients 0, not counted by the mean); one of V
                               or more gives loss NaN and gradients 0 */
    const float *bias;      /* V, or NULL. -inf leaves a point out (its values have to be finite
                               all the same: a NaN or infinity times its probability of 0 is NaN);
                               with every point left out a query's loss is +inf and its gradients
                               are 0. For squared L2 in place of the inner product: scale = 2 t,
                               bias[v] = -t |points[v]|^2 */
    float scale;
    int32_t reduction;      /* of the loss. BOA_REDUCE_MEAN divides by the queries not left out
                               (0 where there is none) */
    float *loss;            /* B floats (BOA_REDUCE_NONE) or one */
    float *lse;             /* B: log of the sum of exponentials, or NULL */
    /* gradients (boa_softmax_xent_grad only) */
    const float *dloss;     /* gradient of `loss`, shaped like it; NULL: 1 */
    void *dh;               /* B x d, dense, or NULL */
    void *dpoints;          /* V x d, dense, or NULL */
    float *dbias;           /* V, or NULL */
} boa_xent;

/* Work memory in bytes of one call with these arguments (grad: of
 * boa_softmax_xent_grad); a negative BOA_E* code for invalid sizes. It holds a
 * copy of points that are not read in place: bfloat16 rows that are not 16-byte
 * aligned or no multiple of 16 wide (all of them up to 128 values a row; wider
 * ones up to 2 GB at a time), and float32 rows of more than 128 values with more
 * than 32 queries (6 bytes a value, up to 2 GB at a time). */
int64_t boa_softmax_xent_workspace(const boa_xent *x, int32_t grad);

/* The losses. Errors: BOA_EINVAL, BOA_EUNSUPPORTED (float16: probabilities of
 * many points fall below its range), BOA_EHIP. */
int boa_softmax_xent(const boa_xent *x, void *workspace, int64_t workspace_bytes, void *stream);

/* The losses and their gradients in one call. */
int boa_softmax_xent_grad(const boa_xent *x, void *workspace, int64_t workspace_bytes, void *stream);

#define BOA_MAX_MATVEC_M 65535
#define BOA_MAX_MATVEC_K (1 << 20)
/*
 * Products of M vectors of K values with rows of 4-bit codes:
 *   y[m][n] = sum_k x[m][k] * w[n][k],
 *   w[n][k] = scales[n][k / group] * q + offsets[n][k / group],
 * or scales * (q - 8) where offsets is NULL. codes: rows x (K + 1) / 2 bytes,
 * byte j holds the code of k = 2j in its low nibble and of 2j + 1 in its high
 * nibble (as in boa_set_pq), codes_stride bytes from row to row. scales and
 * offsets share scale_dtype and scale_stride. x and y have `dtype`, any of the
 * three. A non-finite x makes its vector's results NaN or infinite.
 * Errors: BOA_EINVAL, BOA_EHIP. */
int boa_matvec_fourbit(const void *x, int64_t M, int64_t x_stride, int32_t dtype, const uint8_t *codes, int64_t rows,
                       int32_t K, int64_t codes_stride, const void *scales, const void *offsets, int64_t scale_stride,
                       int32_t scale_dtype, int32_t group, void *y, int64_t y_stride, void *stream);

#define BOA_MAX_LINEAR (1 << 17)
#define BOA_MAX_LINEAR_ROWS 2147483392   /* 2^31 - 256 */
#define BOA_LINEAR_FEW 16   /* rows up to which a forward pass takes no work memory */
enum { BOA_ACT_NONE = 0, BOA_ACT_RELU = 1, BOA_ACT_SILU = 2, BOA_ACT_GELU = 3, BOA_ACT_GELU_TANH = 4 };
/*
 * A linear layer on M rows, with what follows it:
 *   z = x w^T + bias        y = act(z) + residual
 * act: max(z, 0); silu z / (1 + e^-z); gelu z (1 + erf(z / sqrt 2)) / 2;
 * gelu_tanh z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2. And its gradients:
 *   dz = dy act'(z)    dx = dz w    dw = dz^T x    dbias = sum over rows of dz
 * (the residual's is dy). x, w, residual, y and their gradients have one type.
 * Sums are float32. In bfloat16 and float16, z is kept in float16, infinite beyond
 * its range (where every act' is constant) and with an absolute error of 2^-25
 * below 2^-14 (relu: z above 0 stays above 0, so that its slope is 1), and dz is
 * rounded to the layer's type as an operand of the two products, not in dbias
 * (float16's is infinite beyond its range, and its steps are 2^-24 below 2^-14). In
 * float32, with more than 16 to 128 rows (by N and K) and in the gradients, the
 * products' operands are rounded to 22 bits (values far below the largest of their
 * row, or of their column where the sum runs over rows, to 2^-40 of that). A
 * non-finite value makes the results that it takes part in NaN or infinite.
 */
typedef struct {
    int32_t dtype;          /* any of the three */
    int32_t activation;     /* BOA_ACT_* */
    int64_t M;              /* 0 .. BOA_MAX_LINEAR_ROWS */
    int32_t N, K;           /* 1 .. BOA_MAX_LINEAR */
    const void *x;          /* M x K */
    int64_t x_stride;
    const void *w;          /* N x K */
    int64_t w_stride;
    const void *bias;       /* N, or NULL */
    int32_t param_dtype;    /* of bias and dbias: dtype or BOA_T_F32 */
    const void *residual;   /* M x N, or NULL */
    int64_t residual_stride;
    void *y;                /* M x N, dense */
    void *pre;              /* z for the backward pass: M x N, dense, float16 (float32 where dtype is);
                               NULL: not kept. The gradients read it unless the activation is BOA_ACT_NONE */
    /* gradients (boa_linear_grad only); bias, residual and y are not read */
    const void *dy;         /* M x N */
    int64_t dy_stride;
    void *dx;               /* M x K, dense, or NULL */
    void *dw;               /* N x K, dense, or NULL */
    void *dbias;            /* N, or NULL */
} boa_dense;

/* Work memory in bytes of one call with these arguments (grad: of
 * boa_linear_grad); a negative BOA_E* code for invalid ones. It holds copies of
 * operands that cannot be read in place (16-bit rows that are not 16-byte
 * aligned or no multiple of 8 wide, float32 rows as parts), dz, and the shares
 * of sums that are split. */
int64_t boa_linear_workspace(const boa_dense *d, int32_t grad);

/* The layer. Errors: BOA_EINVAL, BOA_EHIP. */
int boa_linear(const boa_dense *d, void *workspace, int64_t workspace_bytes, void *stream);

/* Its gradients. */
int boa_linear_grad(const boa_dense *d, void *workspace, int64_t workspace_bytes, void *stream);

enum { BOA_NORM_LAYER = 0, BOA_NORM_RMS = 1 };
/*
 * What stands between two blocks of a residual tower, on rows of d values: the
 * norm after a block (post), its gate, the residual sum, and the norm before the
 * next block (pre).
 *   u = post ? norm(f) * post_weight + post_bias : f
 *   h = scale * x + gate * u
 *   y = norm(h) * weight + bias
 * norm(v) = (v - mean(v)) / sqrt(mean((v - mean(v))^2) + eps), or without the
 * means (BOA_NORM_RMS). y is formed from h before h is rounded. Any of gate and
 * the parameters may be NULL (ones, zeros).
 */
typedef struct {
    int32_t dtype;          /* of x, f, h, y, their gradients, and a gate per value */
    int32_t param_dtype;    /* of the parameters, their gradients, and a shared gate: dtype or BOA_T_F32 */
    int64_t rows;           /* 0 .. 2^31 - 1 */
    int32_t d;              /* 1 .. BOA_MAX_NORM_D */
    int32_t norm;           /* BOA_NORM_* */
    int32_t post, pre;      /* whether there is the first norm, and the second (without it no y) */
    int32_t gate_rows;      /* 0: gate holds d values for all rows; 1: rows x d */
    float scale, eps;
    const void *x;          /* rows x d: the residual stream */
    int64_t x_stride;
    const void *f;          /* rows x d: the block's output */
    int64_t f_stride;
    const void *gate;
    int64_t gate_stride;    /* of a gate per value */
    const void *post_weight, *post_bias, *weight, *bias;   /* d each */
    void *h, *y;            /* rows x d, dense */
    float *stats;           /* 4 x rows, for the backward pass, or NULL: mean and 1 / deviation of f's
                               rows (where post), then of h's (where pre) */
    /* gradients (boa_block_norm_backward only, which reads h again from x and f;
       y and h are not read, eps neither) */
    const void *dh;         /* rows x d, or NULL (zeros) */
    int64_t dh_stride;
    const void *dy;         /* rows x d, or NULL (nothing comes back through the second norm, whatever h is) */
    int64_t dy_stride;
    void *dx, *df;          /* rows x d, dense, or NULL */
    void *dgate;            /* like gate (dense), or NULL */
    void *dpost_weight, *dpost_bias, *dweight, *dbias;   /* d each, or NULL; zeros without rows */
    void *workspace;        /* where sums over rows are wanted (the last five, but for a gate per value) */
    int64_t workspace_bytes;
} boa_block;

/* Errors of both: BOA_EINVAL, BOA_EHIP. */
int boa_block_norm(const boa_block *b, void *stream);

/* Work memory of boa_block_norm_backward in bytes. */
int64_t boa_block_norm_backward_workspace(int64_t rows, int32_t d);

int boa_block_norm_backward(const boa_block *b, void *stream);

#define BOA_MAX_ORTH (1 << 14)
#define BOA_MAX_ORTH_COUNT 65535
#define BOA_MAX_ORTH_STEPS 32
/*
 * Orthogonalises updates of weight matrices (rows x cols each) by Newton-Schulz
 * products: X = G / (|G| + eps), |G| the root of G's sum of squares, then
 *   X <- a X + (b X X^T + c (X X^T)^2) X
 * for each step's a, b, c: every singular value s of X becomes a s + b s^3 +
 * c s^5, the singular vectors stay. A zero update stays zero. X is held in
 * float32, and the results are rounded once; the products' operands are rounded to
 * f16's 11 bits for bfloat16 updates whose rows and cols are 128 or more, to 22 bits
 * for others (f16's smallest value ends that at 2^-33 where singular values stay
 * around 1), and not at all for the smallest, which a CU's LDS holds: up to 16, 32, 48
 * or 64 rows (or cols) of up to 2,048, 1,024, 672 or 480 values. A value that is
 * not finite makes its matrix NaN, and so may steps that let singular values grow
 * beyond 2^23.
 */
typedef struct {
    int32_t dtype;              /* of update and out: any of the three */
    int32_t rows, cols;         /* 1 .. BOA_MAX_ORTH */
    int64_t count;              /* matrices, 0 .. BOA_MAX_ORTH_COUNT */
    const void *update;
    int64_t update_stride, update_batch;   /* from row to row, from matrix to matrix */
    int32_t steps;              /* 1 .. BOA_MAX_ORTH_STEPS */
    const float *coefficients;  /* HOST, 3 per step; read before the call returns */
    float eps;
    void *out;                  /* count x rows x cols, dense */
} boa_orth;

/* Work memory of one call in bytes (none for the smallest); a negative BOA_E* code for invalid arguments. */
int64_t boa_orthogonalize_workspace(const boa_orth *d);

/* Errors: BOA_EINVAL, BOA_EHIP. */
int boa_orthogonalize(const boa_orth *d, void *workspace, int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* BOA_H */
