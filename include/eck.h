/*
 * eck.h -- C ABI of libeck: batched energy-cost-model evaluation for
 * search-based kernel compilation (arXiv 2411.18873), native to MI355X (gfx950).
 *
 * The paper's search round (Alg. 1) is: reproduce a generation of candidate
 * kernels, keep the low-latency ones, pick among them those of least predicted
 * energy with a learned cost model, measure the picked ones, refit the model,
 * and adapt how many to measure next.  This library runs the data-parallel
 * part of that round on one GPU for millions of candidates at once:
 *
 *   candidate_enumerate -> features_compute -> costmodel_score (energy model,
 *   latency model) -> topk_select            [+ costmodel_update when measured
 *   energies arrive]
 *
 * Conventions
 *   - Plain C, every function returns int32_t: ECK_OK or a negative ECK_E*.
 *   - All arguments are validated on the host before anything is launched; an
 *     error return means nothing was enqueued and no output was touched.
 *   - "device" pointers are HIP device memory owned by the caller (the library
 *     never frees or keeps them); "host" pointers are ordinary memory.
 *   - Kernels are enqueued on `stream` (a hipStream_t passed as void*; NULL is
 *     the default stream).  No call synchronises unless its comment says so.
 *   - Results that depend on device data (count, snr, loss) are written to
 *     device memory, never returned through the host.
 *   - Matrices over candidates are structure-of-arrays: row r of a [R][ld]
 *     array is at base + r*ld elements, candidate i at column i, ld >= n.
 *   - There is no CPU fallback: without a usable GPU the compute calls return
 *     ECK_EDEVICE.
 *   - Handles (eck_space, eck_model, eck_trees) belong to the device that was
 *     current when they were created and are not synchronised internally: a
 *     space uploads its tables on first use, models change under update calls.
 *     Calls on one handle from several host threads must be serialised by the
 *     caller; different handles are independent.
 */
#ifndef ECK_H
#define ECK_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ECK_OK 0
#define ECK_EINVAL (-1)       /* null pointer, zero size, value out of range */
#define ECK_ESHAPE (-2)       /* sizes inconsistent with each other (ld < n, k > segment, widths) */
#define ECK_EUNSUPPORTED (-3) /* valid request this build has no kernel for */
#define ECK_EALIGN (-4)       /* pointer or leading dimension not aligned as required */
#define ECK_EWORKSPACE (-5)   /* workspace missing or too small */
#define ECK_EDEVICE (-6)      /* HIP runtime error (no device, allocation or launch failure) */

/* operator kinds */
#define ECK_OP_GEMM 0   /* dim = {1, M, N, K} */
#define ECK_OP_BGEMM 1  /* dim = {B, M, N, K} */
#define ECK_OP_CONV2D 2 /* dim = {N, C, K, H, W, R, S, stride | pad << 16} (NCHW, square stride/pad) */

/* schedule-space kinds */
#define ECK_SPACE_KNOB 0  /* genes: tile_M, tile_N in {16..256}, tile_K in {8..64}, threads in {64..512},
                             unroll in {1,2,4,8}, vec in {1,2,4,8}; GEMM/BGEMM only */
#define ECK_SPACE_SPLIT 1 /* one gene per split axis (index into the table of ordered 4-way factorisations of
                             the axis extent, lexicographic), then unroll in {1,2,4,8,16}, vec in {1,2,4,8}.
                             Axis order: GEMM (M,N,K); BGEMM (B,M,N,K); CONV2D (N,K,H_out,W_out,C).
                             The reduction axis is staged through shared memory: f0 = stage loop,
                             f1*f2*f3 = elements per stage */
#define ECK_SPACE_SPLIT_XRED 2 /* the same genes and tables as SPLIT, read as a schedule that splits the
                             reduction across threads (the shape reduction-dominated operators need, such as
                             the matrix-vector products of Sec. 7.2): reduction axis f0 = stage loop,
                             f1 = threads sharing one output's reduction, f2*f3 = serial per thread; no
                             staging, every thread loads its own slice; the f1 partial sums of an output are
                             folded by a halving tree in shared memory (fp32).  Same 64 feature slots */

/* enumeration modes */
#define ECK_MODE_EXHAUSTIVE 0
#define ECK_MODE_SAMPLE 1
#define ECK_MODE_MUTATE 2
#define ECK_MODE_CROSSOVER 3

/* element types of feature matrices and models */
#define ECK_F32 0
#define ECK_BF16 1

/* selection modes */
#define ECK_SELECT_THRESHOLD 0
#define ECK_SELECT_RANK 1

#define ECK_MAX_GENES 16
#define ECK_MAX_K 4096 /* largest k topk_select accepts */
#define ECK_MAX_BATCH 128 /* most spaces one *_batch call takes */

/* The tensor operator being compiled plus the parameters of the GPU the
 * candidate kernels are meant for (they enter the occupancy features; the
 * paper's case study, Sec. 8, reasons with the number of multiprocessors). */
typedef struct {
    int32_t op;
    int32_t dim[8];
    int32_t elem_bytes; /* 2 or 4 */
    int32_t hw_num_cu, hw_wave, hw_lds_bytes, hw_max_threads_cu, hw_max_blocks_cu;
} eck_problem;

typedef struct eck_space eck_space; /* schedule space of one problem (host tables + device copy) */
typedef struct eck_model eck_model; /* cost model: fp32 master weights, Adam moments, packed bf16 weights */

/* ------------------------------------------------------------------ spaces */

/* Build the schedule space of `problem` (Sec. 2.2: the hierarchical search
 * space of an auto-scheduler; Sec. 5.3: kernels represented through loops).
 * Host-only work; the device copy of the tables is made lazily by the first
 * call that launches a kernel.  Every axis extent must be in [1, 65535], every
 * factorisation table at most 65535 entries, and 2*outputs*reduction < 2^48.
 * Errors: ECK_EINVAL (null, bad op/kind/elem_bytes/hw fields, zero extents),
 * ECK_EUNSUPPORTED (KNOB space on a convolution, limits above exceeded). */
int32_t eck_space_create(const eck_problem *problem, int32_t kind, eck_space **out);

/* Makes the device copy of the space's parameters and tables now, on the
 * current device, instead of inside the first call that launches a kernel: one
 * hipMalloc and one synchronous host-to-device copy (at most a few hundred KB).
 * For callers that must not allocate or synchronise later on -- code under HIP
 * graph capture, timed loops.  Does nothing when the copy exists already.
 * Errors: ECK_EINVAL (null), ECK_EDEVICE. */
int32_t eck_space_upload(eck_space *space);

/* Frees host tables and the device copy (synchronises the device first). NULL is ignored. */
void eck_space_destroy(eck_space *space);

/* n_genes, the radix of every gene (radix[ECK_MAX_GENES], unused entries 0)
 * and the size of the space (0 when it does not fit 64 bits).  Host only. */
int32_t eck_space_info(const eck_space *space, int32_t *n_genes, uint32_t *radix, uint64_t *size);

/* Copies the factorisation table of split gene `gene` to `out` (host,
 * [capacity][4] uint32); returns the number of entries, or a negative error.
 * out == NULL just returns the count.  Host only. */
int32_t eck_space_table(const eck_space *space, int32_t gene, uint32_t *out, uint32_t capacity);

/* -------------------------------------------------------------- candidates */

/* Generate the genes of candidates first_index .. first_index+n-1
 * (Sec. 6.4: the search starts from many randomly generated kernels; Alg. 1:
 * the reproduction step of the genetic search).
 *   EXHAUSTIVE: candidate index -> genes by mixed radix, first gene most
 *               significant; first_index+n must not exceed the space size.
 *   SAMPLE:     gene g of candidate c = (low32(u) * radix_g) >> 32 with
 *               u = output number 16*c+g+1 of a SplitMix64 generator whose
 *               state starts at mix(seed + gamma*(round+1)).
 *   MUTATE:     child c copies parent (c mod n_parents); gene g is redrawn as
 *               in SAMPLE when high32(u) < p_mut_q32 (probability p*2^32).
 *   CROSSOVER:  two parents: (c mod n_parents) and one drawn uniformly with
 *               word 14 of the child ((low32(u14) * n_parents) >> 32); gene g
 *               comes from the second parent when bit g of word 15 is set;
 *               then every gene mutates as in MUTATE.  (Alg. 1 names the
 *               reproduction step without fixing its operators.)
 * genes_out: device, uint16 [n_genes][ld].  parents: device, uint16
 * [n_genes][n_parents] (MUTATE and CROSSOVER, else NULL).
 * Errors: EINVAL (nulls, n == 0, bad mode, index range), ESHAPE (ld < n),
 * EALIGN (genes_out not 4-byte aligned or ld odd). */
int32_t candidate_enumerate(const eck_space *space, int32_t mode, uint64_t seed, uint32_t round,
                            uint64_t first_index, uint64_t n, const uint16_t *parents, uint32_t n_parents,
                            uint32_t p_mut_q32, uint16_t *genes_out, uint64_t ld, void *stream);

/* candidate_enumerate for several spaces in one launch (many operator
 * shapes searched side by side; Sec. 7.1 lists the shapes the paper evaluates).  Space s
 * draws from stream (seeds[s], round) and writes its n_per_space candidates to
 * columns [s*n_per_space, (s+1)*n_per_space) of genes_out; in MUTATE its
 * parents are columns [s*n_parents_per_space, ...) of parents, uint16
 * [n_genes][n_spaces*n_parents_per_space].  Every space must have the same
 * kind, operator class and number of genes (ESHAPE otherwise).
 * spaces, seeds: host arrays of n_spaces entries, 1 <= n_spaces <=
 * ECK_MAX_BATCH (EUNSUPPORTED above).  ld >= n_spaces*n_per_space.
 * Other arguments and errors as candidate_enumerate. */
int32_t candidate_enumerate_batch(const eck_space *const *spaces, uint32_t n_spaces, int32_t mode,
                                  const uint64_t *seeds, uint32_t round, uint64_t first_index, uint64_t n_per_space,
                                  const uint16_t *parents, uint32_t n_parents_per_space, uint32_t p_mut_q32,
                                  uint16_t *genes_out, uint64_t ld, void *stream);

/* Collect the genes of selected candidates, e.g. the survivors topk_select
 * returned, as the parents of the next generation (Alg. 1: the kernels picked
 * at the end of a round reproduce the next one):
 *   out[g][j] = genes[g][idx[j]]  for j < k.
 * An index of 0xFFFFFFFF (padding of a short selection) copies candidate
 * idx[0] instead, so the output is always a valid parent set; if idx[0] is
 * padding too the column is zero.  genes: device uint16 [n_genes][ld]; idx:
 * device uint32 [k], every valid entry below n; out: device uint16 [n_genes][ld_out].
 * Errors: EINVAL (nulls, k == 0, n_genes outside 1..ECK_MAX_GENES), ESHAPE (ld_out < k). */
int32_t eck_candidates_gather(const uint16_t *genes, uint64_t ld, uint64_t n, int32_t n_genes, const uint32_t *idx,
                              uint32_t k, uint16_t *out, uint64_t ld_out, void *stream);

/* Duplicate removal before scoring (a generation bred from few parents
 * repeats itself; Alg. 1's reproduction step): candidate i is a first
 * occurrence when no candidate of lower index has the same genes.
 *   overwrite != 0: flags[i] = first occurrence ? 1 : 0
 *   overwrite == 0: flags[i] = flags[i] && first occurrence   (e.g. the legal
 *                   flags of features_compute, so that duplicates drop out of
 *                   topk_select)
 * genes: device uint16 [n_genes][ld]; flags: device uint8 [n]; ws: device, at
 * least a hash table of candidate indices (4 bytes for each of the next power of
 * two at or above 2n slots), 4-byte aligned; the query says what is fastest, which
 * is more for 16384 to 2^20 candidates, and wants 16-byte alignment.  The result does not depend on execution order.
 * Errors: EINVAL, ESHAPE (ld < n), EUNSUPPORTED (n > 2^30), EWORKSPACE, EALIGN. */
uint64_t eck_candidates_dedup_workspace_bytes(uint64_t n);
int32_t eck_candidates_dedup(const uint16_t *genes, uint64_t ld, uint64_t n, int32_t n_genes, uint8_t *flags,
                             int32_t overwrite, void *ws, uint64_t ws_bytes, void *stream);

/* ---------------------------------------------------------------- features */

/* High-level kernel features of each candidate, computed analytically from
 * its loop structure (Sec. 5.3; Sec. 5.4: numbers of floating-point and
 * integer operations, vectorisation-, loop- and cache-access features; the
 * grid / block / global-load / shared-store counts are those of Table 5).
 * Feature f of candidate i is the 64-bit integer raw[f][i]; the model input is
 * its fixed-point log2: with v = raw+1 (saturating), e = floor(log2 v) and m =
 * the 10 bits below v's leading one, feat = e + m/1024 (exact in fp32; rounded
 * to nearest-even for bf16).  n_feat = 32 gives features 0..31, 64 all.
 *   genes:     device, uint16 [n_genes][ld] (values >= radix are clamped to radix-1)
 *   feat_out:  device, [n_feat][ld] of out_dtype (ECK_F32 or ECK_BF16); may be NULL
 *   raw_out:   device, uint64 [n_feat][ld] or NULL
 *   legal_out: device, uint8 [n] or NULL; 1 when the schedule can be launched
 *              (32 <= threads <= 1024, staged bytes -- in a SPLIT_XRED space the
 *              partial sums -- fit the LDS, vector width <= 16 bytes and
 *              divides the contiguous per-thread extent)
 * Errors: EINVAL, ESHAPE (ld < n), EUNSUPPORTED (n_feat not 32/64), EALIGN
 * (ld not a multiple of 2). */
int32_t features_compute(const eck_space *space, const uint16_t *genes, uint64_t ld, uint64_t n,
                         int32_t n_feat, int32_t out_dtype, void *feat_out, uint64_t *raw_out,
                         uint8_t *legal_out, void *stream);

/* features_compute for several spaces in one launch: columns
 * [s*n_per_space, (s+1)*n_per_space) of genes, feat_out, raw_out and legal_out
 * belong to spaces[s].  Same restrictions on the batch as
 * candidate_enumerate_batch; ld >= n_spaces*n_per_space. */
int32_t features_compute_batch(const eck_space *const *spaces, uint32_t n_spaces, const uint16_t *genes,
                               uint64_t ld, uint64_t n_per_space, int32_t n_feat, int32_t out_dtype,
                               void *feat_out, uint64_t *raw_out, uint8_t *legal_out, void *stream);

/* ------------------------------------------------------------------ models */

/* A multilayer perceptron widths[0] -> ... -> widths[n_layers] with ReLU
 * between layers and a linear scalar output: the cost model of Sec. 5.4 in the
 * form the workloads prescribe (the paper's own model is a tree ensemble).
 * dtype ECK_F32: fp32 weights and arithmetic.  ECK_BF16: bf16 weights and
 * bf16 first-hidden activations on the matrix cores, fp32 accumulation.
 * Supported: n_layers == 3, widths[3] == 1, widths[0] in {32, 64}, hidden widths
 * at most 512; a BF16 model must be one of the shapes the matrix-core kernels
 * are built for: 64-512-512-1, 64-256-256-1, 64-128-128-1, 32-64-64-1
 * (ECK_EUNSUPPORTED otherwise, here rather than at the first score call).
 * Allocates device memory (parameters, Adam moments, packed weights). */
int32_t eck_model_create(int32_t n_layers, const int32_t *widths, int32_t dtype, eck_model **out);
void eck_model_destroy(eck_model *model);

/* Number of parameters P: sum over layers of fan_in*fan_out + fan_out. Host only. */
int32_t eck_model_param_count(int32_t n_layers, const int32_t *widths, uint64_t *out);

/* State blob (device, fp32): [theta(P) | m(P) | v(P) | t] with theta = per
 * layer W[fan_in][fan_out] row-major then b[fan_out]; m, v Adam moments, t the
 * step count.  set_state accepts n_floats == P (moments and t reset to zero)
 * or 3P+1; get_state needs 3P+1.  The blob is the checkpoint format. */
int32_t eck_model_set_state(eck_model *model, const float *blob, uint64_t n_floats, void *stream);
int32_t eck_model_get_state(const eck_model *model, float *blob, uint64_t n_floats, void *stream);

/* ------------------------------------------------------------------- score */

/* Predicted score of every candidate (Alg. 1: LatencyEvaAndPick /
 * EnergyModelEvaAndPick evaluate the generation with a model; Sec. 5.4: the
 * model outputs a normalised energy score, lower is better).
 *   feat: device [widths[0]][ld] of feat_dtype; score_out: device float [n].
 * A BF16 model takes BF16 or F32 features (F32 is rounded to bf16 on load); an
 * F32 model takes F32 features.  ws/ws_bytes are reserved (pass NULL, 0).
 * A BF16 model reads two (or four) neighbouring candidates per load: ld must
 * be even and feat aligned to two elements (4 bytes for BF16, 8 for F32
 * features), whatever n is; the four-candidate loads are used only when ld is
 * a multiple of 4 and feat 8-byte aligned.  No load crosses the end of a row.
 * Errors: EINVAL, ESHAPE (ld < n), EUNSUPPORTED (dtype combination), EALIGN. */
int32_t costmodel_score(const eck_model *model, const void *feat, int32_t feat_dtype, uint64_t ld, uint64_t n,
                        float *score_out, void *ws, uint64_t ws_bytes, void *stream);

/* costmodel_score that also reduces the scores it writes: min_key_out[s] =
 * the least score among the legal candidates of segment s (n_segments equal
 * consecutive segments, as in topk_select), as an order-preserving key
 *     key(x) = bits(x) ^ (x < 0 ? 0xFFFFFFFF : 0x80000000)
 * (unsigned comparison of keys = comparison of the floats, -0 < +0), or
 * 0xFFFFFFFF when the segment has no legal candidate with a score that is a
 * number.  Run on the latency model it yields the L_min of every segment
 * (Alg. 1 LatencyEvaAndPick; the latency gate of Sec. 4.3) in the pass that
 * produces the latencies, so that topk_select_known_min need not read them a
 * second time.  legal: device uint8 [n] or NULL (all legal); min_key_out:
 * device uint32 [n_segments], overwritten.  The reduction is part of the
 * scoring kernel (integer atomics: the result does not depend on the order of
 * execution).
 * Errors as costmodel_score; also EINVAL (min_key_out NULL, n_segments 0),
 * ESHAPE (n % n_segments, more than 65535 segments), EALIGN (legal odd). */
int32_t costmodel_score_min(const eck_model *model, const void *feat, int32_t feat_dtype, uint64_t ld, uint64_t n,
                            float *score_out, const uint8_t *legal, uint32_t n_segments, uint32_t *min_key_out,
                            void *stream);

/* ------------------------------------------------------------------ select */

/* Bytes of workspace topk_select needs for these sizes in THRESHOLD mode or
 * without latencies, and in RANK mode with m_latency (which adds the lists of
 * the latency stage).  0 on invalid sizes.  Some of it (about a quarter of a
 * byte per candidate, under a finite alpha) only saves time: calls take a
 * workspace without it, too. */
uint64_t topk_select_workspace_bytes(uint64_t n, uint32_t n_segments, uint32_t k);
uint64_t topk_select_rank_workspace_bytes(uint64_t n, uint32_t n_segments, uint32_t k, uint32_t m_latency);

/* Selection under the paper's objective -- low latency first, then least
 * energy (Sec. 4.3, 4.4; Alg. 1).  The n candidates form n_segments equal
 * consecutive segments (one per operator); each is handled independently.
 *   THRESHOLD: L_min = least latency among legal candidates; tau = L_min +
 *              (alpha-1)*|L_min| (fp32, product and sum rounded separately;
 *              +inf when alpha is +inf); feasible = legal and latency <= tau.
 *   RANK:      feasible = the m_latency legal candidates of least latency
 *              (Alg. 1's "fastest M"), ties to the lower index.  m_latency is
 *              at most ECK_MAX_K unless it covers the whole segment.
 *   latency == NULL: feasible = legal.  legal == NULL: all legal.
 * Output per segment: the k feasible candidates of least energy in ascending
 * order (IEEE total order, ties to the lower index): idx_out uint32 [S][k]
 * (index within the segment, 0xFFFFFFFF padding), energy_out float [S][k]
 * (+inf padding), count_out uint32 [S] = min(k, #feasible).  NaN energies or
 * latencies are never feasible.  All pointers device; ws device, 16-byte aligned.
 * The score arrays are read once (THRESHOLD with a finite alpha reads the
 * latencies once more, for L_min; RANK with a partial gate reads the latencies
 * once and the energies of the gated candidates); the result does not depend on
 * the order of execution.
 * Errors: EINVAL (nulls, n == 0, k == 0, bad mode, alpha < 1 or NaN), ESHAPE
 * (n % n_segments, k > n/n_segments, segment longer than 2^32-2), EUNSUPPORTED
 * (k or a partial m_latency > ECK_MAX_K), EWORKSPACE, EALIGN (ws). */
int32_t topk_select(const float *energy, const float *latency, const uint8_t *legal, uint64_t n,
                    uint32_t n_segments, uint32_t k, int32_t mode, float alpha, uint32_t m_latency,
                    uint32_t *idx_out, float *energy_out, uint32_t *count_out, void *ws, uint64_t ws_bytes,
                    void *stream);

/* topk_select in THRESHOLD mode when the least latency of every segment is
 * already known: latency_min_key = what costmodel_score_min wrote for the
 * latency model with the same legal flags and segments (device uint32
 * [n_segments]).  The score arrays are then read exactly once.  Same result as
 * topk_select(..., ECK_SELECT_THRESHOLD, alpha, ...), same workspace
 * (topk_select_workspace_bytes), same errors; EINVAL also for a NULL latency
 * or latency_min_key. */
int32_t topk_select_known_min(const float *energy, const float *latency, const uint8_t *legal, uint64_t n,
                              uint32_t n_segments, uint32_t k, float alpha, const uint32_t *latency_min_key,
                              uint32_t *idx_out, float *energy_out, uint32_t *count_out, void *ws, uint64_t ws_bytes,
                              void *stream);

/* topk_select for callers that cannot allocate device memory and have no
 * workspace to hand over: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  Same arguments, same result, no ws: the
 * intermediate lists live in an array of ECK_TOPK_STATIC_BYTES that is part of
 * the library's device image (one copy per GPU, held until the process ends).
 * The call allocates and frees nothing; its kernels are those of topk_select.
 * Sizes whose workspace (topk_select_workspace_bytes /
 * topk_select_rank_workspace_bytes, without what only saves time) exceeds
 * ECK_TOPK_STATIC_BYTES are refused
 * with ECK_EWORKSPACE before anything is launched.  All calls on one GPU share
 * the one array: calls that overlap in time on the same GPU (different streams
 * or host threads) race and must be serialised by the caller; calls on
 * different GPUs are independent.  Nothing in the array has to be cleared
 * between calls.  Other errors as topk_select; ECK_EUNSUPPORTED also for a
 * device ordinal of 64 or more. */
#define ECK_TOPK_STATIC_BYTES (8u << 20)
int32_t topk_select_static(const float *energy, const float *latency, const uint8_t *legal, uint64_t n,
                           uint32_t n_segments, uint32_t k, int32_t mode, float alpha, uint32_t m_latency,
                           uint32_t *idx_out, float *energy_out, uint32_t *count_out, void *stream);

/* Selection by drawing: parents of the next generation in proportion to what
 * the model thinks of them, so that a generation keeps its variety (Alg. 1's
 * reproduction step does not say how parents are drawn).  In each of n_segments
 * equal consecutive segments candidate i has the weight
 *   w_i = exp(-(energy_i - least) / temperature),  least: the segment's least
 * energy.  Only legal candidates of finite energy are drawn.  In order of
 * energy, equal ones (-0 = +0) by index, the kept ones are a prefix:
 *   the k least (k = 0: all);  of these the fewest that have the share top_p of
 *   their weight (1: all);  of these the ones with w >= min_p (0: all).
 * temperature 0 keeps the least alone.  Draw d of a segment, with the number
 * u = uniform[segment][d] from [0, 1), takes the first kept candidate, by index,
 * at which the running sum of weights passes u times the sum of all kept ones;
 * past the end (u >= 1) the last one of a weight above 0.  Draws are with
 * replacement; the numbers are the caller's.  Weights, sums and the numbers that
 * are drawn with are fp64, but where a share ends: there weights are rounded down
 * to multiples of 2^-60 (the least energy's is 1), whose sums are exact.
 *   uniform: device float [n_segments][draws]; idx_out: device uint32
 *   [n_segments][draws], index within the segment, 0xFFFFFFFF where a segment has
 *   nothing to draw from; logprob_out: device float [n_segments][draws] or NULL,
 *   log(w / sum of the kept weights), -inf there; count_out: device uint32
 *   [n_segments] or NULL, how many are kept.  legal: device uint8 [n] or NULL.
 *   ws: 256-byte aligned, what the query says, for any k and limits (0: may be
 *   NULL; segments of up to 16384 want none, longer ones 0.7 to 4.3 times the
 *   energies' bytes, the most just above that).
 * The result does not depend on the order of execution.  Of segments longer than
 * 16384 the k least are found fastest for k from 1 to 4096, and slower by far
 * where one candidate lies so far below the others that a 2048th of the range
 * between them holds thousands.
 * Errors: EINVAL (nulls, a zero size, temperature negative or not finite, top_p
 * outside (0, 1], min_p outside [0, 1]), ESHAPE (n % n_segments), EUNSUPPORTED
 * (a segment longer than 2^31, more than 2^20 segments, more than 2^31 draws of
 * a segment), EWORKSPACE, EALIGN. */
uint64_t sample_select_workspace_bytes(uint64_t n, uint32_t n_segments, uint32_t draws);
int32_t sample_select(const float *energy, const uint8_t *legal, uint64_t n, uint32_t n_segments, const float *uniform,
                      uint32_t draws, float temperature, uint32_t k, float top_p, float min_p, uint32_t *idx_out,
                      float *logprob_out, uint32_t *count_out, void *ws, uint64_t ws_bytes, void *stream);

/* ------------------------------------------------------------------ update */

uint64_t costmodel_update_workspace_bytes(const eck_model *model, uint64_t n_pairs, int32_t minibatch);

/* ModelUpdate and SNR of Alg. 1 on a buffer of measured kernels.
 *   labels y = energy_measured / max(energy_measured)   ("normalised", Sec. 5.4)
 *   snr  = sum y^2 / sum (pred - y)^2 with the model as it is on entry
 *   then n_steps of Adam (bias-corrected, no weight decay) on the mean of
 *   Eq. (1), (pred - y)^2 / y, over minibatch s = rows [(s mod nb)*minibatch,
 *   +minibatch), nb = n_pairs / minibatch;  loss = the last step's value.
 * BF16 models run forward/backward on bf16 copies of the fp32 master weights.
 *   feat: device [widths[0]][ld]; energy_measured: device float [n_pairs];
 *   snr_out, loss_out: device float (one each).
 * A non-positive or non-finite measured energy is a data error found on the
 * device: snr = loss = NaN and the model is left unchanged.
 * Errors: EINVAL, ESHAPE (n_pairs % minibatch, ld < n_pairs), EUNSUPPORTED,
 * EWORKSPACE, EALIGN (ws not 256-byte aligned; feat / ld as costmodel_score). */
int32_t costmodel_update(eck_model *model, const void *feat, int32_t feat_dtype, uint64_t ld,
                         const float *energy_measured, uint64_t n_pairs, int32_t n_steps, int32_t minibatch,
                         float lr, float beta1, float beta2, float eps, float *snr_out, float *loss_out,
                         void *ws, uint64_t ws_bytes, void *stream);

/* Library version as major*10000 + minor*100 + patch. */
int32_t eck_version(void);

/* The k controller of Alg. 1 (Sec. 6.4): after a round in which round(k*M)
 * kernels were measured and the model updated, a signal-to-noise ratio of the
 * pre-update predictions below mu raises k by 0.2 (more measurements next
 * round), otherwise k falls by 0.2; k stays in [0, 1].  A round that measured
 * nothing (round(k*M) == 0) has no SNR and leaves k unchanged.  Host only;
 * *k_out receives the next k.  EINVAL: nulls, M < 0, k outside [0, 1], NaN. */
int32_t eck_k_step(double k, double snr, double mu, int64_t M, double *k_out);

/* How many of the M fastest kernels a round measures (Alg. 1: "k*M"): round(k*M),
 * halves up.  0 means the round measures nothing.  Host only.  EINVAL: null,
 * M < 0, k outside [0, 1] or NaN. */
int32_t eck_k_count(double k, int64_t M, int64_t *count_out);

/* ------------------------------------------------- boosted-tree cost model */

/* The cost model in the paper's own form (Sec. 5.4 "Approach"): an ensemble of
 * regression trees built one after another by gradient boosting; the
 * prediction is the base score plus the sum of the trees' outputs.  Trees are
 * complete binary trees of one fixed depth d, stored level by level: node j
 * tests x[feature_j] < threshold_j; true -> node 2j+1, false (also NaN) ->
 * node 2j+2; after d tests the walk stands on node (2^d - 1) + leaf.  A node
 * that does not split has threshold +inf.  Arrays (device, per tree):
 *   node_feat uint8 [2^d - 1], node_thr float [2^d - 1], leaf float [2^d].
 * n_feat in 1..256, depth in 1..ECK_MAX_TREE_DEPTH, capacity = most trees the
 * model can hold (<= 65536).  Allocates device memory for `capacity` trees.
 * Errors: EINVAL, EUNSUPPORTED (limits), EDEVICE. */
typedef struct eck_trees eck_trees;
#define ECK_MAX_TREE_DEPTH 8
int32_t eck_trees_create(int32_t n_feat, int32_t depth, int32_t capacity, float base_score, eck_trees **out);
void eck_trees_destroy(eck_trees *trees);

/* Number of trees the model holds now.  Host only. */
int32_t eck_trees_count(const eck_trees *trees, int32_t *n_trees);

/* Replace / read the ensemble (checkpointing).  The arrays are device memory,
 * [n_trees][...] as above; the copies are enqueued on stream.  A feature index
 * >= n_feat is read as n_feat - 1 when scoring.  ESHAPE: n_trees > capacity. */
int32_t eck_trees_set(eck_trees *trees, int32_t n_trees, const uint8_t *node_feat, const float *node_thr,
                      const float *leaf, void *stream);
int32_t eck_trees_get(const eck_trees *trees, uint8_t *node_feat, float *node_thr, float *leaf, void *stream);

/* score_out[i] = base + sum over trees of the leaf candidate i reaches, added in
 * fp32 in tree order.  feat: device, [n_feat][ld] of feat_dtype (ECK_F32 or
 * ECK_BF16; values are compared exactly, never rounded); score_out: device,
 * float [n].  Errors: EINVAL, ESHAPE (ld < n), EUNSUPPORTED (feature tile does
 * not fit the LDS: n_feat * 1 KB fp32 / 512 B bf16 above ~140 KB). */
int32_t treemodel_score(const eck_trees *trees, const void *feat, int32_t feat_dtype, uint64_t ld, uint64_t n,
                        float *score_out, void *stream);

/* Gradient boosting on the loss of Eq. (1) (Sec. 5.4; Alg. 1 ModelUpdate):
 * appends n_rounds trees fitted to the measured pairs.
 *   labels      y = energy_measured / max(energy_measured) in fp32
 *   prediction  p in fp32: base, then the trees in order
 *   per round   g = 2 (p - y) / y, h = 2 / y (derivatives of Eq. (1) in p),
 *               computed in fp64 and rounded to integers of resolution 2^-20
 *               (|g|, h clamped to 2^20); all sums are exact integer sums
 *   growth      level by level; features are binned into 256 bins of width 1/4
 *               on [0, 64) (the range of the transformed features); a split
 *               "feature f, bins <= b go left" has threshold (b + 1) / 4 and
 *               gain GL^2/(HL+lam) + GR^2/(HR+lam) - G^2/(H+lam), fp64, lam =
 *               lambda * 2^20; both sides non-empty; largest gain > 0 wins, ties
 *               to the lower feature then the lower bin; else no split
 *   leaves      w = -eta * G / (H + lam), fp64 -> fp32; empty leaf 0
 * The result is identical to a sequential evaluation of these steps: nothing
 * depends on the order of execution.
 * snr_out (device float): sum y^2 / sum (p - y)^2 of the ensemble on entry;
 * loss_out (device float): mean Eq. (1) loss after the last round.
 * Any energy <= 0 or not finite: snr = loss = NaN and the appended trees are
 * empty (no split, all leaves 0), so predictions do not change.
 * n_pairs <= 2^20 (EUNSUPPORTED above); ESHAPE: ld < n_pairs or capacity
 * exceeded; EWORKSPACE / EALIGN (256 B) for ws. */
uint64_t treemodel_update_workspace_bytes(const eck_trees *trees, uint64_t n_pairs);
int32_t treemodel_update(eck_trees *trees, const void *feat, int32_t feat_dtype, uint64_t ld,
                         const float *energy_measured, uint64_t n_pairs, int32_t n_rounds, float eta, float lambda,
                         float *snr_out, float *loss_out, void *ws, uint64_t ws_bytes, void *stream);

/* --------------------------------------- operators of gated cost models
 *
 * What a deeper cost model over the same candidates is made of: residual
 * blocks  x <- x + dropout(feedforward(layernorm(x)))  on rows of activations.
 * A matrix of activations is row-major: row i of an [n][ld] array, ld >= width
 * elements apart, is candidate i.  Elements are ECK_F32 or ECK_BF16; sums,
 * statistics and products accumulate in fp32 or more, results are rounded once.
 * Pointers are aligned to their elements, nothing more is asked for (rows that
 * start on 16 bytes are fastest); workspaces start on 256 bytes.  Outputs and
 * workspaces overlap neither each other nor inputs, but for what a call says.
 * Nothing depends on the order of execution: equal calls give equal bits. */

#define ECK_ROWS 0    /* x is an [n][ld] matrix of activations */
#define ECK_COLUMNS 1 /* x is a [width][ld] matrix with a candidate per column, as features_compute writes it */

#define ECK_ACT_SILU 0 /* a(g) = g / (1 + exp(-g)) */
#define ECK_ACT_GELU 1 /* a(g) = g (1 + erf(g / sqrt 2)) / 2 */
#define ECK_ACT_RELU 2 /* a(g) = max(g, 0); derivative 0 at g = 0 */

/* Layer norm of every candidate's `width` values:
 *   mean = sum x / width,  rstd = 1 / sqrt(sum (x - mean)^2 / width + eps),
 *   y = (x - mean) rstd gamma + beta.
 *   x: device, of dtype, in x_order; gamma, beta: device float [width], NULL
 *   reads as ones and zeros; y: device [n][ld_y] of dtype;
 *   mean_out, rstd_out: device float [n], both or neither NULL (what
 *   layernorm_backward wants to know).  In ROWS order y may be x.
 *   Squares of differences from a row's mean have to be in fp32's range, and
 *   with eps = 0 not all of them below it.
 * Errors: EINVAL (x or y NULL, one of mean_out / rstd_out alone, n or width 0,
 * bad x_order or dtype, eps negative or not finite), ESHAPE (ld_x, ld_y too
 * small), EUNSUPPORTED (COLUMNS with width > ECK_MAX_COLUMNS_WIDTH, n > 2^31,
 * width > 2^24), EALIGN. */
#define ECK_MAX_COLUMNS_WIDTH 256
int32_t layernorm_forward(const void *x, int32_t x_order, int32_t dtype, uint64_t ld_x, uint64_t n, uint32_t width,
                          const float *gamma, const float *beta, float eps, void *y, uint64_t ld_y, float *mean_out,
                          float *rstd_out, void *stream);

/* Its backward pass, from dy = dL/dy ([n][ld_dy] of dtype, rows), the x of the
 * forward call and its statistics.  With g = dy gamma and xh = (x - mean) rstd:
 *   dx = rstd (g - mean(g) - xh mean(g xh)),
 *   dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy   (fp32).
 *   dx_out: device, of dtype, in x_order (ld_dx), or NULL (features need none);
 *   dgamma_out, dbeta_out: device float [width], overwritten; both or neither
 *   NULL.  dx_out may be dy or x in ROWS order.  ws may be NULL where dgamma_out is.
 * Errors: EINVAL (nulls; nothing to compute), ESHAPE, EUNSUPPORTED (as
 * layernorm_forward), EWORKSPACE, EALIGN. */
uint64_t layernorm_backward_workspace_bytes(uint64_t n, uint32_t width, int32_t dtype);
int32_t layernorm_backward(const void *x, int32_t x_order, int32_t dtype, uint64_t ld_x, const void *dy, uint64_t ld_dy,
                           uint64_t n, uint32_t width, const float *gamma, const float *mean, const float *rstd,
                           void *dx_out, uint64_t ld_dx, float *dgamma_out, float *dbeta_out, void *ws,
                           uint64_t ws_bytes, void *stream);

/* Dropout from the counter-based generator that draws the candidates' genes:
 * no mask is stored, the same (seed, round, row, column) gives the same one.
 *   out = residual + (dropped ? 0 : x * 2^32 / (2^32 - p_drop_q32))
 * Element (r, c) is dropped iff its 32-bit draw is below p_drop_q32 (the
 * probability times 2^32): the low (even c) or high (odd c) half of output
 * number (first_row + r) * ceil(width / 2) + c / 2 + 1 of a SplitMix64 generator
 * whose state starts at mix(seed + gamma*(round+1)), as in candidate_enumerate.
 * The backward pass is the same call on the gradient, without a residual.
 * A dropped element is 0 whatever x holds there (NaN too).
 *   x, residual (or NULL), out: device, [n][ld] of dtype; out may be x or
 *   residual.  first_row: the number of row 0, for matrices handled in pieces.
 * Errors: EINVAL (x or out NULL, n or width 0, bad dtype), ESHAPE (an ld <
 * width), EUNSUPPORTED (n > 2^31, width > 2^24), EALIGN. */
int32_t dropout_apply(const void *x, int32_t dtype, uint64_t ld_x, uint64_t n, uint32_t width, uint32_t p_drop_q32,
                      uint64_t seed, uint32_t round, uint64_t first_row, const void *residual, uint64_t ld_residual,
                      void *out, uint64_t ld_out, void *stream);

/* A gated feed-forward block:
 *   [g | u] = x W_gate_up,   h = a(g) u,   y = h W_down.
 *   x: device [n][ld_x]; w_gate_up: device [n_in][2*n_hidden] (gate columns,
 *   then up columns), w_down: device [n_hidden][n_out], contiguous ([fan_in]
 *   [fan_out] row-major, as in a model's state); y: device [n][ld_y]; all of
 *   dtype.  act: ECK_ACT_*.  pre_out: device float [n][2*n_hidden], receives
 *   [g | u] for gatedffn_backward, or NULL (narrow blocks of many rows are
 *   fastest then).
 * h is rounded to dtype before the second product.
 * Few rows (up to 16 of fp32, up to 4 of bf16) may be multiplied in fp32
 * instructions; more are on the matrix cores, fp32 ones as sums of six
 * products of bfloat16 parts, as good as fp32 products for magnitudes of
 * 2^-100 to 2^127 (and zeros; an infinite input gives NaN or infinities in
 * its row, smaller numbers lose low bits).  So a row's last bits, and in fp32
 * its range, depend on how many rows go with it.
 * ws: room for h, for shares of sums, and for copies of the operands of an
 * fp32 block or of matrices that do not start on 16 bytes or whose rows are
 * no multiple of eight elements.  The queries say 0 for sizes that are refused.
 * Errors: EINVAL (nulls, a zero size, bad dtype or act), ESHAPE (an ld too
 * small), EUNSUPPORTED (n > 2^31, a width > 2^20, or more than 2^22 tiles of
 * 64 x 64 in a product's result), EWORKSPACE, EALIGN. */
uint64_t gatedffn_forward_workspace_bytes(uint64_t n, uint32_t n_in, uint32_t n_hidden, uint32_t n_out, int32_t dtype);
int32_t gatedffn_forward(const void *x, int32_t dtype, uint64_t ld_x, uint64_t n, uint32_t n_in, uint32_t n_hidden,
                         uint32_t n_out, const void *w_gate_up, const void *w_down, int32_t act, void *y,
                         uint64_t ld_y, float *pre_out, void *ws, uint64_t ws_bytes, void *stream);

/* Its backward pass, from dy = dL/dy ([n][ld_dy]) and the pre of the forward call:
 *   dh = dy W_down^T,  du = dh a(g),  dg = dh u a'(g),
 *   dx = [dg | du] W_gate_up^T,  dW_gate_up = x^T [dg | du],  dW_down = h^T dy.
 * The gradients are of dtype and overwritten; each may be NULL, not all.
 * dg, du and h are rounded to dtype before the products they enter.
 * Errors: as gatedffn_forward. */
uint64_t gatedffn_backward_workspace_bytes(uint64_t n, uint32_t n_in, uint32_t n_hidden, uint32_t n_out, int32_t dtype);
int32_t gatedffn_backward(const void *x, int32_t dtype, uint64_t ld_x, uint64_t n, uint32_t n_in, uint32_t n_hidden,
                          uint32_t n_out, const void *w_gate_up, const void *w_down, int32_t act, const float *pre,
                          const void *dy, uint64_t ld_dy, void *dx_out, uint64_t ld_dx, void *dw_gate_up_out,
                          void *dw_down_out, void *ws, uint64_t ws_bytes, void *stream);

/* --------------------------------------------- scoring in 8-bit integers
 *
 * A matrix of 8-bit integers is row-major like one of activations, [rows][ld],
 * and has a scale for each row (float): element k of row r stands for
 * scale[r] q[r][k].  Rows start on 16 bytes (ld a multiple of 16), and what
 * lies between a row's width and the next multiple of 16 belongs to it:
 * quantise_rows writes zeros there, and product_int8 wants them in x or in w. */

/* Rows in 8-bit integers, each by its largest magnitude m:
 *   scale = m / 127,  q = x (127 / m) rounded to the nearest, halves to even,
 * quotients and product in fp32.  A row whose m is below 2^-100 is all zeros, its
 * scale too; one that holds a NaN or an infinity is zeros with the scale NaN.
 *   x: device, of dtype, in x_order (ECK_COLUMNS: [width][ld_x], a row of the
 *   result per column, as features_compute writes candidates; so the columns
 *   of weights [fan_in][fan_out] become rows); q_out: device [n][ld_q];
 *   scale_out: device float [n].
 * Errors: EINVAL (nulls, a zero size, bad x_order or dtype), ESHAPE (an ld too
 * small), EUNSUPPORTED (n > 2^31, width > 131071), EALIGN (also q_out not on 16
 * bytes, ld_q no multiple of 16). */
int32_t quantise_rows(const void *x, int32_t x_order, int32_t dtype, uint64_t ld_x, uint64_t n, uint32_t width,
                      int8_t *q_out, uint64_t ld_q, float *scale_out, void *stream);

#define ECK_ACT_NONE (-1) /* product_int8: no gate */

/* Products of rows of 8-bit integers, and gates of them:
 *   ECK_ACT_NONE: y[i][c] = ((sum_k x[i][k] w[c][k]) x_scale[i]) w_scale[c]
 *   ECK_ACT_*:    y[i][c] = a(g) u, g so from w's row c, u from row n_out + c
 * (the first product of a gated feed-forward block, gate rows then up rows).
 * Sums are exact, what follows is fp32, y is rounded once.
 *   x: device [n][ld_x], w: device [n_out or 2 n_out][ld_w], int8 matrices of
 *   width n_in; x_scale, w_scale: device float, one for each of their rows;
 *   y: device [n][ld_y] of dtype.  ws: where the query says 0, it may be NULL.
 * Errors: EINVAL (nulls, a zero size, bad act or dtype), ESHAPE (an ld too
 * small), EUNSUPPORTED (n > 2^31, n_in > 131071, n_out > 2^20, an ld of x or w
 * above 2^22, more than 2^22 tiles of 64 x 64 in all products), EWORKSPACE,
 * EALIGN (also x or w not on 16 bytes, their ld no multiple of 16). */
uint64_t product_int8_workspace_bytes(uint64_t n, uint32_t n_in, uint32_t n_out, int32_t act);
int32_t product_int8(const int8_t *x, uint64_t ld_x, const float *x_scale, uint64_t n, uint32_t n_in, uint32_t n_out,
                     const int8_t *w, uint64_t ld_w, const float *w_scale, int32_t act, int32_t dtype, void *y,
                     uint64_t ld_y, void *ws, uint64_t ws_bytes, void *stream);

/* ------------------------------------------- refits of models of many tensors */

/* A parameter tensor with its gradient and Adam's states.  Everything but the
 * struct is device memory; elements are contiguous and aligned to their type.
 * A tensor of no elements is passed over. */
#define ECK_STATE_F32 0  /* m, v: float [n] */
#define ECK_STATE_8BIT 1 /* m, v: uint8 [n], with a power of two for every ECK_STATE_BLOCK elements */
#define ECK_STATE_BLOCK 128
typedef struct {
    float *param;         /* [n], updated */
    const void *grad;     /* [n] of grad_dtype */
    void *m, *v;          /* [n], updated: the gradient's mean and its square's */
    uint8_t *m_scale;     /* 8BIT: [ceil(n / ECK_STATE_BLOCK)], updated; F32: not looked at */
    uint8_t *v_scale;
    void *bf16_out;       /* bf16 [n]: the new parameters, rounded; or NULL */
    uint64_t n;
    int32_t grad_dtype;   /* ECK_F32 or ECK_BF16 */
    float weight_decay;
} eck_parameter;

/* One step of AdamW (decoupled weight decay; of Adam where that is 0) over all
 * tensors, number t = step (the first is 1):
 *   g = s grad,  m <- beta1 m + (1 - beta1) g,  v <- beta2 v + (1 - beta2) g^2,
 *   w <- w (1 - lr decay) - lr / (1 - beta1^t) m / (sqrt(v / (1 - beta2^t)) + eps)
 * in fp32.  step_more: device uint32 or NULL, added to step modulo 2^32 (a
 * captured step that is replayed counts there, or steps that were left out are
 * taken off; where t is 0, the call changes nothing).  grad_scale: device float
 * s or NULL (1), as gradients_norm writes it; where it is not finite, the call
 * changes nothing.
 * 8BIT states: m in the float8 format e4m3, v in e5m2 (all bytes 0: a state of
 * zeros), times 2^(scale - 127) of the block of ECK_STATE_BLOCK elements, which
 * brings its largest finite one into [2^7, 2^8) or [2^14, 2^15) (scales of 27 to
 * 247).  They are rounded up or down to the format's next number by 16-bit
 * draws d: up iff d / 2^16 + (the way to the next lower one, in steps) >= 1; a v
 * that is not 0 does not become 0, what is not finite becomes NaN.  Elements are
 * numbered over the list, every tensor from a multiple of ECK_STATE_BLOCK on;
 * those of 2j and 2j + 1 have the low and the high half of output number j + 1 of
 * a SplitMix64 generator whose state starts at mix(seed + gamma*(t+1)), as in
 * candidate_enumerate: the low half of that m's draw, the high half v's.
 * parameters: host, read during the call.  No tensor that is written may
 * overlap another, or a gradient, unless that is of the same entry and, element
 * for element, the same memory.  A launch takes up to 200 tensors.
 * Errors: EINVAL (nulls, no element at all, a bad dtype or state, lr, eps or a
 * decay negative or not finite, a beta outside [0, 1), step 0 without
 * step_more), EUNSUPPORTED (n > 2^34), EALIGN. */
int32_t adamw_step(const eck_parameter *parameters, uint32_t count, int32_t state, double lr, double beta1, double beta2,
                   double eps, uint32_t step, const uint32_t *step_more, const float *grad_scale, uint64_t seed, void *stream);

/* The norm of all gradients of a list (its grad, grad_dtype and n; nothing else
 * of it is looked at), sqrt(sum g^2), summed in fp64 in a fixed order, and what
 * they are to be multiplied with so that it is max_norm at most:
 *   *norm_out = norm,  *scale_out = min(1, max_norm / norm), NaN where the norm
 *   is not finite (device float; one may be NULL).
 * The query says 0 for lists that are refused.
 * Errors: EINVAL (nulls, no element at all, a bad dtype, max_norm not above 0),
 * EUNSUPPORTED (n > 2^34), EWORKSPACE, EALIGN (ws: 256 bytes). */
uint64_t gradients_norm_workspace_bytes(const eck_parameter *parameters, uint32_t count);
int32_t gradients_norm(const eck_parameter *parameters, uint32_t count, float max_norm, float *norm_out, float *scale_out,
                       void *ws, uint64_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ECK_H */
