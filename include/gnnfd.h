/*
 * gnnfd — feature-decomposed GNN aggregation on one CUDA device (sm_100a).
 *
 * The library computes the Aggregation phase of message-passing GNN inference
 * (Algorithm 1, the loop over decomposition layers p with its Message,
 * Aggregate and Concat steps): the feature dimension is cut into chunks of
 * `chunk_width` columns, every chunk is aggregated over all vertices, and each
 * chunk's result is written into its own columns of the output.  The
 * Combination (dense) phase comes first (Section III: combination is run ahead
 * of aggregation); its output is the aggregation's input, whether the caller
 * computed it or gnnfd_combine did.
 *
 * Conventions
 *   - Every pointer named d_* is DEVICE memory owned by the caller.  The library
 *     never allocates or frees device memory; it carves what it needs out of
 *     the buffers it is handed.  Host pointers are named without the prefix.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the default stream).
 *   - All entry points return a gnnfd_status_t (0 = success, negative = error);
 *     nothing throws, aborts or traps.  Device-side problems (a vertex id out of
 *     range) are counted on the device and reported as a status.
 *   - Matrices are row-major with a leading dimension in ELEMENTS (ld >= width).
 *     Padding columns are never written and never influence a result.
 *   - Same inputs give bit-identical outputs from run to run: no floating-point
 *     atomics are used anywhere.
 *   - Graph structure is int32 on the device: n and nnz must stay below 2^31.
 */
#ifndef GNNFD_H
#define GNNFD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gnnfd_csr gnnfd_csr_t; /* opaque host-side handle; holds device pointers into caller memory */

typedef enum { GNNFD_F32 = 0, GNNFD_BF16 = 1 } gnnfd_dtype_t;
typedef enum { GNNFD_I32 = 0, GNNFD_I64 = 1 } gnnfd_itype_t;

/* gnnfd_build_csr flags */
enum {
    GNNFD_CSR_ADD_SELF_LOOPS = 1, /* drop every input loop, then add exactly one (v,v) per vertex */
    GNNFD_CSR_DEDUP = 2,          /* keep the first (lowest edge id) of equal (dst, src) pairs */
    GNNFD_CSR_SYMMETRIZE = 4,     /* add the reverse of every non-loop edge, with edge id e + i */
    GNNFD_CSR_INPUT_ORDER = 8     /* light build: sort by destination only; the entries of a row keep the order of
                                     their edge ids instead of ascending source ids (not with DEDUP) */
};

typedef enum {
    GNNFD_OK = 0,
    GNNFD_INVALID_ARG = -1,         /* null pointer, non-positive size, ld < width, heads*dim mismatch */
    GNNFD_BAD_INDEX = -2,           /* a vertex id outside [0, n) was found in the edge list */
    GNNFD_TOO_LARGE = -3,           /* n, e or the resulting nnz does not fit the int32 structure */
    GNNFD_WORKSPACE_TOO_SMALL = -4, /* a caller-provided buffer is smaller than the size query says */
    GNNFD_UNSUPPORTED = -5,         /* unknown dtype / itype enum; an operand layout gnnfd_combine cannot take */
    GNNFD_CUDA_ERROR = -6,          /* a CUDA runtime call failed; see gnnfd_last_cuda_error() */
    GNNFD_STATIC_SCRATCH_EXCEEDED = -7 /* the built-in workspace of a *_static entry point is too small for this call */
} gnnfd_status_t;

/* ------------------------------------------------------------------ graph set-up
 *
 * CSR by destination from a COO edge list (Section II-C: the aggregation's input
 * is the edge set in COO form plus the vertex features).  Edge i goes from
 * src[i] to dst[i]; row v of the CSR lists the sources of the edges that end in
 * v.  Steps, in this order: reject ids outside [0,n); SYMMETRIZE; ADD_SELF_LOOPS;
 * order by (dst, src), ties by ascending edge id; DEDUP.  Besides row_ptr /
 * col_idx the build stores perm (CSR slot -> input edge id; e + i for the
 * reverse of edge i; -1 for an added self-loop), the degree normalisers
 * deg^-1/2 and 1/deg (0 for empty rows, deg = entries in the row), the GCN edge
 * weight deg(src)^-1/2 * deg(dst)^-1/2 per slot, and the launch schedule (rows
 * grouped by degree, rows above GNNFD_HUB_DEGREE cut into segments of at most
 * GNNFD_HUB_SEGMENT edges; see gnnfd_csr_schedule).
 *
 * GNNFD_CSR_INPUT_ORDER is for graphs that are aggregated once or a few times at a narrow width, where the
 * conversion would cost more than the aggregation it serves (Section III, the discussion of format-conversion
 * latency: a conversion can cancel the gain of the format).  The sort then runs over the destination bits only
 * (half the passes), rows list their sources in edge-id order, and everything else (perm, weights, schedule)
 * is as above, so every aggregation entry point takes the handle; results differ from the fully ordered
 * build only in the order of the fp32 additions inside a row.
 */
#define GNNFD_HUB_DEGREE 2048
#define GNNFD_HUB_SEGMENT 1024
#ifndef GNNFD_HUB_RANGE_ROWS
#define GNNFD_HUB_RANGE_ROWS 524288
#endif

/* Sizes (bytes) of the two device buffers gnnfd_build_csr needs for n vertices and e input edges.
 * persistent: must stay alive and untouched while the handle is in use.
 * scratch:    only during the call. */
int gnnfd_csr_workspace_bytes(int64_t n, int64_t e, uint32_t flags, size_t* persistent_bytes,
                              size_t* scratch_bytes);

/* Builds the CSR.  d_src / d_dst: device arrays of e vertex ids of type `itype`, not modified.
 * d_persistent / d_scratch: device buffers, 256-byte aligned, at least as large as the size query
 * says.  Enqueues on `stream` and synchronises it once before returning (the host needs nnz and
 * the bad-index count).  On success *out receives a new handle (release with gnnfd_csr_destroy;
 * the device memory stays the caller's).  On GNNFD_BAD_INDEX no handle is produced. */
int gnnfd_build_csr(int64_t n, int64_t e, const void* d_src, const void* d_dst, gnnfd_itype_t itype,
                    uint32_t flags, void* d_persistent, size_t persistent_bytes, void* d_scratch,
                    size_t scratch_bytes, void* stream, gnnfd_csr_t** out);

/* Reads the handle.  Any output pointer may be NULL.  The d_* results point into d_persistent:
 * row_ptr[n+1], col_idx[nnz], perm[nnz], dinv_sqrt[n], rdeg[n], edge_weight[nnz]. */
int gnnfd_csr_info(const gnnfd_csr_t* csr, int64_t* n, int64_t* nnz, const int32_t** d_row_ptr,
                   const int32_t** d_col_idx, const int32_t** d_perm, const float** d_dinv_sqrt,
                   const float** d_rdeg, const float** d_edge_weight, int32_t* max_degree);

/* The launch schedule.  (The paper has no counterpart: its CPU scatter walks the edge list as it comes.
 * This is how the library balances power-law rows over the GPU; exposed for inspection and tests.)
 * bin_count[5]: rows with degree <= 8, <= 32, <= 128, <= GNNFD_HUB_DEGREE, and
 * hub rows.  d_row_order[n]: row ids sorted by degree class, ascending id inside a class; a class is
 * the exact degree up to 8, then a quarter octave of (degree - 1) up to GNNFD_HUB_DEGREE, then one
 * class for all hub rows, so every bin is a contiguous range and neighbouring rows have near-equal
 * lengths.  Hub rows are cut at the boundaries of source ranges of GNNFD_HUB_RANGE_ROWS vertex ids (doubled
 * until at most 64 ranges cover the graph; one range for a GNNFD_CSR_INPUT_ORDER build) and then into segments of
 * at most GNNFD_HUB_SEGMENT entries.  The segment arrays are in launch order, which goes range by range over all
 * hub rows, so that the hub rows in flight gather from one band of source rows: d_seg_row[n_segments],
 * d_seg_begin / d_seg_end (CSR slots [begin, end) of the segment), d_seg_slot (the segment's number when a row's
 * segments are counted in ascending source order, row after row: partial results are stored by slot).
 * d_hub_seg_ptr[n_hub+1]: the slots of the i-th hub row (i-th row of the last bin) are [ptr[i], ptr[i+1]). */
int gnnfd_csr_schedule(const gnnfd_csr_t* csr, int64_t bin_count[5], const int32_t** d_row_order,
                       int64_t* n_segments, const int32_t** d_seg_row, const int32_t** d_seg_begin,
                       const int32_t** d_seg_end, const int32_t** d_seg_slot, const int32_t** d_hub_seg_ptr);

/* Frees the host-side handle only. */
void gnnfd_csr_destroy(gnnfd_csr_t* csr);

/* ------------------------------------------------------------------ GCN / GraphSAGE aggregation
 *
 * out[v, j] = s_v * sum over the CSR entries k of row v of w_k * x[col_idx[k], j]
 *   GCN : w_k = deg(col_idx[k])^-1/2 * deg(v)^-1/2, s_v = 1   (with the self-loop flag this is
 *         the symmetric normalisation D^-1/2 (A + I) D^-1/2 X of the cited GCN model)
 *   SAGE: w_k = 1, s_v = 1/deg(v)                              (neighbourhood mean)
 * Empty rows give 0.  Products and sums are fp32 (bf16 inputs are widened exactly).
 *
 * chunk_width (>= 1) is the width of one decomposition layer: P = ceil(f / chunk_width) chunks, the
 * last one narrower; chunk_width >= f means no decomposition.  Chunks are swept one after the other
 * over all rows, so the gathered working set of a sweep is n * chunk_width elements.  The result
 * does not depend on chunk_width beyond fp32 rounding (the order of the additions inside a row
 * depends on how many lanes a chunk occupies).
 *
 * d_x: [n, ldx] of xdt.  d_out: [n, ldo] of odt (must not alias d_x).  d_scratch: per-call buffer
 * of gnnfd_aggregate_workspace_bytes(csr, f) bytes (holds the per-segment partial sums of hub rows;
 * 0 bytes when the graph has no hub row, NULL is then accepted).  The call only enqueues work.
 * 16-byte-aligned pointers with ldx*sizeof(x) and chunk offsets multiples of 16 bytes take the
 * 128-bit load path; anything else is still correct through narrower loads.  Where the features are not aligned
 * like that, a scratch buffer of gnnfd_aggregate_best_workspace_bytes(csr, d_x, ldx, xdt, f, chunk_width) bytes lets
 * the call gather from an aligned copy of them wherever that is faster (the same sums in another order);
 * elsewhere that size equals gnnfd_aggregate_workspace_bytes. */
int gnnfd_aggregate_workspace_bytes(const gnnfd_csr_t* csr, int32_t f, size_t* scratch_bytes);

int gnnfd_aggregate_best_workspace_bytes(const gnnfd_csr_t* csr, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t f,
                                         int32_t chunk_width, size_t* scratch_bytes);

int gnnfd_aggregate_gcn(const gnnfd_csr_t* csr, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt,
                        void* d_out, int64_t ldo, gnnfd_dtype_t odt, int32_t f, int32_t chunk_width,
                        void* d_scratch, size_t scratch_bytes, void* stream);

int gnnfd_aggregate_sage(const gnnfd_csr_t* csr, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt,
                         void* d_out, int64_t ldo, gnnfd_dtype_t odt, int32_t f, int32_t chunk_width,
                         void* d_scratch, size_t scratch_bytes, void* stream);

/* Choice of the chunk width.  The paper leaves the number of decomposition layers to the user: it
 * depends on the device's memory capacity and on the dataset (Section II-B; the granularity sweep of
 * Section III).  gnnfd_default_chunk_candidates fills `candidates` with f (no decomposition) and the
 * powers of two below f from 256 down to two 16-byte vectors, and returns how many it wrote.
 * gnnfd_tune_chunk_width runs the aggregation (model 0 = GCN, 1 = SAGE) twice per candidate on the
 * caller's own graph and features, times the second call with CUDA events on `stream`, and returns the
 * fastest width in *best_width (its time in *best_ms, may be NULL).  It synchronises the stream;
 * d_out holds the result for the last candidate tried.  Other arguments as for gnnfd_aggregate_gcn. */
int gnnfd_default_chunk_candidates(int32_t f, gnnfd_dtype_t xdt, int32_t* candidates, int capacity);

int gnnfd_tune_chunk_width(const gnnfd_csr_t* csr, int model, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt,
                           void* d_out, int64_t ldo, gnnfd_dtype_t odt, int32_t f, const int32_t* candidates,
                           int n_candidates, void* d_scratch, size_t scratch_bytes, void* stream,
                           int32_t* best_width, float* best_ms);

/* GCN aggregation without a caller workspace and without any allocation.  (The paper has no
 * counterpart to this entry point; it exists for the library's users.)
 *
 * Who needs it: a host that gave the whole device to its own memory pool at start-up, or that calls
 * from a loop where cudaMalloc's device-wide synchronisation is not acceptable, and that has no spare
 * buffer to hand over.  Such a caller cannot obtain the hub-row workspace gnnfd_aggregate_gcn asks
 * for.  Here that workspace is a fixed array of GNNFD_STATIC_SCRATCH_BYTES inside the library image;
 * every device that loads the library carries it until the process exits.  The call itself performs
 * no cudaMalloc / cudaFree and calls no allocating routine -- with one exception: while the optional
 * per-kernel timing is switched on (gnnfd_kernel_timing_enable(1), a diagnostic that is off by
 * default) every launch of the library creates a pair of CUDA events, this entry point's included;
 * leave the timing off where allocation is not allowed.
 *
 * Same arguments and same results (bit for bit: it runs the same kernels on the same data) as
 * gnnfd_aggregate_gcn with gnnfd_aggregate_workspace_bytes of scratch, minus the scratch pair.
 * Limits and rules:
 *   - returns GNNFD_STATIC_SCRATCH_EXCEEDED when gnnfd_aggregate_workspace_bytes(csr, f) is larger
 *     than GNNFD_STATIC_SCRATCH_BYTES (hub segments x f rounded up to 4, x 4 bytes); nothing is launched;
 *   - the first call on each device looks up the array's device address (one runtime query, with that
 *     device current); make that first call outside any stream capture;
 *   - all calls on a device share the one array and it keeps whatever the previous call left.  The
 *     kernels overwrite every element before reading it, so nothing needs clearing, but two calls
 *     whose kernels may overlap on the GPU (different streams, no ordering between them) race on it:
 *     serialise them, or use gnnfd_aggregate_gcn with separate buffers. */
#define GNNFD_STATIC_SCRATCH_BYTES (32u << 20)

int gnnfd_aggregate_gcn_static(const gnnfd_csr_t* csr, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt,
                               void* d_out, int64_t ldo, gnnfd_dtype_t odt, int32_t f, int32_t chunk_width,
                               void* stream);

/* ------------------------------------------------------------------ one-shot aggregation of a COO edge list
 *
 * Edge list in, aggregated features out, for a graph that is used once (or at a narrow width, where a full
 * conversion costs several times the aggregation it serves; Section III of the paper makes that point about
 * conversion latency, its own method taking the COO edge set as it is).  The call does the light build
 * (GNNFD_CSR_INPUT_ORDER: half the sort passes; with GNNFD_CSR_DEDUP in `flags` the fully ordered build instead)
 * and the GCN / SAGE aggregation defined above out of ONE caller buffer, and returns no handle.  Still no
 * atomics: the stable destination sort fixes the order of every row's additions, so results are bit-identical
 * from run to run.  d_scratch: gnnfd_oneshot_workspace_bytes(n, e, flags, f) bytes, 256-byte aligned; it holds the
 * CSR, the sort buffers and the hub-row partial sums (sized for the worst case, because the graph is not known
 * yet).  Other arguments as for gnnfd_build_csr and gnnfd_aggregate_gcn.  Synchronises the stream once (the build
 * reads its counters), then enqueues the aggregation. */
int gnnfd_oneshot_workspace_bytes(int64_t n, int64_t e, uint32_t flags, int32_t f, size_t* scratch_bytes);

int gnnfd_oneshot_gcn(int64_t n, int64_t e, const void* d_src, const void* d_dst, gnnfd_itype_t itype, uint32_t flags,
                      const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, void* d_out, int64_t ldo, gnnfd_dtype_t odt,
                      int32_t f, int32_t chunk_width, void* d_scratch, size_t scratch_bytes, void* stream);

int gnnfd_oneshot_sage(int64_t n, int64_t e, const void* d_src, const void* d_dst, gnnfd_itype_t itype, uint32_t flags,
                       const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, void* d_out, int64_t ldo, gnnfd_dtype_t odt,
                       int32_t f, int32_t chunk_width, void* d_scratch, size_t scratch_bytes, void* stream);

/* The same for the attention aggregator (defined in the GAT section below; arguments as for gnnfd_aggregate_gat). */
int gnnfd_oneshot_gat_workspace_bytes(int64_t n, int64_t e, uint32_t flags, int32_t heads, int32_t dim,
                                      size_t* scratch_bytes);

int gnnfd_oneshot_gat(int64_t n, int64_t e, const void* d_src, const void* d_dst, gnnfd_itype_t itype, uint32_t flags,
                      const void* d_z, int64_t ldz, gnnfd_dtype_t zdt, const float* d_a_src, const float* d_a_dst,
                      int32_t heads, int32_t dim, float negative_slope, void* d_out, int64_t ldo, gnnfd_dtype_t odt,
                      int32_t chunk_width, void* d_scratch, size_t scratch_bytes, void* stream);

/* ------------------------------------------------------------------ GAT
 *
 * The attention aggregator is the third model the paper evaluates (Section II-A lists it with GCN and
 * GraphSAGE as the message-passing models under study; Section III runs it with a decomposition
 * granularity of 8 columns, one head, and studies that granularity against the hidden width).  The
 * paper gives no formula; the definition below is the cited GAT model's, evaluated on the
 * destination-indexed edge list as Section II-C describes the framework's chunked `propagate`: the
 * attention coefficients belong to the Message step and depend on whole heads, the weighted sum is the
 * Aggregate step and is what Algorithm 1 decomposes.
 *
 * Scores (full head width, computed once, never per chunk):
 *   s_src[u, h] = sum_d a_src[h, d] * z[u, h*dim + d],   s_dst[v, h] likewise with a_dst.
 * Logit of CSR entry k of row v, head h: LeakyReLU(s_src[col_idx[k], h] + s_dst[v, h]) with the given
 * negative slope.  alpha = softmax of the logits over the entries of the row (multi-edges are
 * separate terms).  out[v, h*dim + d] = sum_k alpha[k, h] * z[col_idx[k], h*dim + d]; empty row -> 0.
 * The fused kernel evaluates logits, a running (max, sum) softmax and the weighted sum in one pass
 * over the row; chunk_width decomposes the flattened heads*dim columns (column j uses head j / dim).
 */

/* The per-vertex halves of the attention logit (the linear part of the cited model's Message step,
 * Section II-A), computed once per layer from the full head width.
 * d_z [n, ldz] of zdt; d_a_src / d_a_dst [heads, dim] fp32; d_s_src / d_s_dst [n, heads] fp32 out. */
int gnnfd_gat_scores(int64_t n, const void* d_z, int64_t ldz, gnnfd_dtype_t zdt, const float* d_a_src,
                     const float* d_a_dst, int32_t heads, int32_t dim, float* d_s_src, float* d_s_dst,
                     void* stream);

/* Scratch for gnnfd_aggregate_gat: the two score arrays plus hub-row partials.
 * gnnfd_aggregate_gat is Algorithm 1's loop over decomposition layers for the attention model: Message
 * (coefficient times source feature) and Aggregate (sum over the row) per chunk of chunk_width columns,
 * Concat by writing each chunk into its own output columns. */
int gnnfd_gat_workspace_bytes(const gnnfd_csr_t* csr, int32_t heads, int32_t dim, size_t* scratch_bytes);

/* As gnnfd_aggregate_best_workspace_bytes: with this much scratch gnnfd_aggregate_gat can gather from a copy of z whose heads are
 * padded to whole 16-byte vectors, where they are not and it is faster. */
int gnnfd_gat_best_workspace_bytes(const gnnfd_csr_t* csr, const void* d_z, int64_t ldz, gnnfd_dtype_t zdt, int32_t heads,
                                   int32_t dim, int32_t chunk_width, size_t* scratch_bytes);

int gnnfd_aggregate_gat(const gnnfd_csr_t* csr, const void* d_z, int64_t ldz, gnnfd_dtype_t zdt,
                        const float* d_a_src, const float* d_a_dst, int32_t heads, int32_t dim,
                        float negative_slope, void* d_out, int64_t ldo, gnnfd_dtype_t odt,
                        int32_t chunk_width, void* d_scratch, size_t scratch_bytes, void* stream);

/* Materialised edge softmax (the normalisation inside the cited attention model's Message step,
 * Section II-A, written out instead of fused; Section II-C's gather-scatter framework materialises it
 * the same way): alpha[k, h] for every CSR slot k, [nnz, heads] fp32 in CSR order, from
 * caller-supplied scores d_s_src / d_s_dst [n, heads] fp32 (logit and softmax as defined above).
 * d_scratch: per-call buffer of gnnfd_edge_softmax_workspace_bytes(csr, heads) bytes (the running
 * maximum and sum of every hub-row segment; 0 bytes when the graph has no hub row, NULL is then
 * accepted), 8-byte aligned.  16-byte-aligned pointers with heads a multiple of 4 take the 128-bit
 * path; anything else is still correct through narrower accesses.  The call only enqueues work. */
int gnnfd_edge_softmax_workspace_bytes(const gnnfd_csr_t* csr, int32_t heads, size_t* scratch_bytes);

int gnnfd_edge_softmax(const gnnfd_csr_t* csr, const float* d_s_src, const float* d_s_dst, int32_t heads,
                       float negative_slope, float* d_alpha, void* d_scratch, size_t scratch_bytes, void* stream);

/* ------------------------------------------------------------------ Combination ahead of aggregation
 *
 * z[v, j] = sum_k x[v, k] * w_t[j, k]: the dense transform of a layer, applied to the input features
 * before the aggregation so that the aggregation runs on the f_out transformed columns (Section III of
 * the paper: the Combination phase is executed ahead of Aggregation; Algorithm 1 then decomposes the
 * transformed features).  Not part of the aggregation path proper; offered so that a whole layer stays
 * on the device.
 *
 * d_x [n, ldx] and d_w_t [f_out, ldw] (the weight matrix transposed: one row per output column) both of
 * type xdt; d_z [n, ldz] of type zdt.  The product runs on the tensor cores with fp32 sums:
 *   xdt = GNNFD_F32, mode GNNFD_COMBINE_TF32: both operands are read as tf32 (the low 13 mantissa bits of each
 *                     fp32 value are ignored), products are exact, so |z - exact| <= 2^-9 * sum_k |x[v,k] * w_t[j,k]|
 *                     plus fp32 summation error;
 *   xdt = GNNFD_F32, mode GNNFD_COMBINE_FP32: fp32-faithful.  Each operand is used as a tf32 pair (hi, lo) and
 *                     the three products that matter are accumulated, so the result meets the library's fp32
 *                     bar |z - exact| <= 1e-5 * sum_k |x[v,k] * w_t[j,k]| + 1e-6 (the paper's framework runs
 *                     the Combination in fp32);
 *   xdt = GNNFD_BF16: operands are used as they are, products are exact in fp32 (mode is ignored).
 * zdt = GNNFD_BF16 rounds the fp32 result to nearest even.
 * d_x and d_w_t must be 16-byte aligned with row pitches that are multiples of 16 bytes
 * (GNNFD_UNSUPPORTED otherwise); d_z has no alignment rule.  d_status (may be NULL): one int32 the caller
 * has set to 0; it becomes 1 if a block gave up waiting for its own copies or matrix instructions (each
 * wait is limited to one second), in which case d_z is incomplete.  The calls only enqueue work.
 *
 * gnnfd_combine is the tf32 product alone.  gnnfd_combine_ex adds the mode and, optionally, the GAT scores of
 * the result as part of the same pass (all four of d_a_src, d_a_dst [heads, dim] and d_s_src, d_s_dst
 * [n, heads] given, heads * dim == f_out; all four NULL to leave them out): the scores are formed from the
 * values written to d_z while a thread still holds its output row, so z is not read again.  With more than 256
 * output columns the columns are processed in tiles, which must then hold whole heads (GNNFD_UNSUPPORTED
 * otherwise; use gnnfd_gat_scores on the result instead). */
typedef enum { GNNFD_COMBINE_TF32 = 0, GNNFD_COMBINE_FP32 = 1 } gnnfd_combine_mode_t;

int gnnfd_combine(int64_t n, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t f_in, const void* d_w_t,
                  int64_t ldw, int32_t f_out, void* d_z, int64_t ldz, gnnfd_dtype_t zdt, int32_t* d_status,
                  void* stream);

int gnnfd_combine_ex(int64_t n, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t f_in, const void* d_w_t,
                     int64_t ldw, int32_t f_out, void* d_z, int64_t ldz, gnnfd_dtype_t zdt, int mode,
                     const float* d_a_src, const float* d_a_dst, int32_t heads, int32_t dim, float* d_s_src,
                     float* d_s_dst, int32_t* d_status, void* stream);

/* ------------------------------------------------------------------ a whole layer on a built CSR
 *
 * Combination, then Aggregation of the transformed features (Section III: the Combination phase is run ahead
 * of the Aggregation phase, so that Algorithm 1's decomposed aggregation works on the f_out transformed columns
 * instead of the f_in input columns): out = Aggregate(x * W), with the aggregators defined above.
 *   gnnfd_layer_gcn / gnnfd_layer_sage : gnnfd_combine_ex, then gnnfd_aggregate_gcn / gnnfd_aggregate_sage.
 *   gnnfd_layer_gat : gnnfd_combine_ex with the attention scores formed in its epilogue, then the fused GAT
 *                     aggregation on those scores (no separate scores pass; heads * dim output columns).
 * x, w_t, mode, d_status as for gnnfd_combine_ex; out, chunk_width as for the aggregation calls (chunk_width
 * decomposes the f_out transformed columns).  The transformed features z [n, f_out rounded up to 8] are kept in
 * the scratch buffer in the dtype of x.  d_scratch: gnnfd_layer_workspace_bytes(csr, model, f_out, heads, dim,
 * xdt) bytes, 256-byte aligned (model 0 = GCN, 1 = SAGE, 2 = GAT; heads and dim are ignored for 0 and 1).
 * d_out must not alias d_x.  The calls only enqueue work. */
int gnnfd_layer_workspace_bytes(const gnnfd_csr_t* csr, int model, int32_t f_out, int32_t heads, int32_t dim,
                                gnnfd_dtype_t xdt, size_t* scratch_bytes);

/* As gnnfd_gat_best_workspace_bytes: room for a copy of z with padded heads, where gnnfd_layer_gat is faster with one. */
int gnnfd_layer_best_workspace_bytes(const gnnfd_csr_t* csr, int model, int32_t f_out, int32_t heads, int32_t dim,
                                     gnnfd_dtype_t xdt, int32_t chunk_width, size_t* scratch_bytes);

int gnnfd_layer_gcn(const gnnfd_csr_t* csr, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t f_in,
                    const void* d_w_t, int64_t ldw, int32_t f_out, int mode, void* d_out, int64_t ldo, gnnfd_dtype_t odt,
                    int32_t chunk_width, void* d_scratch, size_t scratch_bytes, int32_t* d_status, void* stream);

int gnnfd_layer_sage(const gnnfd_csr_t* csr, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t f_in,
                     const void* d_w_t, int64_t ldw, int32_t f_out, int mode, void* d_out, int64_t ldo, gnnfd_dtype_t odt,
                     int32_t chunk_width, void* d_scratch, size_t scratch_bytes, int32_t* d_status, void* stream);

int gnnfd_layer_gat(const gnnfd_csr_t* csr, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t f_in,
                    const void* d_w_t, int64_t ldw, int32_t heads, int32_t dim, const float* d_a_src,
                    const float* d_a_dst, float negative_slope, int mode, void* d_out, int64_t ldo, gnnfd_dtype_t odt,
                    int32_t chunk_width, void* d_scratch, size_t scratch_bytes, int32_t* d_status, void* stream);

/* ------------------------------------------------------------------ dot-product attention over a graph
 *
 * The attention of transformer layers with the graph as its mask: vertex v attends to the sources of the edges that end in it, so the graphs
 * of a batch (or documents) do not see one another, and a batch of small graphs that are attended as wholes is the CSR of
 * all their pairs.  (The paper's attention model scores an edge by a sum of two halves instead: gnnfd_aggregate_gat.)  For CSR entry k of row v with
 * source u and head h
 *   t = scale * <q[v, h], key[u, h]>,   s[k, h] = (softcap > 0 ? softcap * tanh(t / softcap) : t) + bias[dist[k], h]
 *   p = softmax of s[., h] over the entries of the row,   out[v, h] = sum_k p[k, h] * value[u, h]
 * Multi-edges are separate terms.  q, key, value, out: [n, ld] with heads * dim columns (column j belongs to head j / dim; dim up to
 * 256 for fp32, 512 for bf16); the three inputs have type dt.  d_dist [nnz] int32, in CSR slot order: the bucket of every entry, say the distance of its ends;
 * buckets below 0 or past the last one count as the first or last.  d_bias [buckets, heads] fp32.  Both NULL (buckets 0): no bias.  A bias of
 * -infinity takes an entry out, whatever q, key and value hold for it.  Rows without entries, or with none left, give 0.
 * d_lse (may be NULL): [n, heads, 2] fp32, 8-byte aligned, receives each row's largest score and the sum of e^(s - largest): the
 * logarithm of the softmax's denominator in two parts, as the gradient needs it ((-infinity, 0) for rows without entries).
 * chunk_width: as for the other aggregations, but a multiple of dim (or >= heads * dim): a chunk holds whole heads.
 * GNNFD_TOO_LARGE: more than 4,194,240 columns, 2^31 - 65536 entries or a pitch of 2^30; for d_dbias also more than 2,621,400 buckets.
 * d_scratch: gnnfd_attention_workspace_bytes(csr, heads, dim) bytes, 256-byte aligned (0 and NULL where the graph has no hub row).  fp32 sums and
 * softmax; tanh is within 8 * 2^-24 of its value, for bf16 features and results of a call without d_lse and a cap of up to 64 within as much
 * of 1 (a weight is then off by 2^-14 of itself at most).  The call only enqueues work. */
int gnnfd_attention_workspace_bytes(const gnnfd_csr_t* csr, int32_t heads, int32_t dim, size_t* scratch_bytes);

int gnnfd_aggregate_attention(const gnnfd_csr_t* csr, const void* d_q, int64_t ldq, const void* d_k, int64_t ldk, const void* d_v,
                              int64_t ldv, gnnfd_dtype_t dt, int32_t heads, int32_t dim, float scale, float softcap,
                              const int32_t* d_dist, const float* d_bias, int32_t buckets, void* d_out, int64_t ldo, gnnfd_dtype_t odt,
                              float* d_lse, int32_t chunk_width, void* d_scratch, size_t scratch_bytes, void* stream);

/* The gradients of the above for d_dout [n, lddo] of type dt, the gradient of out: d_dq, d_dk, d_dv [n, ld*] of type gdt and, where d_dbias is not NULL,
 * d_dbias [buckets, heads] fp32.  csr_t: the CSR of the reversed edges, gnnfd_build_csr of the same edge list with d_src and d_dst exchanged and
 * the same flags; d_dist_t: the buckets in csr_t's slot order.  d_lse as written by the forward call with the same arguments.  Nothing is
 * added with atomics: gradients of vertices that many edges share are sums over the rows of csr_t.
 * d_scratch: gnnfd_attention_backward_workspace_bytes(csr, csr_t, heads, dim, buckets) bytes (buckets may be 0 there where d_dbias is NULL;
 * with it, nnz * heads floats of it and up to 740 * buckets * heads more). */
int gnnfd_attention_backward_workspace_bytes(const gnnfd_csr_t* csr, const gnnfd_csr_t* csr_t, int32_t heads, int32_t dim, int32_t buckets,
                                             size_t* scratch_bytes);

int gnnfd_aggregate_attention_backward(const gnnfd_csr_t* csr, const gnnfd_csr_t* csr_t, const void* d_q, int64_t ldq, const void* d_k,
                                       int64_t ldk, const void* d_v, int64_t ldv, const void* d_dout, int64_t lddo, gnnfd_dtype_t dt,
                                       const float* d_lse, int32_t heads, int32_t dim, float scale, float softcap, const int32_t* d_dist,
                                       const int32_t* d_dist_t, const float* d_bias, int32_t buckets, void* d_dq, int64_t lddq, void* d_dk,
                                       int64_t lddk, void* d_dv, int64_t lddv, gnnfd_dtype_t gdt, float* d_dbias, int32_t chunk_width,
                                       void* d_scratch, size_t scratch_bytes, void* stream);

/* ------------------------------------------------------------------ group norm with an activation, over the graphs of a batch
 *
 * The step between two layers (the Update of Algorithm 1 is left to the user by the paper): rows graph_ptr[b] .. graph_ptr[b + 1] - 1 are the
 * vertices of graph b, a group is f / groups neighbouring columns, and over the rows of a graph and the columns of a group
 *   out = act((x - mean) * rstd * weight + bias),   rstd = (variance + eps)^-1/2  (the variance of all values there, not corrected).
 * groups = 1 normalises a graph as a whole, groups = f each column of a graph by itself.
 * d_x [n, ldx] of type xdt, d_out [n, ldo] of type odt (may be d_x itself, with ldo = ldx and odt = xdt).  d_graph_ptr [graphs + 1] of type itype, ascending
 * from 0; NULL: one graph of n rows (graphs = 1).  Rows behind the last offset are left as they are; graphs may be empty (mean 0,
 * rstd eps^-1/2).  Offsets outside [0, n] or not ascending are cut to what is inside: nothing outside of the arrays is touched.  d_weight, d_bias [f] fp32,
 * either may be NULL (1 and 0).  d_mean, d_rstd [graphs, groups] fp32 receive the statistics; both may be NULL.  f up to 8192.
 * Statistics, sums and the activation are fp32 or wider, squares of distances from the mean included; the result is rounded once.  d_scratch:
 * gnnfd_group_norm_workspace_bytes(n, f, groups, graphs, 0) bytes, 256-byte aligned.  The call only enqueues work. */
typedef enum {
    GNNFD_ACT_NONE = 0,
    GNNFD_ACT_RELU = 1,
    GNNFD_ACT_ELU = 2,   /* z > 0 ? z : e^z - 1 */
    GNNFD_ACT_SILU = 3,  /* z / (1 + e^-z) */
    GNNFD_ACT_GELU = 4   /* z / 2 * (1 + erf(z / sqrt 2)) */
} gnnfd_activation_t;

int gnnfd_group_norm_workspace_bytes(int64_t n, int32_t f, int32_t groups, int64_t graphs, int backward, size_t* scratch_bytes);

int gnnfd_group_norm(int64_t n, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t f, int32_t groups, int64_t graphs,
                     const void* d_graph_ptr, gnnfd_itype_t itype, const float* d_weight, const float* d_bias, float eps, int activation,
                     void* d_out, int64_t ldo, gnnfd_dtype_t odt, float* d_mean, float* d_rstd, void* d_scratch, size_t scratch_bytes,
                     void* stream);

/* The gradients of the above for d_dout [n, ldd] of type xdt: d_dx [n, lddx] of type gdt (rows behind the last offset are left as they
 * are), and d_dweight, d_dbias [f] fp32, sums over the rows of all graphs (both NULL: not wanted).  d_mean, d_rstd as the forward call
 * gave them; the other arguments as there.  relu's slope at 0 is 0.  d_dx may be d_dout itself (same pitch and type).  d_scratch:
 * gnnfd_group_norm_workspace_bytes(n, f, groups, graphs, 1) bytes. */
int gnnfd_group_norm_backward(int64_t n, const void* d_dout, int64_t ldd, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t f,
                              int32_t groups, int64_t graphs, const void* d_graph_ptr, gnnfd_itype_t itype, const float* d_weight,
                              const float* d_bias, const float* d_mean, const float* d_rstd, int activation, void* d_dx, int64_t lddx,
                              gnnfd_dtype_t gdt, float* d_dweight, float* d_dbias, void* d_scratch, size_t scratch_bytes, void* stream);

/* ------------------------------------------------------------------ layer norm
 *
 * Every row by itself, where gnnfd_group_norm takes the rows of a graph together: a vertex's result does not depend on the vertices beside
 * it, nor a token's on its batch.  (Like that call a step between layers, which the paper leaves to the user.)  Over the f columns of a row
 *   out = (x - mean) * rstd * weight + bias,   rstd = (variance + eps)^-1/2  (not corrected)
 * d_x [n, ldx] of type xdt, d_out [n, ldo] of type odt (may be d_x itself, with ldo = ldx and odt = xdt).  d_weight, d_bias [f] fp32, either may be NULL (1 and 0).
 * d_mean, d_rstd [n] fp32 receive the statistics; both may be NULL.  f up to 8192.  Sums and statistics are fp32, the variance is the mean of squared
 * distances from the mean, and what a rounded sum leaves in the mean is taken off it and them; the result is rounded once.  Rows that hold an infinity or NaN, or whose
 * sum is beyond fp32, give NaN (where only the squares' sum is, rstd is 0); others are not touched by them.
 *
 * gnnfd_layer_norm_backward: for d_dout [n, ldd] of type xdt, d_dx [n, lddx] of type gdt (may be d_dout itself: same pitch and type; not d_x) and d_dweight,
 * d_dbias [f] fp32, sums over all rows (both NULL: not wanted; d_scratch may then be NULL), in fp32 over 16 rows at most and beyond that in 64 bits.  d_mean, d_rstd as the forward call gave
 * them, so distances from the mean are those from its fp32 value.  d_scratch: gnnfd_layer_norm_backward_workspace_bytes(n, f) bytes, 256-byte aligned.  The calls only enqueue work. */
int gnnfd_layer_norm(int64_t n, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t f, const float* d_weight, const float* d_bias,
                     float eps, void* d_out, int64_t ldo, gnnfd_dtype_t odt, float* d_mean, float* d_rstd, void* stream);

int gnnfd_layer_norm_backward_workspace_bytes(int64_t n, int32_t f, size_t* scratch_bytes);

int gnnfd_layer_norm_backward(int64_t n, const void* d_dout, int64_t ldd, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t f,
                              const float* d_weight, const float* d_mean, const float* d_rstd, void* d_dx, int64_t lddx, gnnfd_dtype_t gdt,
                              float* d_dweight, float* d_dbias, void* d_scratch, size_t scratch_bytes, void* stream);

/* ------------------------------------------------------------------ rotary positions
 *
 * Ahead of gnnfd_aggregate_attention: queries and keys are turned by angles that grow with their vertices' positions (in a document, along a
 * path), so that a score depends on how far apart the positions are.  (The paper's models know no positions.)  In each of `heads` heads of `dim` columns the first rotary_dim
 * columns (even, up to dim, up to 4096) are turned in pairs,
 *   angle = position[row] * freq[i],   (u, v) -> scale * (u cos(angle) - v sin(angle), u sin(angle) + v cos(angle)),   i < rotary_dim / 2
 * with (u, v) the columns (i, i + rotary_dim / 2) of the head or, with interleaved != 0, (2 i, 2 i + 1).  The other columns are copied.  inverse != 0 turns by the
 * opposite angle (the scale stays): this is the gradient, out's for x's.  A matrix that holds queries, keys and values side by side is turned in one call: `heads` counts
 * those of the queries and keys, and ldx goes on to the values.
 * d_positions [n] of type itype, any value (an angle is exact to 2^-51 of itself; beyond 2^50 radians it has no meaning, results stay finite); NULL: the row's number.  d_freq [rotary_dim / 2] fp64, radians per position:
 * gnnfd_rotary_frequencies or any other.  d_x [n, ldx] of type xdt, d_out [n, ldo] of type odt (d_x itself with ldo = ldx and odt = xdt; columns of
 * heads that are not turned and columns past heads * dim then stay as they are).  fp32 arithmetic on cosines and sines within 3 * 2^-24; one rounding at the end.
 * GNNFD_TOO_LARGE: more than 2^20 columns.  The call only enqueues work.
 *
 * gnnfd_rotary_frequencies (host memory, no device): freq[i] = base^(-2 i / rotary_dim), for contexts beyond the length that a model was trained on
 *   GNNFD_ROTARY_POSITION  divided by factor (positions are squeezed),
 *   GNNFD_ROTARY_BASE      with base * factor^(rotary_dim / (rotary_dim - 2)): the last frequency is divided by factor, the first stays (rotary_dim > 2),
 *   GNNFD_ROTARY_RAMP      divided by factor where a frequency makes fewer than low_turns turns over `length` positions, kept where it makes more than
 *                          high_turns, in between kept * freq + (1 - kept) * freq / factor with kept = (turns - low_turns) / (high_turns - low_turns).
 * GNNFD_INVALID_ARG where a frequency is beyond fp64. */
typedef enum { GNNFD_ROTARY_NONE = 0, GNNFD_ROTARY_POSITION = 1, GNNFD_ROTARY_BASE = 2, GNNFD_ROTARY_RAMP = 3 } gnnfd_rotary_scaling_t;

int gnnfd_rotary_frequencies(int32_t rotary_dim, double base, int scaling, double factor, int64_t length, double low_turns, double high_turns,
                             double* freq);

int gnnfd_rotary(int64_t n, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t heads, int32_t dim, int32_t rotary_dim, int interleaved,
                 const void* d_positions, gnnfd_itype_t itype, const double* d_freq, float scale, int inverse, void* d_out, int64_t ldo,
                 gnnfd_dtype_t odt, void* stream);

/* ------------------------------------------------------------------ gated linear recurrence over the rows of a graph
 *
 * A mixer of linear cost beside the attention, for vertices that have an order (the tokens of a document, a walk): every column keeps a state that decays by a
 * gate of its own from row to row.  (An aggregation over the rows ahead with weights that are products of gates; not in the paper.)  Per column
 *   h[t] = a[t] * h[t - 1] + b[t],   out[t] = h[t]        GNNFD_GATE_FACTOR: a = gate, b = x (gates of -1 to 1 are meant)
 *                                                         GNNFD_GATE_SIGMOID: a = 1 / (1 + e^-gate), b = (1 - a) * x
 * Rows graph_ptr[b] .. graph_ptr[b + 1] - 1 are graph b, in order; its first row's h[t - 1] is d_initial[b] (fp32 [graphs, f]; NULL: 0).  d_graph_ptr [graphs + 1]
 * of type itype, ascending from 0; NULL: graphs of n / graphs rows each (n must be a multiple), so graphs = n is one token for each of n sequences.  Rows
 * behind the last offset are left as they are; graphs may be empty (their last state is the first one).  Offsets outside [0, n] or not ascending are cut to what is
 * inside: nothing outside of the arrays is touched.  d_x, d_gate [n, ld] of type dt, d_out [n, ldo] of type odt, not overlapping them nor d_initial (a
 * copy of the last row of a stretch that goes on in the same buffer will do; for single tokens, graphs = n without d_graph_ptr, d_initial may be d_out itself, fp32 with ldo = f).  d_final (fp32
 * [graphs, f], may be NULL) receives the last state of each graph; it may be d_initial itself where graphs = n and d_graph_ptr is NULL, and does not overlap it otherwise.  d_states
 * (may be NULL): fp32 [(n + 7) / 8, f], states that the gradient starts from.  States and products of gates are fp32 or wider; of
 * sigmoid gates a and 1 - a are within (10 + |gate| / 20) * 2^-24 of themselves (a above 2^-100).
 * d_scratch: gnnfd_linear_recurrence_workspace_bytes(n, f, graphs, d_graph_ptr == NULL, 0) bytes, 256-byte aligned (0
 * and NULL for up to GNNFD_RECURRENCE_FEW_ROWS rows, in the gradient half as many and of up to
 * GNNFD_RECURRENCE_FEW_VALUES values).
 *
 * gnnfd_linear_recurrence_backward: for d_dout [n, ldd] of type dt and d_dfinal (fp32 [graphs, f]; NULL: 0), the gradients of out and the last states, d_dx and
 * d_dgate [n, ld*] of type gdt and d_dinitial (fp32 [graphs, f]; NULL: not wanted), none of which overlaps another or what is read.  d_states as written by the forward call with the same arguments.  Rows
 * behind the last offset are left as they are.  Scratch: the same query with backward = 1.
 * GNNFD_TOO_LARGE: more than 2^31 - 65536 rows or 2^20 columns.  The calls only enqueue work. */
typedef enum { GNNFD_GATE_FACTOR = 0, GNNFD_GATE_SIGMOID = 1 } gnnfd_gate_t;

#define GNNFD_RECURRENCE_FEW_ROWS 4096
#define GNNFD_RECURRENCE_FEW_VALUES 524288
int gnnfd_linear_recurrence_workspace_bytes(int64_t n, int32_t f, int64_t graphs, int equal_lengths, int backward, size_t* scratch_bytes);

int gnnfd_linear_recurrence(int64_t n, const void* d_x, int64_t ldx, const void* d_gate, int64_t ldg, gnnfd_dtype_t dt, int32_t f, int form,
                            int64_t graphs, const void* d_graph_ptr, gnnfd_itype_t itype, const float* d_initial, void* d_out, int64_t ldo,
                            gnnfd_dtype_t odt, float* d_final, float* d_states, void* d_scratch, size_t scratch_bytes, void* stream);

int gnnfd_linear_recurrence_backward(int64_t n, const void* d_dout, int64_t ldd, const void* d_x, int64_t ldx, const void* d_gate, int64_t ldg,
                                     gnnfd_dtype_t dt, int32_t f, int form, int64_t graphs, const void* d_graph_ptr, gnnfd_itype_t itype,
                                     const float* d_initial, const float* d_states, const float* d_dfinal, void* d_dx, int64_t lddx,
                                     void* d_dgate, int64_t lddg, gnnfd_dtype_t gdt, float* d_dinitial, void* d_scratch, size_t scratch_bytes,
                                     void* stream);

/* ------------------------------------------------------------------ learned vertex features
 *
 * For graphs whose vertices have no features of their own (or a type, a degree, a name instead): a table with a learned row per
 * id, looked up ahead of the first layer, and the table's gradient for its training.  (The paper's graphs come with features.)
 *
 * gnnfd_embedding: out[i, :] = scale * table[ids[i], :] for i < n (n may be 0).  d_ids [n] of type itype; d_table [vocab, ldt] of type tdt;
 * d_out [n, ldo] of type odt, not overlapping the table.  An id outside [0, vocab) gives a row of zeros and sets bit 0 of
 * *d_status (d_status may be NULL; the caller has set it to 0).
 *
 * gnnfd_embedding_backward: grad[r, :] = scale * sum of dout[i, :] over the i with ids[i] == r, for all vocab rows; rows that no id
 * names become 0.  Sums are fp32 in an order that depends on the ids, the sizes, and the operands' alignment and pitches: equal calls give equal bits.  With accumulate != 0 the
 * sums are added to what d_grad holds (of type gdt, rounded once) and rows that no id names are left as they are.  Ids equal to `padding`
 * (-1: none) take no part: their row is treated as one that no id names.  Ids outside [0, vocab) take no part and set bit 0 of *d_status;
 * bit 1 is set if a block of the sort gave up waiting for another one (grad is then incomplete).  d_dout [n, ldd] of type ddt;
 * d_grad [vocab, ldg], not overlapping it.  d_scratch: gnnfd_embedding_backward_workspace_bytes(n, vocab, f) bytes, 256-byte
 * aligned (0 bytes for no ids, and up to GNNFD_EMBEDDING_FEW_IDS ids of a table of up to GNNFD_EMBEDDING_FEW_ROWS rows; NULL is then accepted).  GNNFD_TOO_LARGE:
 * 2^31 - 15 or more ids or rows (2^31 in the lookup), more than 65535 * 256 columns in the gradient (65535 * 128 where rows do not all start on two
 * elements of their type), 2^31 - 4096 in the lookup.  Both calls only enqueue work. */
#define GNNFD_EMBEDDING_FEW_IDS 16384
#define GNNFD_EMBEDDING_FEW_ROWS 3629056
int gnnfd_embedding(int64_t n, const void* d_ids, gnnfd_itype_t itype, int64_t vocab, const void* d_table, int64_t ldt,
                    gnnfd_dtype_t tdt, int32_t f, float scale, void* d_out, int64_t ldo, gnnfd_dtype_t odt, int32_t* d_status,
                    void* stream);

int gnnfd_embedding_backward_workspace_bytes(int64_t n, int64_t vocab, int32_t f, size_t* scratch_bytes);

int gnnfd_embedding_backward(int64_t n, const void* d_ids, gnnfd_itype_t itype, const void* d_dout, int64_t ldd, gnnfd_dtype_t ddt,
                             int64_t vocab, int32_t f, float scale, int64_t padding, int accumulate, void* d_grad, int64_t ldg,
                             gnnfd_dtype_t gdt, void* d_scratch, size_t scratch_bytes, int32_t* d_status, void* stream);

/* ------------------------------------------------------------------ diagnostics */

const char* gnnfd_status_string(int status);

/* cudaError_t of the most recent failed runtime call made by this library on this thread (0 if none). */
int gnnfd_last_cuda_error(void);

/* Kernels launched by this library since it was loaded. */
int64_t gnnfd_launch_count(void);

/* Optional per-kernel timing.  While enabled every launch is bracketed by CUDA events on its stream.
 * gnnfd_kernel_timing_read synchronises the recorded events, clears them, and fills up to `capacity`
 * entries: names[i] (static strings), ms[i] (total milliseconds), launches[i].  Returns the number of
 * distinct kernels seen (may exceed capacity), or a negative status. */
int gnnfd_kernel_timing_enable(int on);
int gnnfd_kernel_timing_read(const char** names, double* ms, int64_t* launches, int capacity);

/* Drill of gnnfd_combine's give-up path, for tests.  (The paper has no counterpart.)  It arms the NEXT
 * gnnfd_combine / gnnfd_combine_ex / gnnfd_layer_gcn / _sage / _gat call made by this host thread, and only that one: every
 * barrier wait of that launch is limited to wait_ns nanoseconds (0 keeps the usual second; at most 10^9) and the
 * loads of K block skip_k_block (32 fp32 or 64 bf16 columns of x per block; -1: none) are never issued.
 * Nothing is in flight for the block that was left out, so the waits of the other lanes run out, every thread
 * block sets *d_status to 1, releases its tensor memory and returns; the device stays usable and d_z is
 * incomplete. */
int gnnfd_debug_combine_fault(int64_t wait_ns, int32_t skip_k_block);

/* Drill of the CSR build's give-up path, for tests.  It arms the NEXT gnnfd_build_csr, gnnfd_oneshot_* or gnnfd_embedding_backward
 * (digits only; it reports through *d_status) call made by this host thread, and only that one: a block of the sort gives up after max_polls reads (rounded up to 256; 0 keeps the usual million)
 * of a word that another block has not written yet, and in sweep `sweep` (0 ..: the digits; one past the last digit: the row
 * order; two past it, in gnnfd_oneshot_* calls without duplicate removal: the row pointers' sums) nobody takes the first tile, so all others wait for it and give up.  The kernels that follow do nothing, the
 * call returns GNNFD_CUDA_ERROR and no handle, nothing outside the call's buffers is touched and the device stays usable.
 * Where the sweep does not exist, has a single tile, or sorts buckets that need not hold a second one (all but the first of a large
 * graph's, where ids and edge numbers together need more than 64 bits), the armed call returns GNNFD_INVALID_ARG and launches nothing. */
int gnnfd_debug_build_fault(int32_t max_polls, int32_t sweep);

#ifdef __cplusplus
}
#endif
#endif /* GNNFD_H */
