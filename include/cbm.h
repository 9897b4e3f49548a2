/*
 * libcbm -- Compressed Binary Matrix (CBM) products on one AMD MI355X (gfx950).
 *
 * C ABI.  A binary m x n matrix A, given as CSR without values (each row a
 * sorted list of column indices: the paper's adjacency-list input, Section 2),
 * is compressed once into a CBM handle; the handle then multiplies any number
 * of dense fp32 matrices (the "compressed once, multiplied many times" use of
 * Section 1.2).  All dense operands are row-major fp32 in DEVICE memory; all
 * index arrays passed to cbm_build are in HOST memory.
 *
 * Every function returns a cbm_status; nothing throws or aborts across this
 * boundary, and output arguments are left untouched on failure.
 */
#ifndef CBM_H
#define CBM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct cbm_handle cbm_handle; /* opaque; owns its host and device arrays */

typedef enum {
    CBM_OK = 0,
    CBM_ERR_INVALID_ARG = 1, /* null pointer, k <= 0, ld < k, bad option value      */
    CBM_ERR_INVALID_CSR = 2, /* row offsets not monotone, columns unsorted, repeated
                                or out of [0, n)                                     */
    CBM_ERR_ALLOC = 3,       /* host or device allocation failed                     */
    CBM_ERR_HIP = 4,         /* a HIP runtime call failed                            */
    CBM_ERR_UNSUPPORTED = 5, /* size beyond what the index types can hold            */
    CBM_ERR_STATE = 6        /* handle cannot do this (host-only handle, normalised
                                product on a handle built without self-loops, ...)   */
} cbm_status;

/* cbm_build_opts.flags */
#define CBM_FLAG_HOST_ONLY 1u /* build the format but upload nothing to a GPU:
                                 cbm_stats / cbm_get_tree / cbm_decompress work,
                                 products return CBM_ERR_STATE                      */
#define CBM_FLAG_EXACT_TREE 2u /* the chain of compression is a minimum-cost arborescence
                                  of the pruned candidate digraph rooted at the virtual
                                  vertex (Section 2.2, "Edge Pruning"), found exactly by
                                  Edmonds' algorithm; max_depth and seed_roots are
                                  ignored.  With hub_cap = max_candidates = -1 the
                                  candidate digraph is the whole pruned distance graph. */

#define CBM_FLAG_DEVICE_BUILD 4u /* run the builder's candidate search (which rows share columns
                                    with which, the pattern of A A^T) on the GPU instead of the
                                    host threads; the chain of compression is the same.  Needs
                                    1 <= max_candidates <= 16 (the default qualifies); not with
                                    CBM_FLAG_HOST_ONLY or CBM_FLAG_HOST_SEARCH.  Without this
                                    flag a matrix of 65536 rows or more is searched on the GPU
                                    too when those conditions hold, and on the host threads if
                                    the GPU cannot take it (the search needs up to 24 GB of
                                    device memory while it runs); with it, that is an error.   */
#define CBM_FLAG_HOST_SEARCH 16u /* keep the candidate search on the host threads              */

#define CBM_FLAG_TRANSPOSE 8u /* compress the transpose: the handle holds A^T (n x m; (A v I)^T with
                                 add_self_loops) and every product and query works on that matrix.
                                 The normalised product keeps D = the row sums of A v I as given, so
                                 it computes (D^-1/2 (A + I) D^-1/2)^T X: the backward pass of the
                                 normalised product for a directed graph (for a symmetric one the
                                 transpose is the matrix itself and this flag changes nothing).   */

/*
 * Build options.  A NULL pointer means all zeros, i.e. the defaults below.
 *
 * alpha          Edge-pruning threshold of Section 2.2 ("Edge Pruning"): row x may
 *                be compressed against row y only if that saves at least alpha
 *                scalar operations, w(y,x) <= nnz(a_x) - alpha.  alpha = 0 keeps
 *                every compression that strictly beats storing the row in full
 *                (draws go to the virtual vertex, Section 2.2 after Eq. (5)).
 * add_self_loops Compress A v I instead of A (needs m == n).  Required by
 *                cbm_spmm_normalized, whose matrix is D^-1/2 (A + I) D^-1/2.
 * max_depth      Cap on the depth of the compression tree (a row stored in full
 *                has depth 1).  -1 = unlimited.  0 = automatic: cap 16, and a
 *                cost model of the kernels (launch overhead, latency of the
 *                longest work item, bandwidth) decides whether the tree pays
 *                for its extra dependent launches at all; on small graphs it
 *                does not, and every row is then stored in full (the paper's
 *                own finding for its small citation graphs, Section 3.3); the
 *                same model drops a trailing round of dependent work when
 *                storing its rows in full is cheaper than its launch, and on a
 *                matrix of 65536 rows or more the candidate search first looks
 *                at every 64th row: if their best candidates would save under
 *                2 % of their entries, the search stops there and every row is
 *                stored in full.  On a square matrix of 512 rows or more whose
 *                neighbouring rows share most of their columns the same model may
 *                let the products run in row blocks: one walk over the columns of
 *                128 alike rows, on the matrix cores, in one launch.  The tree and
 *                its counters stay what they are; the device then holds the blocks
 *                only, and bytes_cbm counts them (a small matrix whose rows are all
 *                stored in full keeps these beside its blocks or sums, and the width of
 *                a product decides which it runs on).  Where every row is stored in
 *                full, rows long enough to be split share their popular columns in
 *                such blocks too (num_tasks and bytes_cbm count what is left of
 *                them, bytes_cbm also the blocks).  On a square matrix whose rows
 *                share whole column sets (the cliques of a collaboration network)
 *                the same model may sum each set once and make the rows of those
 *                sums; bytes_cbm counts these lists too.  A row that does not hold its
 *                own column is then its sets' sums less its own row of X as often as
 *                they hold it, unless that is more than 32 times the largest other value
 *                of a column: what rounding leaves of it stays below 1e-5 of the row's
 *                terms, whatever value the row itself has.  A host-only handle has no
 *                blocks or shared sums: num_tasks and bytes_cbm are those of the
 *                paths.  The
 *                tree is cut into vertical paths, one work item each;
 *                dependent kernel launches per product = rounds of paths
 *                (cbm_stats), at most the depth.  Any value yields a valid CBM
 *                (exact product).
 * hub_cap        Candidate search: columns with more than hub_cap entries are
 *                not expanded when counting shared columns (their rows are still
 *                compared exactly once they are candidates).  0 = default (512);
 *                -1 = expand everything (exact shared-column search).
 * max_candidates Candidate parents kept per row.  0 = default (8); -1 = keep all
 *                (with hub_cap = -1, max_depth = -1 and alpha = 0 the tree is then
 *                a true minimum spanning tree of the extended distance graph).
 * seed_roots     Rows forced to be stored in full before the tree is grown, spread
 *                evenly over the row range.  With a depth cap, growing from many
 *                seeds at once gives wider levels (more parallel work per dependent
 *                launch) and often fewer deltas.  0 = automatic (the cost model
 *                picks among 0, m/128, m/32, m/8); -1 = none; > 0 = that many.
 * num_threads    Host threads for the build.  0 = all hardware threads.
 * device         HIP device that will own the arrays.  -1 = current device.
 * flags          CBM_FLAG_* bits.
 * column_blocks  0 or 1 = the format of the paper: one tree over whole rows.  B > 1 = column-blocked CBM (the
 *                column-splitting idea that Section 1.1 credits to a related format): the columns are cut
 *                into B equal ranges, the part of every row inside a range is a row of its own, and the
 *                compression tree is grown over all B m part-rows, so two rows that are alike only inside one
 *                range can still share; a product sums the B partial rows of each row in a last launch.  Costs B
 *                partial rows (written, then read) per matrix row and product.  Not with CBM_FLAG_TRANSPOSE.
 */
typedef struct {
    int32_t alpha;
    int32_t add_self_loops;
    int32_t max_depth;
    int32_t hub_cap;
    int32_t max_candidates;
    int32_t seed_roots;
    int32_t num_threads;
    int32_t device;
    uint32_t flags;
    int32_t column_blocks;
} cbm_build_opts;

typedef struct {
    int64_t m, n;
    int64_t nnz;             /* nonzeros of the compressed matrix (A, or A v I)      */
    int64_t num_delta_plus;  /* sum over rows of |Delta+|                            */
    int64_t num_delta_minus; /* sum over rows of |Delta-|                            */
    int64_t num_roots;       /* rows compressed against the virtual null row         */
    int64_t num_internal;    /* rows that some other row is compressed against       */
    int64_t scalar_ops;      /* Section 2.2: nnz(a_x) for a root, 1+|D+|+|D-| else   */
    int64_t num_tasks;       /* GPU work items (rows, plus segments of split rows)   */
    int64_t num_split_rows;  /* rows whose delta list is cut into several segments   */
    int64_t bytes_csr;       /* int64 row offsets + int32 columns, no values         */
    int64_t bytes_cbm;       /* packed device arrays of this handle (host-only: the
                                arrays that it would upload without blocks or sums)   */
    int32_t depth;           /* number of tree levels                                */
    int32_t alpha;
    int32_t add_self_loops;
    int32_t rounds;          /* dependent kernel launches per product (<= depth)      */
    double build_seconds;
    int32_t column_blocks;   /* 1, or B for a column-blocked handle: the tree then spans
                                B m part-rows; num_roots, num_internal, depth and the
                                delta counts are those of the part-rows, and scalar_ops
                                includes the (B - 1) m additions of the block sum        */
    int32_t bundled_rounds;  /* rounds whose paths are gathered in one sweep per path
                                (long work items of more than one row)                 */
} cbm_stats_t;

/*
 * cbm_build -- compress a binary CSR matrix (Section 2).
 *   m, n      matrix shape; 0 <= m, n < 2^29.
 *   rowptr    host, m + 1 entries, rowptr[0] = 0, non-decreasing.
 *   colidx    host, rowptr[m] entries; within a row strictly increasing, in [0, n).
 *   opts      host, or NULL for defaults.
 *   out       receives the handle.
 * The CSR arrays are only read during the call (copied, not retained).
 * Builder = extended distance graph restricted to row pairs that share a column
 * (only those can beat the virtual edge), Prim growth from the virtual vertex
 * with the draw rule and the alpha rule, delta lists by list merge (Eq. (2)).
 */
cbm_status cbm_build(int64_t m, int64_t n, const int64_t* rowptr, const int32_t* colidx,
                     const cbm_build_opts* opts, cbm_handle** out);

/*
 * cbm_spmm -- Y = A . X  (Eq. (5), Algorithm 1).
 *   X   device, n x k row-major fp32, leading dimension ldx >= k (in floats).
 *   Y   device, m x k row-major fp32, leading dimension ldy >= k.  Fully
 *       overwritten (it need not be zeroed).  The byte ranges spanned by X and
 *       Y must be disjoint (CBM_ERR_INVALID_ARG otherwise, also for column
 *       slices interleaved in one buffer).  The tree update runs in place in Y
 *       (Property 3).
 *   hip_stream  a hipStream_t (NULL = default stream).  The call only enqueues
 *       kernels and returns; the caller synchronises.
 * If the handle was built with add_self_loops the product is (A v I) . X.
 * k not a multiple of 4, or pointers / leading dimensions that are not 16-byte
 * multiples, select a variant of the same kernel that moves 32 bits per lane
 * and access instead of 128, not an error; it takes about 1.7x the time per
 * byte on a large graph, so pad the feature dimension to a multiple of 4 where
 * speed matters.
 * Rows with very long delta lists are summed in pieces through a scratch array owned
 * by the handle (cbm_stats.num_split_rows > 0 says the handle has such rows).  Hence:
 *  - one product at a time per handle: two products of one handle that run at the same
 *    time (two host threads, or two streams) would share that scratch and race;
 *  - the scratch is sized for the widest k seen so far.  A product with a wider k than
 *    any before it frees and reallocates it (the free waits for the device), which is
 *    not allowed under HIP-graph capture: call cbm_reserve(h, widest k) once beforehand;
 *    after that, products with k <= that width only launch kernels and can be captured.
 * A handle whose products take shared sums (launch records of kind 6) keeps an array of at most 32 MiB (128 columns of
 * sums where that is more; a quarter more without self-loops) for each of up to sixteen streams and captures, of these
 * fourteen captures at most.  The first is there from cbm_build on; the others are allocated when a product first needs
 * them, also under capture.  Where more than four streams have one, a stream that asks is given that of another whose
 * products are done; those of captures come back by cbm_release_captures; cbm_free frees them all (bytes_cbm leaves them
 * out, as it does all scratch).  A product for which there is none sums each row's sets in place: one launch (level 3 of
 * kind 6), the same bits, two to four times the time.  Neither way touches the scratch of split rows, so such products
 * may overlap freely, whatever num_split_rows says (those of cbm_spmm_noalloc may not).  A stream may be destroyed once
 * what it was given is done.
 * Per-launch profiling (cbm_profile_enable) records events and must be off during capture.
 */
cbm_status cbm_spmm(const cbm_handle* h, const float* X, int64_t ldx, int32_t k, float* Y, int64_t ldy,
                    void* hip_stream);

/*
 * cbm_spmm_noalloc -- cbm_spmm for callers that cannot allocate device memory: code under HIP-graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels and the
 * same result as cbm_spmm, but the partial sums of split rows go to a 64 MiB array that is part of the
 * library's device code instead of a scratch the handle allocates; the call makes no hipMalloc / hipFree
 * and no other allocating call.
 *   Limit: (segments the handle's split rows are cut into at the column ranges, one scratch row each)
 *   x (k rounded up to a multiple of 4) floats must fit 64 MiB = 16,777,216 floats,
 *   else CBM_ERR_UNSUPPORTED (cbm_last_error_detail gives the numbers); a handle without split rows
 *   (cbm_stats.num_split_rows == 0) always fits.  Where long rows share their popular columns in blocks
 *   (see max_depth) and that takes more scratch rows, the columns of X go through in several goes; so
 *   they do where shared sums need more.
 *   CBM_ERR_STATE while per-launch profiling is on (it creates events).
 * Every GPU the library runs on holds one such array until the process ends, and every call on that GPU
 * shares it, whatever the handle: calls that overlap in time on one GPU (two streams, two host threads, two
 * replayed graphs) race on it -- run them one after the other.  That holds for a handle without split rows too: where
 * its products take shared sums, these are written to the array.  Nothing in it has to be cleared between calls: a
 * product writes every scratch row and every sum it later reads.
 */
cbm_status cbm_spmm_noalloc(const cbm_handle* h, const float* X, int64_t ldx, int32_t k, float* Y, int64_t ldy,
                            void* hip_stream);

/*
 * cbm_reserve -- size the handle's split-row scratch for products of up to max_k columns now, so
 * that no later product with k <= max_k allocates (see cbm_spmm).  The handle's device must be
 * current.  A handle without split rows needs no scratch: the call then does nothing.
 */
cbm_status cbm_reserve(cbm_handle* h, int32_t max_k);

/*
 * cbm_release_captures -- the caller's word that no graph with products of this handle captured so far runs or will
 * be launched again (nor an instance updated from one): their arrays of sums (see cbm_spmm) are there for
 * later captures and streams.  For programs that capture anew many times in a handle's life; not while a capture with
 * products of the handle is under way.  A handle whose products take no shared sums has none: the call then does nothing.
 */
cbm_status cbm_release_captures(cbm_handle* h);

/*
 * cbm_spmm_normalized -- Y = D^-1/2 (A + I) D^-1/2 . X  (Eq. (1); Section 2.2,
 * "Extending SpMM with CBM to normalized adjacency matrices"), D = row sums of
 * A v I.  Same arguments as cbm_spmm.  Needs a square handle built with
 * add_self_loops, else CBM_ERR_STATE.  The column scale d_j^-1/2 is applied to
 * each gathered row of X, the row scale d_x^-1/2 when a row is written.
 */
cbm_status cbm_spmm_normalized(const cbm_handle* h, const float* X, int64_t ldx, int32_t k, float* Y,
                               int64_t ldy, void* hip_stream);

/* Same as cbm_spmm_normalized followed by an element-wise max(., 0): the
 * sigma(A_hat . Z) step of Eq. (1) with sigma = ReLU, fused into the row write. */
cbm_status cbm_spmm_normalized_relu(const cbm_handle* h, const float* X, int64_t ldx, int32_t k, float* Y,
                                    int64_t ldy, void* hip_stream);

/*
 * Two more aggregators of the GNN layers the paper names as targets (Section 1: GraphSAGE, GIN), as
 * epilogues of the same kernels; M is the compressed matrix (A, or A v I if built with add_self_loops).
 *   cbm_spmm_mean  Y = D^-1 M X, D = row sums of M: the mean of each row's entries (GraphSAGE's mean
 *                  aggregator); a row of M with no entry gives a zero row.
 *   cbm_spmm_gin   Y = M X + (1 + eps) X (GIN's aggregator); needs m == n.
 * Arguments as for cbm_spmm.  For a symmetric M the backward pass of all products here is the
 * same product applied to the output gradient (M^T = M).
 */
cbm_status cbm_spmm_mean(const cbm_handle* h, const float* X, int64_t ldx, int32_t k, float* Y, int64_t ldy,
                         void* hip_stream);
cbm_status cbm_spmm_gin(const cbm_handle* h, float eps, const float* X, int64_t ldx, int32_t k, float* Y, int64_t ldy,
                        void* hip_stream);

/*
 * cbm_dense_matmul -- C = A . B for dense row-major fp32 device matrices
 * (the X . W products of Eq. (1)), fp32 accumulation: on the fp32 matrix cores, or, where that is faster, on the bf16 ones
 * with each operand split into three bf16 parts that add up to it exactly (the products of parts that are left out are
 * below 2^-24 of a term).  Infinities, NaN and subnormal values are what they are in fp32.
 *   A  M x K (lda >= K),  B  K x N (ldb >= N),  C  M x N (ldc >= N), no overlap.
 */
cbm_status cbm_dense_matmul(int64_t M, int32_t N, int32_t K, const float* A, int64_t lda, const float* B,
                            int64_t ldb, float* C, int64_t ldc, void* hip_stream);

/*
 * cbm_gcn2_forward -- two-layer GCN inference, Eq. (1):
 *   out = A_hat . relu(A_hat . (X . W0)) . W1
 * evaluated as Z0 = X W0, H = relu(A_hat Z0), Z1 = H W1, out = A_hat Z1.
 *   X n x f_in, W0 f_in x hidden, W1 hidden x f_out, out n x f_out: device,
 *   row-major, densely packed (leading dimension = number of columns).
 *   workspace  device scratch of at least cbm_gcn2_workspace_bytes() bytes,
 *              caller-owned, 16-byte aligned.
 * X, W0, W1, the workspace and out must not overlap one another where one is written
 * (CBM_ERR_INVALID_ARG).  The handle's split-row scratch is sized for max(hidden, f_out)
 * before the first kernel is enqueued (as cbm_reserve does).
 */
cbm_status cbm_gcn2_forward(const cbm_handle* h, const float* X, int32_t f_in, const float* W0, int32_t hidden,
                            const float* W1, int32_t f_out, float* out, void* workspace, size_t workspace_bytes,
                            void* hip_stream);
size_t cbm_gcn2_workspace_bytes(const cbm_handle* h, int32_t f_in, int32_t hidden, int32_t f_out);

/*
 * What stands between the products of a training step.  Matrices here are row-major device matrices of one of three types with any
 * leading dimension (in elements, >= the row); statistics and the sums of gradients are fp32.  Pointers need the alignment of one element
 * (a workspace 16 bytes).  What is written must not overlap anything else of the same call (CBM_ERR_INVALID_ARG; also for
 * column slices interleaved in one buffer) unless the call says so.  The calls only enqueue kernels on the stream, allocate nothing and
 * keep nothing from one call to the next, so they can be captured and may overlap as long as they have workspaces of
 * their own; sums are added in a fixed order, so the same call gives the same bits.  n = 0 is a call without rows.  Rows of up to 2^24 columns.
 */
typedef enum { CBM_F32 = 0, CBM_BF16 = 1, CBM_F16 = 2 } cbm_dtype;

/*
 * cbm_layer_norm -- y = (x - m) r gamma + beta along each row, m = mean(x), r = (mean((x - m)^2) + eps)^-1/2.
 *   X, Y         n x k, of `type`.
 *   gamma, beta  k fp32 values each; NULL stands for ones, zeros.
 *   eps          >= 0 and finite.  A row of equal values has y = beta; with eps = 0 r = infinity and a y of NaN, as the formula says (both exactly for values
 *                of 2^-50 to 2^70 in size in rows of up to 2^16 columns: squares of what rounded sums leave of them are neither lost nor too large).
 *   mean, rstd   receive m and r (n fp32 values each), which the backward pass reads; either may be NULL.
 */
cbm_status cbm_layer_norm(int64_t n, int32_t k, int32_t type, const void* X, int64_t ldx, const float* gamma, const float* beta,
                          float eps, void* Y, int64_t ldy, float* mean, float* rstd, void* hip_stream);

/*
 * cbm_layer_norm_backward -- with h = (x - mean) rstd and u = dy gamma, along each row
 *   dX = rstd (u - mean(u) - h mean(u h)),  and over the rows  dgamma = sum(dy h),  dbeta = sum(dy).
 *   dY, X, dX    n x k, of `type`.  dX may be NULL (nothing before the layer learns).
 *   gamma        as forward; mean, rstd as the forward pass gave them.
 *   dgamma, dbeta  k fp32 values each, overwritten (zeros for n = 0); either may be NULL, not all three outputs.
 *   workspace    cbm_layer_norm_workspace_bytes(n, k) bytes; may be NULL where dgamma and dbeta are.
 */
cbm_status cbm_layer_norm_backward(int64_t n, int32_t k, int32_t type, const void* dY, int64_t lddy, const void* X, int64_t ldx,
                                   const float* gamma, const float* mean, const float* rstd, void* dX, int64_t lddx,
                                   float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t cbm_layer_norm_workspace_bytes(int64_t n, int32_t k);

/*
 * Activations kept in 8 bits until the backward pass.  Each 32 columns of a row (the last block of a row may be shorter) share a step 2^e:
 *   e = max(floor(log2(largest |x| of them)) - 6, -126);  q = sign(x) min(127, max(1, round-to-even(|x| 2^-e))), 0 for x = 0;  x~ = q 2^e.
 * So |x~ - x| <= 2^e (half of that but for the smallest values and the topmost 1 / 128 of a binade), x~ is never larger than its type's largest value, a
 * value other than zero keeps its sign, and x~ is a bf16 value.  A block with a value that is not finite comes back as NaN throughout.
 *   Q   n x k int8, leading dimension ldq >= k: the q.
 *   E   n x ceil(k / 32) uint8, leading dimension lde: e + 127; 255 for a block that is not finite (its q are 0).
 * k may be any number of columns; a row of Q may start at any byte.
 *   cbm_checkpoint_save           X (n x k, of `type`) -> Q, E.
 *   cbm_checkpoint_restore        Q, E -> X (rounded to `type`; exact in fp32 and bf16).
 *   cbm_checkpoint_relu_backward  dX = dY where q > 0, else 0 (n x k, of `type`; NaN in a block that is not finite): the backward pass of a
 *                                 ReLU whose output, or input, was kept.  dX may be dY itself with lddx = lddy.
 *   cbm_checkpoint_weight_grad    dW = X~^T dY (k x c, fp32, leading dimension lddw, overwritten; zeros for n = 0): the weights' gradient of Y = X W.
 *                                 dY n x c of `type`.  On the bf16 matrix cores with dY in parts that add up to it: exact products (parts
 *                                 below 2^-126 are taken for zero), fp32 sums.  workspace: cbm_checkpoint_workspace_bytes(n, k, c) bytes (may be 0).
 */
cbm_status cbm_checkpoint_save(int64_t n, int32_t k, int32_t type, const void* X, int64_t ldx, int8_t* Q, int64_t ldq, uint8_t* E,
                               int64_t lde, void* hip_stream);
cbm_status cbm_checkpoint_restore(int64_t n, int32_t k, const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int32_t type,
                                  void* X, int64_t ldx, void* hip_stream);
cbm_status cbm_checkpoint_relu_backward(int64_t n, int32_t k, const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int32_t type,
                                        const void* dY, int64_t lddy, void* dX, int64_t lddx, void* hip_stream);
cbm_status cbm_checkpoint_weight_grad(int64_t n, int32_t k, int32_t c, const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde,
                                      int32_t type, const void* dY, int64_t lddy, float* dW, int64_t lddw, void* workspace,
                                      size_t workspace_bytes, void* hip_stream);
size_t cbm_checkpoint_workspace_bytes(int64_t n, int32_t k, int32_t c);

/*
 * cbm_log_probs -- along each row z of scores, with m = max z, l = log sum exp(z - m) and log p = z - m - l:
 *   Z            n x c, of `type`.  A score of -infinity rules its class out.
 *   labels       n whole numbers of label_bits 32 or 64; a row whose label is outside [0, c) has none.  May be NULL where logp is.
 *   logp         log p[label], 0 for a row without a label.
 *   entropy      -sum p log p.
 *   stats        n x 2: m and l, which the backward pass reads.
 *   top          0 to 32 alternatives: top_values (n x top) receives the largest log p in descending order, top_columns (n x top) their classes, the
 *                lower one first among equal scores; where fewer classes are not ruled out, -infinity and -1.
 *   workspace    cbm_log_probs_workspace_bytes(n, c, top) bytes; 0 but for few rows of over 1,024 columns (those of over 49,152 are shared by several workgroups).
 * logp, entropy and stats may be NULL; fp32, packed.  A row with every class ruled out has m = l = log p[label] = -infinity and entropy 0.  A row
 * with NaN or +infinity has NaN for all of it (0 without a label, classes -1).
 *
 * cbm_log_probs_backward -- dZ = a (1[label] - p) - b p (log p + entropy), a = dlogp, the gradient of log p[label] (0 without a label), and
 * b = dentropy, that of the entropy.  labels may be NULL where dlogp is, entropy where dentropy is; one of the two gradients has to be there.
 * Zeros in a row with every class ruled out.  dZ (n x c, of `type`) may be Z itself with lddz = ldz.
 */
cbm_status cbm_log_probs(int64_t n, int32_t c, int32_t type, const void* Z, int64_t ldz, const void* labels, int32_t label_bits,
                         float* logp, float* entropy, float* stats, int32_t top, float* top_values, int32_t* top_columns,
                         void* workspace, size_t workspace_bytes, void* hip_stream);
size_t cbm_log_probs_workspace_bytes(int64_t n, int32_t c, int32_t top);
cbm_status cbm_log_probs_backward(int64_t n, int32_t c, int32_t type, const void* Z, int64_t ldz, const void* labels, int32_t label_bits,
                                  const float* stats, const float* entropy, const float* dlogp, const float* dentropy, void* dZ,
                                  int64_t lddz, void* hip_stream);

/*
 * cbm_gated_linear -- H = a(X Wg) o (X Wu), the gated layer (o: value by value), both projections, the activation and the product in one call:
 *   X            n x k, Wg and Wu k x m, H n x m, of `type`, any leading dimension.
 *   activation   a(g) = g / (1 + exp(-g)) (CBM_SILU), g Phi(g) with the normal distribution's Phi (CBM_GELU), max(g, 0) (CBM_RELU).
 *   G, U         receive X Wg and X Wu (n x m, of `type`), which the backward pass reads; either may be NULL.  H is made of the sums before they are rounded.
 *   workspace    cbm_gated_linear_workspace_bytes(n, k, m, type) bytes (may be 0).
 *
 * cbm_gated_linear_backward -- with dU = dH o a(G) and dG = dH o U o a'(G) (a'(0) = 0 for CBM_RELU), each rounded to `type` unless the products are small (fp16: at a power of two that puts the largest finite one between 2^3
 * and 65504, so that what is 2^-28 of it and less may be lost):
 *   dX = dG Wg^T + dU Wu^T (n x k),  dWg = X^T dG,  dWu = X^T dU (k x m), of `type`; each may be NULL, not all three.  dWg and dWu are zeros for n = 0.
 *   workspace    cbm_gated_linear_backward_workspace_bytes(n, k, m, type) bytes.
 *
 * Products of 16-bit types are exact, those of fp32 are made of three bf16 parts of each value (left out is at most 2^-24 of a term; parts below 2^-126 are taken for zero); sums
 * are fp32.  (Small products of fp32: in fp32 throughout.)  In fp32, a value that is not finite leaves no finite sum that it is part of, one from 2^127 on may leave none.
 * Workspaces hold copies of operands and shares of sums, or slopes in fp32, whatever the sizes ask for: a smaller call may need more than a larger one.
 * Up to 2^31 rows; CBM_ERR_UNSUPPORTED (and a workspace of 0 bytes) where a product has 2^24 tiles of 128 x 128 values or more: n x 2 m forward, n x k and k x 2 m backward.
 */
typedef enum { CBM_SILU = 0, CBM_GELU = 1, CBM_RELU = 2 } cbm_activation;
cbm_status cbm_gated_linear(int64_t n, int32_t k, int32_t m, int32_t type, int32_t activation, const void* X, int64_t ldx, const void* Wg, int64_t ldwg,
                            const void* Wu, int64_t ldwu, void* H, int64_t ldh, void* G, int64_t ldg, void* U, int64_t ldu, void* workspace,
                            size_t workspace_bytes, void* hip_stream);
size_t cbm_gated_linear_workspace_bytes(int64_t n, int32_t k, int32_t m, int32_t type);
cbm_status cbm_gated_linear_backward(int64_t n, int32_t k, int32_t m, int32_t type, int32_t activation, const void* dH, int64_t lddh, const void* X,
                                     int64_t ldx, const void* Wg, int64_t ldwg, const void* Wu, int64_t ldwu, const void* G, int64_t ldg, const void* U,
                                     int64_t ldu, void* dX, int64_t lddx, void* dWg, int64_t lddwg, void* dWu, int64_t lddwu, void* workspace,
                                     size_t workspace_bytes, void* hip_stream);
size_t cbm_gated_linear_backward_workspace_bytes(int64_t n, int32_t k, int32_t m, int32_t type);

/*
 * cbm_linear_log_probs -- cbm_log_probs of the scores Z = X W of many classes, without Z in memory: along each row z of it, with m = max z and
 * l = log sum exp(z - m), log p = z - m - l.
 *   X            n x d, W d x c, of `type`.  Products and sums as for cbm_gated_linear; Z is not rounded.
 *   labels, label_bits, logp, stats   as for cbm_log_probs (log p[label], 0 without a label; m and l); logp and stats may be NULL, labels where logp is.
 *   workspace    cbm_linear_log_probs_workspace_bytes(n, d, c, type) bytes: up to 512 MiB of maxima and sums, by rows, and copies of operands.
 * A row with a score of NaN or +infinity has NaN for all of it (0 without a label).
 *
 * cbm_linear_log_probs_backward -- with dZ = dlogp (1[label] - p), and nothing for rows without a label or a distribution (m of -infinity), whatever dlogp has there; rounded to `type` unless the products are
 * small (16 bits: at 2^15 over the largest finite |dlogp| of the other rows of its size, so that in fp16 what is 2^-40 of that and less is lost),
 *   dX = dZ W^T (n x d),  dW = X^T dZ (d x c; zeros for n = 0), of `type`; either may be NULL.  Values of X must be finite in rows without a label, too.
 *   The scores are made again from X and W, a piece of the classes at a time, with m and l from `stats`.
 *   workspace    cbm_linear_log_probs_backward_workspace_bytes(n, d, c, type) bytes: dZ of a piece (512 MiB or 1,024 classes), and sums.
 *                CBM_ERR_UNSUPPORTED (and 0 bytes) where a product, n x the classes of a piece, n x d or d x those, has 2^24 tiles of 128 x 128 values or more.
 */
cbm_status cbm_linear_log_probs(int64_t n, int32_t d, int32_t c, int32_t type, const void* X, int64_t ldx, const void* W, int64_t ldw, const void* labels,
                                int32_t label_bits, float* logp, float* stats, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t cbm_linear_log_probs_workspace_bytes(int64_t n, int32_t d, int32_t c, int32_t type);
cbm_status cbm_linear_log_probs_backward(int64_t n, int32_t d, int32_t c, int32_t type, const void* X, int64_t ldx, const void* W, int64_t ldw,
                                         const void* labels, int32_t label_bits, const float* stats, const float* dlogp, void* dX, int64_t lddx, void* dW,
                                         int64_t lddw, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t cbm_linear_log_probs_backward_workspace_bytes(int64_t n, int32_t d, int32_t c, int32_t type);

/*
 * cbm_orthogonalise -- the update that a weights' gradient X (m x n, of `type`) stands for where all its directions are to count alike: with
 * Z = X / (|X| + eps), |X| the root of the sum of squares, and `steps` times
 *   A = Z Z^T,  Z <- a Z + (b A + c A^2) Z        (of Z^T where m > n, which is the same),
 * Y = scale Z (of `type`).  Five steps with the usual coefficients bring singular values from 1 / 500 of |X| up to between 0.7 and 1.2.
 *   steps          0 to 100.  coefficients: a, b and c, on the host; NULL stands for 3.4445, -4.7750, 2.0315.
 *   eps            >= 0 and finite; a matrix of zeros stays one with eps > 0, and is NaN with eps = 0.
 *   Y              may be X itself with ldy = ldx.
 *   workspace      cbm_orthogonalise_workspace_bytes(m, n, type) bytes.
 * m and n up to 65,536.  Between X and Y values are held in two parts of 16 bits each, 22 bits together, at powers of two that follow from the coefficients; sums are fp32.  (A value of Z is held to 2^-38 at
 * best: where eps is far above |X|, so that Z is small, it and Y keep as many bits fewer as its values are below 2^-16.)  Coefficients are refused
 * (CBM_ERR_UNSUPPORTED) where, on what the steps before may make of [0, 1], |a + b s^2 + c s^4| passes 16 |a| or 2^100, or s passes 2^24.  A value that is not finite makes NaN of all of Y.
 */
cbm_status cbm_orthogonalise(int32_t m, int32_t n, int32_t type, const void* X, int64_t ldx, int32_t steps, const float* coefficients, float eps, float scale,
                             void* Y, int64_t ldy, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t cbm_orthogonalise_workspace_bytes(int32_t m, int32_t n, int32_t type);

/* Counters of the built format (Properties 1 and 2, Lemma 2.2). */
cbm_status cbm_stats(const cbm_handle* h, cbm_stats_t* out);

/*
 * cbm_get_tree -- the chain of compression, host arrays of m entries each (any
 * may be NULL): parent[x] = row that x is compressed against, -1 for the virtual
 * null row; nplus / nminus = |Delta+|, |Delta-| of the edge (parent[x], x);
 * level[x] = depth of x, 1 for rows stored in full.  For a column-blocked handle (column_blocks = B > 1)
 * every array has B m entries: entry b m + i is the part of row i inside column range b, and parents are
 * part-row indices.
 */
cbm_status cbm_get_tree(const cbm_handle* h, int32_t* parent, int32_t* nplus, int32_t* nminus, int32_t* level);

/*
 * cbm_decompress -- rebuild the compressed matrix from the tree and the delta
 * lists alone, a_x = (a_y u Delta+) \ Delta- (Eq. (2)).  Host outputs: rowptr
 * (m + 1) and colidx (stats.nnz entries, sorted within rows).  Returns A v I
 * when the handle was built with add_self_loops.
 */
cbm_status cbm_decompress(const cbm_handle* h, int64_t* rowptr, int32_t* colidx);

/*
 * Per-launch timing of the product kernels.  With profiling on, every kernel a
 * product call enqueues is bracketed by HIP events on the caller's stream.
 * on = 1 changes what is launched: segments of split rows and rows stored in full,
 * which share a launch otherwise, are launched one after the other (kinds 1 and 0), so
 * that each has a time.  on = 2 leaves the launches as they are (kind 7 where the two
 * share one).  The results are the same.
 * After synchronising the stream, cbm_profile_read returns, for the most
 * recent product call, up to `cap` records and the total count in *count.
 */
typedef struct {
    int32_t kind;           /* 0 = gather/update round, 1 = segments of split rows,
                               2 = split-row combine, 3 = deferred finish of rows that
                               other work items read (row weight, self term, ReLU),
                               4 = sum of the partial rows of a column-blocked handle,
                               5 = row blocks: the whole product, or the popular columns of
                               split rows (tasks = blocks, deltas = columns gathered, each
                               once per block), 6 = shared sums: level 1 the sets, level 2
                               the rows made of them, level 3 rows that sum their sets in place
                               (tasks = sets or rows, deltas = rows of X and sums gathered),
                               7 = segments of split rows and rows stored in full (on = 2) */
    int32_t level;          /* round for kinds 0, 2 and 7, launch for kind 6, else 0   */
    int64_t tasks;          /* work items in the launch                               */
    int64_t deltas;         /* delta entries gathered by the launch                   */
    int64_t algorithmic_bytes; /* bytes the method itself must move in this launch    */
    float milliseconds;
    int32_t per_xcd;        /* 1 = the launch hands every XCD a work list of its own (segments
                               by column range; a round in graph-locality order), else 0     */
} cbm_launch_record;
cbm_status cbm_profile_enable(cbm_handle* h, int32_t on); /* 0 off, 1 (or any other value) apart, 2 as they are */
cbm_status cbm_profile_read(cbm_handle* h, cbm_launch_record* records, int32_t cap, int32_t* count);

void cbm_free(cbm_handle* h); /* NULL-safe; releases everything the handle owns */
const char* cbm_status_string(cbm_status s);
/* Text naming the HIP call and runtime error behind the calling thread's most recent
 * CBM_ERR_HIP / CBM_ERR_ALLOC ("" if none).  Valid until that thread's next failing call. */
const char* cbm_last_error_detail(void);

#ifdef __cplusplus
}
#endif
#endif /* CBM_H */
