/*
 * libstream: C ABI of the B200 (sm_100a) implementation of Stream sparse-mask estimation and
 * the block-sparse attention pass that consumes the mask.
 *
 * Conventions for every entry point
 *   - Plain C types only. Unless a parameter says HOST, every data pointer is a DEVICE pointer
 *     owned by the caller; the library never allocates or frees device memory. The state it
 *     keeps between calls is: the thread-local error text; per device, the two copy streams and
 *     the events of stream_run_host (created at its first call, kept until the process ends);
 *     per device, the built-in scratch array of stream_build_mask_static and its address; and
 *     the status words of the tensor-core attention kernels (stream_check_device_status).
 *   - Work is enqueued on `cuda_stream` (a cudaStream_t passed as void*; NULL = default stream)
 *     and the call returns after enqueue unless stated otherwise.
 *   - Every failure is a returned status; nothing aborts or throws. Arguments are validated on
 *     the host before anything is launched. stream_last_error() gives the text of the last
 *     failure on the calling thread.
 *   - Tensors: Q is [batch, n_q_heads, T, d], K and V are [batch, n_kv_heads, T, d], addressed
 *     with the element strides in the problem struct (innermost stride 1). Query head h reads
 *     kv head h / (n_q_heads / n_kv_heads). dtype is fp32 or bf16 for Q, K, V and the attention
 *     output alike. Inputs must be finite, all of them: a kernel may multiply keys and values
 *     that a row does not keep by a weight of zero (the tcgen05 and mma.sync kernels do), and zero
 *     times an infinity or a NaN is a NaN.
 *   - A "row" is one (batch, query head, query block); there are ceil(T / block_q) query
 *     blocks. The mask is int32 [batch, n_q_heads, ceil(T / block_q), k_top], contiguous: per
 *     row the kept key-block indices (0-based; block r covers tokens r*block_k ..), strictly
 *     ascending, then -1 padding.
 */
#ifndef STREAM_H_
#define STREAM_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    STREAM_OK = 0,
    STREAM_ERR_INVALID_ARG = 1, /* null pointer, non-positive size, bad stride, bad enum */
    STREAM_ERR_UNSUPPORTED = 2, /* valid request that no kernel here covers (see stream_problem) */
    STREAM_ERR_WORKSPACE = 3,   /* workspace or staging buffer missing, misaligned or too small */
    STREAM_ERR_CUDA = 4,        /* a CUDA runtime/driver call failed; text in stream_last_error */
    STREAM_ERR_DEVICE_CHECK = 5 /* a kernel gave up on a bounded wait or met an out-of-range mask
                                   entry; see stream_read_stats */
} stream_status;

typedef enum { STREAM_F32 = 0, STREAM_BF16 = 1 } stream_dtype;

typedef enum {
    STREAM_IMPL_AUTO = 0,    /* tcgen05 kernels when the shape allows, else mma.sync for bf16 with d in
                                {64, 128, 256} and 16-byte aligned rows, else the generic ones */
    STREAM_IMPL_GENERIC = 1, /* fp32-FMA kernels: any dtype, d in {16,32,64,128,256}, blocks 1..64 */
    STREAM_IMPL_TENSOR = 2   /* tcgen05 kernels only: bf16, d = 128, block_q = block_k = 64, strides
                                that are multiples of 8 elements, 16-byte aligned pointers (and
                                k_top <= 32 for the mask build); the mask build also takes
                                block_q = 1 (per-token masks) with block_k = 64, one k, and at most
                                32768 key blocks; otherwise STREAM_ERR_UNSUPPORTED */
} stream_impl;

typedef struct {
    int32_t batch;          /* independent problems (e.g. layers); >= 1 */
    int32_t n_q_heads;      /* >= 1 */
    int32_t n_kv_heads;     /* >= 1 and divides n_q_heads */
    int64_t T;              /* tokens, >= 1; need not be a multiple of the block sizes */
    int32_t d;              /* head dimension: 16, 32, 64, 128 or 256 */
    int32_t block_q;        /* b_q */
    int32_t block_k;        /* b_k */
    int32_t k_top;          /* k: key blocks kept per query block = row width of the mask; 1..1024 */
    int32_t causal;         /* 1: C is lower triangular; 0: C is all ones (Algorithm 1) */
    int32_t dtype;          /* stream_dtype */
    int32_t impl;           /* stream_impl */
    int64_t q_stride_b, q_stride_h, q_stride_t;    /* elements */
    int64_t kv_stride_b, kv_stride_h, kv_stride_t; /* elements; K and V share them */
} stream_problem;

/* Counters a mask build leaves in the first bytes of its workspace. */
typedef struct {
    uint64_t tiles_scored; /* (row, representative key block) tiles that the method scores. (A row with no more
                              allowed blocks than k keeps them all whatever their scores: where these are
                              not asked for it may be written without computing them. Its tiles
                              are counted all the same.) */
    uint64_t rows;         /* rows finished */
    uint32_t error;        /* 0, or a code saying which bounded wait ran out (kernel returned early) */
    uint32_t error_info;
    uint64_t tile_products; /* 64 x 64 x d tile products the per-token tensor-core kernel computed (it
                               multiplies every fetched key tile with 128 tokens at once, so this exceeds
                               what its tokens' scored tiles / 64 would be; none for groups of tokens
                               that keep all they may); 0 from the other kernels, whose products are
                               the tiles scored, but for rows written without them */
    uint64_t tiles_fetched; /* key and query tiles (block x d) the tensor-core block kernel copied into
                               shared memory: fewer than tiles_scored where a fetched key tile serves
                               several rows, none for rows written without products; 0 from the
                               kernels that do not count them */
} stream_stats;

/* Library version: major * 10000 + minor * 100 + patch. */
int stream_version(void);

/* Text of the most recent failure on this thread ("" if none). The pointer stays valid until the
 * thread's next failing call. */
const char *stream_last_error(void);

/*
 * Bytes of device workspace stream_build_mask needs for this problem (a small header holding
 * stream_stats and the work counter of the persistent kernels; O(1), never grows with T).
 * Returns 0 if the problem is invalid or unsupported.
 */
size_t stream_workspace_bytes(const stream_problem *p);

/*
 * Stream mask estimation (Algorithm 2 of the paper; Algorithm 1 when causal == 0).
 *
 * For every row: start from k_top nodes tiling the N_k key blocks, and for ceil(log2 N_k) levels
 * split every node in two, score each branch by the masked maximum token-level dot product
 * (Eq. 4) between the query block and the branch's first allowed key block, keep the k_top best
 * branches (higher fp32 score, then lower block index), and finally emit the first allowed block
 * of every surviving node. Levels that cannot change the result (all nodes single blocks) are
 * skipped, and a left branch reuses its parent's score (same tile, same value).
 *
 *   q, k       device, dtype of the problem, strided as described above; read only
 *   mask_out   device int32 [batch, n_q_heads, ceil(T/block_q), k_top]; fully overwritten
 *   score_out  device float32, same shape, or NULL: block score of every kept block, -inf padded
 *   workspace  device, 256-byte aligned, >= stream_workspace_bytes(p); overwritten. After the
 *              stream has drained, stream_read_stats(workspace, ...) returns this call's counters.
 *              If workspace_bytes >= stream_workspace_bytes(p) + 4 * rows (rows = batch *
 *              n_q_heads * ceil(T/block_q)), the build also writes, as uint32 [rows] right behind
 *              the first stream_workspace_bytes(p) bytes, how many tiles each row scored (their
 *              sum is stream_stats.tiles_scored). stream_build_mask and stream_build_mask_var only.
 *
 * Errors: INVALID_ARG, UNSUPPORTED, WORKSPACE before any launch; CUDA if a launch fails.
 */
stream_status stream_build_mask(const stream_problem *p, const void *q, const void *k, int32_t *mask_out,
                                float *score_out, void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * stream_build_mask with a sparsity constant of its own for every query block ("variable k": the
 * paper's discussion of needle depth, Section 4.2, and the fourth item of its Limitations name it
 * as the remedy for the stronger pruning of late rows under a causal mask, and leave it
 * undefined). The reading taken: the row of query block qb is Algorithm 2, unchanged, run with
 * k = k_row[qb]; rows stay k_top wide (the row's blocks ascending, then -1; scores -inf padded),
 * so the result feeds stream_sparse_attention, stream_vertical_scores and stream_mask_difference
 * as it is.
 *
 *   k_row      device int32 [ceil(T/block_q)], shared by all heads and batch entries; read only.
 *              Entries outside 1 .. k_top are clamped into that range.
 * Everything else as stream_build_mask (p->k_top is the row width and the largest k).
 */
stream_status stream_build_mask_var(const stream_problem *p, const void *q, const void *k, const int32_t *k_row,
                                    int32_t *mask_out, float *score_out, void *workspace, size_t workspace_bytes,
                                    void *cuda_stream);

/*
 * The masks of the same inputs for several sparsity constants in one call: the search over k of
 * Section 3 (binary search for the smallest k that keeps the model's behaviour) and the
 * k_success / k_fail comparison of Section 4.2 need them. Mask i is Algorithm 2 with
 * k = k_list_host[i]. A block's score does not depend on k, so where the kernel can keep a row's
 * scores (the generic kernel, while ceil(T/block_k) floats fit in shared memory beside its tiles)
 * every (row, block) tile is scored once for all k. The tensor-core kernel does the same when the
 * workspace has room for its score memory (stream_workspace_bytes_multi: 8 bytes per key block, row
 * of a group and SM, i.e. O(T)); with only stream_workspace_bytes it is launched once per k and
 * shares nothing. stream_read_stats then reports the tiles actually scored over the whole call.
 *
 *   n_k          1 .. 8
 *   k_list_host  HOST int32 [n_k], each 1 .. p->k_top (p->k_top is the row width), any order
 *   mask_out     device int32 [n_k, batch, n_q_heads, ceil(T/block_q), k_top]; mask i is one
 *                contiguous slab, its rows -1 padded beyond k_list_host[i] entries
 *   score_out    device float32, same shape, or NULL
 * Everything else, and the errors, as stream_build_mask.
 */
size_t stream_workspace_bytes_multi(const stream_problem *p, int32_t n_k);  /* 0 = invalid problem or n_k */
stream_status stream_build_mask_multi(const stream_problem *p, const void *q, const void *k, int32_t n_k,
                                      const int32_t *k_list_host, int32_t *mask_out, float *score_out, void *workspace,
                                      size_t workspace_bytes, void *cuda_stream);

/*
 * A schedule for stream_build_mask_var, computed on the host: the effective-sparsity formula of
 * Section 4.2, k = floor(1 + (n - 1) s), applied per query block with n = the number of key
 * blocks that row may look at (qb + 1 blocks under a causal mask with equal block sizes; the
 * paper applies the formula once, with n = T / b_q, which is what prunes late rows harder).
 * Clamped to 1 .. p->k_top.
 *
 *   s           0 < s < 1, else INVALID_ARG
 *   k_row_host  HOST int32 [ceil(T/block_q)], overwritten; copy it to the device for the build
 */
stream_status stream_k_schedule(const stream_problem *p, double s, int32_t *k_row_host);

/*
 * The effective-sparsity formula of Section 4.2 as printed: k = floor(1 + (T / b_q - 1) s), kept
 * inside k's range 1 .. floor(T / b_q) (at least 1). T / b_q is taken as the real quotient. As
 * printed, a larger s keeps MORE blocks (the prose beside the formula says the opposite; the
 * formula is followed). Host-only arithmetic; nothing is launched.
 *
 *   s           0 <= s <= 1, else INVALID_ARG
 *   k_out_host  HOST int32, one value
 */
stream_status stream_effective_k(int64_t T, int32_t block_q, double s, int32_t *k_out_host);

/*
 * stream_build_mask without a caller-provided workspace and without any allocation. (The paper
 * has no counterpart to this entry point; it exists for deployment.)
 *
 * For callers that cannot get device memory when they call: a host application that reserved all
 * of HBM for its own pool at start-up, or a latency-critical loop that must not hit the implicit
 * synchronisation of cudaMalloc / cudaFree. The kernel's scratch (work counter and counters, see
 * stream_stats) lives in a 4096-byte device array built into the library, which each GPU that
 * loads the library holds until the process exits. Same arguments, results and errors as
 * stream_build_mask otherwise (an invalid or unsupported problem gets exactly the status
 * stream_build_mask gives it); a problem whose scratch need exceeded 4096 bytes would be refused
 * with STREAM_ERR_WORKSPACE (no current problem does). The call allocates and frees nothing.
 *
 *   - The first call on each device looks up the array's device address (a one-time host-side
 *     query, made with that device current). Make that first call outside any stream capture.
 *   - All calls on a device share the one array and it keeps the previous call's contents; each
 *     call clears what it needs on `cuda_stream` before its kernel. Two calls that can overlap on
 *     the GPU (different streams, no dependency) race on it: serialise them, or give the
 *     overlapping calls stream_build_mask with workspaces of their own.
 *   - The counters are not readable through this entry point.
 */
stream_status stream_build_mask_static(const stream_problem *p, const void *q, const void *k, int32_t *mask_out,
                                       float *score_out, void *cuda_stream);

/*
 * Block-sparse attention under a Stream mask (Eq. 2 of the paper; the product QK^T * C * M of
 * Figure 1): for every query token, softmax(scale * q.k) over the keys of the row's kept blocks
 * that C allows (element-level causal test inside a block, keys beyond T excluded), times V.
 * Softmax statistics and the output accumulate in fp32; a token that no kept key is allowed for
 * gets zeros.
 *
 *   q, k, v    device, dtype of the problem; read only
 *   mask       device int32 [batch, n_q_heads, ceil(T/block_q), k_top] as written by
 *              stream_build_mask; entries < 0 are skipped; valid entries must be < ceil(T/block_k)
 *   scale      logit scale; <= 0 selects 1/sqrt(d)
 *   out        device, dtype of the problem, contiguous [batch, n_q_heads, T, d]; overwritten
 */
stream_status stream_sparse_attention(const stream_problem *p, const void *q, const void *k, const void *v,
                                      const int32_t *mask, float scale, void *out, void *cuda_stream);

/*
 * Vertical attention scores of a mask and their kurtosis (Section 4.1 of the paper: the column
 * sums of a head's sparse mask show which key blocks attract the later queries; heads whose
 * vertical scores have a high kurtosis are the "receiver heads").
 *
 *   vertical[b, h, r] = sum over the head's query blocks q and slots j with mask[b, h, q, j] == r
 *                       of scores[b, h, q, j]   (of 1 if scores is NULL: the binary mask)
 *   kurtosis[b, h]    = m4 / m2^2 of vertical[b, h, :], m2 and m4 the second and fourth central
 *                       moments over the ceil(T / block_k) key blocks (Pearson, not excess); 0
 *                       if all vertical scores of the head are equal
 *
 *   mask          device int32 [batch, n_q_heads, ceil(T/block_q), k_top]; entries < 0 are skipped
 *   scores        device float32, same shape (score_out of stream_build_mask), or NULL; -inf
 *                 padding is never read because its mask entry is < 0
 *   vertical_out  device float32 [batch, n_q_heads, ceil(T/block_k)]; overwritten
 *   kurtosis_out  device float32 [batch, n_q_heads], or NULL
 *   workspace     as for stream_build_mask; stream_read_stats afterwards returns
 *                 STREAM_ERR_DEVICE_CHECK if a mask entry was >= ceil(T/block_k) (such entries
 *                 are ignored). Sums are fp32 and added in no fixed order.
 * Only T, block_k, block_q, k_top, batch and n_q_heads of *p matter. Up to 49152 key blocks per
 * head; more gives STREAM_ERR_UNSUPPORTED.
 */
stream_status stream_vertical_scores(const stream_problem *p, const int32_t *mask, const float *scores, float *vertical_out,
                                     float *kurtosis_out, void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Mask subtraction (Section 4.2 of the paper, "Exploring Information Flow": the sparse masks
 * found with a smaller budget k are subtracted from those found with a larger one; what is left,
 * weighted by the larger mask's block scores, are the connections only the larger budget keeps).
 * Row by row: the entries of mask_a that are >= 0 and do not occur in the same row of mask_b, in
 * mask_a's order, then -1 padding (their scores, then -inf padding).
 *
 *   n_rows           rows of both masks (batch * n_q_heads * query blocks)
 *   mask_a, mask_b   device int32 [n_rows, k_a] and [n_rows, k_b], 1 <= k_a, k_b <= 1024; any order
 *   scores_a         device float32 [n_rows, k_a] or NULL
 *   diff_out         device int32 [n_rows, k_a]; overwritten; must not alias the inputs
 *   diff_scores_out  device float32 [n_rows, k_a] or NULL (needs scores_a)
 */
stream_status stream_mask_difference(int64_t n_rows, int32_t k_a, const int32_t *mask_a, const float *scores_a, int32_t k_b,
                                     const int32_t *mask_b, int32_t *diff_out, float *diff_scores_out, void *cuda_stream);

/*
 * Synchronous read-back of the counters left by the last stream_build_mask that used this
 * workspace. Waits for `cuda_stream` to drain, copies the header to *out (HOST pointer) and
 * returns STREAM_ERR_DEVICE_CHECK if the kernel recorded a failed device-side check (a bounded
 * wait that ran out; an out-of-range mask entry in stream_vertical_scores).
 */
stream_status stream_read_stats(const void *workspace, stream_stats *out, void *cuda_stream);

/*
 * Synchronous health check of the kernels that have no workspace to report into (the tensor-core
 * attention kernel). Waits for `cuda_stream` to drain and returns STREAM_ERR_DEVICE_CHECK if, on
 * the current device and since the library was loaded, such a kernel gave up on one of its
 * bounded waits and left early (its output is then incomplete); STREAM_OK otherwise.
 */
stream_status stream_check_device_status(void *cuda_stream);

/*
 * Diagnostic (the paper has no counterpart): runs the bounded wait that every mbarrier wait of the
 * tensor-core kernels goes through to its limit once, in a one-warp kernel of its own that waits
 * on a barrier nothing arrives at, with no copy or tensor-core operation in flight. After
 * limit_cycles SM clock cycles the wait gives up exactly as it would in a product kernel: it
 * records code 901 in the workspace header, raises the abort flag, all lanes leave together and
 * the kernel returns. stream_read_stats(workspace, ...) then returns STREAM_ERR_DEVICE_CHECK with
 * error = 901 (rows = 0: the wait did not succeed; tiles_scored = 1: the abort flag was raised).
 * The product kernels use the same code path with a limit of 2^31 cycles (about a second).
 *
 *   limit_cycles  1 .. 2^31, else INVALID_ARG
 *   workspace     device, 256-byte aligned, >= 256 bytes; overwritten
 */
stream_status stream_selftest_bounded_wait(int64_t limit_cycles, void *workspace, size_t workspace_bytes,
                                           void *cuda_stream);

/* What stream_probe_unit_rates measured. */
typedef struct {
    double tma_bytes_per_clk;   /* bytes per SM clock that one SM's TMA unit brought from L2 into its shared
                                   memory (16 KiB bulk copies of L2-resident data, two issuing warps with
                                   four copies in flight each, every SM busy at once; CTA 0's figure) */
    double mma_cycles_m128n64;  /* SM clocks per tcgen05.mma of M = 128, N = 64, K = 16, bf16, shared-memory
                                   operands, issued back to back (32 would be the tensor core's own time) */
    uint32_t error;             /* 0, or the code of a bounded wait that ran out (911 copies, 912 MMAs) */
    uint32_t reserved;
} stream_unit_rates;

/*
 * Measurement aid (the paper has no counterpart): the two unit rates that bound the tensor-core
 * mask and attention kernels on the device at hand, so that a measured throughput can be set
 * against what the SM delivers rather than against a data-sheet figure. Launches two short
 * kernels (one CTA per SM, a few hundred microseconds), waits for `cuda_stream` and fills
 * *out_host. Every wait inside is bounded like the product kernels' (STREAM_ERR_DEVICE_CHECK and
 * out_host->error if one ran out).
 *
 *   scratch       device, 256-byte aligned, >= stream_probe_scratch_bytes(); overwritten (zeros:
 *                 the source of the copies and a result record)
 *   out_host      host
 */
size_t stream_probe_scratch_bytes(void);
stream_status stream_probe_unit_rates(void *scratch, size_t scratch_bytes, stream_unit_rates *out_host, void *cuda_stream);

/*
 * Bytes of device staging stream_run_host and stream_run_host_var need: room for Q, K, V, the mask,
 * the output, the mask workspace and one k per query block, each 256-byte aligned. 0 if the problem
 * is invalid or unsupported.
 */
size_t stream_host_staging_bytes(const stream_problem *p);

/*
 * The whole path from HOST memory: copy Q, K, V to the device, build the mask, run the sparse
 * attention, copy mask and output back. Strides in *p describe the HOST tensors, which must be
 * dense ([batch, heads, T, d] contiguous). The work is cut into one chunk per (batch entry, kv
 * head) - nothing else depends on a chunk - and chunk c + 1's copy in, chunk c's kernels and
 * chunk c - 1's copy out run at the same time: the copies on two streams the library creates
 * once per device at the first call (with a few events; kept until the process ends), the
 * kernels on cuda_stream. Pinned host memory is what makes the copies asynchronous.
 *
 *   q_host, k_host, v_host   HOST, read only
 *   mask_host                HOST int32 [batch, n_q_heads, ceil(T/block_q), k_top]
 *   out_host                 HOST, dtype of the problem, [batch, n_q_heads, T, d]
 *   staging                  DEVICE, 256-byte aligned, >= stream_host_staging_bytes(p)
 * Everything is ordered after what cuda_stream already holds, and cuda_stream is made to wait
 * for the last copy out: the host buffers are valid once cuda_stream has been synchronised. Two
 * calls that share a device must not overlap in time (they share the internal streams' events).
 */
stream_status stream_run_host(const stream_problem *p, const void *q_host, const void *k_host, const void *v_host,
                              int32_t *mask_host, void *out_host, float scale, void *staging,
                              size_t staging_bytes, void *cuda_stream);

/*
 * stream_run_host with a sparsity constant of its own for every query block (the variable-k build
 * of stream_build_mask_var, Section 4.2's remedy for the harder pruning of late rows, followed by
 * the sparse attention on its masks), from HOST memory and pipelined the same way.
 *
 *   k_row_host   HOST int32 [ceil(T/block_q)], e.g. from stream_k_schedule; entries outside
 *                1 .. k_top are clamped. It is copied to the staging buffer ahead of the first chunk.
 * Everything else as stream_run_host (same staging size).
 */
stream_status stream_run_host_var(const stream_problem *p, const void *q_host, const void *k_host, const void *v_host,
                                  const int32_t *k_row_host, int32_t *mask_host, void *out_host, float scale, void *staging,
                                  size_t staging_bytes, void *cuda_stream);

/*
 * ------------------------------------------------------------------------------------------------
 * Dense attention, and the key-value cache of chains that are being generated: what the masks and the
 * sparse pass above are set against, the layers that stay dense, and how the chains that are traced
 * come about (one prompt, several chains forked from it, one token after the other).
 * ------------------------------------------------------------------------------------------------
 */

/* Prompts packed one behind the other. Q is [total_q, n_q_heads, d], K and V are [total_k, n_kv_heads, d]
 * (innermost stride 1, K and V share their strides). */
typedef struct {
    int32_t n_seqs;         /* >= 1 */
    int32_t n_q_heads;      /* >= 1 */
    int32_t n_kv_heads;     /* >= 1 and divides n_q_heads */
    int32_t d;              /* 16, 32, 64, 128 or 256 */
    int64_t total_q;        /* rows of Q and of the output, 0 .. 2^31 - 4096 */
    int64_t total_k;        /* rows of K and V, 0 .. 2^31 - 4096 */
    int32_t causal;         /* 1: a sequence's last query sees all its keys, the one before it all but the last, ...; 0: all see all */
    int32_t dtype;          /* stream_dtype */
    int64_t q_stride_t, q_stride_h, kv_stride_t, kv_stride_h; /* elements; a stride whose extent is 1 does not matter */
} stream_prompt;

/*
 * Attention of whole prompts. Sequence s has the queries cu_q[s] .. cu_q[s+1] - 1 and the keys
 * cu_k[s] .. cu_k[s+1] - 1; with n queries and m keys, query i sees the keys j <= i + m - n if causal
 * (m > n: a prompt whose first part was computed before; m < n: the first n - m queries see nothing).
 *     out[i, h] = sum_j softmax_j(scale q_i.k_j) v_j,     lse[h, i] = log sum_j exp(scale q_i.k_j)
 * A query that sees nothing gets zeros and -inf. What K and V hold outside a query's own sequence, or beyond
 * the last one, does not matter, whatever it is (NaN included); Q, K and V of the sequences must be finite, and the logits in fp32, times log2(e).
 *
 *   q, k, v     device, read only
 *   cu_q, cu_k  device int32 [n_seqs + 1], ascending; an entry outside 0 .. total_q (total_k) counts as the nearest
 *               inside, and a sequence whose end lies before its beginning is empty
 *   scale       logit scale, up to 2.3e38 (fp32 holds scale log2(e)); <= 0 selects 1/sqrt(d)
 *   out         device, dtype of the problem, contiguous [total_q, n_q_heads, d]; rows of no sequence stay as they are. Must
 *               not overlap an input
 *   lse_out     device float32 [n_q_heads, total_q] or NULL; likewise
 * Softmax statistics and the output accumulate in fp32, with weights of up to 2^30 before the division by their sum: |V| up to
 * 2^64 cannot overflow, whatever the logits and the length.
 */
stream_status stream_prompt_attention(const stream_prompt *p, const void *q, const void *k, const void *v, const int32_t *cu_q,
                                      const int32_t *cu_k, float scale, void *out, float *lse_out, void *cuda_stream);

/* A paged key-value cache. Token t of the sequence in slot s lies in row t % page_size of page
 * page_table[s][t / page_size]; K and V are each [n_layers, n_pages, page_size, n_kv_heads, d] with the
 * strides below (in elements; innermost 1; K and V share them; any order of the dimensions).
 *
 * The ledger, three device arrays that all layers share and only the calls below change:
 *   page_table  int32 [n_slots, max_pages]: a slot's first ceil(seq_len / page_size) entries are pages, the rest -1
 *   seq_len     int32 [n_slots]: tokens, 0 = the slot is empty
 *   ref_count   int32 [n_pages]: how many entries of the table name the page, 0 = it is free
 * A new cache has -1, 0 and 0 everywhere. A page that is not full belongs to one slot alone (a fork copies it);
 * full pages may be shared, and are not written again. The lowest-numbered free pages are taken first. */
typedef struct {
    int32_t n_slots;        /* 1 .. 2^30; n_slots * max_pages < 2^31 */
    int32_t n_pages;        /* 1 .. 2^30 */
    int32_t page_size;      /* tokens; >= 1; max_pages * page_size <= 2^31 - 4096 */
    int32_t max_pages;      /* >= 1 */
    int32_t n_kv_heads;     /* >= 1 */
    int32_t d;              /* 16, 32, 64, 128 or 256 */
    int32_t n_layers;       /* >= 1 */
    int32_t dtype;          /* stream_dtype */
    int64_t stride_l, stride_p, stride_t, stride_h; /* layer, page, token, head; one whose extent is 1 does not matter */
} stream_cache;

/* Bytes of device workspace that the ledger calls (reserve, fork, free, compact) need; 0 = invalid cache. */
size_t stream_cache_workspace_bytes(const stream_cache *c);

/*
 * The ledger calls. Each is done as a whole or not at all, and writes info_out, device int32 [4], 16-byte aligned:
 *   [0] 1 = done, 0 = refused: nothing was changed
 *   [1] pages taken (reserve, fork: and copies due), given back (free) or to be moved (compact); what it would
 *       have taken where it was refused
 *   [2] free pages after the call
 *   [3] slots that the call has to refuse for (an index or a length out of range; see each call); free: entries of the
 *       table or counts that cannot be, passed over
 * workspace: device, 256-byte aligned, >= stream_cache_workspace_bytes(c); overwritten, nothing is kept in it. Calls on
 * one cache, or with one workspace, must not overlap on the GPU.
 *
 * reserve: room for n_new[s] >= 0 more tokens in every slot s, and seq_len[s] grows by as many (their keys and
 * values are then written with stream_cache_write, layer by layer). Refused if pages are missing, if an n_new is negative
 * or if a row of the table would have to be longer than max_pages.
 */
stream_status stream_cache_reserve(const stream_cache *c, const int32_t *n_new, int32_t *page_table, int32_t *seq_len,
                                   int32_t *ref_count, int32_t *info_out, void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * fork: every slot s with parent[s] >= 0 becomes another chain with the tokens that slot parent[s] has: it shares
 * the full pages, and a last page that is not full gets a copy of its own. The copies are due before
 * anything is written: pairs_out, device int32 [n_slots, 2], 8-byte aligned, gets their {from, to}, by ascending s, then -1;
 * hand it with info_out + 1 to stream_cache_copy_pages. (Where the call was refused all of it is -1.) Refused if pages are
 * missing, if such a slot is not empty, if its parent is no slot, is itself to become a copy in this call, or has an
 * impossible length.
 */
stream_status stream_cache_fork(const stream_cache *c, const int32_t *parent, int32_t *page_table, int32_t *seq_len,
                                int32_t *ref_count, int32_t *pairs_out, int32_t *info_out, void *workspace, size_t workspace_bytes,
                                void *cuda_stream);

/* free: every slot s with done[s] != 0 is empty afterwards; pages that nobody names any more are free. Never refused. */
stream_status stream_cache_free(const stream_cache *c, const int32_t *done, int32_t *page_table, int32_t *seq_len,
                                int32_t *ref_count, int32_t *info_out, void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * compact: with n pages in use, those of them with a number of n or more move to the free ones below n, the lowest to
 * the lowest, so that 0 .. n - 1 are in use. pairs_out, device int32 [n_pages / 2, 2], 8-byte aligned: {from, to} by ascending
 * number, then -1, for stream_cache_copy_pages (before anything is written or read).
 */
stream_status stream_cache_compact(const stream_cache *c, int32_t *page_table, int32_t *seq_len, int32_t *ref_count,
                                   int32_t *pairs_out, int32_t *info_out, void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Copies whole pages, in all layers, of K and V: for i < *count (device; at most n_pairs) page pairs[i][0] to page
 * pairs[i][1]. Pairs with a number outside the cache are passed over. No page may be written that another pair reads or
 * writes. k_pages and v_pages are the caches' first elements.
 */
stream_status stream_cache_copy_pages(const stream_cache *c, void *k_pages, void *v_pages, const int32_t *pairs,
                                      const int32_t *count, int32_t n_pairs, void *cuda_stream);

/*
 * Keys and values of new tokens into the pages of one layer, after stream_cache_reserve. The rows cu_new[s] ..
 * cu_new[s+1] - 1 of k and v are the last tokens of slot s, up to seq_len[s] - 1. Rows of no slot, and tokens whose
 * position or page cannot be, are passed over.
 *   k, v     device, [total, n_kv_heads, d] with the strides given (elements, innermost 1); read only
 *   cu_new   device int32 [n_slots + 1], ascending, clamped like cu_q
 *   done     device int32, or NULL: nothing is written where it is 0. The first word of reserve's info_out: a reserve that was
 *            refused has left the lengths as they were, and the last tokens that there are would be overwritten
 *   k_pages, v_pages  the caches' first elements (layer 0); written: layer `layer`
 */
stream_status stream_cache_write(const stream_cache *c, int32_t layer, const void *k, const void *v, int64_t total,
                                 int64_t stride_t, int64_t stride_h, const int32_t *cu_new, const int32_t *page_table,
                                 const int32_t *seq_len, const int32_t *done, void *k_pages, void *v_pages, void *cuda_stream);

/*
 * Attention of one new token of every slot over its cached tokens (its own among them, if it has been written):
 *     out[s, h] = sum_{t < seq_len[s]} softmax_t(scale q_s.k_t) v_t,     lse[s, h] = log sum_t exp(scale q_s.k_t)
 * An empty slot gets zeros and -inf. Sums as in stream_prompt_attention (|v| up to 2^64). The tokens of all slots and
 * heads are dealt evenly to the SMs, and pieces of a long slot are joined in a fixed order: the same call gives the same bits.
 * What the pages hold beyond a slot's tokens does not matter (NaN included). Tokens whose page number is outside the cache are left out, and recorded:
 * stream_read_stats(workspace, ...) then returns STREAM_ERR_DEVICE_CHECK with error = 701 and error_info = such a slot. A seq_len below 0
 * counts as 0, one above max_pages * page_size as that.
 *
 *   n_q_heads   a multiple of n_kv_heads
 *   q           device [n_slots, n_q_heads, d] with the strides given (elements, innermost 1); read only
 *   scale       logit scale, up to 2.3e38 (fp32 holds scale log2(e)); <= 0 selects 1/sqrt(d)
 *   out         device, dtype of the cache, contiguous [n_slots, n_q_heads, d]; overwritten. Must not overlap an input
 *   lse_out     device float32 [n_slots, n_q_heads] or NULL
 *   workspace   device, 256-byte aligned, >= stream_decode_workspace_bytes(c, n_q_heads); overwritten, nothing is kept
 *               in it but the record. Calls that can overlap on the GPU need one each.
 */
size_t stream_decode_workspace_bytes(const stream_cache *c, int32_t n_q_heads);  /* 0 = invalid */
stream_status stream_decode_attention(const stream_cache *c, int32_t layer, int32_t n_q_heads, const void *q, int64_t q_stride_s,
                                      int64_t q_stride_h, const void *k_pages, const void *v_pages, const int32_t *page_table,
                                      const int32_t *seq_len, float scale, void *out, float *lse_out, void *workspace,
                                      size_t workspace_bytes, void *cuda_stream);

/*
 * The keys and values of slots read back as packed rows: what stream_prompt_attention needs of a prompt that comes in pieces. The rows cu[s] ..
 * cu[s+1] - 1 of k_out and v_out become the last tokens of slot s, up to seq_len[s] - 1 (all of them where there are as many
 * rows as tokens). Rows of no slot stay as they are; tokens whose position or page cannot be are zeros.
 *   cu              device int32 [n_slots + 1], ascending, clamped like cu_q
 *   k_out, v_out    device, dtype of the cache, contiguous [total, n_kv_heads, d]
 */
stream_status stream_cache_read(const stream_cache *c, int32_t layer, const void *k_pages, const void *v_pages, const int32_t *cu,
                                int64_t total, const int32_t *page_table, const int32_t *seq_len, void *k_out, void *v_out, void *cuda_stream);

/*
 * Attention with a sliding window and sinks: a query at position p of its sequence sees the keys j <= p with j > p - window or j < sinks, that
 * is the last `window` keys, its own among them, and the first `sinks` ones. (The fixed pattern that a searched mask is set against, and
 * what models do whose layers look back only so far.) window >= 1, sinks >= 0, and both may be larger than any sequence.
 *
 * stream_prompt_window_attention: as stream_prompt_attention with causal = 1 (else INVALID_ARG); query i of a sequence with n queries and m keys
 * is at position i + m - n. Keys that no query of a sequence sees are not read, but for those that share a tile with others.
 *
 * stream_decode_window_attention: as stream_decode_attention; a slot's query is at position seq_len[s] - 1. Pages all of whose tokens lie
 * between the sinks and the window are not read, and their entries of the table may be anything.
 */
stream_status stream_prompt_window_attention(const stream_prompt *p, int32_t window, int32_t sinks, const void *q, const void *k,
                                             const void *v, const int32_t *cu_q, const int32_t *cu_k, float scale, void *out,
                                             float *lse_out, void *cuda_stream);
stream_status stream_decode_window_attention(const stream_cache *c, int32_t layer, int32_t n_q_heads, int32_t window, int32_t sinks,
                                             const void *q, int64_t q_stride_s, int64_t q_stride_h, const void *k_pages,
                                             const void *v_pages, const int32_t *page_table, const int32_t *seq_len, float scale,
                                             void *out, float *lse_out, void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * A paged cache in 8 bits: K and V are e4m3 (sign, four bits of exponent, three of mantissa; up to 448), and the tokens of a block, in one kv
 * head, share a scale: a key is its e4m3 numbers times its block's scale. The scales of K and V are each float32 [n_layers, n_pages,
 * page_size / block, n_kv_heads] with the strides below, which are positive. The ledger is that of any cache: its calls take &c->cache.
 *
 * A block's scale is the smallest power of two 2^e, -90 <= e <= 120, of which no element is more than 448 times: e4m3's relative precision, 2^-4 at most, does
 * not depend on a scale, powers of two make the division exact, and what is rounded again when a block's scale grows stays
 * what it was, but for elements below 2^-6 of the new scale. */
typedef struct {
    stream_cache cache;     /* dtype: of queries, outputs and new keys and values; strides: of the e4m3 arrays, in elements (bytes) */
    int32_t block;          /* tokens that share a scale; divides page_size */
    int32_t reserved;       /* 0 */
    int64_t scale_stride_l, scale_stride_p, scale_stride_b, scale_stride_h; /* layer, page, block, head; elements; one whose extent is 1 does not matter */
} stream_cache8;

/*
 * stream_cache_write for a cache in 8 bits. A block whose first token is among the new ones gets a scale for its new tokens. One that
 * has tokens in front of them keeps its scale or takes the one that the new tokens ask for, whichever is larger; where it grows, those
 * tokens are rounded again: rn(x old / new). The sum of a block's roundings is so at most a step of its last scale. Infinities become +-448
 * scales, with e = 120, and as that is more than fp32 holds they are read as infinities (what is rounded to 2^128 too); NaN stays NaN and
 * asks for no scale. Everything else as stream_cache_write.
 *   k_scale, v_scale  the scales' first elements (layer 0); written: layer `layer`
 */
stream_status stream_cache8_write(const stream_cache8 *c, int32_t layer, const void *k, const void *v, int64_t total, int64_t stride_t,
                                  int64_t stride_h, const int32_t *cu_new, const int32_t *page_table, const int32_t *seq_len,
                                  const int32_t *done, void *k_pages, void *v_pages, float *k_scale, float *v_scale, void *cuda_stream);

/* stream_cache_read for a cache in 8 bits: the rows of k_out and v_out, of dtype c->cache.dtype, are e4m3 numbers times their scales. */
stream_status stream_cache8_read(const stream_cache8 *c, int32_t layer, const void *k_pages, const void *v_pages, const float *k_scale,
                                 const float *v_scale, const int32_t *cu, int64_t total, const int32_t *page_table, const int32_t *seq_len,
                                 void *k_out, void *v_out, void *cuda_stream);

/* stream_cache_copy_pages for a cache in 8 bits: pages and their scales. */
stream_status stream_cache8_copy_pages(const stream_cache8 *c, void *k_pages, void *v_pages, float *k_scale, float *v_scale,
                                       const int32_t *pairs, const int32_t *count, int32_t n_pairs, void *cuda_stream);

/*
 * stream_decode_attention over a cache in 8 bits, with a window and sinks where window > 0 (stream_decode_window_attention; 0: every key is
 * seen, whatever sinks says). Any scales of 0 to 2^120 for keys (with logits that fp32 holds) and of 0 to 2^100 for values (of which those up
 * to 2^64 cannot overflow) will do, powers of two or not; a token whose key scale is 0 counts as not there, whatever its bytes and its value's scale are. Products are those of
 * e4m3 numbers, which fp16 holds, with queries and weights in fp16 (bf16 caches: 2^-11 of a weight; fp32 ones: two fp16 numbers each, 2^-22). Everything
 * else, the workspace too (stream_decode_workspace_bytes of &c->cache), as stream_decode_attention.
 */
stream_status stream_decode_attention8(const stream_cache8 *c, int32_t layer, int32_t n_q_heads, int32_t window, int32_t sinks,
                                       const void *q, int64_t q_stride_s, int64_t q_stride_h, const void *k_pages, const void *v_pages,
                                       const float *k_scale, const float *v_scale, const int32_t *page_table, const int32_t *seq_len,
                                       float scale, void *out, float *lse_out, void *workspace, size_t workspace_bytes, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* STREAM_H_ */
