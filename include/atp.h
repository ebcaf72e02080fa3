/*
 * atp.h -- C ABI of the MI355X (gfx950) ATP shard-block library.
 *
 * One device's share of a transformer layer under ATP's row-first /
 * column-first 2D tensor parallelism (Cheng, Liu, Du, You, "ATP: Adaptive
 * Tensor Parallelism for Foundation Models", arXiv 2301.08658):
 * the sharded QKV, out-projection, fc1 (+bias+GeLU) and fc2 GEMMs, the
 * reduction of their Partial(SUM) outputs, and the token-chunk pipeline
 * that overlaps each chunk's reduction with the next chunk's GEMM.
 *
 * Conventions shared by every call
 * --------------------------------
 *  - Mesh (Sec. 3.1): DeviceMesh(d1, d2); this device sits at (i1, i2),
 *    rank = i1 * d2 + i2.
 *  - Y = X W with X [tokens, k] and W [k, n] (Sec. 3.2, "Y = XW").
 *      ATP_ROW_FIRST: W spec [Shard(0), Shard(1)]: local W rows
 *        [i1*k/d1, (i1+1)*k/d1), columns [i2*n/d2, (i2+1)*n/d2); X holds
 *        the matching k/d1 columns; the output block is Partial(SUM) over
 *        the d1 devices that share i2 (mesh axis 0).
 *      ATP_COL_FIRST: W spec [Shard(1), Shard(0)]: local W rows
 *        [i2*k/d2, ...), columns [i1*n/d1, ...); the output is Partial(SUM)
 *        over the d2 devices that share i1 (mesh axis 1).
 *    In the backward pass (Sec. 4.2) the input gradient dX = dY W^T is
 *    partial over the other axis (the one that split n).
 *  - Tensors are row-major device buffers owned by the caller: element
 *    (r, c) of a matrix with leading dimension ld is at base[r * ld + c].
 *    bf16 = IEEE bfloat16 bits (uint16), f32 = IEEE binary32.
 *    Every device pointer must be 16-byte aligned, every leading dimension
 *    and every local column count a multiple of 8 elements, and leading
 *    dimensions at most 4M (2^22) elements.
 *  - Streams and events are hipStream_t / hipEvent_t passed as void*;
 *    NULL means the default stream.  Calls only enqueue work and return.
 *  - Chunks (Sec. 4.1): the token rows are split into `chunks` contiguous
 *    equal parts; tokens % chunks must be 0.  Chunking never changes a
 *    value: every output element is computed by the same instructions in
 *    the same order whatever the chunk count.
 *  - Reductions sum the group's buffers in group order 0..d-1, so every
 *    member of a group obtains bit-identical results.
 *  - Errors: all arguments are checked before anything is enqueued; a
 *    non-OK status means nothing was enqueued.  atp_last_error() returns
 *    a per-thread message for the last failure.  A HIP launch failure
 *    after checks passed returns ATP_ERR_DEVICE (work enqueued before it
 *    may have run).
 *  - The library never allocates device memory.
 */
#ifndef ATP_H
#define ATP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    ATP_OK = 0,
    ATP_ERR_INVALID_ARGUMENT = 1, /* null pointer, coordinate out of range, bad enum, ld < cols */
    ATP_ERR_SHAPE = 2,            /* k or n not divisible by the mesh, tokens % chunks != 0 */
    ATP_ERR_UNSUPPORTED = 3,      /* alignment, multiple-of-8 rule, group larger than ATP_MAX_GROUP */
    ATP_ERR_DEVICE = 4            /* a HIP call failed */
} atp_status;

typedef enum { ATP_ROW_FIRST = 0, ATP_COL_FIRST = 1 } atp_mode;

/* ATP_BLOCK_COL: the layer of Sec. 3.2.1 -- QKV and fc1 column-first,
 * out-proj and fc2 row-first.  ATP_BLOCK_ROW: the transposed arrangement
 * (QKV and fc1 row-first, out-proj and fc2 column-first); on mesh (d1, d2)
 * it has the local shapes of ATP_BLOCK_COL on (d2, d1). */
typedef enum { ATP_BLOCK_COL = 0, ATP_BLOCK_ROW = 1 } atp_block_mode;

/* Epilogues (Sec. 2.1 and 3.2.1).  With s the reduced sum:
 *   NONE: s;  BIAS: s + b[n];  BIAS_GELU: GeLU(s + b[n]) with the exact erf
 *   form, optionally saving s + b[n];  GELU_BWD: s * GeLU'(pre[t, n]). */
typedef enum {
    ATP_EPI_NONE = 0,
    ATP_EPI_BIAS = 1,
    ATP_EPI_BIAS_GELU = 2,
    ATP_EPI_GELU_BWD = 3
} atp_epilogue;

typedef enum { ATP_F32 = 0, ATP_BF16 = 1 } atp_dtype;

#define ATP_MAX_GROUP 64   /* largest reduction group (d1 or d2) */
#define ATP_MAX_CHUNKS 64

typedef struct { int32_t d1, d2, i1, i2; } atp_mesh;

/* Local block of one linear (Sec. 3.2): W rows [k_off, k_off + k_loc),
 * columns [n_off, n_off + n_loc); forward reduction over mesh axis
 * red_axis (group size red_size, this device at red_index); backward
 * input-gradient reduction over bwd_axis (bwd_size, bwd_index). */
typedef struct {
    int64_t k_loc, n_loc, k_off, n_off;
    int32_t red_axis, red_size, red_index;
    int32_t bwd_axis, bwd_size, bwd_index;
} atp_shard;

/* Shard geometry of Y = XW, Sec. 3.2 (local sizes [b, h1/d1] x [h1/d1, h2/d2]
 * for row-first; communicated block [b, h2/d1] for column-first).
 * Host only, no device work.  Errors: INVALID_ARGUMENT (null, d <= 0,
 * coordinate out of range, bad mode), SHAPE (k or n not divisible). */
atp_status atp_shard_geometry(const atp_mesh* mesh, int32_t mode, int64_t k, int64_t n,
                              atp_shard* out);

/* Local GEMM of one shard linear, chunked (Sec. 3.2, Sec. 4.1):
 *   y[t, :] = epi( x_loc[t, :] . w_loc )   for t in each chunk, in order.
 * x_loc  bf16 [tokens, k_loc], ld ldx.   w_loc bf16 [k_loc, n_loc], ld ldw.
 * If the reduction group has more than one member, y is this device's
 * Partial(SUM) block: epi must be ATP_EPI_NONE (the bias and GeLU belong
 * after the reduction); y_dtype ATP_F32, or ATP_BF16 for partials kept in
 * the training precision as the paper all-reduces them (Sec. 5: FP16),
 * reduced by atp_chunked_partial_reduce_bf16.  With a group of one, epi may
 * be NONE, BIAS or BIAS_GELU and y f32 or bf16; bias_loc bf16 [n_loc]
 * (the block n_off..), preact (nullable, bf16, ld ldy) receives s + b for
 * BIAS_GELU.  chunk_done (nullable) holds `chunks` caller-created events;
 * event c is recorded on `stream` once chunk c's rows of y are written
 * (chunks with no event between them run as one launch). */
atp_status atp_shard_linear_fwd(const atp_mesh* mesh, int32_t mode, int64_t tokens,
                                int64_t k, int64_t n, int32_t chunks,
                                const void* x_loc, int64_t ldx,
                                const void* w_loc, int64_t ldw,
                                const void* bias_loc, int32_t epi,
                                void* y, int32_t y_dtype, int64_t ldy, void* preact,
                                void* stream, void* const* chunk_done);

/* Reduction of a group's Partial(SUM) blocks -- the arithmetic of the
 * grouped all-reduce of Sec. 3.2 (Sec. 3.1, Partial(SUM)) -- chunked so
 * that chunk c can start as soon as its partials are ready (Sec. 4.1):
 *   out[t, n] = epi( sum_{j=0..red_size-1} partials[j][t * ldp + n] ).
 * partials: host array of red_size device pointers, f32 [tokens, ldp];
 * on one GPU the other members' buffers stand in for the peers' data.
 * bias_loc bf16 [n_loc] for BIAS / BIAS_GELU.  preact_in (bf16, ld ldo)
 * for GELU_BWD; preact_out (nullable, bf16, ld ldo) for BIAS_GELU.
 * out is f32 or bf16 (round to nearest even).  chunk_ready (nullable):
 * `chunks` events; the stream waits for event c before reducing chunk c.
 * Errors: INVALID_ARGUMENT for red_size < 1, a null entry, missing bias or
 * preact_in; UNSUPPORTED for red_size > ATP_MAX_GROUP. */
atp_status atp_chunked_partial_reduce(int32_t red_size, int64_t tokens, int64_t n_loc,
                                      int32_t chunks, const float* const* partials,
                                      int64_t ldp, const void* bias_loc, int32_t epi,
                                      const void* preact_in, void* out, int32_t out_dtype,
                                      int64_t ldo, void* preact_out, void* stream,
                                      void* const* chunk_ready);

/* The same reduction over bf16 Partial(SUM) blocks (partials: red_size
 * device pointers, bf16 [tokens, ldp]): each value widened to f32 and
 * summed in group order, then epi as above.  This is the variant of Sec. 5's
 * half-precision training, where the all-reduced activations are 16-bit;
 * it halves the bytes each reduction reads.  Errors as above. */
atp_status atp_chunked_partial_reduce_bf16(int32_t red_size, int64_t tokens, int64_t n_loc,
                                           int32_t chunks, const void* const* partials,
                                           int64_t ldp, const void* bias_loc, int32_t epi,
                                           const void* preact_in, void* out, int32_t out_dtype,
                                           int64_t ldo, void* preact_out, void* stream,
                                           void* const* chunk_ready);

/* One shard linear with the group's reduction fused into the GEMM's
 * epilogue: the fused GEMM-and-all-reduce design that Sec. 4.1 contrasts
 * with chunked overlapping.  In one launch, unchunked:
 *   out[t, :] = epi( sum_{j=0..red_size-1} P_j[t, :] ),
 * with P_own = x_loc[t, :] . w_loc formed in the tile's registers and never
 * stored, and P_j (j != red_index) read from peers[j] (f32 [tokens, ldp],
 * the other members' partials; peers[red_index] is not read and may be
 * NULL).  The terms are summed in group order, so out has the same bits as
 * atp_shard_linear_fwd + atp_chunked_partial_reduce on the same inputs.
 * x_loc, w_loc, bias_loc, epi (NONE, BIAS, BIAS_GELU), preact (nullable,
 * bf16, ld ldo) as for atp_shard_linear_fwd; out f32 or bf16.
 * Errors: as atp_shard_linear_fwd; UNSUPPORTED for a group of more than 8;
 * INVALID_ARGUMENT for a missing peer or GELU_BWD. */
atp_status atp_shard_linear_fwd_fused(const atp_mesh* mesh, int32_t mode, int64_t tokens,
                                      int64_t k, int64_t n, const void* x_loc, int64_t ldx,
                                      const void* w_loc, int64_t ldw,
                                      const float* const* peers, int64_t ldp,
                                      const void* bias_loc, int32_t epi, void* out,
                                      int32_t out_dtype, int64_t ldo, void* preact,
                                      void* stream);

/* Backward of one shard linear (Sec. 4.2): with dy the gradient of this
 * device's reduced output block (bf16 [tokens, n_loc], ld lddy),
 *   dx_partial = dy . w_loc^T   f32 [tokens, k_loc], ld lddx -- partial over
 *                               the backward group (bwd_size members);
 *   dw         = x_loc^T . dy   f32 [k_loc, n_loc], ld lddw (complete);
 *   db         = sum_t dy       f32 [n_loc] (nullable).
 * dX is computed first, chunk by chunk, recording dx_chunk_done[c]
 * (nullable) so its reduction can overlap the dW GEMM that follows on the
 * same stream. */
atp_status atp_shard_linear_bwd(const atp_mesh* mesh, int32_t mode, int64_t tokens,
                                int64_t k, int64_t n, int32_t chunks,
                                const void* x_loc, int64_t ldx,
                                const void* w_loc, int64_t ldw,
                                const void* dy, int64_t lddy,
                                float* dx_partial, int64_t lddx,
                                float* dw, int64_t lddw, float* db,
                                void* stream, void* const* dx_chunk_done);

/* Storage order of a local weight block.  ATP_W_KN: [k_loc][n_loc], the
 * paper's Y = XW orientation (Sec. 3.2).  ATP_W_NK: [n_loc][k_loc], W^T, the
 * way torch.nn.Linear keeps its weight ([out_features, in_features]). */
typedef enum { ATP_W_KN = 0, ATP_W_NK = 1 } atp_weight_layout;

/* Local weights of the block; index 0..3 = qkv [h,3h], out [h,h],
 * fc1 [h,4h], fc2 [4h,h] (Sec. 2.1).  Each w[i] is the device's bf16
 * block, [k_loc][n_loc] or [n_loc][k_loc] as `layout` says (ld ldw[i]);
 * b[i] its bf16 bias block [n_loc].  A zero-filled struct means ATP_W_KN. */
typedef struct {
    const void* w[4];
    int64_t ldw[4];
    const void* b[4];
    int32_t layout;   /* atp_weight_layout, the same for all four */
} atp_block_weights;

/* Forward inputs and outputs of the block (Sec. 3.2.1).
 *  x_loc   bf16 [tokens, h_x]: the layer-input columns QKV and fc1
 *          contract over (h/d2 for COL, h/d1 for ROW).
 *  attn_loc bf16 [tokens, h_a]: the attention-core output columns that
 *          feed out-proj (h/d1 for COL, h/d2 for ROW).
 *  partials[i]: host array of the red_size device pointers of linear i's
 *          group ([tokens, ldp[i]] of partial_dtype); entry red_index is
 *          this device's own buffer and is written, the others are read.
 *          Unused (may be NULL) when the group has one member.
 *  partial_dtype: ATP_F32 (a zero-filled struct), or ATP_BF16 for the
 *          16-bit Partial(SUM) blocks of Sec. 5's half-precision training:
 *          the own partial is rounded once to bf16 (nearest even) and the
 *          group's bf16 values are summed in f32, halving the bytes every
 *          reduction reads.
 *  qkv, o, h, z: bf16 reduced outputs (+bias; h = GeLU(...)); pre: bf16
 *          fc1 pre-activation saved for the backward, ld ld_h. */
typedef struct {
    const void* x_loc;
    int64_t ldx;
    const void* attn_loc;
    int64_t lda;
    void* const* partials[4];
    int64_t ldp[4];
    void* qkv; int64_t ld_qkv;
    void* o;   int64_t ld_o;
    void* h;   int64_t ld_h;
    void* pre;
    void* z;   int64_t ld_z;
    int32_t partial_dtype;
} atp_block_fwd_io;

/* Backward inputs and outputs of the block (Sec. 4.2).
 *  x_loc, attn_loc, h, pre: the forward's inputs and saved activations.
 *  dz, dqkv, d_o: bf16 gradients of the reduced outputs z, qkv, o.
 *  dx_partials[i]: host array of the bwd_size device pointers of linear
 *          i's backward group ([tokens, ld_dxp[i]] of partial_dtype, f32 or
 *          bf16 as in atp_block_fwd_io), own entry written.
 *  dh_pre: bf16 fc1 upstream gradient = (reduced fc2 dX) * GeLU'(pre).
 *  dx_qkv, dx_fc1, d_attn: bf16 reduced input gradients.
 *  dw[i] f32 in the weights' layout and leading dimension ([k_loc][n_loc]
 *  for ATP_W_KN, [n_loc][k_loc] for ATP_W_NK), db[i] f32 [n_loc]. */
typedef struct {
    const void* x_loc;    int64_t ldx;
    const void* attn_loc; int64_t lda;
    const void* h;        int64_t ld_h;
    const void* pre;
    const void* dz;   int64_t ld_dz;
    const void* dqkv; int64_t ld_dqkv;
    const void* d_o;  int64_t ld_do;
    void* const* dx_partials[4];
    int64_t ld_dxp[4];
    void* dh_pre;
    void* dx_qkv; int64_t ld_dx_qkv;
    void* dx_fc1; int64_t ld_dx_fc1;
    void* d_attn; int64_t ld_d_attn;
    float* dw[4];
    float* db[4];
    int32_t partial_dtype;
} atp_block_bwd_io;

/* Workspace for the block calls' transposed-layout path (bytes): the larger
 * of the forward's need and the backward's for weights in `weight_layout`
 * (atp_weight_layout).  The forward keeps W^T of a weight stored
 * [k_loc][n_loc] (n_loc rows of k_loc + 64 bf16 values) when, at some
 * valid chunk count, its products are split over k or are not shaped for
 * the 256 x 256 tiles that stream W as stored as fast as W^T; weights
 * stored [n_loc][k_loc] need no copy.  The backward keeps X^T of x, the attention
 * block and H, and dY^T of the four linears (cols rows of tokens + 64 bf16
 * values each), for weights stored [n_loc][k_loc] one copy of the largest
 * weight in [k_loc][n_loc] order (k_loc rows of n_loc + 64 values, reused
 * linear by linear), and the fp32 column partials of dY that the
 * transposes leave for db (ceil(tokens / 64) rows of the widest linear's
 * columns).  Each side adds the fp32 split-K slabs of the chunked products
 * that feed a reduction (S * chunk rows * cols * 4 bytes for the largest
 * split plan S over every valid chunk count).  The 64 values of padding
 * keep row pitches off memory-channel-aligned strides; every piece is
 * rounded up to 256 bytes.  `chunks` does not change the size.
 * Returns 0 for invalid arguments. */
size_t atp_block_workspace_bytes(const atp_mesh* mesh, int32_t block_mode, int64_t tokens,
                                 int64_t h, int32_t chunks, int32_t weight_layout);

/* Which path a block call takes (pass 0: atp_block_fwd, 1: atp_block_bwd)
 * for a workspace of ws_bytes bytes: 1 the transposed-layout path (the
 * workspace holds the pass's need, and for the backward tokens % 8 == 0),
 * 0 the direct path, -1 for invalid arguments.  Host only.  A block call
 * that would take the direct path refuses a compute stream under HIP graph
 * capture (see atp_block_fwd). */
int32_t atp_block_workspace_path(const atp_mesh* mesh, int32_t block_mode, int64_t tokens,
                                 int64_t h, int32_t weight_layout, size_t ws_bytes, int32_t pass);

/* Shard geometry of the block's four linears, out[0..3] = qkv, out, fc1,
 * fc2, each as atp_shard_geometry gives it for the linear's mode in
 * block_mode (Sec. 3.2.1: ATP_BLOCK_COL runs QKV and fc1 column-first,
 * out-proj and fc2 row-first).  Host only.  Errors: those of
 * atp_shard_geometry; UNSUPPORTED when a local size is not a multiple
 * of 8. */
atp_status atp_block_geometry(const atp_mesh* mesh, int32_t block_mode, int64_t h,
                              atp_shard out[4]);

/* The device's heads of the attention block (Sec. 3.2.1): its QKV block
 * holds *per_block whole heads of dimension h / heads; the block is
 * scattered over the group that reduced it, and the device attends over
 * heads [*first, *first + *count) of the block (block-local indices).
 * Host only.  Errors: those of atp_block_geometry; SHAPE when h is not a
 * multiple of heads, the QKV block does not hold whole heads or its heads
 * do not divide over the group. */
atp_status atp_attention_heads(const atp_mesh* mesh, int32_t block_mode, int64_t h,
                               int32_t heads, int32_t* first, int32_t* count,
                               int32_t* per_block);

/* Transpose a bf16 matrix: dst[c * ldd + r] = src[r * lds + c] for r < rows,
 * c < cols.  A data-layout step for the products of Sec. 3.2 / 4.2 (it turns
 * an operand contiguous along its M/N side into one contiguous along the
 * contraction), not part of the paper's arithmetic.  src [rows][lds] and dst
 * [cols][ldd] are 16-byte aligned with leading dimensions that are multiples
 * of 8 (at most 2^22); rows and cols may be any size (with either 0 nothing
 * is read or written and the pointers may be NULL); the buffers must not be
 * the same.
 * Errors: INVALID_ARGUMENT for negative sizes, NULL or aliased buffers,
 * leading dimensions below the row length; UNSUPPORTED for alignment. */
atp_status atp_transpose_bf16(int64_t rows, int64_t cols, const void* src, int64_t lds, void* dst,
                              int64_t ldd, void* stream);

/* One device's forward share of the layer (Sec. 3.2.1) with chunk-based
 * overlapping (Sec. 4.1).  Each linear's GEMM runs chunk by chunk; each
 * chunk's reduction runs on comm_stream as soon as that chunk's partial is
 * written (one that moves at most 8 MB is too short to hide anything and runs
 * on compute_stream, except under graph capture: still after comm_stream's
 * earlier work, behind the products that need no result of it, and
 * comm_stream is ordered after it when the call returns);
 * fc2's chunk c waits for fc1's reduced chunk c.  A group of one
 * needs no reduction: its bias (and GeLU) are applied in the GEMM epilogue
 * and it runs as one launch.  The GEMMs are issued on compute_stream in the
 * order out-proj, fc1, then QKV and fc2 (the one whose reductions read fewer
 * bytes last); with chunks > 1, comm_stream != compute_stream and outside
 * HIP graph capture, every other chunk product of a linear whose chunks do
 * not split over k runs on a second stream the library keeps per host
 * thread and device (default priority, never destroyed), so a chunk's
 * product can start on the CUs the previous chunk leaves idle; the call
 * joins that stream back into compute_stream before it returns.  With
 * comm_stream == compute_stream nothing overlaps.
 * workspace (nullable, 256-byte aligned): when ws_bytes is at least the
 * forward's need (atp_block_workspace_path) the products run with both
 * operands contiguous along k, the faster layout (weights stored
 * [k_loc][n_loc] are first copied there as W^T, except for a linear whose
 * products, at this chunk count, run unsplit on the 256 x 256 tiles that
 * stream W as stored as fast; weights stored [n_loc][k_loc] already are
 * contiguous along k), and a chunk product with too few output
 * tiles to fill the chip is split over its contraction, the splits' fp32
 * slabs summed in split order into the own partial before the chunk's
 * reduction reads it.  Without the workspace the products read W as
 * stored.  Every layout sums each element's products in the same order:
 * the paths give the same bits except where a product splits (then they
 * agree to fp32 rounding).  Results do not depend on the streams used, and
 * are the same for every chunk count that gives each chunk product the same
 * split plan (without a workspace: every chunk count).  compute_stream's
 * earlier work happens before the block's, and on return compute_stream is
 * ordered after all of it and after comm_stream's earlier work; the workspace
 * may be reused once compute_stream reaches that point.  comm_stream is
 * ordered after compute_stream's earlier work, with or without reductions.  A call that would take the direct path refuses a
 * compute_stream under HIP graph capture (UNSUPPORTED) before enqueueing
 * anything, and every block call refuses a comm_stream under capture whose
 * compute_stream is not.  Concurrent calls from different host threads are safe (each
 * thread keeps its own synchronisation events). */
atp_status atp_block_fwd(const atp_mesh* mesh, int32_t block_mode, int64_t tokens, int64_t h,
                         int32_t chunks, const atp_block_weights* w,
                         const atp_block_fwd_io* io, void* workspace, size_t ws_bytes,
                         void* compute_stream, void* comm_stream);

/* One device's backward share of the layer (Sec. 4.2): dX = dY W^T per
 * linear, chunked and reduced on comm_stream where its group has more than
 * one member, dW = X^T dY and db = column sums of dY; fc1's dY is fc2's
 * reduced dX times GeLU'(pre).  Issue order on compute_stream: fc2's dX
 * (fc1 waits for it), QKV's and out-proj's dX, fc1's dX, then the four dW
 * largest first, so the dX reductions overlap the later GEMMs.
 * workspace: when ws_bytes is at least the backward's need and tokens % 8
 * == 0 (atp_block_workspace_path), X^T and dY^T are written there and dW
 * runs from them where that is faster than reading X and dY as given, weights
 * stored [n_loc][k_loc] are copied there in [k_loc][n_loc] order for the dX
 * products, and the chunked dX products are split over their contraction as
 * in atp_block_fwd; otherwise every product reads its operands as stored.  The paths give the same bits except where
 * a product splits (as in atp_block_fwd).  On return compute_stream is
 * ordered after all work.  Graph capture and threads as atp_block_fwd. */
atp_status atp_block_bwd(const atp_mesh* mesh, int32_t block_mode, int64_t tokens, int64_t h,
                         int32_t chunks, const atp_block_weights* w,
                         const atp_block_bwd_io* io, void* workspace, size_t ws_bytes,
                         void* compute_stream, void* comm_stream);

/* One device's attention core (Sec. 2.1 Formula (mha), causal; the
 * attention block of Sec. 3.2.1).  qkv is the device's reduced QKV output
 * block for block_mode on the mesh (bf16 [batch*seq, ld_qkv], token rows
 * sequence-major, the n_loc columns atp_block_fwd's QKV linear produces).
 * The block holds n_loc / 384 whole heads of dimension h / heads, which
 * must be 128, each as [q | k | v] columns.  The block is replicated over
 * the group that reduced it; the attention block scatters it over that
 * group, so the device attends over the r-th of g equal runs of heads,
 * r = its index in the group, g = the group's size.  The output goes to
 * out (bf16 [batch*seq, ld_out], at least n_loc / 3 columns: the gathered
 * input of out-proj): the device writes its heads' columns, the r-th run of
 * h/heads-wide column blocks, and leaves the other members' columns (the
 * all-gather) alone.  lse (fp32 [heads_of_device][batch*seq]) receives the
 * natural-log softmax denominator of every row, for the backward.  The
 * caller owns every buffer; work is enqueued on `stream`.
 * Errors: INVALID_ARGUMENT for a bad mesh, negative sizes, NULL buffers,
 * qkv and out sharing memory, ld below the row length; SHAPE when h is not
 * a multiple of heads or the heads do not divide over the group;
 * UNSUPPORTED for a head dimension other than 128, sizes above 2^24,
 * misalignment. */
atp_status atp_attention_fwd(const atp_mesh* mesh, int32_t block_mode, int64_t batch, int64_t seq,
                             int64_t h, int32_t heads, const void* qkv, int64_t ld_qkv,
                             void* out, int64_t ld_out, float* lse, void* stream);

/* Gradient of atp_attention_fwd (Sec. 2.1 Formula (mha), the backward of
 * Sec. 4.2 applied to the attention core).  qkv, out and lse are the
 * forward's input, output (the gathered block; the device's columns are
 * read) and saved row log-sum-exps; d_out (bf16, same shape and columns as
 * out) is the gradient of the gathered out-proj input.  The device writes
 * dq, dk, dv of its heads into d_qkv (bf16, the QKV block's shape and
 * column order) at its heads' columns and leaves the other members'
 * columns alone (the conjugate of the scatter).  delta is caller-owned fp32
 * scratch of heads_of_device * batch * seq values.  P is recomputed from
 * lse; with delta_t = dO_t . O_t: dV = P^T dO, dS = P o (dO V^T - delta),
 * dQ = dS K / sqrt(d), dK = dS^T Q / sqrt(d), each accumulated by one
 * workgroup (deterministic).  Errors as atp_attention_fwd; d_qkv must not
 * share memory with qkv, out or d_out (INVALID_ARGUMENT). */
atp_status atp_attention_bwd(const atp_mesh* mesh, int32_t block_mode, int64_t batch, int64_t seq,
                             int64_t h, int32_t heads, const void* qkv, int64_t ld_qkv,
                             const void* out, int64_t ld_out, const float* lse, const void* d_out,
                             int64_t ld_dout, void* d_qkv, int64_t ld_dqkv, float* delta,
                             void* stream);

/* The attention block of one device (Sec. 3.2.1, with Sec. 2.1 Formula
 * (mha) as its core), chained: QKV (chunked, reduced with its bias over its
 * group) -> scatter of the reduced QKV block's heads over that group ->
 * causal attention core on the device's run of heads -> all-gather of the
 * heads' outputs (the out-proj input block) -> out-proj (chunked, reduced
 * with its bias).  One GPU holds one device: the all-gather's other columns
 * are the peers' data, as the partial tables are.
 *  x_loc        bf16 [tokens, k_loc of QKV]: the layer input block.
 *  qkv_partials host table of the QKV group's red_size buffers
 *               ([tokens, ldp_qkv] of partial_dtype; own entry written).
 *  qkv          bf16 [tokens, n_loc of QKV]: reduced QKV block (+ bias),
 *               written; token rows sequence-major (b * seq + t).
 *  attn         bf16 [tokens, k_loc of out-proj]: the gathered out-proj
 *               input.  The call writes its heads' columns (as
 *               atp_attention_fwd); the other columns must hold the other
 *               group members' outputs when the call is made.
 *  lse          fp32 [heads of the device][tokens], written.
 *  o_partials / o: out-proj's partial table and reduced output (+ bias).
 * Weights: entries 0 (qkv) and 1 (out) of w, in w->layout; 2 and 3 are
 * not read.  The attention core starts once the whole QKV block is reduced
 * (a causal sequence spans chunks), out-proj's chunks follow on
 * compute_stream and their reductions overlap the next chunk's GEMM on
 * comm_stream (Sec. 4.1).
 * workspace / ws_bytes: optional, caller-owned device memory (256-byte
 * aligned; atp_block_workspace_bytes() for the same mesh, mode, tokens, h,
 * chunks and weight layout is enough).  With it, as in atp_block_fwd, a
 * chunk product with too few tiles to fill the chip is split over k into
 * fp32 slabs there, summed in split order (so its bits can differ from the
 * unsplit product's by fp32 rounding), and weights stored [k][n] are copied
 * there as W^T where the products stream faster from it; without it the
 * products read the weights as stored.  Nothing in the workspace is read
 * before the call writes it.
 * Without such a workspace the call refuses a compute_stream under HIP
 * graph capture (as the block calls do).  Errors as atp_block_fwd and
 * atp_attention_fwd. */
typedef struct {
    const void* x_loc; int64_t ldx;
    void* const* qkv_partials; int64_t ldp_qkv;
    void* qkv; int64_t ld_qkv;
    void* attn; int64_t ld_attn;
    float* lse;
    void* const* o_partials; int64_t ldp_o;
    void* o; int64_t ld_o;
    int32_t partial_dtype;
} atp_attn_block_fwd_io;

atp_status atp_attention_block_fwd(const atp_mesh* mesh, int32_t block_mode, int64_t batch,
                                   int64_t seq, int64_t h, int32_t heads, int32_t chunks,
                                   const atp_block_weights* w, const atp_attn_block_fwd_io* io,
                                   void* workspace, size_t ws_bytes, void* compute_stream,
                                   void* comm_stream);

/* Backward of atp_attention_block_fwd (Sec. 4.2 through the chain):
 * out-proj's dX (chunked, reduced over its backward group) gives d_attn;
 * out-proj's dW and db; the attention core's backward on the device's heads
 * writes their dq, dk, dv columns of d_qkv (the conjugate of the scatter);
 * QKV's dX (chunked, reduced over its backward group), dW and db follow.
 *  x_loc, qkv, attn, lse: the forward's input, outputs and saved lse.
 *  d_o          bf16 gradient of o.
 *  d_attn_partials / d_attn: out-proj's backward table and the reduced
 *               gradient of the gathered block (bf16, written).
 *  delta        fp32 scratch of heads-of-device * tokens values.
 *  d_qkv        bf16 [tokens, n_loc of QKV]: the device's heads' columns are
 *               written; the other columns must hold the other group
 *               members' (the all-gather of the QKV block's gradient).
 *  dx_partials / dx: QKV's backward table and reduced input gradient.
 *  dw[0], db[0] (qkv), dw[1], db[1] (out): f32, as atp_block_bwd_io
 *               (dw in the weights' layout and leading dimension; db
 *               nullable).
 * workspace / ws_bytes: optional, caller-owned device memory (256-byte
 * aligned).  A workspace of atp_block_workspace_bytes() bytes for the same
 * mesh, mode, tokens, h and weight layout (or larger), with tokens a
 * multiple of 8, runs the dW products from transposed copies of X and dY
 * kept there (both operands contiguous along the tokens), with db from the
 * dY transpose, where that is the faster way; otherwise dW reads X and dY as
 * given.  Both paths give the same bits.  The workspace is scratch: nothing in it is read before
 * the call writes it.
 * Without such a workspace (or with tokens not a multiple of 8) the call
 * refuses a compute_stream under HIP graph capture.  Errors as
 * atp_block_bwd and atp_attention_bwd. */
typedef struct {
    const void* x_loc; int64_t ldx;
    const void* qkv; int64_t ld_qkv;
    const void* attn; int64_t ld_attn;
    const float* lse;
    const void* d_o; int64_t ld_do;
    void* const* d_attn_partials; int64_t ldp_da;
    void* d_attn; int64_t ld_d_attn;
    float* delta;
    void* d_qkv; int64_t ld_dqkv;
    void* const* dx_partials; int64_t ldp_dx;
    void* dx; int64_t ld_dx;
    float* dw[2];
    float* db[2];
    int32_t partial_dtype;
} atp_attn_block_bwd_io;

atp_status atp_attention_block_bwd(const atp_mesh* mesh, int32_t block_mode, int64_t batch,
                                   int64_t seq, int64_t h, int32_t heads, int32_t chunks,
                                   const atp_block_weights* w, const atp_attn_block_bwd_io* io,
                                   void* workspace, size_t ws_bytes, void* compute_stream,
                                   void* comm_stream);

/* atp_attention_bwd without the delta argument, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc): delta lives in a scratch array
 * the library holds on each GPU it runs on (4 MiB, 2^20 fp32 values, kept
 * until the process ends; its address is looked up once per device, on the
 * first call there).  The call allocates nothing.  heads-of-device * batch *
 * seq must be at most 2^20, else ATP_ERR_UNSUPPORTED before any work.  Every
 * call on one GPU shares that GPU's array (the backward writes each value
 * before reading it, so nothing needs clearing): calls that overlap on one
 * GPU -- on different streams, or from different threads -- race.  Other
 * arguments, results and errors as atp_attention_bwd. */
atp_status atp_attention_bwd_noalloc(const atp_mesh* mesh, int32_t block_mode, int64_t batch,
                                     int64_t seq, int64_t h, int32_t heads, const void* qkv,
                                     int64_t ld_qkv, const void* out, int64_t ld_out,
                                     const float* lse, const void* d_out, int64_t ld_dout,
                                     void* d_qkv, int64_t ld_dqkv, void* stream);

/* ------------------------------------------------------------------------
 * Position, cache and cached attention of one device's run of heads.
 *
 * What a layer needs around the attention core to be trained with positions
 * and to answer with: the norms of queries and keys with the position
 * rotation, a paged cache of keys and values, and the attention that reads
 * it.  The calls take the device's run of heads itself (atp_attention_heads
 * gives its first head: pass the buffer at that head's column).
 *
 * Head layout of a QKV row: for each of kv_heads key/value heads its `group`
 * query heads, the key and the value, 128 columns each ([q .. q | k | v];
 * group 1 is the block of atp_attention_fwd).  Rows of queries and of
 * attention outputs hold the kv_heads * group query heads in that order.
 * group is at most ATP_MAX_QUERY_GROUP.
 *
 * Lists, lengths and tables live in device memory (int32, 16-byte aligned),
 * so a step can be captured once and replayed as the lengths grow.  What the
 * host cannot see is checked by the kernels: a table entry outside
 * [0, n_pages) holds no tokens, rows and columns stay inside the sizes given
 * here, and nothing is read or written elsewhere.
 *
 * Buffers overlap when their bytes from the first element of the first row to
 * the last of the last do, with what lies between the rows: two column runs of
 * one buffer count as overlapping.
 * ------------------------------------------------------------------------ */
#define ATP_MAX_QUERY_GROUP 64
#define ATP_MAX_FORKS 4096

/* What is done to every query and key head row x (128 values), in fp32 and
 * rounded once:
 *   u = norm ? w o x / sqrt(mean(x^2) + eps) : x     (w: q_weight or k_weight)
 *   y = u with the pairs of its first rotary_dims values turned by the angle
 *       position * inv_freq[i], i = 0 .. rotary_dims / 2 - 1:
 *       (a, b) -> (a cos - b sin, b cos + a sin)
 * with pair i = (u[i], u[i + rotary_dims / 2]), or (u[2 i], u[2 i + 1]) when
 * interleaved.  The angle is formed and reduced in 64 bits.
 * q_weight, k_weight: bf16 [128], nullable (ones).  inv_freq: fp32
 * [rotary_dims / 2], radians per position.  rotary_dims: a multiple of 8 up
 * to 128, 0 for no rotation (inv_freq may be NULL).
 * Errors: INVALID_ARGUMENT for a NULL struct, negative or non-finite eps, eps
 * and norm flags out of range, weights without norm, rotary_dims outside [0,
 * 128], a missing inv_freq; UNSUPPORTED for rotary_dims not a multiple of 8,
 * misalignment. */
typedef struct {
    const void* q_weight;
    const void* k_weight;
    const float* inv_freq;
    float eps;
    int32_t norm;
    int32_t rotary_dims;
    int32_t interleaved;
} atp_qk_norm_rope;

/* The rows of a QKV block normed and turned: out = the block with its query
 * and key heads replaced, values copied (the input of atp_attention_fwd).
 * qkv, out: bf16 [batch*seq, kv_heads * (group + 2) * 128], token rows
 * sequence-major.  positions: int32 [batch*seq], or NULL for t % seq.  out
 * may be qkv itself (same pointer and ld; values are then not touched), else
 * they must not overlap.
 * Errors: INVALID_ARGUMENT for negative sizes, kv_heads or group < 1, NULL
 * buffers, overlap; UNSUPPORTED for more than 2^24 tokens, a group above
 * ATP_MAX_QUERY_GROUP, misalignment. */
atp_status atp_qk_norm_rope_fwd(int64_t batch, int64_t seq, int32_t kv_heads, int32_t group,
                                const atp_qk_norm_rope* params, const int32_t* positions,
                                const void* qkv, int64_t ld_qkv, void* out, int64_t ld_out,
                                void* stream);

/* Gradient of atp_qk_norm_rope_fwd.  qkv: the forward's input; d_out: the
 * gradient of its output (what atp_attention_bwd writes); d_qkv receives the
 * gradient of qkv and may be d_out itself (same pointer and ld), else it must
 * not overlap it, and never qkv.  With u' = y's gradient turned back and
 * r = 1 / sqrt(mean(x^2) + eps): dw = sum over rows of u' o x r (fp32 [128]
 * for the queries, shared by all their heads, and for the keys; nullable,
 * refused without norm), dx = r (g - x r mean(g o x r)) with g = w o u'.
 * The sums are formed in a fixed order.  workspace: caller-owned device
 * memory of atp_qk_norm_rope_workspace_bytes(batch*seq) bytes, scratch;
 * needed when a weight gradient is asked for.  Errors as
 * atp_qk_norm_rope_fwd; INVALID_ARGUMENT for a missing or short workspace. */
atp_status atp_qk_norm_rope_bwd(int64_t batch, int64_t seq, int32_t kv_heads, int32_t group,
                                const atp_qk_norm_rope* params, const int32_t* positions,
                                const void* qkv, int64_t ld_qkv, const void* d_out,
                                int64_t ld_dout, void* d_qkv, int64_t ld_dqkv, float* dq_weight,
                                float* dk_weight, void* workspace, size_t ws_bytes, void* stream);
/* 0 for a negative number of tokens. */
size_t atp_qk_norm_rope_workspace_bytes(int64_t tokens);

/* One layer's cache: bf16 pages[n_pages][2][kv_heads][page_size][128], the
 * keys then the values of page_size consecutive tokens of one sequence.
 * page_size: a power of two from 16 to 1024. */
typedef struct {
    void* pages;
    int32_t n_pages, kv_heads, page_size;
} atp_kv_cache;

/* A batch of n_seqs sequences.  Token i of sequence s is in page
 * table[s * ld_table + i / page_size] (columns [0, max_pages), at most 2^30
 * tokens); an entry outside [0, n_pages) is empty.  ctx[s]: tokens cached
 * before this step.  Rows [cu_new[s], cu_new[s + 1]) of the step's buffers
 * are the sequence's new tokens (cu_new: n_seqs + 1 ascending values, a
 * sequence may have none); token j of them goes to place ctx[s] + j of the
 * cache.  Rows behind cu_new[n_seqs] are padding, neither read nor written.
 * At most 65536 sequences. */
typedef struct {
    int32_t* table;
    int64_t ld_table;
    int32_t max_pages, n_seqs;
    const int32_t* ctx;
    const int32_t* cu_new;
} atp_kv_batch;

/* The new tokens of a step: queries normed and turned into q (bf16 [tokens,
 * kv_heads * group * 128]), keys normed and turned and values as they are into
 * the cache.  qkv: bf16 [tokens, kv_heads * (group + 2) * 128], the step's rows.
 * positions: int32 [tokens] (a drafted tree's depths), or NULL for the place
 * in the cache.  A row whose page is empty or beyond the table is not cached.
 * kv_heads is the cache's.  Errors as atp_qk_norm_rope_fwd, and those of the
 * cache and the batch: INVALID_ARGUMENT for NULL structs or members, sizes < 1
 * (n_seqs < 0), ld_table < max_pages; UNSUPPORTED for page sizes, alignment
 * and sizes beyond the limits above. */
atp_status atp_qk_norm_rope_cache(const atp_kv_cache* cache, const atp_kv_batch* batch,
                                  int64_t tokens, int32_t group, const atp_qk_norm_rope* params,
                                  const int32_t* positions, const void* qkv, int64_t ld_qkv,
                                  void* q, int64_t ld_q, void* stream);

/* Pages.  refs[n_pages] counts the table entries that name a page; 0 is
 * free.  The bookkeeping is one for all layers that share a table; the data
 * of a layer's cache moves by atp_cache_copy_pages and atp_cache_compact.
 * Calls that change refs or a table are ordered by their stream: run them on
 * one stream, or order the streams.
 *
 * atp_cache_reserve gives every sequence the pages that its new tokens go to.
 * An empty entry gets a free page; a page that other sequences hold too
 * (refs > 1) is replaced by a free one, and when it holds some of the
 * sequence's cached tokens (the page of place ctx[s] - 1 and ctx[s]) they have
 * to be copied: copy_src[s], copy_dst[s] name the pages and copy_rows[s] =
 * ctx[s] % page_size the tokens (-1, -1, 0 for no copy), for
 * atp_cache_copy_pages on every layer before the next call that gives pages
 * out.  Pages are given in ascending order to the sequences in ascending
 * order.  What is shared is decided by the counts at the call's start: all
 * holders of a page that write to it get a copy, the last one too, and the page
 * falls free.  A sequence gets all it needs or nothing: missing[s] is 0, or how
 * many pages it needs (all of them, free ones counted) when the pool (after the
 * sequences before it) or the table's columns cannot hold it; such a sequence
 * changes nothing, and the sequences behind it that need pages get none either
 * if it was the pool.  The time grows with the pages in front of the last free
 * one that is given.
 * workspace: atp_cache_workspace_bytes(n_pages, n_seqs) bytes, scratch.
 * missing, copy_src, copy_dst, copy_rows: int32 [n_seqs], written. */
atp_status atp_cache_reserve(int32_t n_pages, int32_t page_size, int32_t* refs,
                             const atp_kv_batch* batch, int32_t* missing, int32_t* copy_src,
                             int32_t* copy_dst, int32_t* copy_rows, void* workspace,
                             size_t ws_bytes, void* stream);
/* 0 for sizes below 1 (n_seqs below 0). */
size_t atp_cache_workspace_bytes(int32_t n_pages, int32_t n_seqs);

/* children[f] becomes a copy of parents[f], f < n_forks: it holds the pages of
 * the parent's ctx[parent] cached tokens too (no data moves: a shared page is
 * copied by atp_cache_reserve when one of its holders writes to it).  done[f]
 * (int32, written) is 0, or 1 for a fork that is refused and changes nothing:
 * an index outside the batch, a child that is a parent or an earlier child
 * of the call, or a child whose row still holds pages.  A parent may appear any
 * number of times.  The lengths (ctx) are the caller's.  n_forks is at most
 * ATP_MAX_FORKS. */
atp_status atp_cache_fork(int32_t n_pages, int32_t page_size, int32_t* refs,
                          const atp_kv_batch* batch, int32_t n_forks, const int32_t* parents,
                          const int32_t* children, int32_t* done, void* stream);

/* Every sequence with keep[s] >= 0 gives back the pages behind its first
 * keep[s] tokens (all of them for 0): their entries become -1 and their
 * reference counts fall by one.  keep: int32 [n_seqs].  ctx and cu_new are not
 * read. */
atp_status atp_cache_release(int32_t n_pages, int32_t page_size, int32_t* refs,
                             const atp_kv_batch* batch, const int32_t* keep, void* stream);

/* For i < n: the first rows[i] tokens (all for rows NULL) of page src[i], keys
 * and values of every head, are copied to page dst[i].  An entry with rows[i]
 * <= 0, an index outside the pool or src[i] == dst[i] does nothing.  A page
 * that is a destination must not appear a second time among src and dst (its
 * content is undefined then).  n is at most 2^23. */
atp_status atp_cache_copy_pages(const atp_kv_cache* cache, int32_t n, const int32_t* src,
                                const int32_t* dst, const int32_t* rows, void* stream);

/* Chosen rows behind ctx[s] are moved together: token ctx[s] + keep[cu_keep[s]
 * + i] goes to place ctx[s] + i, for i < cu_keep[s + 1] - cu_keep[s] (the
 * accepted path of a drafted tree, or the tokens of a context that are kept).
 * The indices of a sequence must ascend strictly.  moved (int32 [n_seqs],
 * nullable) receives the number of rows, or -1 for a sequence that is left
 * as it was: indices that do not ascend or are negative, or a place without
 * a page.  cu_keep: int32 [n_seqs + 1]; keep: int32 [n_keep].  The pages
 * written to must be held by this sequence alone.  cu_new is not read. */
atp_status atp_cache_compact(const atp_kv_cache* cache, const atp_kv_batch* batch,
                             const int32_t* cu_keep, const int32_t* keep, int32_t n_keep,
                             int32_t* moved, void* stream);

/* Attention of the step's new tokens over the cache, which holds them already
 * (atp_qk_norm_rope_cache): softmax(q k^T / sqrt(128)) v over what each token
 * sees, in fp32 (for the product with v weights are rounded to 16 significant
 * bits, to 8 where group * max_new is above 32).  New token
 * j of sequence s sees the ctx[s] cached tokens and, of the new ones, 0 .. j
 * (tree_mask NULL: a decode step, a chunk of a prompt) or those whose bit is
 * set in its row of tree_mask (uint64 [tokens][mask_words]; bit i % 64 of word
 * i / 64 is new token i of its sequence, itself included; tokens beyond the
 * words are not seen).  Whatever a masked or empty place holds does not reach
 * the result; an infinity or NaN among the values that a token sees reaches that
 * value of its result alone (a weight below 2^-100 of the largest may count as
 * 0, which gives NaN there).  A token that sees nothing gets zeros and a
 * log-sum-exp of -inf.
 * q, out: bf16 [tokens, kv_heads * group * 128], no overlap.  lse (nullable):
 * fp32 [kv_heads * group][tokens], the natural log-sum-exp of each row's
 * scaled scores.  max_new: the most new tokens a sequence is expected to have;
 * it chooses the kernel's tile (a sequence may have more).  workspace: caller-owned,
 * atp_attention_cache_workspace_bytes(kv_heads, group, max_new) bytes,
 * scratch.  Long contexts are split over workgroups and joined in a fixed
 * order: repeats give the same bits; another batch around a sequence or
 * another max_new can change its results by the roundings above.
 * Errors as atp_qk_norm_rope_cache; INVALID_ARGUMENT for max_new < 1,
 * mask_words < 1 with a mask, a short workspace. */
atp_status atp_attention_cache_fwd(const atp_kv_cache* cache, const atp_kv_batch* batch,
                                   int64_t tokens, int32_t group, int32_t max_new, const void* q,
                                   int64_t ld_q, const uint64_t* tree_mask, int32_t mask_words,
                                   void* out, int64_t ld_out, float* lse, void* workspace,
                                   size_t ws_bytes, void* stream);
/* 0 for sizes below 1 or a group above ATP_MAX_QUERY_GROUP. */
size_t atp_attention_cache_workspace_bytes(int32_t kv_heads, int32_t group, int32_t max_new);

/* ------------------------------------------------------------------------
 * Around the layers, for training on packed documents: the embedding of the
 * tokens, layer norms, the attention within documents, and the norm and
 * clipping of the gradients.
 *
 * Tables of a group's buffers (stats, sums) are host arrays of red_size device
 * pointers, as the partial tables are: this device's entry is written by its
 * own call before, the others hold the peers' data.  They are added in group
 * order, so every member gets the same bits.  Nothing is added by atomics:
 * repeats give the same bits.
 * ------------------------------------------------------------------------ */

/* Embedding on this device's rows [vocab_off, vocab_off + vocab_loc) of the
 * vocabulary and `cols` of its columns: Y = X W with one-hot rows X, W
 * row-first (Sec. 3.2), so where the vocabulary lies on several devices out is
 * Partial(SUM) over them (atp_chunked_partial_reduce):
 *   out[t, :] = scale * table[ids[t] - vocab_off, :], formed in fp32 and rounded
 *   once; zeros for a token outside this device's rows.
 * ids: int32 [tokens], any value.  table: bf16 [vocab_loc, cols].  out: fp32 or
 * bf16 [tokens, cols].
 * Errors: INVALID_ARGUMENT for negative sizes, vocab_loc or cols < 1, a negative
 * vocab_off, a non-finite scale, NULL buffers, out sharing memory with table or ids;
 * UNSUPPORTED for more than 2^24 tokens or rows, 2^37 values of out, cols not a multiple
 * of 8, misalignment. */
atp_status atp_embedding_fwd(int64_t tokens, const int32_t* ids, int64_t vocab_loc,
                             int64_t vocab_off, int64_t cols, const void* table, int64_t ld_table,
                             float scale, void* out, int32_t out_dtype, int64_t ld_out,
                             void* stream);

/* Gradient of the table (Sec. 4.2, dW = X^T dY):
 *   dtable[v, :] = scale * sum over t with ids[t] = vocab_off + v of dy[t, :],
 * the sum in fp32 over ascending t, in pieces that depend on the sizes and the ids
 * alone.  dy: bf16 [tokens, cols].  dtable: fp32 [vocab_loc, cols]; accumulate 0:
 * every row is written (zeros for rows without tokens); 1: the sums are added to
 * it and rows without tokens are not touched (a table that is the output
 * layer's weight too).  workspace: atp_embedding_workspace_bytes() bytes,
 * scratch.  Errors as atp_embedding_fwd; INVALID_ARGUMENT for another accumulate,
 * a short workspace, dtable or the workspace sharing memory with another buffer. */
atp_status atp_embedding_bwd(int64_t tokens, const int32_t* ids, int64_t vocab_loc,
                             int64_t vocab_off, int64_t cols, const void* dy, int64_t ld_dy,
                             float scale, float* dtable, int64_t ld_dtable, int32_t accumulate,
                             void* workspace, size_t ws_bytes, void* stream);
/* 0 for sizes that the call refuses (and for 0 tokens); what is enough for a number of
 * tokens is enough for fewer. */
size_t atp_embedding_workspace_bytes(int64_t tokens, int64_t vocab_loc, int64_t cols);

/* Layer norm of rows: y = (x - mean(x)) / sqrt(mean((x - mean(x))^2) + eps) o weight
 * + bias.  weight, bias: bf16 [cols], this device's columns, nullable (ones,
 * zeros). */
typedef struct {
    const void* weight;
    const void* bias;
    float eps;
} atp_layer_norm;

/* The norm of x (atp_dtype `dtype`, [tokens, cols], the residual stream), or with
 * add (bf16 [tokens, cols], a linear's reduced output) of x_out = x + add, which is
 * formed in fp32, rounded to `dtype` and stored; the norm is that of the stored
 * values.  x_out may be x itself (same pointer and ld).  y: bf16 [tokens, cols].
 * mean, rstd: fp32 [tokens], written for the backward.
 * Rows whose columns lie on several devices (h / d2 or h / d1 columns each, all the
 * same number): red_size devices, `cols` the local columns, stats the table of their
 * statistics (fp32 [tokens][2]: mean and sum of centred squares of the local
 * columns), each written by atp_layer_norm_stats, which also forms the sum: add
 * and x_out are then NULL and x is the stored sum.  red_size 1 and stats NULL:
 * whole rows, one call.
 * Statistics in fp32, of values centred first.  An infinity or NaN stays in its row.
 * Errors: INVALID_ARGUMENT for negative sizes, cols < 1, a bad dtype, a negative or
 * non-finite eps, NULL buffers, add without x_out or with stats, buffers that
 * overlap otherwise than above, red_size < 1; UNSUPPORTED for more than 2^24
 * tokens or 32768 columns, 2^32 threads of 16 to 32 columns each in the two calls below
 * (13.4 million rows of 4104 columns), cols not a multiple of 8, misalignment, red_size
 * above ATP_MAX_GROUP. */
atp_status atp_layer_norm_fwd(int64_t tokens, int64_t cols, int32_t dtype,
                              const atp_layer_norm* norm, const void* x, int64_t ldx,
                              const void* add, int64_t ld_add, void* x_out, int64_t ld_xout,
                              int32_t red_size, const float* const* stats, void* y, int64_t ld_y,
                              float* mean, float* rstd, void* stream);
atp_status atp_layer_norm_stats(int64_t tokens, int64_t cols, int32_t dtype, const void* x,
                                int64_t ldx, const void* add, int64_t ld_add, void* x_out,
                                int64_t ld_xout, float* stats, void* stream);

/* Gradient of atp_layer_norm_fwd.  x: the normed values (x, or x_out where there was an
 * add); mean, rstd: the forward's; dy: bf16 gradient of y.  With xh = (x - mean) rstd
 * and g = weight o dy, over the whole row:
 *   dx = rstd (g - mean(g) - xh mean(g o xh)) + d_res,
 *   dweight = sum over rows of dy o xh,  dbias = sum over rows of dy.
 * d_res: the gradient that reaches x_out past the norm (`dtype`, nullable).  dx:
 * `dtype`, may be d_res itself (same pointer and ld); it is the gradient of x and of
 * add.  d_add (nullable): dx rounded to bf16 from fp32, for the linear that add came
 * from.  dweight, dbias: fp32 [cols], nullable, overwritten (batches are added up by the
 * caller); they need a workspace of atp_layer_norm_workspace_bytes(tokens, cols) bytes.
 * Rows on several devices: sums is the table of the devices' two row sums (fp32
 * [tokens][2]: g and g o xh over the local columns), each written by
 * atp_layer_norm_bwd_sums.  Errors as atp_layer_norm_fwd; INVALID_ARGUMENT for a
 * short workspace. */
atp_status atp_layer_norm_bwd(int64_t tokens, int64_t cols, int32_t dtype,
                              const atp_layer_norm* norm, const void* x, int64_t ldx,
                              const float* mean, const float* rstd, const void* dy, int64_t ld_dy,
                              const void* d_res, int64_t ld_dres, int32_t red_size,
                              const float* const* sums, void* dx, int64_t ld_dx, void* d_add,
                              int64_t ld_dadd, float* dweight, float* dbias, void* workspace,
                              size_t ws_bytes, void* stream);
atp_status atp_layer_norm_bwd_sums(int64_t tokens, int64_t cols, int32_t dtype,
                                   const atp_layer_norm* norm, const void* x, int64_t ldx,
                                   const float* mean, const float* rstd, const void* dy,
                                   int64_t ld_dy, float* sums, void* stream);
/* 0 for sizes that the call refuses (and for 0 tokens); what is enough for a number of
 * tokens is enough for fewer. */
size_t atp_layer_norm_workspace_bytes(int64_t tokens, int64_t cols);

/* Documents of packed rows.  Rows [cu_docs[d], cu_docs[d + 1]) are document d (int32
 * [n_docs + 1], ascending, device memory; a document may be empty); rows outside
 * all documents are padding, neither read nor written.  Row i of a document of n
 * rows sees its rows j <= i, and the first prefix[d] rows (int32 [n_docs], nullable;
 * cut to [0, n]).  Scores: x = q . k / sqrt(128), with cap > 0 cap * tanh(x / cap), then
 * minus slopes[head] * |i - j| (fp32 [kv_heads * group], nullable; constants: they
 * get no gradient).  A cap of up to 64 moves a score by up to 6 * 2^-24 of the cap beside
 * fp32's roundings of the product, a larger one, up to 2^100, by up to 2^-18 of the
 * score.  At most 65536 documents.  Lists that do not ascend or leave
 * the rows give undefined results, but no access outside the buffers. */
typedef struct {
    const int32_t* cu_docs;
    const int32_t* prefix;
    const float* slopes;
    int32_t n_docs;
    float cap;
} atp_attention_docs;

/* Attention of the device's run of heads within documents, for training.  qkv: bf16
 * [tokens, kv_heads * (group + 2) * 128] in the head layout of
 * atp_qk_norm_rope_fwd (what it writes).  out: bf16 [tokens, kv_heads * group *
 * 128]; lse: fp32 [kv_heads * group][tokens], the natural log-sum-exp of each row's
 * scores.  Scores, softmax and sums in fp32; weights are rounded to bf16 for the
 * product with v.  Whatever other documents, padding or, in the forward, rows that a
 * row does not see hold does not reach its result.
 * Errors: INVALID_ARGUMENT for negative sizes, kv_heads or group < 1, NULL buffers,
 * a negative or non-finite cap, overlap; UNSUPPORTED for more than 2^24 tokens, the
 * limits above, a cap above 2^100, 2^24 tiles of 64 rows of all documents (empty ones count
 * one) and heads, misalignment. */
atp_status atp_attention_docs_fwd(int64_t tokens, int32_t kv_heads, int32_t group,
                                  const atp_attention_docs* docs, const void* qkv, int64_t ld_qkv,
                                  void* out, int64_t ld_out, float* lse, void* stream);

/* Gradient of atp_attention_docs_fwd: out and lse are the forward's, d_out (bf16) the
 * gradient of out, d_qkv (bf16) receives dq, dk, dv of the documents' rows in qkv's
 * layout and must not overlap qkv, out or d_out.  dk and dv are summed in fp32 over the
 * group's query heads.  The weights are formed again from lse, whose last bit moves
 * them by |lse| 2^-23 of themselves; scores of 2^30 and more have no defined gradient.
 * Weights are rounded to bf16 for dv's product with d_out, and the scores' gradients
 * for those with k and q that give dq and dk.  An infinity or NaN in a document may
 * reach all gradients of that document, and no other.  workspace:
 * atp_attention_docs_workspace_bytes() bytes, scratch.  Errors as
 * atp_attention_docs_fwd; INVALID_ARGUMENT for a short workspace. */
atp_status atp_attention_docs_bwd(int64_t tokens, int32_t kv_heads, int32_t group,
                                  const atp_attention_docs* docs, const void* qkv, int64_t ld_qkv,
                                  const void* out, int64_t ld_out, const float* lse,
                                  const void* d_out, int64_t ld_dout, void* d_qkv, int64_t ld_dqkv,
                                  void* workspace, size_t ws_bytes, void* stream);
/* 0 for sizes that the call refuses (and for 0 tokens); what is enough for a number of
 * tokens is enough for fewer. */
size_t atp_attention_docs_workspace_bytes(int64_t tokens, int32_t kv_heads, int32_t group);

/* One gradient: src [rows, cols], fp32 or bf16 (ld_src elements between rows; for one
 * row, or rows without gaps, cols and ld may be any number, else leading dimensions
 * are multiples of 8), and where its clipped values go: dst, of either type, or src
 * itself. */
typedef struct {
    const void* src;
    void* dst;
    int64_t rows, cols, ld_src, ld_dst;
    int32_t src_dtype, dst_dtype;
} atp_grad;

/* *sum = sum of the squares of all values of n gradients, in 64 bits and a fixed
 * order (device memory, 8-byte aligned, written; 0 for none).  dst is not looked
 * at.  Where a gradient is held by several devices, list it on one of them.
 * grads is read during the call only.  workspace:
 * atp_grad_workspace_bytes(n, grads) bytes, scratch.
 * Errors: INVALID_ARGUMENT for NULL pointers, negative sizes, bad dtypes, ld < cols, a
 * short workspace; UNSUPPORTED for misalignment, leading dimensions above, more than
 * 2^31 - 1 rows or 2^40 values. */
atp_status atp_grad_sq_sum(int32_t n, const atp_grad* grads, double* sum, void* workspace,
                           size_t ws_bytes, void* stream);
/* 0 for a list that the calls refuse (and for no values). */
size_t atp_grad_workspace_bytes(int32_t n, const atp_grad* grads);

/* Clipping by the norm over all devices: with S the sum of the red_size devices' sums
 * (sums: host table of device pointers, 8-byte aligned, added in group order),
 *   norm = scale * sqrt(S),  factor = scale * (norm > max_norm ? max_norm / norm : 1),
 *   dst = factor * src, rounded once, for each gradient.
 * scale: what the gradients are to be multiplied by in any case (1 / loss scale, 1 /
 * number of accumulated batches).  norm: fp32 [2], 8-byte aligned, receives norm and
 * factor.  An infinite norm gives factor 0 (NaN where the gradient is infinite) unless
 * max_norm is infinite too, a NaN one NaN everywhere: look at norm before using dst.
 * A dst must be its src itself (type and leading dimension too) or overlap no src, and
 * no other dst (the call looks at pairs of one gradient alone, from the first value to
 * the last).  Errors as atp_grad_sq_sum; INVALID_ARGUMENT for scale or max_norm not
 * positive (max_norm may be infinite), red_size < 1; UNSUPPORTED for red_size above
 * ATP_MAX_GROUP. */
atp_status atp_grad_clip(int32_t n, const atp_grad* grads, int32_t red_size,
                         const double* const* sums, float scale, float max_norm, float* norm,
                         void* stream);

/* Per-kernel timing of the library's own launches.  When enabled, every
 * kernel the library enqueues is bracketed by HIP events on its stream;
 * atp_profile_collect synchronises those events, fills up to `max`
 * records (one per kernel name: launches, total milliseconds, total
 * algorithmic FLOPs and bytes) and clears the log.  Returns the number of
 * records, or -1 on a HIP error. */
typedef struct {
    char name[64];
    int64_t launches;
    double total_ms;
    double flops;
    double bytes;
} atp_kernel_stat;

/* on: 0 = off, 1 = one record per kernel, 2 = one record per kernel and
 * problem shape (names carry M x N x K and the epilogue). */
void atp_profile_enable(int32_t on);
int32_t atp_profile_collect(atp_kernel_stat* out, int32_t max);

const char* atp_status_string(int32_t status);
const char* atp_last_error(void);
const char* atp_version(void);

/* ------------------------------------------------------------------------
 * Mesh planner (host only; no GPU needed, nothing is enqueued).
 *
 * Picks the DeviceMesh(d1, d2) of least tensor-parallel communication time
 * for N devices on an interconnect described by a hierarchical
 * communication matrix (HCM, Sec. 3.4): the search space is every (d1, d2)
 * with d1 * d2 = N (Sec. 3.2), the per-axis all-reduce bandwidths come from
 * Eq. (bwd) and Eq. (allreduce) (Sec. 3.5), the time from Eq. (tcomm)
 * (Sec. 3.3).
 *
 * HCM: `n_layers` layers, outermost first (e.g. nodes, then GPUs in a
 * node).  Device r of the mesh (r = i1 * d2 + i2) has, at layer j, the rank
 * index (r / D_j) % R_j, with D_j the product of the rank counts of the
 * layers inside j.  Axis 1 all-reduces run among the devices with equal i2,
 * axis 2 among those with equal i1.
 *
 * B1' / B2' (Eq. (bwd)): at every layer an axis group spans with more than
 * one rank of one parent, each spanned rank u offers the group
 * min(group_bw, sum of p2p[u][v] over the group's other ranks v there),
 * divided by the number of that axis's groups spanning the layer through u;
 * B' is the least such value over the group's layers.  This is the paper's
 * division by d2 when a node hosts d2 groups, its P2P correction of
 * DeviceMesh(8, 2), and no division when ranks are single devices (its
 * switch and torus cases).  B = d / (2 (d - 1)) B' (Eq. (allreduce)); an
 * axis of size 1 has no all-reduce (B' = 0, B = +inf, its Eq. (tcomm) term
 * is 0).  T_comm = 2 L b s elem_bytes (7 h / (d1 B2) + 2 h / (d2 B1)) / 1e9
 * seconds for bandwidths in GB/s; +inf when a spanned rank has no
 * bandwidth to the rest of its group.
 *
 * Errors: ATP_ERR_INVALID_ARGUMENT for NULL pointers, n_layers outside
 * 1..ATP_PLAN_MAX_LAYERS, a rank count < 1, a group_bw <= 0 or not finite, a
 * negative or non-finite p2p entry, model sizes < 1, elem_bytes < 1, a
 * bandwidth given to atp_tcomm that is not > 0 (+inf is allowed), or a
 * `costs` array too small; ATP_ERR_SHAPE when d1 * d2 differs from the
 * HCM's device count; ATP_ERR_UNSUPPORTED above ATP_PLAN_MAX_DEVICES devices.
 * ------------------------------------------------------------------------ */
#define ATP_PLAN_MAX_LAYERS 16
#define ATP_PLAN_MAX_DEVICES 65536

typedef struct {
    int32_t ranks;       /* ranks of this layer under one parent, >= 1 */
    double group_bw;     /* GB/s from one rank of this layer to outside it */
    const double* p2p;   /* [ranks][ranks] row-major GB/s between ranks of one
                            parent (diagonal ignored); NULL = every pair at
                            group_bw, as behind a switch.  Host memory, read
                            during the call only. */
} atp_hcm_layer;

typedef struct {
    int64_t layers;      /* L, transformer layers */
    int64_t batch;       /* b */
    int64_t seq;         /* s */
    int64_t hidden;      /* h */
    int32_t elem_bytes;  /* bytes per all-reduced element (2 for fp16 / bf16) */
} atp_model_dims;

typedef struct {
    int32_t d1, d2;
    double b1_eff, b2_eff;  /* B1', B2' in GB/s (0 for an axis of size 1) */
    double b1, b2;          /* Eq. (allreduce) bandwidths, GB/s (+inf for size 1) */
    double t_comm;          /* Eq. (tcomm), seconds */
} atp_mesh_cost;

/* Eq. (tcomm) for given algorithm bandwidths b1, b2 (GB/s, > 0, +inf = no
 * all-reduce on that axis), e.g. calibrated from measured all-reduces
 * (Sec. 5.3).  *t_out in seconds. */
atp_status atp_tcomm(const atp_model_dims* dims, int32_t d1, int32_t d2, double b1, double b2,
                     double* t_out);

/* B1', B2', B1, B2 and T_comm of DeviceMesh(d1, d2) on the HCM. */
atp_status atp_hcm_mesh_cost(const atp_hcm_layer* hcm, int32_t n_layers,
                             const atp_model_dims* dims, int32_t d1, int32_t d2,
                             atp_mesh_cost* out);

/* Every candidate mesh of the HCM's N devices, largest d1 first: when
 * `costs` is not NULL their costs go to costs[0 .. n-1] (max_costs must be
 * >= n); *n_meshes (if not NULL) receives n; *best receives the cost of the
 * mesh of least T_comm (ties: the larger d1). */
atp_status atp_plan_mesh(const atp_hcm_layer* hcm, int32_t n_layers, const atp_model_dims* dims,
                         atp_mesh_cost* best, atp_mesh_cost* costs, int32_t max_costs,
                         int32_t* n_meshes);

#ifdef __cplusplus
}
#endif
#endif
