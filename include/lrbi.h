/*
 * lrbi -- inference with a layer pruned by a tiled low-rank binary index (B200, sm_100a).
 *
 * Plain C ABI.  The pruning index of a layer W [rows x cols] (rows = output features,
 * cols = input features) is not stored; it is rebuilt from two small binary factors per
 * tile.  The index matrix is cut into equal tiles of tile_rows x tile_cols (Section 3.1
 * of the paper: each block is factorised, hence decoded, independently, all with the same
 * rank k).  For tile (tr, tc) with factors Ip (tile_rows x k) and Iz (k x tile_cols) the
 * decoded index is the Boolean matrix product of Eq. 3,
 *
 *        Ia[i][j] = OR_{l=1..k} ( Ip[i][l] AND Iz[l][j] ),
 *
 * where a 1 keeps the weight and a 0 prunes it to zero (Section 2, Eq. 1-2).  Ia is the
 * masking layer of the layer (Sections 2 and 2.2), so the layer computes
 * Y = X * (W .* Ia)^T.
 *
 * Packed factor format (KW = ceil(k / 32) 32-bit words per row of Ip / per column of Iz,
 * GR = ceil(rows / tile_rows), GC = ceil(cols / tile_cols), tile index t = tr * GC + tc):
 *
 *   ip[(t * tile_rows + i) * KW + w]   bit (l % 32) of word w = l / 32   is  Ip_t[i][l]
 *   iz[(t * tile_cols + j) * KW + w]   bit (l % 32) of word w = l / 32   is  Iz_t[l][j]
 *
 * Edge tiles still hold tile_rows row words and tile_cols column words; those that fall
 * outside the matrix are ignored.  Bits at positions >= k of the last word are ignored.
 *
 * Unless an argument says "host", every pointer is a DEVICE pointer owned by the caller,
 * valid on the current device, 16-byte aligned.  Calls are asynchronous and ordered on
 * `stream` (a cudaStream_t passed as void*, NULL = the legacy default stream).  Inputs are
 * only read.  Nothing outside the stated output extent is written.  Argument errors are
 * detected on the host before anything is launched and reported by the return code; no
 * call aborts, throws or traps.  There is no CPU fallback: without a usable sm_100 device
 * a compute call returns LRBI_ERR_CUDA.
 *
 * Timeouts.  Every wait inside a kernel is bounded (about two seconds); a wait that runs out
 * leaves a code in a per-device status word, the kernel ends early and its output is
 * incomplete.  The asynchronous calls (lrbi_decode_mask, lrbi_masked_gemm, ..._static) cannot
 * know this when they return.  The contract is: a call that synchronises
 * (lrbi_layer_forward_host, lrbi_device_status, lrbi_last_device_error) reads the word; once
 * it has been seen non-zero, every compute call on that device returns LRBI_ERR_TIMEOUT and
 * launches nothing until lrbi_device_status(1) clears it.  A caller of the asynchronous calls
 * checks lrbi_device_status after synchronising its stream.
 *
 * Threads.  Entry points may be called from several host threads; the library's own lazily
 * built state is guarded by one lock.  Two calls that use the K-split buffer of
 * lrbi_masked_gemm (or the fixed array of lrbi_masked_gemm_static) at the same time on
 * different streams race on the device: order them.
 *
 * Non-finite values.  A NaN/Inf stored in a PRUNED weight never reaches Y (the weight is
 * selected away).  Activations must be finite: the tensor-core kernels zero the pruned weight
 * and still multiply, so an Inf/NaN in X at a pruned column gives NaN there, while the
 * CUDA-core kernels skip the product; which kernel runs depends on the batch.
 */
#ifndef LRBI_H_
#define LRBI_H_

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define LRBI_API __attribute__((visibility("default")))
#else
#define LRBI_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    LRBI_OK = 0,
    LRBI_ERR_INVALID_ARG = 1, /* null pointer, non-positive size, misaligned pointer          */
    LRBI_ERR_UNSUPPORTED = 2, /* a shape, dtype or kernel choice this library does not cover   */
    LRBI_ERR_CUDA = 3,        /* a CUDA runtime/driver call failed (see lrbi_last_cuda_error)  */
    LRBI_ERR_TIMEOUT = 4,     /* a bounded device-side wait gave up earlier on this device and has
                                 been seen by a synchronising call; cleared by lrbi_device_status(1) */
    LRBI_ERR_TOO_LARGE = 5    /* the problem needs more fixed scratch than the library carries   */
} lrbi_status;

/* Geometry of one pruned layer (Section 3.1: equal tiles, one rank). */
typedef struct {
    int32_t rows;      /* output features: rows of W and of the index          */
    int32_t cols;      /* input features: columns of W and of the index        */
    int32_t tile_rows; /* tm >= 1                                               */
    int32_t tile_cols; /* tn >= 1                                               */
    int32_t rank;      /* k >= 1, the same for every tile                       */
} lrbi_layout;

/* Output element type of lrbi_masked_gemm. */
enum { LRBI_Y_BF16 = 0, LRBI_Y_F32 = 1 };

/* Kernel choice for lrbi_masked_gemm / lrbi_decode_mask (LRBI_ALGO_AUTO picks by shape). */
enum {
    LRBI_ALGO_AUTO = 0,
    LRBI_ALGO_GENERIC = 1,   /* any shape; one thread per output, slow                         */
    LRBI_ALGO_GEMV = 2,      /* small batch, bandwidth-bound, CUDA-core FMA                    */
    LRBI_ALGO_TENSOR = 3,    /* tcgen05 MMA with TMEM accumulators                             */
    LRBI_ALGO_DECODE_BALLOT = 4, /* decode: one __ballot_sync per 32-bit mask word             */
    LRBI_ALGO_DECODE_PLANES = 5, /* decode: Iz transposed into bit-planes, OR per 32 columns (variant by size) */
    LRBI_ALGO_DECODE_PLANES_WIDE = 6, /* decode: the 1024-column bit-plane variant, whatever the mask size */
    LRBI_ALGO_STREAM = 7,    /* batch <= 32, bandwidth-bound, warp-level tensor-core MMAs              */
    /* The next two force an instantiation that LRBI_ALGO_TENSOR otherwise picks from the problem size
       (any shape LRBI_ALGO_TENSOR covers; small problems just leave most of a tile empty). */
    LRBI_ALGO_TENSOR_PAIR = 8,  /* tcgen05 CTA pairs (cta_group::2), 256 rows x 256 batch rows per pair  */
    LRBI_ALGO_TENSOR_PAIR2 = 9, /* CTA pairs with two accumulators: 256 rows x 512 batch rows per pair   */
    LRBI_ALGO_TENSOR_PAIR192 = 10 /* CTA pairs, one accumulator of 192 batch rows (few rows, long batch)   */
};

/* Element counts of the packed arrays for a layout (0 if the layout is invalid). */
LRBI_API size_t lrbi_packed_ip_words(const lrbi_layout *layout); /* GR*GC*tile_rows*KW */
LRBI_API size_t lrbi_packed_iz_words(const lrbi_layout *layout); /* GR*GC*tile_cols*KW */
LRBI_API size_t lrbi_mask_words(const lrbi_layout *layout);      /* rows*ceil(cols/32) */

/*
 * Decode the whole index (Eq. 3 per tile, Section 3.1) into a bit-packed mask.
 *   ip, iz    device, packed factors as above (read only)
 *   mask_out  device, rows x ceil(cols/32) uint32, row-major; bit (c % 32) of word c / 32
 *             of row r is Ia[r][c]; bits beyond `cols` in the last word of a row are 0.
 *   algo      LRBI_ALGO_AUTO, LRBI_ALGO_DECODE_BALLOT, LRBI_ALGO_DECODE_PLANES (needs
 *             tile_cols % 32 == 0) or LRBI_ALGO_DECODE_PLANES_WIDE (needs rank <= 256 and tiles of 128, 256,
 *             512 or a multiple of 1024 columns, or a single tile column of a multiple of 128 columns);
 *             a variant that does not cover the layout returns LRBI_ERR_UNSUPPORTED
 * Every word of mask_out is written; nothing else is.
 */
LRBI_API lrbi_status lrbi_decode_mask(const lrbi_layout *layout, const uint32_t *ip, const uint32_t *iz,
                             uint32_t *mask_out, int32_t algo, void *stream);

/*
 * Fused decode + prune + dense product (Eq. 3; masking layer of Sections 2 and 2.2):
 *       Y[b][o] = sum_i  Ia[o][i] ? X[b][i] * W[o][i] : 0      (fp32 accumulation)
 * The decoded index never reaches device memory.  A pruned weight is selected away (its bf16
 * pattern is replaced by +0 or its product is skipped), so a NaN/Inf stored in a pruned
 * position does not reach Y.  X must be finite (see "Non-finite values" above).
 *   W      device, bf16 bit patterns, [rows][cols] row-major
 *   X      device, bf16 bit patterns, [batch][cols] row-major
 *   Y      device, [batch][rows] row-major, bf16 (round to nearest even) or fp32 per y_dtype
 *   algo   LRBI_ALGO_AUTO, _GENERIC, _GEMV (batch <= 8), _STREAM (batch <= 32), _TENSOR, _TENSOR_PAIR or
 *          _TENSOR_PAIR2 / _TENSOR_PAIR192; a kernel that does not
 *          cover the shape returns LRBI_ERR_UNSUPPORTED and launches nothing.
 * The tensor-core path may split the reduction over several thread blocks; it then keeps
 * fp32 partial sums in a library-owned device buffer that grows (cudaMalloc) on the first
 * call that needs more, so such a first call must not be made during stream capture.
 * Calls that use that buffer concurrently on different streams are not supported.
 */
LRBI_API lrbi_status lrbi_masked_gemm(const lrbi_layout *layout, const uint16_t *W, const uint32_t *ip,
                             const uint32_t *iz, const uint16_t *X, int32_t batch, void *Y,
                             int32_t y_dtype, int32_t algo, void *stream);

/*
 * lrbi_masked_gemm for callers that must not allocate device memory.  (The paper has no
 * counterpart to this call; it exists for the library's users.)
 *
 * Who needs it: code that runs inside a memory-pool or arena discipline where every device byte
 * is accounted for up front (an inference server that sizes its pool at start-up and treats a
 * later cudaMalloc as a bug), code that runs where cudaMalloc may block or fail at a bad moment
 * (it takes a device-wide lock and can synchronise; under memory pressure it returns an error in
 * the middle of a request), and plug-ins that are simply not given the right to allocate.
 * lrbi_masked_gemm may allocate: when it splits the reduction over K it keeps fp32 partial sums
 * in a buffer that it grows with cudaMalloc.  This call never does.  It always runs the
 * tensor-core kernel (LRBI_ALGO_TENSOR shapes only, else LRBI_ERR_UNSUPPORTED) and keeps the
 * partial sums in a fixed array that is part of the library image: LRBI_STATIC_SCRATCH_BYTES
 * (8 MiB) of device memory on every GPU that loads the library, held until the process exits.
 *
 *   - If splits * batch * rows * 4 bytes exceeds that array the call returns LRBI_ERR_TOO_LARGE
 *     and launches nothing (lrbi_masked_gemm_static_bytes tells the need in advance; 0 = no
 *     scratch needed).  Problems with enough output tiles to fill the GPU do not split K and need none.
 *   - It calls no cudaMalloc, cudaFree or any other allocating routine.
 *   - The first call on a device looks up the array's device address (once per device, with that
 *     device current) and caches it; make that first call before starting any stream capture.
 *   - All calls on a device share the one array, and it keeps whatever the last call left in it.
 *     Nothing has to be cleared: every word the reduction reads was written earlier in the same
 *     call.  But two calls that overlap on the GPU (different streams) race on it and give wrong
 *     results: keep calls to this entry point on one stream, or order them with events.
 * Arguments, layouts and results are those of lrbi_masked_gemm with LRBI_ALGO_TENSOR.
 */
#define LRBI_STATIC_SCRATCH_BYTES (8u * 1024u * 1024u)
LRBI_API lrbi_status lrbi_masked_gemm_static(const lrbi_layout *layout, const uint16_t *W, const uint32_t *ip,
                                             const uint32_t *iz, const uint16_t *X, int32_t batch, void *Y,
                                             int32_t y_dtype, void *stream);
LRBI_API size_t lrbi_masked_gemm_static_bytes(const lrbi_layout *layout, int32_t batch);

/*
 * Same computation for callers whose activations live in host memory (the index and the
 * weights are uploaded once, activations and results cross the bus on every call).
 *   lrbi_layer_create   copies W, ip, iz (HOST pointers) to the current device and reserves
 *                       staging for up to max_batch rows.  *out owns device memory.
 *   lrbi_layer_forward_host   X_host [batch][cols] bf16 and Y_host [batch][rows] are HOST
 *                       pointers (pinned memory makes the copies asynchronous and overlapped
 *                       with the kernels, chunk by chunk); returns after Y_host is complete.
 *   lrbi_layer_destroy  frees everything the handle owns.
 */
typedef struct lrbi_layer lrbi_layer;
LRBI_API lrbi_status lrbi_layer_create(const lrbi_layout *layout, const uint16_t *W_host,
                              const uint32_t *ip_host, const uint32_t *iz_host,
                              int32_t max_batch, lrbi_layer **out);
LRBI_API lrbi_status lrbi_layer_forward_host(lrbi_layer *layer, const uint16_t *X_host, int32_t batch,
                                    void *Y_host, int32_t y_dtype, int32_t algo);
LRBI_API lrbi_status lrbi_layer_destroy(lrbi_layer *layer);

/*
 * Inner loop of Algorithm 1 (Section 2.1: "binary pruning-index-data matrix factorization").  The NMF of
 * |W| and the search over S_p stay with the caller; these two calls are the steps the search repeats.
 *
 * lrbi_threshold_pack: binary conversion of the NMF factors (the sentence under Eq. 4; Eq. 4 -> Eq. 5),
 *       (Ip)[i][l] = 1 if (Mp)[i][l] >= T_p else 0,     (Iz)[l][j] = 1 if (Mz)[l][j] >= T_z else 0,
 * written in the packed factor format above.  Every tile is its own factorisation (Section 3.1) and has its
 * own pair of thresholds.
 *   mp   device, fp32, [GR*GC][tile_rows][rank]   row-major per tile
 *   mz   device, fp32, [GR*GC][rank][tile_cols]   row-major per tile
 *   tp, tz   device, fp32, [GR*GC]   thresholds of each tile (+inf gives an empty factor)
 *   ip_out, iz_out   device, lrbi_packed_ip_words / lrbi_packed_iz_words words; bits >= rank are written as 0
 *
 * lrbi_index_cost: what the search looks at for one candidate (ip, iz), per tile, tiles in row-major grid order:
 *   kept_i = number of ones of the magnitude index I = (|W| >= theta)            (Eq. 1 -> Eq. 2)
 *   kept_a = number of ones of the decoded index Ia = Ip (x) Iz                  (Eq. 3; S_a = 1 - kept_a / size)
 *   lost   = number of positions with I = 1 and Ia = 0
 *   cost   = sum of |W| over those positions                                    (the Cost line of Algorithm 1)
 * W is read once, Ia is decoded on the fly and never stored.  A NaN weight counts as pruned (I = 0).  cost is
 * summed in fp32 per 8 weights and in fp64 beyond; blocks add to a tile's record with atomics, so the last bits
 * of cost may differ between calls.
 *   W    device, bf16 bit patterns, [rows][cols]
 *   out  device, GR*GC records, 8-byte aligned; overwritten
 * Only positions inside the matrix are counted (edge tiles are smaller).
 */
typedef struct {
    uint64_t kept_i;
    uint64_t kept_a;
    uint64_t lost;
    double cost;
} lrbi_tile_cost;
LRBI_API lrbi_status lrbi_threshold_pack(const lrbi_layout *layout, const float *mp, const float *mz, const float *tp,
                                         const float *tz, uint32_t *ip_out, uint32_t *iz_out, void *stream);
LRBI_API lrbi_status lrbi_index_cost(const lrbi_layout *layout, const uint16_t *W, float theta, const uint32_t *ip,
                                     const uint32_t *iz, lrbi_tile_cost *out, void *stream);

/*
 * Generalised layouts (Section 3.1, last paragraph: "each submatrix can optimally choose a different rank").
 *
 * Ranked layout: tile t (row-major grid order) has its own rank k_t, 0 <= k_t <= layout->rank (the layout's rank is
 * then only the upper bound), and is packed with KW_t = ceil(k_t / 32) words per row of Ip / column of Iz:
 *       ip[ip_offset[t] + i * KW_t + w],      iz[iz_offset[t] + j * KW_t + w]
 * so a tile of low rank takes less room (k_t (tile_rows + tile_cols) bits, the index size of Section 2 for that
 * tile).  A tile of rank 0 is empty: everything in it is pruned.  The three arrays are DEVICE arrays of GR*GC
 * entries; offsets count 32-bit words.  Tile bases need only 4-byte alignment.
 *   lrbi_decode_mask_ranked   Eq. 3 per tile with the tile's rank -> bit-packed mask (as lrbi_decode_mask)
 *   lrbi_masked_gemm_ranked   the fused product (as lrbi_masked_gemm); the tensor-core kernel runs when the shape
 *                             allows it (LRBI_ALGO_TENSOR's conditions), else a one-thread-per-output kernel
 *
 * lrbi_decode_mask_batch: the indices of n layers decoded by ONE launch per 32 layers (many small layers, e.g. the
 * blocks of a network, cost one launch latency instead of n).  layouts, ip, iz, mask_out are HOST arrays of n
 * entries; the pointers they hold are device pointers as for lrbi_decode_mask.
 */
typedef struct {
    const int32_t *ranks;     /* device, [GR*GC]                                   */
    const int64_t *ip_offset; /* device, [GR*GC], first word of tile t in ip       */
    const int64_t *iz_offset; /* device, [GR*GC], first word of tile t in iz       */
} lrbi_tile_ranks;
LRBI_API lrbi_status lrbi_decode_mask_ranked(const lrbi_layout *layout, const lrbi_tile_ranks *ranks, const uint32_t *ip,
                                             const uint32_t *iz, uint32_t *mask_out, void *stream);
LRBI_API lrbi_status lrbi_masked_gemm_ranked(const lrbi_layout *layout, const lrbi_tile_ranks *ranks, const uint16_t *W,
                                             const uint32_t *ip, const uint32_t *iz, const uint16_t *X, int32_t batch,
                                             void *Y, int32_t y_dtype, int32_t algo, void *stream);
LRBI_API lrbi_status lrbi_decode_mask_batch(int32_t n, const lrbi_layout *layouts, const uint32_t *const *ip,
                                            const uint32_t *const *iz, uint32_t *const *mask_out, void *stream);

/*
 * NMF of the magnitude matrix (Section 2.1: M[i][j] = |W[i][j]| "is factorized by an NMF library" into Mp, Mz,
 * Eq. 4; first two steps of Algorithm 1), every tile on its own (Section 3.1).  The paper names no solver; this is
 * the multiplicative update rule for the Frobenius objective ||M - Mp Mz||^2 of the NMF reference it cites, from
 * the caller's starting factors: per iteration
 *       Mz <- Mz * (Mp^T M) / (Mp^T Mp Mz + eps),   then   Mp <- Mp * (M Mz^T) / (Mp Mz Mz^T + eps),
 * in fp32.  Positions of an edge tile outside the matrix count as zeros of M.  rank <= 256.
 *   W     device, bf16 bit patterns, [rows][cols]
 *   mp    device, fp32, [GR*GC][tile_rows][rank], in and out (start from positive values)
 *   mz    device, fp32, [GR*GC][rank][tile_cols], in and out
 *   workspace   device, lrbi_nmf_workspace(layout) bytes, 16-byte aligned, scratch for the call
 * The results feed lrbi_threshold_pack.
 */
LRBI_API size_t lrbi_nmf_workspace(const lrbi_layout *layout);
LRBI_API lrbi_status lrbi_nmf_update(const lrbi_layout *layout, const uint16_t *W, float *mp, float *mz, int32_t iterations,
                                     float eps, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Backward pass of the masked layer (Section 2.2: the pruned network is retrained "using a masking layer" Ia, so
 * gradients flow through kept weights only).  With Y = X (W .* Ia)^T and dY = dL/dY [batch][rows]:
 *       dX[b][i] = sum_o  Ia[o][i] ? dY[b][o] * W[o][i] : 0          dW[o][i] = Ia[o][i] ? sum_b dY[b][o] * X[b][i] : 0
 * fp32 accumulation; outputs bf16 (round to nearest even) or fp32 as the dtype argument says (LRBI_Y_*).
 *
 * lrbi_masked_gemm_dx   needs the weights TRANSPOSED: Wt [cols][rows] bf16 (keep that copy beside W and refresh it with
 *       lrbi_transpose_bf16 when W changes).  It is the forward product of the transposed layer, so it runs on the same
 *       kernels: the packed factors are used as they are (a row word of Ip is a column word of Ip^T).  algo:
 *       LRBI_ALGO_AUTO, _GENERIC or _TENSOR / _TENSOR_PAIR / _TENSOR_PAIR2 / _TENSOR_PAIR192 (tensor-core shapes: rows % 8 == 0, and
 *       tile_cols % 128 == 0 and tile_rows % 64 == 0 unless the grid has one tile in that direction).
 * lrbi_masked_gemm_dw   dY [batch][rows], X [batch][cols] -> dW [rows][cols].  Large aligned layers (rows, cols and
 *       batch multiples of 8; tile_cols % 128 == 0 and tile_rows % 256 == 0 unless the grid has one tile in that
 *       direction) run as ONE launch of the tensor-core kernel on dY and X as they are (the operands are read
 *       MN-major): nothing is pruned inside the contraction and the index, decoded on the fly and never stored, is
 *       applied as dW is written; `workspace` is not touched and may be NULL.  Other tensor-core shapes use
 *       `workspace` (DEVICE memory of at least lrbi_masked_gemm_dw_workspace(layout, batch) bytes, 16-byte aligned,
 *       owned by the caller, scratch for the call) for transposed copies of dY and X and apply the index to dW in
 *       place afterwards; batch % 8 != 0, or a NULL workspace on such a shape, falls back to a slow
 *       one-thread-per-weight kernel.
 * lrbi_transpose_bf16   dst [cols][rows] = transpose of src [rows][cols] (bf16 bit patterns; dst must not overlap src).
 */
LRBI_API lrbi_status lrbi_transpose_bf16(const uint16_t *src, int32_t rows, int32_t cols, uint16_t *dst, void *stream);
LRBI_API lrbi_status lrbi_masked_gemm_dx(const lrbi_layout *layout, const uint16_t *Wt, const uint32_t *ip, const uint32_t *iz,
                                         const uint16_t *dY, int32_t batch, void *dX, int32_t dx_dtype, int32_t algo, void *stream);
LRBI_API size_t lrbi_masked_gemm_dw_workspace(const lrbi_layout *layout, int32_t batch);
LRBI_API lrbi_status lrbi_masked_gemm_dw(const lrbi_layout *layout, const uint16_t *dY, const uint16_t *X, int32_t batch,
                                         const uint32_t *ip, const uint32_t *iz, void *dW, int32_t dw_dtype,
                                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * Around the pruned layers of a feed-forward block: layer norm, the nonlinearity, activations kept in 8 bits for the
 * backward pass, and (further down) 4-bit weights for a few rows of activations.  (The paper has no counterpart to
 * these calls: it retrains and serves whole networks, and they are what stands between two masked layers.)
 *
 * Matrices of these calls are [rows][cols] with unit column stride; element (r, c) is at data[r * stride + c], stride in
 * elements, at least cols and less than 2^32 bytes, so a slice of a wider array is passed as it is.  Each has its own element
 * type (LRBI_Y_BF16 or LRBI_Y_F32) and needs that type's alignment only; rows that start on 16-byte boundaries (32-byte ones
 * in fp32) and a multiple of 8 columns are read and written in vectors.  rows may be 0 (nothing is read; gradients of
 * parameters are written as zeros), cols is 1 .. LRBI_MAX_ROW_COLS.  All sums and statistics are fp32, each output is rounded
 * once.  Outputs must not overlap inputs or one another.
 * Results of a call have the same bits every time it is made on the same GPU model.
 */
#define LRBI_MAX_ROW_COLS (1 << 24)

/*
 * 8-bit copy ("checkpoint") of a matrix: columns are cut into groups of LRBI_CHECKPOINT_GROUP, and a group of a row has
 *       top = max |x|,   scale = top / 127,   q = round_to_even(x * (127 / top))       (each step one fp32 operation)
 * and stands for q * scale, so a value is off by at most top / 254 (and rounding).  A group whose top is below 2^-118 is kept
 * as zeros (scale 0); a group that holds a NaN or an infinity has scale NaN and q = 0, and loads as NaN.
 *   q      device, int8, [rows][lrbi_checkpoint_pitch(cols)], 16-byte aligned; bytes past the last column are written as 0
 *   scale  device, fp32, [rows][lrbi_checkpoint_groups(cols)]
 * lrbi_checkpoint_store writes the copy of x, lrbi_checkpoint_load writes what a copy stands for.
 */
#define LRBI_CHECKPOINT_GROUP 128
LRBI_API int32_t lrbi_checkpoint_pitch(int32_t cols);  /* cols rounded up to 16; 0 for cols out of range  */
LRBI_API int32_t lrbi_checkpoint_groups(int32_t cols); /* ceil(cols / LRBI_CHECKPOINT_GROUP)              */
LRBI_API lrbi_status lrbi_checkpoint_store(const void *x, int32_t x_dtype, int64_t x_stride, int32_t rows, int32_t cols,
                                           int8_t *q, float *scale, void *stream);
LRBI_API lrbi_status lrbi_checkpoint_load(const int8_t *q, const float *scale, int32_t rows, int32_t cols, void *x,
                                          int32_t x_dtype, int64_t x_stride, void *stream);

/*
 * Layer norm over the columns of each row:
 *       mean = sum x / cols,  rstd = 1 / sqrt(sum (x - mean)^2 / cols + eps),  y = (x - mean) * rstd * gamma + beta
 *   gamma, beta   device, [cols], param_dtype each; beta may be NULL (no offset)
 *   mean, rstd    device, fp32, [rows], for the backward pass; both or neither NULL
 *   q, scale      8-bit copy of x, taken on the way; both or neither NULL
 *
 * lrbi_layer_norm_backward: with n = (x - mean) * rstd and g = dy * gamma,
 *       dx = dres + rstd * (g - mean_c(g) - n * mean_c(g * n)),   dgamma = sum over rows of dy * n,   dbeta = sum of dy
 *   x             the forward input, or NULL where its 8-bit copy q, scale is given: n is then taken from what the copy
 *                 stands for, with the statistics that the forward pass saved (those of x itself)
 *   dres          in dx's type, or NULL: the gradient that reaches x past the norm (the residual connection)
 *   y             in dy's type, or NULL: n * gamma + beta, the forward result, restored for the weight gradient of the
 *                 layer that it went into
 *   dgamma, dbeta device, fp32, [cols]; either may be NULL
 *   workspace     device, lrbi_layer_norm_backward_workspace(rows, cols) bytes, 16-byte aligned, scratch for the call
 */
LRBI_API lrbi_status lrbi_layer_norm(const void *x, int32_t x_dtype, int64_t x_stride, int32_t rows, int32_t cols,
                                     const void *gamma, const void *beta, int32_t param_dtype, float eps, void *y,
                                     int32_t y_dtype, int64_t y_stride, float *mean, float *rstd, int8_t *q, float *scale,
                                     void *stream);
LRBI_API size_t lrbi_layer_norm_backward_workspace(int32_t rows, int32_t cols);
LRBI_API lrbi_status lrbi_layer_norm_backward(const void *dy, int32_t dy_dtype, int64_t dy_stride, const void *x,
                                              int32_t x_dtype, int64_t x_stride, const int8_t *q, const float *scale,
                                              int32_t rows, int32_t cols, const void *gamma, const void *beta,
                                              int32_t param_dtype, const float *mean, const float *rstd, const void *dres,
                                              int64_t dres_stride, void *dx, int32_t dx_dtype, int64_t dx_stride, void *y,
                                              int64_t y_stride, float *dgamma, float *dbeta, void *workspace,
                                              size_t workspace_bytes, void *stream);

/*
 * The nonlinearity between two layers: a = act(h), optionally with the 8-bit copy of h (q, scale: both or neither NULL).
 *       LRBI_ACT_RELU max(h, 0)      LRBI_ACT_GELU h * Phi(h), Phi the normal distribution      LRBI_ACT_SILU h / (1 + exp(-h))
 * lrbi_activation_backward: dh = da * act'(h), from h, or (h NULL) from its 8-bit copy; `a`, in da's type, or NULL,
 * receives act(h) again, for the weight gradient of the layer that it went into.  At h = 0 relu has slope 0.
 * Before it is rounded to its output's type a result is off by at most 2^-20 (1 + h^2 / 8) of itself for gelu (2^-13 more
 * for an output in bf16) and 2^-20 (1 + |h|) for silu (below 2^-100 it may come as 0), a slope by as much of the larger of
 * its two terms.
 * An infinite h gives what the formula gives: +inf for +inf; for -inf 0 (relu) or NaN (gelu, silu: infinity times zero); the
 * slopes of gelu and silu are NaN there.
 */
enum { LRBI_ACT_RELU = 0, LRBI_ACT_GELU = 1, LRBI_ACT_SILU = 2 };
LRBI_API lrbi_status lrbi_activation(const void *h, int32_t h_dtype, int64_t h_stride, int32_t rows, int32_t cols,
                                     int32_t act, void *a, int32_t a_dtype, int64_t a_stride, int8_t *q, float *scale,
                                     void *stream);
LRBI_API lrbi_status lrbi_activation_backward(const void *da, int32_t da_dtype, int64_t da_stride, const void *h,
                                              int32_t h_dtype, int64_t h_stride, const int8_t *q, const float *scale,
                                              int32_t rows, int32_t cols, int32_t act, void *dh, int32_t dh_dtype,
                                              int64_t dh_stride, void *a, int64_t a_stride, void *stream);

/*
 * 4-bit weights with a scale and a zero point for each group of columns of a row (groups of 32, 64 or 128):
 *       W[o][i] = s[o][g] * (q[o][i] - z[o][g]),     q and z whole numbers 0 .. 15, s bf16,  g = i / group
 * A weight that the index prunes is stored with q = z, which is exactly zero: the index is applied once, when the layer is
 * quantised, and costs nothing afterwards.
 *
 * Layout (RT = ceil(rows / 16), U = ceil(cols / 64), G = ceil(cols / group)):
 *   packed  device, uint32, [RT][U][32][4], 16-byte aligned.  Word (tile, u, 4 * g + t, s) holds eight values of rows
 *           16 * tile + g and + g + 8; its bits 4j .. 4j + 3 are row g + 8 * (j & 1), column
 *           64 * u + 32 * (s / 2) + 8 * t + 4 * (s & 1) + i with i = 2 * (j / 2 & 1) + j / 4.  Rows past the last hold anything; columns past the last hold their group's z
 *           (where they belong to no group, anything).
 *   meta    device, uint32, [RT][G][16], 16-byte aligned: row 16 * tile + r of group g has the bits of s in the upper half
 *           and z in the lowest four bits of word (tile, g, r).
 * lrbi_w4_quantize  W [rows][cols] bf16 -> packed, meta.  Over the kept weights of a group: lo = min(0, W), hi = max(0, W),
 *           s = bf16((hi - lo) / 15), z = clamp(round(-lo / s)), q = clamp(round(W / s) + z), each step one fp32 operation,
 *           rounding to nearest even, clamped to 0 .. 15.  A group without a non-zero kept weight (or with a range below
 *           2^-130, whose s is rounded to 0) has s = 0, z = 8; a kept weight that is not finite, or a range beyond fp32, gives
 *           s = NaN.  What the array holds at pruned places is not looked at.  ip, iz: the layer's packed factors, or both
 *           NULL (nothing is pruned; only rows and cols of the layout are looked at).
 *           Columns up to 65535 * 128; LRBI_ERR_UNSUPPORTED beyond.
 * lrbi_w4_gemv  Y [batch][rows] (bf16 or fp32) = X W^T for X [batch][cols] bf16, contiguous, sums in fp32.  Made for a few
 *           rows of X: up to 16 go through the weights together, and each further 16 read them again.  batch may be 0, and up
 *           to 16 * 65535; LRBI_ERR_UNSUPPORTED beyond.
 */
LRBI_API size_t lrbi_w4_packed_words(int32_t rows, int32_t cols);             /* RT*U*128; 0 if a size is out of range */
LRBI_API size_t lrbi_w4_meta_words(int32_t rows, int32_t cols, int32_t group); /* RT*G*16; 0 also for other groups      */
LRBI_API lrbi_status lrbi_w4_quantize(const lrbi_layout *layout, const uint16_t *W, const uint32_t *ip, const uint32_t *iz,
                                      int32_t group, uint32_t *packed, uint32_t *meta, void *stream);
LRBI_API lrbi_status lrbi_w4_gemv(const uint32_t *packed, const uint32_t *meta, int32_t rows, int32_t cols, int32_t group,
                                  const uint16_t *X, int32_t batch, void *Y, int32_t y_dtype, void *stream);

/* Which kernel LRBI_ALGO_AUTO would run for this layout and batch (an LRBI_ALGO_* value). */
LRBI_API int32_t lrbi_masked_gemm_choice(const lrbi_layout *layout, int32_t batch);

/*
 * How lrbi_masked_gemm would run a call on the current device (nothing is launched).  For
 * LRBI_ALGO_TENSOR the fields say which instantiation of the tcgen05 kernel runs; for the other
 * kernels only `algo` is meaningful (k_splits = 1, the rest 0).
 */
typedef struct {
    int32_t algo;          /* the LRBI_ALGO_* value that runs (LRBI_ALGO_AUTO resolved)             */
    int32_t batch_tile;    /* batch rows per output tile (512: a CTA pair with two accumulators)    */
    int32_t cta_pair;      /* 1: two CTAs of a cluster share a 256-row tile (tcgen05 cta_group::2)  */
    int32_t panel_columns; /* columns of the index decoded per step inside the kernel (256 or 64)   */
    int32_t k_splits;      /* thread blocks along the reduction; > 1 means fp32 partial sums + a second kernel */
    int32_t stages;        /* operand stages in shared memory                                       */
    uint64_t scratch_bytes;/* bytes of partial sums (what lrbi_masked_gemm_static_bytes reports)    */
} lrbi_gemm_plan;
LRBI_API lrbi_status lrbi_masked_gemm_plan(const lrbi_layout *layout, int32_t batch, int32_t algo,
                                           lrbi_gemm_plan *plan);

/* Kernels launched by this library since it was loaded (all entry points, this process). */
LRBI_API uint64_t lrbi_launch_count(void);

/*
 * Device-side status word of the current device: 0, or a code left by a kernel whose bounded
 * wait (pipeline barrier) ran out.  Synchronises the device.  `clear` != 0 resets it and
 * lifts the LRBI_ERR_TIMEOUT refusal of later calls.  Returns -1 if a CUDA call failed.
 */
LRBI_API int32_t lrbi_device_status(int32_t clear);
LRBI_API int32_t lrbi_last_device_error(void); /* lrbi_device_status(0) */

/*
 * Self-test of the timeout path (no counterpart in the paper).  Launches one tiny kernel whose single
 * thread waits, with the same bounded wait the pipeline kernels use but a limit of `limit_us`
 * microseconds (at most 100 000), on a barrier that nothing signals.  The wait gives up, the kernel
 * returns normally and the status word of the device then holds 0x600.  Nothing hangs or traps; it is
 * how the tests show that a timeout is recorded, reported (LRBI_ERR_TIMEOUT) and cleared.
 */
LRBI_API lrbi_status lrbi_selftest_bounded_wait(uint32_t limit_us, void *stream);

LRBI_API const char *lrbi_status_string(lrbi_status s);
LRBI_API int32_t lrbi_last_cuda_error(void); /* cudaError_t / CUresult of the last failed call, else 0 */

#ifdef __cplusplus
}
#endif
#endif /* LRBI_H_ */
