// Activations kept in 8 bits for the backward pass, and the nonlinearity between two layers, which takes its copy on the
// way forward and computes its gradient from that copy.
//
//   store      x -> (q, scale)                     load      (q, scale) -> x^ = q * scale
//   forward    a = act(h), optionally (q, scale)   backward  dh = da * act'(h^), optionally a^ = act(h^)
//
// One pass, and memory bounds it: 4096 x 16384 bf16, gelu forward with the copy and backward from it, 137 us of 124 at the
// rate of a plain copy; 16384 x 4096 bf16: stored in 34.4 us (31.1), loaded in 33.4 (31.1), gelu 43.7 (41.0), with the copy
// 60 (51.6); fp32: stored in 51.2 us (51.5), loaded in 53.6, gelu 82.3 (82.0), with the copy 93.9 (92.6).  The arithmetic of gelu and of the copy takes nearly as long as memory in bf16, which
// is why values go in pairs and four groups share one division (a chunk at a time the copy was stored in 46 us).  Rows that
// are not whole vectors are bound by their accesses, one a value: 4096 x 8191 bf16, gelu step, 108 us (62).
#include "activation.cuh"

namespace lrbi {

struct KeepArgs {
    RowsIn h, da;      // h unused when the copy is read
    KeptIn from;
    RowsOut a, dh;     // data null: not written
    KeptOut kept;
    int rows, cols;
    int shift;         // log2 of the spans of a row that a block takes side by side
};

constexpr int KEEP_THREADS = 256;

// Rows that a warp takes together: four groups' divisions are one, else what keeps memory busy.
template <bool COPY, bool STRIDED>
constexpr int KEEP_ROWS = COPY && !STRIDED ? 4 : 2;

// The place of row `row` of a matrix of rows `bytes` apart: one multiply-add.
template <class T>
__device__ __forceinline__ T *row_at(T *base, uint32_t row, long long bytes) { return base + (uint64_t)row * (uint32_t)bytes; }

// Block (x: rows, y: spans of a row).  A warp takes a span of U rows, the loads of all of them first.  COPY: h is kept in 8 bits.
// OUT: type of a (forward) or dh (backward); the backward pass writes a in da's type.
template <int SRC, int ACT, bool BACK, int DA, int OUT, bool COPY, bool STRIDED>
__global__ void __launch_bounds__(KEEP_THREADS) keep_kernel(KeepArgs k)
{
    begin();
    constexpr int WARPS = KEEP_THREADS / 32, U = KEEP_ROWS<COPY, STRIDED>;
    constexpr int HSIZE = SRC == SRC_F32 ? 4 : 2, ASIZE = (BACK ? DA : OUT) == SRC_F32 ? 4 : 2, DSIZE = DA == SRC_F32 ? 4 : 2, OSIZE = OUT == LRBI_Y_F32 ? 4 : 2;
    const int warp = threadIdx.x >> 5, lane = kept_lane();
    const int c0 = ((blockIdx.y << k.shift) + (warp & ((1 << k.shift) - 1))) * SPAN, c = lane_column<STRIDED>(c0, lane), left = k.cols - c;
    if (c0 >= k.cols) return;               // the whole warp
    const uint32_t down = WARPS >> k.shift;     // rows of a block at a time
    const uint32_t row0 = blockIdx.x * down * U + (warp >> k.shift), rows = k.rows;
    const bool whole = c0 + SPAN <= k.cols;
    Raw<SRC, STRIDED> raw[U];
    Raw<DA, STRIDED> raw_da[BACK ? U : 1];
    const char *h0 = static_cast<const char *>(k.h.data) + c * HSIZE, *da0 = static_cast<const char *>(k.da.data) + c * DSIZE;
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const uint32_t row = row0 + i * down;
        if (row < rows) {                   // the whole warp
            if constexpr (SRC == SRC_KEPT) raw[i].load(k.h, k.from, row, c, k.cols);
            else raw[i].load_at(row_at(h0, row, k.h.stride * HSIZE), left, whole);
            if constexpr (BACK) raw_da[i].load_at(row_at(da0, row, k.da.stride * DSIZE), left, whole);
        } else raw[i].clear();
    }
    let_next();
    if constexpr (COPY) {
        using Keeper = Keep<STRIDED>;
        static_assert(U == Keeper::CHUNKS, "");
        uint32_t tops[4];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            uint32_t t[STRIDED ? 2 : 1];
            raw[i].tops(t);
            tops[STRIDED ? 2 * i : i] = t[0];
            if (STRIDED) tops[STRIDED ? 2 * i + 1 : 0] = t[STRIDED ? 1 : 0];
        }
        const Keeper keep(tops, lane);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const uint32_t row = row0 + i * down;
            F2 h[PAIRS];
            raw[i].get(h);
            keep.bytes(i, row_at(k.kept.q + c, row, k.kept.pitch), row < rows ? k.kept.pitch - c : 0, h);
        }
        const uint32_t row = row0 + Keeper::chunk(lane) * down;
        const int group = c0 / KEEP_GROUP + Keeper::group(lane);
        if (Keeper::stores(lane) && row < rows && group < k.kept.groups) k.kept.scale[(uint64_t)row * (uint32_t)k.kept.groups + group] = keep.quotient;
        if (ACT == ACT_NONE) return;
    }
    char *a0 = static_cast<char *>(k.a.data) + c * ASIZE, *dh0 = static_cast<char *>(k.dh.data) + c * OSIZE;
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const uint32_t row = row0 + i * down;
        if (row >= rows) break;
        F2 h[PAIRS], v[PAIRS], d[PAIRS];
        raw[i].get(h);
        if constexpr (ACT == ACT_NONE) store_at<ASIZE, STRIDED>(row_at(a0, row, k.a.stride * ASIZE), left, h, whole);
        else {
#pragma unroll
            for (int j = 0; j < PAIRS; ++j) activate<ACT, BACK, ASIZE == 4, OSIZE == 4>(h[j], v[j], d[j]);
            if constexpr (BACK) {
                F2 da[PAIRS];
                raw_da[i].get(da);
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) d[j] = d[j] * da[j];
                store_at<OSIZE, STRIDED>(row_at(dh0, row, k.dh.stride * OSIZE), left, d, whole);
            }
            if (!BACK || k.a.data) store_at<ASIZE, STRIDED>(row_at(a0, row, k.a.stride * ASIZE), left, v, whole);
        }
    }
}

namespace {

template <int SRC, int ACT, bool BACK, int DA, int OUT, bool COPY, bool STRIDED>
lrbi_status keep_launch(KeepArgs k, cudaStream_t s)
{
    const int spans = (k.cols + SPAN - 1) / SPAN, warps = KEEP_THREADS / 32;
    k.shift = 0;
    while ((1 << k.shift) < spans && (1 << k.shift) < warps) ++k.shift;
    const int wide = 1 << k.shift;
    const long long down = (long long)(warps >> k.shift) * KEEP_ROWS<COPY, STRIDED>;
    const dim3 grid((unsigned)((k.rows + down - 1) / down), (unsigned)((spans + wide - 1) / wide));
    return launch_kernel(keep_kernel<SRC, ACT, BACK, DA, OUT, COPY, STRIDED>, grid, dim3(KEEP_THREADS), 0, s, 1, k);
}

template <int SRC, bool BACK, int DA, int OUT, bool COPY>
lrbi_status act_launch(const KeepArgs &k, int act, bool strided, cudaStream_t s)
{
#define ACT(A) strided ? keep_launch<SRC, A, BACK, DA, OUT, COPY, true>(k, s) : keep_launch<SRC, A, BACK, DA, OUT, COPY, false>(k, s)
    if (act == LRBI_ACT_RELU) return ACT(LRBI_ACT_RELU);
    if (act == LRBI_ACT_SILU) return ACT(LRBI_ACT_SILU);
    return ACT(LRBI_ACT_GELU);
#undef ACT
}

}  // namespace

lrbi_status launch_checkpoint_store(const void *x, int dtype, long long stride, int rows, int cols, int8_t *q, float *scale, cudaStream_t s)
{
    KeepArgs k = {};
    k.h = {x, stride};
    k.kept = {q, scale, checkpoint_pitch(cols), checkpoint_groups(cols)};
    k.rows = rows; k.cols = cols;
    const bool strided = cols % CHUNK != 0 || !vector_rows(x, stride, dtype);
#define STORE(SRC) strided ? keep_launch<SRC, ACT_NONE, false, SRC_BF16, LRBI_Y_BF16, true, true>(k, s) : keep_launch<SRC, ACT_NONE, false, SRC_BF16, LRBI_Y_BF16, true, false>(k, s)
    return dtype == LRBI_Y_BF16 ? (STORE(SRC_BF16)) : (STORE(SRC_F32));
#undef STORE
}

lrbi_status launch_checkpoint_load(const int8_t *q, const float *scale, int rows, int cols, void *x, int dtype, long long stride, cudaStream_t s)
{
    KeepArgs k = {};
    k.from = {q, scale, checkpoint_pitch(cols), checkpoint_groups(cols)};
    k.a = {x, stride, dtype};
    k.rows = rows; k.cols = cols;
    const bool strided = cols % CHUNK != 0 || !vector_rows(x, stride, dtype);
#define LOAD(OUT) strided ? keep_launch<SRC_KEPT, ACT_NONE, false, SRC_BF16, OUT, false, true>(k, s) : keep_launch<SRC_KEPT, ACT_NONE, false, SRC_BF16, OUT, false, false>(k, s)
    return dtype == LRBI_Y_BF16 ? (LOAD(LRBI_Y_BF16)) : (LOAD(LRBI_Y_F32));
#undef LOAD
}

lrbi_status launch_activation(const ActArgs &n, cudaStream_t s)
{
    KeepArgs k = {};
    k.h = {n.h, n.h_stride};
    k.a = {n.a, n.a_stride, n.a_dtype};
    k.kept = {n.q_out, n.scale_out, checkpoint_pitch(n.cols), checkpoint_groups(n.cols)};
    k.rows = n.rows; k.cols = n.cols;
    const bool strided = n.cols % CHUNK != 0 || !vector_rows(n.h, n.h_stride, n.h_dtype) || !vector_rows(n.a, n.a_stride, n.a_dtype);
#define FORWARD(SRC, OUT) n.q_out ? act_launch<SRC, false, SRC_BF16, OUT, true>(k, n.act, strided, s) : act_launch<SRC, false, SRC_BF16, OUT, false>(k, n.act, strided, s)
    if (n.h_dtype == LRBI_Y_BF16) return n.a_dtype == LRBI_Y_BF16 ? (FORWARD(SRC_BF16, LRBI_Y_BF16)) : (FORWARD(SRC_BF16, LRBI_Y_F32));
    return n.a_dtype == LRBI_Y_BF16 ? (FORWARD(SRC_F32, LRBI_Y_BF16)) : (FORWARD(SRC_F32, LRBI_Y_F32));
#undef FORWARD
}

lrbi_status launch_activation_backward(const ActArgs &n, cudaStream_t s)
{
    KeepArgs k = {};
    k.h = {n.h, n.h_stride};
    k.da = {n.da, n.da_stride};
    k.from = {n.q, n.scale, checkpoint_pitch(n.cols), checkpoint_groups(n.cols)};
    k.dh = {n.dh, n.dh_stride, n.dh_dtype};
    k.a = {n.a, n.a_stride, n.a_dtype};
    k.rows = n.rows; k.cols = n.cols;
    const bool strided = n.cols % CHUNK != 0 || (!n.q && !vector_rows(n.h, n.h_stride, n.h_dtype)) || !vector_rows(n.da, n.da_stride, n.da_dtype) ||
                       !vector_rows(n.dh, n.dh_stride, n.dh_dtype) || (n.a && !vector_rows(n.a, n.a_stride, n.a_dtype));
    const int src = n.q ? SRC_KEPT : n.h_dtype;
#define BACKWARD(SRC, DA) n.dh_dtype == LRBI_Y_BF16 ? act_launch<SRC, true, DA, LRBI_Y_BF16, false>(k, n.act, strided, s) : act_launch<SRC, true, DA, LRBI_Y_F32, false>(k, n.act, strided, s)
    if (n.da_dtype == LRBI_Y_BF16) {
        if (src == SRC_BF16) return BACKWARD(SRC_BF16, SRC_BF16);
        if (src == SRC_F32) return BACKWARD(SRC_F32, SRC_BF16);
        return BACKWARD(SRC_KEPT, SRC_BF16);
    }
    if (src == SRC_BF16) return BACKWARD(SRC_BF16, SRC_F32);
    if (src == SRC_F32) return BACKWARD(SRC_F32, SRC_F32);
    return BACKWARD(SRC_KEPT, SRC_F32);
#undef BACKWARD
}

}  // namespace lrbi
