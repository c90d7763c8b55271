// Activations kept in 8 bits for the backward pass, and the nonlinearity between two layers, which takes its copy on the
// way forward and computes its gradient from that copy.
//
//   store      x -> (q, scale)                     load      (q, scale) -> x^ = q * scale
//   forward    a = act(h), optionally (q, scale)   backward  dh = da * act'(h^), optionally a^ = act(h^)
//
// One pass, a group of 128 columns per half warp (or warp): all of it streams, the arithmetic is about 20 operations a
// value at most, so memory is the bound.
#include "row_ops.cuh"

namespace lrbi {

enum { ACT_NONE = -1 };

// Value and slope of the nonlinearity.  gelu(h) = h Phi(h), Phi the normal distribution; slope Phi(h) + h phi(h).
// Phi comes from Abramowitz and Stegun 7.1.26, erfc(z) = t (a1 + t (a2 + ...)) exp(-z^2) with t = 1 / (1 + p z), z >= 0,
// off by at most 1.5e-7; for h < 0 it is taken without a difference, so small values keep their leading digits.
template <int ACT>
__device__ __forceinline__ void activate(float h, float &value, float &slope)
{
    if (ACT == LRBI_ACT_RELU) {
        value = h < 0.f ? 0.f : h;                       // a NaN stays
        slope = h > 0.f ? 1.f : (h <= 0.f ? 0.f : h);
    } else if (ACT == LRBI_ACT_SILU) {
        const float s = __fdividef(1.f, 1.f + __expf(-h));
        value = h * s;
        slope = fmaf(value, 1.f - s, s);
    } else {
        const float z = fabsf(h) * 0.70710678f, e = __expf(-0.5f * h * h);
        const float t = __fdividef(1.f, fmaf(0.3275911f, z, 1.f));
        const float p = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
        const float tail = 0.5f * p * e;                 // the normal distribution's tail beyond |h|
        const float phi = h < 0.f ? tail : 1.f - tail;
        value = h * phi;
        slope = fmaf(h * 0.39894228f, e, phi);
    }
}

struct KeepArgs {
    RowsIn h, da;      // h unused when the copy is read
    KeptIn from;
    RowsOut a, dh;     // data null: not written
    KeptOut kept;      // q null: no copy
    int rows, cols;
    int shift;         // log2 of the groups of a row that a block takes side by side
    int tall;          // rows that a block takes one after the other, per thread
};

constexpr int KEEP_THREADS = 256;

// Block (x: rows, y: groups of columns).  A unit is what takes a group: 16 lanes with 8 columns each, or 32 with 4.
template <int SRC, int ACT, bool BACK, int DA, bool VEC, int U>
__global__ void __launch_bounds__(KEEP_THREADS) keep_kernel(KeepArgs k)
{
    constexpr int E = Chunk<VEC>::E, LANES = VEC ? 16 : 32, UNITS = KEEP_THREADS / LANES;
    const int unit = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const int wide = 1 << k.shift;
    const int group = blockIdx.y * wide + (unit & (wide - 1));
    const int c = group * KEEP_GROUP + (VEC ? lane * 8 : lane);
    const int down = UNITS >> k.shift;      // rows of a block at a time
    const long long row0 = (long long)blockIdx.x * down * U + (unit >> k.shift);
    Raw<SRC, VEC> raw[U];
    Raw<DA, VEC> raw_da[BACK ? U : 1];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const long long row = row0 + i * down;
        if (row < k.rows) {
            raw[i].load(k.h, k.from, row, c, k.cols);
            if (BACK) raw_da[BACK ? i : 0].load(k.da, k.from, row, c, k.cols);
        }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const long long row = row0 + i * down;
        const bool in = row < k.rows;
        float h[E], v[E], d[E];
        raw[i].get(h);
        if (!in) {
#pragma unroll
            for (int e = 0; e < E; ++e) h[e] = 0.f;
        }
        if (!BACK && k.kept.q) {
            // lanes of rows past the end take part in the group's maximum, and store nothing
            KeptOut to = k.kept;
            if (!in) { to.pitch = 0; to.groups = 0; }
            keep_chunk<VEC>(to, in ? row : 0, c, h);
        }
        if (!in) continue;
        if (ACT == ACT_NONE) {
            if (k.a.data) store_chunk<VEC>(k.a, row, c, k.cols, h);
            continue;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) activate<ACT>(h[e], v[e], d[e]);
        if (BACK) {
            float da[E];
            raw_da[BACK ? i : 0].get(da);
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] *= da[e];
            store_chunk<VEC>(k.dh, row, c, k.cols, d);
            if (k.a.data) store_chunk<VEC>(k.a, row, c, k.cols, v);
        } else {
            store_chunk<VEC>(k.a, row, c, k.cols, v);
        }
    }
}

namespace {

template <int SRC, int ACT, bool BACK, int DA>
lrbi_status keep_launch(KeepArgs k, bool vec, cudaStream_t s)
{
    constexpr int U = 2;
    const int groups = (k.cols + KEEP_GROUP - 1) / KEEP_GROUP, units = KEEP_THREADS / (vec ? 16 : 32);
    k.shift = 0;
    while ((1 << k.shift) < groups && (1 << k.shift) < units) ++k.shift;
    const int wide = 1 << k.shift;
    const long long down = (long long)(units >> k.shift) * U;
    const dim3 grid((unsigned)((k.rows + down - 1) / down), (unsigned)((groups + wide - 1) / wide));
    if (grid.y > 65535) return LRBI_ERR_UNSUPPORTED;
    if (vec) keep_kernel<SRC, ACT, BACK, DA, true, U><<<grid, KEEP_THREADS, 0, s>>>(k);
    else keep_kernel<SRC, ACT, BACK, DA, false, U><<<grid, KEEP_THREADS, 0, s>>>(k);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) { note_cuda_error((int)e); return LRBI_ERR_CUDA; }
    count_launch(1);
    return LRBI_OK;
}

template <int SRC, bool BACK, int DA>
lrbi_status act_launch(const KeepArgs &k, int act, bool vec, cudaStream_t s)
{
    if (act == LRBI_ACT_RELU) return keep_launch<SRC, LRBI_ACT_RELU, BACK, DA>(k, vec, s);
    if (act == LRBI_ACT_SILU) return keep_launch<SRC, LRBI_ACT_SILU, BACK, DA>(k, vec, s);
    return keep_launch<SRC, LRBI_ACT_GELU, BACK, DA>(k, vec, s);
}

}  // namespace

lrbi_status launch_checkpoint_store(const void *x, int dtype, long long stride, int rows, int cols, int8_t *q, float *scale, cudaStream_t s)
{
    KeepArgs k = {};
    k.h = {x, stride};
    k.kept = {q, scale, checkpoint_pitch(cols), checkpoint_groups(cols)};
    k.rows = rows; k.cols = cols;
    const bool vec = cols % 8 == 0 && rows16(x, stride, dtype);
    return dtype == LRBI_Y_BF16 ? keep_launch<SRC_BF16, ACT_NONE, false, SRC_BF16>(k, vec, s) : keep_launch<SRC_F32, ACT_NONE, false, SRC_BF16>(k, vec, s);
}

lrbi_status launch_checkpoint_load(const int8_t *q, const float *scale, int rows, int cols, void *x, int dtype, long long stride, cudaStream_t s)
{
    KeepArgs k = {};
    k.from = {q, scale, checkpoint_pitch(cols), checkpoint_groups(cols)};
    k.a = {x, stride, dtype};
    k.rows = rows; k.cols = cols;
    return keep_launch<SRC_KEPT, ACT_NONE, false, SRC_BF16>(k, cols % 8 == 0 && rows16(x, stride, dtype), s);
}

lrbi_status launch_activation(const ActArgs &n, cudaStream_t s)
{
    KeepArgs k = {};
    k.h = {n.h, n.h_stride};
    k.a = {n.a, n.a_stride, n.a_dtype};
    k.kept = {n.q_out, n.scale_out, checkpoint_pitch(n.cols), checkpoint_groups(n.cols)};
    k.rows = n.rows; k.cols = n.cols;
    const bool vec = n.cols % 8 == 0 && rows16(n.h, n.h_stride, n.h_dtype) && rows16(n.a, n.a_stride, n.a_dtype);
    return n.h_dtype == LRBI_Y_BF16 ? act_launch<SRC_BF16, false, SRC_BF16>(k, n.act, vec, s) : act_launch<SRC_F32, false, SRC_BF16>(k, n.act, vec, s);
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
    const bool vec = n.cols % 8 == 0 && (n.q || rows16(n.h, n.h_stride, n.h_dtype)) && rows16(n.da, n.da_stride, n.da_dtype) &&
                     rows16(n.dh, n.dh_stride, n.dh_dtype) && (!n.a || rows16(n.a, n.a_stride, n.a_dtype));
    const int src = n.q ? SRC_KEPT : n.h_dtype;
    if (n.da_dtype == LRBI_Y_BF16) {
        if (src == SRC_BF16) return act_launch<SRC_BF16, true, SRC_BF16>(k, n.act, vec, s);
        if (src == SRC_F32) return act_launch<SRC_F32, true, SRC_BF16>(k, n.act, vec, s);
        return act_launch<SRC_KEPT, true, SRC_BF16>(k, n.act, vec, s);
    }
    if (src == SRC_BF16) return act_launch<SRC_BF16, true, SRC_F32>(k, n.act, vec, s);
    if (src == SRC_F32) return act_launch<SRC_F32, true, SRC_F32>(k, n.act, vec, s);
    return act_launch<SRC_KEPT, true, SRC_F32>(k, n.act, vec, s);
}

}  // namespace lrbi
