// Activations kept in 8 bits for the backward pass, and the nonlinearity between two layers, which takes its copy on the
// way forward and computes its gradient from that copy.
//
//   store      x -> (q, scale)                     load      (q, scale) -> x^ = q * scale
//   forward    a = act(h), optionally (q, scale)   backward  dh = da * act'(h^), optionally a^ = act(h^)
//
// One pass; all of it streams.
#include "row_ops.cuh"

namespace lrbi {

enum { ACT_NONE = -1 };

__device__ __forceinline__ F2 exp2_2(F2 p)      // the hardware's estimate, 2^-22 off
{
    float a, b;
    split(p, a, b);
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
    return f2(a, b);
}
__device__ __forceinline__ F2 inverse2(F2 p)    // 2^-23 off
{
    float a, b;
    split(p, a, b);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
    return f2(a, b);
}

// Value and slope of the nonlinearity.  gelu(h) = h Phi(h), Phi the normal distribution; slope Phi(h) + h phi(h).
// With tail = Phi(-|h|): value = max(h, 0) - |h| tail, slope = [h >= 0] - sign(h) tail + h phi(h), no branch and no lost
// leading digits for h < 0.  The tail comes from Abramowitz and Stegun 7.1.26, erfc(z) = t (a1 + t (a2 + ...)) exp(-z^2)
// with t = 1 / (1 + p z), z >= 0, off by at most 1.5e-7; z = |h| / sqrt(2), tail = erfc(z) / 2, phi = exp(-z^2) / sqrt(2 pi).
template <int ACT, bool SLOPE>
__device__ __forceinline__ void activate(F2 h, F2 &value, F2 &slope)
{
    constexpr float LOG2E = 1.44269504f;
    float a, b;
    split(h, a, b);
    if (ACT == LRBI_ACT_RELU) {
        value = f2(a < 0.f ? 0.f : a, b < 0.f ? 0.f : b);                       // a NaN stays
        if (SLOPE) slope = f2(a > 0.f ? 1.f : (a <= 0.f ? 0.f : a), b > 0.f ? 1.f : (b <= 0.f ? 0.f : b));
    } else if (ACT == LRBI_ACT_SILU) {
        const F2 s = inverse2(exp2_2(h * f2(-LOG2E)) + f2(1.f));
        value = h * s;
        if (SLOPE) slope = fma2(value, fma2(s, f2(-1.f), f2(1.f)), s);
    } else {
        const F2 m = f2(fabsf(a), fabsf(b)), e = exp2_2(h * h * f2(-0.5f * LOG2E));
        const F2 t = inverse2(fma2(m, f2(0.3275911f * 0.70710678f), f2(1.f)));
        F2 p = fma2(t, f2(0.5f * 1.061405429f), f2(0.5f * -1.453152027f));
        p = fma2(t, p, f2(0.5f * 1.421413741f));
        p = fma2(t, p, f2(0.5f * -0.284496736f));
        p = fma2(t, p, f2(0.5f * 0.254829592f));
        const F2 tail = t * p * e;
        float x, y;
        split(tail, x, y);
        value = fma2(f2(-fabsf(a), -fabsf(b)), tail, f2(fmaxf(a, 0.f), fmaxf(b, 0.f)));
        if (SLOPE) slope = fma2(h * f2(0.39894228f), e, f2((a >= 0.f ? 1.f : 0.f) - copysignf(x, a), (b >= 0.f ? 1.f : 0.f) - copysignf(y, b)));
    }
}

struct KeepArgs {
    RowsIn h, da;      // h unused when the copy is read
    KeptIn from;
    RowsOut a, dh;     // data null: not written
    KeptOut kept;      // q null: no copy
    int rows, cols;
    int shift;         // log2 of the spans of a row that a block takes side by side
};

constexpr int KEEP_THREADS = 256, KEEP_ROWS = 2;

// Block (x: rows, y: spans of a row).  A warp takes a span of KEEP_ROWS rows, the loads of all of them first.
template <int SRC, int ACT, bool BACK, int DA, bool STRIDED>
__global__ void __launch_bounds__(KEEP_THREADS) keep_kernel(KeepArgs k)
{
    begin();
    constexpr int WARPS = KEEP_THREADS / 32, U = KEEP_ROWS;
    const int warp = threadIdx.x >> 5, lane = kept_lane();
    const int c0 = ((blockIdx.y << k.shift) + (warp & ((1 << k.shift) - 1))) * SPAN, c = lane_column<STRIDED>(c0, lane);
    if (c0 >= k.cols) return;
    const int down = WARPS >> k.shift;      // rows of a block at a time
    const long long row0 = (long long)blockIdx.x * down * U + (warp >> k.shift);
    Raw<SRC, STRIDED> raw[U];
    Raw<DA, STRIDED> raw_da[BACK ? U : 1];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const long long row = row0 + i * down;
        if (row < k.rows) {                 // the whole warp
            raw[i].load(k.h, k.from, row, c, k.cols);
            if constexpr (BACK) raw_da[i].load(k.da, k.from, row, c, k.cols);
        }
    }
    let_next();
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const long long row = row0 + i * down;
        if (row >= k.rows) break;
        F2 h[PAIRS], v[PAIRS], d[PAIRS];
        raw[i].get(h);
        if constexpr (!BACK && SRC != SRC_KEPT) {
            if (k.kept.q) {
                uint32_t tops[STRIDED ? 2 : 1];
                raw[i].tops(tops);
                keep_chunk<STRIDED>(k.kept, row, c0, lane, h, tops);
            }
        }
        if constexpr (ACT == ACT_NONE) {
            if (k.a.data) store_chunk<STRIDED>(k.a, row, c, k.cols, h);
        } else {
#pragma unroll
            for (int j = 0; j < PAIRS; ++j) activate<ACT, BACK>(h[j], v[j], d[j]);
            if constexpr (BACK) {
                F2 da[PAIRS];
                raw_da[i].get(da);
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) d[j] = d[j] * da[j];
                store_chunk<STRIDED>(k.dh, row, c, k.cols, d);
            }
            if (!BACK || k.a.data) store_chunk<STRIDED>(k.a, row, c, k.cols, v);
        }
    }
}

namespace {

template <int SRC, int ACT, bool BACK, int DA>
lrbi_status keep_launch(KeepArgs k, bool strided, cudaStream_t s)
{
    const int spans = (k.cols + SPAN - 1) / SPAN, warps = KEEP_THREADS / 32;
    k.shift = 0;
    while ((1 << k.shift) < spans && (1 << k.shift) < warps) ++k.shift;
    const int wide = 1 << k.shift;
    const long long down = (long long)(warps >> k.shift) * KEEP_ROWS;
    const dim3 grid((unsigned)((k.rows + down - 1) / down), (unsigned)((spans + wide - 1) / wide));
    if (grid.y > 65535) return LRBI_ERR_UNSUPPORTED;
    if (strided) return launch_kernel(keep_kernel<SRC, ACT, BACK, DA, true>, grid, dim3(KEEP_THREADS), 0, s, 1, k);
    return launch_kernel(keep_kernel<SRC, ACT, BACK, DA, false>, grid, dim3(KEEP_THREADS), 0, s, 1, k);
}

template <int SRC, bool BACK, int DA>
lrbi_status act_launch(const KeepArgs &k, int act, bool strided, cudaStream_t s)
{
    if (act == LRBI_ACT_RELU) return keep_launch<SRC, LRBI_ACT_RELU, BACK, DA>(k, strided, s);
    if (act == LRBI_ACT_SILU) return keep_launch<SRC, LRBI_ACT_SILU, BACK, DA>(k, strided, s);
    return keep_launch<SRC, LRBI_ACT_GELU, BACK, DA>(k, strided, s);
}

}  // namespace

lrbi_status launch_checkpoint_store(const void *x, int dtype, long long stride, int rows, int cols, int8_t *q, float *scale, cudaStream_t s)
{
    KeepArgs k = {};
    k.h = {x, stride};
    k.kept = {q, scale, checkpoint_pitch(cols), checkpoint_groups(cols)};
    k.rows = rows; k.cols = cols;
    const bool strided = cols % CHUNK != 0 || !rows16(x, stride, dtype);
    return dtype == LRBI_Y_BF16 ? keep_launch<SRC_BF16, ACT_NONE, false, SRC_BF16>(k, strided, s) : keep_launch<SRC_F32, ACT_NONE, false, SRC_BF16>(k, strided, s);
}

lrbi_status launch_checkpoint_load(const int8_t *q, const float *scale, int rows, int cols, void *x, int dtype, long long stride, cudaStream_t s)
{
    KeepArgs k = {};
    k.from = {q, scale, checkpoint_pitch(cols), checkpoint_groups(cols)};
    k.a = {x, stride, dtype};
    k.rows = rows; k.cols = cols;
    return keep_launch<SRC_KEPT, ACT_NONE, false, SRC_BF16>(k, cols % CHUNK != 0 || !rows16(x, stride, dtype), s);
}

lrbi_status launch_activation(const ActArgs &n, cudaStream_t s)
{
    KeepArgs k = {};
    k.h = {n.h, n.h_stride};
    k.a = {n.a, n.a_stride, n.a_dtype};
    k.kept = {n.q_out, n.scale_out, checkpoint_pitch(n.cols), checkpoint_groups(n.cols)};
    k.rows = n.rows; k.cols = n.cols;
    const bool strided = n.cols % CHUNK != 0 || !rows16(n.h, n.h_stride, n.h_dtype) || !rows16(n.a, n.a_stride, n.a_dtype);
    return n.h_dtype == LRBI_Y_BF16 ? act_launch<SRC_BF16, false, SRC_BF16>(k, n.act, strided, s) : act_launch<SRC_F32, false, SRC_BF16>(k, n.act, strided, s);
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
    const bool strided = n.cols % CHUNK != 0 || (!n.q && !rows16(n.h, n.h_stride, n.h_dtype)) || !rows16(n.da, n.da_stride, n.da_dtype) ||
                       !rows16(n.dh, n.dh_stride, n.dh_dtype) || (n.a && !rows16(n.a, n.a_stride, n.a_dtype));
    const int src = n.q ? SRC_KEPT : n.h_dtype;
    if (n.da_dtype == LRBI_Y_BF16) {
        if (src == SRC_BF16) return act_launch<SRC_BF16, true, SRC_BF16>(k, n.act, strided, s);
        if (src == SRC_F32) return act_launch<SRC_F32, true, SRC_BF16>(k, n.act, strided, s);
        return act_launch<SRC_KEPT, true, SRC_BF16>(k, n.act, strided, s);
    }
    if (src == SRC_BF16) return act_launch<SRC_BF16, true, SRC_F32>(k, n.act, strided, s);
    if (src == SRC_F32) return act_launch<SRC_F32, true, SRC_F32>(k, n.act, strided, s);
    return act_launch<SRC_KEPT, true, SRC_F32>(k, n.act, strided, s);
}

}  // namespace lrbi
