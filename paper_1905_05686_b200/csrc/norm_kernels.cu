// Layer norm over the columns of each row, forward and backward.
//
//   forward   y = (x - mean) * rstd * gamma + beta, statistics in fp32, optionally an 8-bit copy of x on the way
//   backward  with n = (x - mean) * rstd and g = dy * gamma:
//             dx = dres + rstd * (g - mean(g) - n * mean(g * n)),  dgamma = sum over rows of dy * n,  dbeta = sum of dy
//             x as it was, or its 8-bit copy; optionally writes n * gamma + beta, the forward result of that copy
//
// A row belongs to one warp (up to 256 columns) or to one block; its values stay in registers between the statistics
// and the result, so memory is read once and written once.  Each warp takes its own mean and the sum of squares about
// it (two passes over registers), the warps' pairs are joined by their counts: no cancellation, one barrier per row.
#include "row_ops.cuh"

namespace lrbi {

struct Params {            // gamma and beta, fp32 or bf16; beta may be null
    const void *gamma, *beta;
    int dtype;
};

template <bool VEC>
__device__ __forceinline__ void load_param(const void *p, int dtype, int c, int cols, float other, float (&v)[Chunk<VEC>::E])
{
    constexpr int E = Chunk<VEC>::E;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = other;
    if (!p) return;
    if (dtype == LRBI_Y_F32) {
        const float *f = static_cast<const float *>(p);
        if constexpr (VEC) {
            if (c < cols) {
                const float4 a = __ldg(reinterpret_cast<const float4 *>(f + c)), b = __ldg(reinterpret_cast<const float4 *>(f + c + 4));
                v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) if (c + 32 * e < cols) v[e] = __ldg(f + c + 32 * e);
        }
    } else {
        const uint16_t *h = static_cast<const uint16_t *>(p);
        if constexpr (VEC) {
            if (c < cols) {
                const uint4 a = __ldg(reinterpret_cast<const uint4 *>(h + c));
                const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_lo(w[i]); v[2 * i + 1] = bf16_hi(w[i]); }
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) if (c + 32 * e < cols) v[e] = __uint_as_float((uint32_t)__ldg(h + c + 32 * e) << 16);
        }
    }
}

// Columns of the row that this warp holds (all of its chunks).
template <bool VEC, int NV>
__device__ __forceinline__ int warp_columns(int warp, int warps, int cols)
{
    int n = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) n += min(max(cols - (j * warps + warp) * Chunk<VEC>::SPAN, 0), Chunk<VEC>::SPAN);
    return n;
}

__device__ __forceinline__ float inverse_root(float a)   // one Newton step on the hardware's estimate
{
    const float r = rsqrtf(a);
    return a < 3e38f ? r * fmaf(-0.5f * a * r, r, 1.5f) : r;
}

struct NormForward {
    RowsIn x;
    Params p;
    RowsOut y;
    KeptOut kept;          // q null: no copy
    float *mean, *rstd;    // both or neither
    float eps;
    int rows, cols;
};

// blockDim = (32 * warps of a row, rows of a block); more than one warp per row means one row per block.
template <int SRC, bool VEC, int NV, bool HOLD>
__global__ void __launch_bounds__(1024) norm_forward_kernel(NormForward a)
{
    constexpr int E = Chunk<VEC>::E;
    __shared__ float2 part[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const float n_warp = (float)warp_columns<VEC, NV>(warp, warps, a.cols);
    const float n_lane = lane < warps ? (float)warp_columns<VEC, NV>(lane, warps, a.cols) : 0.f;
    const float over = 1.f / (float)a.cols;
    int c[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) c[j] = Chunk<VEC>::first((j * warps + warp) * Chunk<VEC>::SPAN, lane);
    float gamma[HOLD ? NV : 1][E], beta[HOLD ? NV : 1][E];
    if (HOLD) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            load_param<VEC>(a.p.gamma, a.p.dtype, c[j], a.cols, 1.f, gamma[j]);
            load_param<VEC>(a.p.beta, a.p.dtype, c[j], a.cols, 0.f, beta[j]);
        }
    }
    const long long step = (long long)gridDim.x * blockDim.y;
    long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const KeptIn none = {nullptr, nullptr, 0, 0};
    Raw<SRC, VEC> raw[NV];
    if (row < a.rows) {
#pragma unroll
        for (int j = 0; j < NV; ++j) raw[j].load(a.x, none, row, c[j], a.cols);
    }
    int turn = 0;
    for (; row < a.rows; row += step, turn ^= 1) {
        float v[NV][E];
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            raw[j].get(v[j]);
#pragma unroll
            for (int e = 0; e < E; ++e) s += v[j][e];
        }
        if (row + step < a.rows) {
#pragma unroll
            for (int j = 0; j < NV; ++j) raw[j].load(a.x, none, row + step, c[j], a.cols);
        }
        if (a.kept.q) {
#pragma unroll
            for (int j = 0; j < NV; ++j) keep_chunk<VEC>(a.kept, row, c[j], v[j]);
        }
        s = warp_sum(s);
        float mean = n_warp > 0.f ? s / n_warp : 0.f, m2 = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float d = Chunk<VEC>::column(c[j], e) < a.cols ? v[j][e] - mean : 0.f;
                m2 = fmaf(d, d, m2);
            }
        m2 = warp_sum(m2);
        if (warps > 1) {
            if (lane == 0) part[turn][warp] = make_float2(mean, m2);
            __syncthreads();
            const float2 o = lane < warps ? part[turn][lane] : make_float2(0.f, 0.f);
            mean = warp_sum(n_lane * o.x) * over;
            const float d = o.x - mean;
            m2 = warp_sum(fmaf(n_lane * d, d, o.y));
        }
        const float rstd = inverse_root(fmaf(m2, over, a.eps));
        if (a.mean && threadIdx.x == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!HOLD) {
                load_param<VEC>(a.p.gamma, a.p.dtype, c[j], a.cols, 1.f, gamma[0]);
                load_param<VEC>(a.p.beta, a.p.dtype, c[j], a.cols, 0.f, beta[0]);
            }
            float y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = fmaf((v[j][e] - mean) * rstd, gamma[HOLD ? j : 0][e], beta[HOLD ? j : 0][e]);
            store_chunk<VEC>(a.y, row, c[j], a.cols, y);
        }
    }
}

// Sum over the block of two values, in every thread.  `turn` alternates between calls.
__device__ __forceinline__ float2 block_sum2(float u, float v, float2 (&part)[2][32], int turn, int lane, int warp, int warps)
{
    u = warp_sum(u);
    v = warp_sum(v);
    if (warps > 1) {
        if (lane == 0) part[turn][warp] = make_float2(u, v);
        __syncthreads();
        const float2 o = lane < warps ? part[turn][lane] : make_float2(0.f, 0.f);
        u = warp_sum(o.x);
        v = warp_sum(o.y);
    }
    return make_float2(u, v);
}

// Rows wider than the registers of a block: the row is read three times (the second and third time mostly from L2).
template <int SRC, bool VEC>
__global__ void __launch_bounds__(1024) norm_forward_wide_kernel(NormForward a)
{
    constexpr int E = Chunk<VEC>::E;
    __shared__ float2 part[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int span = warps * Chunk<VEC>::SPAN;
    const float over = 1.f / (float)a.cols;
    const KeptIn none = {nullptr, nullptr, 0, 0};
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        Raw<SRC, VEC> raw;
        float v[E], s = 0.f;
        for (int c0 = warp * Chunk<VEC>::SPAN; c0 < a.cols; c0 += span) {
            raw.load(a.x, none, row, Chunk<VEC>::first(c0, lane), a.cols);
            raw.get(v);
#pragma unroll
            for (int e = 0; e < E; ++e) s += v[e];
        }
        const float mean = block_sum2(s, 0.f, part, 0, lane, warp, warps).x * over;
        s = 0.f;
        for (int c0 = warp * Chunk<VEC>::SPAN; c0 < a.cols; c0 += span) {
            const int c = Chunk<VEC>::first(c0, lane);
            raw.load(a.x, none, row, c, a.cols);
            raw.get(v);
            if (a.kept.q) keep_chunk<VEC>(a.kept, row, c, v);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float d = Chunk<VEC>::column(c, e) < a.cols ? v[e] - mean : 0.f;
                s = fmaf(d, d, s);
            }
        }
        const float rstd = inverse_root(fmaf(block_sum2(s, 0.f, part, 1, lane, warp, warps).x, over, a.eps));
        if (a.mean && threadIdx.x == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
        for (int c0 = warp * Chunk<VEC>::SPAN; c0 < a.cols; c0 += span) {
            const int c = Chunk<VEC>::first(c0, lane);
            float gamma[E], beta[E];
            load_param<VEC>(a.p.gamma, a.p.dtype, c, a.cols, 1.f, gamma);
            load_param<VEC>(a.p.beta, a.p.dtype, c, a.cols, 0.f, beta);
            raw.load(a.x, none, row, c, a.cols);
            raw.get(v);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = fmaf((v[e] - mean) * rstd, gamma[e], beta[e]);
            store_chunk<VEC>(a.y, row, c, a.cols, v);
        }
    }
}

struct NormBackward {
    RowsIn dy, x, dres;    // dres.data null: nothing added; x unused when the copy is given
    KeptIn kept;
    Params p;
    const float *mean, *rstd;
    RowsOut dx, y;         // y.data null: the forward result is not restored
    int dres_dtype;
    float *part;           // [gridDim.x][2][cols]: sums over the rows of a block
    int rows, cols;
};

template <bool VEC>
__device__ __forceinline__ void add_residual(const NormBackward &a, long long row, int c, float (&v)[Chunk<VEC>::E])
{
    if (!a.dres.data) return;
    constexpr int E = Chunk<VEC>::E;
    const KeptIn none = {nullptr, nullptr, 0, 0};
    float r[E];
    if (a.dres_dtype == LRBI_Y_BF16) { Raw<SRC_BF16, VEC> w; w.load(a.dres, none, row, c, a.cols); w.get(r); }
    else { Raw<SRC_F32, VEC> w; w.load(a.dres, none, row, c, a.cols); w.get(r); }
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] += r[e];
}

// The sums over rows stay with the thread that owns the column: in registers (HOLD), or in shared memory where a thread
// has more columns than registers.  Rows go round the blocks in a fixed order and blocks are summed in order by the
// next kernel, so the parameters' gradients have the same bits in every run.
template <int DY, int SRC, bool VEC, int NV, bool HOLD>
__global__ void __launch_bounds__(1024) norm_backward_kernel(NormBackward a)
{
    constexpr int E = Chunk<VEC>::E;
    extern __shared__ float sums[];   // !HOLD: [2][NV][E][blockDim.x]; rows of several warps per block: [warps][2][SPAN * NV]
    __shared__ float2 part[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const float over = 1.f / (float)a.cols;
    int c[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) c[j] = Chunk<VEC>::first((j * warps + warp) * Chunk<VEC>::SPAN, lane);
    float dgamma[HOLD ? NV : 1][E], dbeta[HOLD ? NV : 1][E];
    auto held = [&](int which, int j, int e) -> float & { return sums[((which * NV + j) * E + e) * blockDim.x + threadIdx.x]; };
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (HOLD) { dgamma[j][e] = 0.f; dbeta[j][e] = 0.f; }
            else { held(0, j, e) = 0.f; held(1, j, e) = 0.f; }
        }
    const long long step = (long long)gridDim.x * blockDim.y;
    long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const KeptIn none = {nullptr, nullptr, 0, 0};
    Raw<DY, VEC> raw_dy[NV];
    Raw<SRC, VEC> raw_x[NV];
    if (row < a.rows) {
#pragma unroll
        for (int j = 0; j < NV; ++j) { raw_dy[j].load(a.dy, none, row, c[j], a.cols); raw_x[j].load(a.x, a.kept, row, c[j], a.cols); }
    }
    int turn = 0;
    for (; row < a.rows; row += step, turn ^= 1) {
        float g[NV][E], n[NV][E];
        const float mean = __ldg(a.mean + row), rstd = __ldg(a.rstd + row);
        float sg = 0.f, sgn = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float gamma[E];
            load_param<VEC>(a.p.gamma, a.p.dtype, c[j], a.cols, 1.f, gamma);
            raw_dy[j].get(g[j]);
            raw_x[j].get(n[j]);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float dy = g[j][e];
                n[j][e] = Chunk<VEC>::column(c[j], e) < a.cols ? (n[j][e] - mean) * rstd : 0.f;
                if (HOLD) { dgamma[j][e] = fmaf(dy, n[j][e], dgamma[j][e]); dbeta[j][e] += dy; }
                else { held(0, j, e) = fmaf(dy, n[j][e], held(0, j, e)); held(1, j, e) += dy; }
                g[j][e] = dy * gamma[e];
                sg += g[j][e];
                sgn = fmaf(g[j][e], n[j][e], sgn);
            }
        }
        if (row + step < a.rows) {
#pragma unroll
            for (int j = 0; j < NV; ++j) { raw_dy[j].load(a.dy, none, row + step, c[j], a.cols); raw_x[j].load(a.x, a.kept, row + step, c[j], a.cols); }
        }
        const float2 both = block_sum2(sg, sgn, part, turn, lane, warp, warps);
        const float mg = both.x * over, mgn = both.y * over;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float d[E];
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] = rstd * (g[j][e] - mg - n[j][e] * mgn);
            add_residual<VEC>(a, row, c[j], d);
            store_chunk<VEC>(a.dx, row, c[j], a.cols, d);
            if (a.y.data) {
                float gamma[E], beta[E];
                load_param<VEC>(a.p.gamma, a.p.dtype, c[j], a.cols, 1.f, gamma);
                load_param<VEC>(a.p.beta, a.p.dtype, c[j], a.cols, 0.f, beta);
#pragma unroll
                for (int e = 0; e < E; ++e) d[e] = fmaf(n[j][e], gamma[e], beta[e]);
                store_chunk<VEC>(a.y, row, c[j], a.cols, d);
            }
        }
    }
    float *out = a.part + (long long)blockIdx.x * 2 * a.cols;
    if (blockDim.y > 1) {   // several rows at a time (one warp each): sum over the warps first
        constexpr int W = Chunk<VEC>::SPAN * NV;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int k = Chunk<VEC>::column(c[j], e);
                sums[(threadIdx.y * 2 + 0) * W + k] = HOLD ? dgamma[j][e] : 0.f;
                sums[(threadIdx.y * 2 + 1) * W + k] = HOLD ? dbeta[j][e] : 0.f;
            }
        __syncthreads();
        for (int k = threadIdx.y * 32 + lane; k < 2 * a.cols; k += 32 * blockDim.y) {
            const int which = k >= a.cols, at = which ? k - a.cols : k;
            float s = 0.f;
            for (int w = 0; w < (int)blockDim.y; ++w) s += sums[(w * 2 + which) * W + at];
            out[k] = s;
        }
        return;
    }
    const RowsOut to = {out, a.cols, LRBI_Y_F32};
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            // rows of `part` start on 8-column boundaries only when cols does; single stores otherwise
            float s[E];
#pragma unroll
            for (int e = 0; e < E; ++e) s[e] = HOLD ? (which ? dbeta[j][e] : dgamma[j][e]) : held(which, j, e);
            store_chunk<VEC>(to, which, c[j], a.cols, s);
        }
}

template <int DY, int SRC, bool VEC>
__global__ void __launch_bounds__(1024) norm_backward_wide_kernel(NormBackward a)
{
    constexpr int E = Chunk<VEC>::E;
    __shared__ float2 part[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int span = warps * Chunk<VEC>::SPAN;
    const float over = 1.f / (float)a.cols;
    const KeptIn none = {nullptr, nullptr, 0, 0};
    float *out = a.part + (long long)blockIdx.x * 2 * a.cols;
    for (int k = threadIdx.x; k < 2 * a.cols; k += blockDim.x) out[k] = 0.f;
    __syncthreads();
    int turn = 0;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const float mean = __ldg(a.mean + row), rstd = __ldg(a.rstd + row);
        Raw<DY, VEC> raw_dy;
        Raw<SRC, VEC> raw_x;
        float g[E], n[E], gamma[E], sg = 0.f, sgn = 0.f;
        for (int c0 = warp * Chunk<VEC>::SPAN; c0 < a.cols; c0 += span) {
            const int c = Chunk<VEC>::first(c0, lane);
            raw_dy.load(a.dy, none, row, c, a.cols);
            raw_x.load(a.x, a.kept, row, c, a.cols);
            load_param<VEC>(a.p.gamma, a.p.dtype, c, a.cols, 1.f, gamma);
            raw_dy.get(g);
            raw_x.get(n);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int k = Chunk<VEC>::column(c, e);
                const float dy = g[e];
                n[e] = (n[e] - mean) * rstd;
                if (k < a.cols) { out[k] = fmaf(dy, n[e], out[k]); out[a.cols + k] += dy; }   // this thread's columns alone
                g[e] = dy * gamma[e];
                sg += g[e];
                sgn = fmaf(g[e], n[e], sgn);
            }
        }
        const float2 both = block_sum2(sg, sgn, part, turn, lane, warp, warps);
        const float mg = both.x * over, mgn = both.y * over;
        for (int c0 = warp * Chunk<VEC>::SPAN; c0 < a.cols; c0 += span) {
            const int c = Chunk<VEC>::first(c0, lane);
            float d[E], beta[E];
            raw_dy.load(a.dy, none, row, c, a.cols);
            raw_x.load(a.x, a.kept, row, c, a.cols);
            load_param<VEC>(a.p.gamma, a.p.dtype, c, a.cols, 1.f, gamma);
            raw_dy.get(g);
            raw_x.get(n);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                n[e] = (n[e] - mean) * rstd;
                d[e] = rstd * (g[e] * gamma[e] - mg - n[e] * mgn);
            }
            add_residual<VEC>(a, row, c, d);
            store_chunk<VEC>(a.dx, row, c, a.cols, d);
            if (a.y.data) {
                load_param<VEC>(a.p.beta, a.p.dtype, c, a.cols, 0.f, beta);
#pragma unroll
                for (int e = 0; e < E; ++e) d[e] = fmaf(n[e], gamma[e], beta[e]);
                store_chunk<VEC>(a.y, row, c, a.cols, d);
            }
        }
    }
}

// Sums the blocks' parts in order: 32 columns a block, 32 threads along the parts of each.
__global__ void __launch_bounds__(1024) norm_param_sum_kernel(const float *__restrict__ part, int parts, int cols, float *dgamma, float *dbeta)
{
    __shared__ float s[32][33];
    const int k = blockIdx.x * 32 + threadIdx.x;
    float v = 0.f;
    if (k < 2 * cols)
        for (int p = threadIdx.y; p < parts; p += 32) v += part[(long long)p * 2 * cols + k];
    s[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    v = warp_sum(s[threadIdx.x][threadIdx.y]);
    const int at = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0 && at < 2 * cols) {
        if (at < cols) { if (dgamma) dgamma[at] = v; }
        else if (dbeta) dbeta[at - cols] = v;
    }
}

// -----------------------------------------------------------------------------------------------------------------
// Host side
// -----------------------------------------------------------------------------------------------------------------
namespace {

constexpr int NORM_SMS = 148;

struct Shape {
    dim3 block;
    int chunks;     // chunks of a lane in units of 8 values (1 or 2); 0: the wide kernel
};

// A lane holds 8 values of a row while that takes at most 1024 threads, then 16 values.
Shape norm_shape(int cols, bool vec)
{
    const int span = 256;   // columns of a warp with 8 values a lane, in either way of taking them
    const int warps = (cols + span - 1) / span;
    (void)vec;
    if (warps == 1) return {dim3(32, 8), 1};
    if (warps <= 32) return {dim3(32 * warps, 1), 1};
    if (warps <= 64) return {dim3(32 * ((warps + 1) / 2), 1), 2};
    return {dim3(1024, 1), 0};
}

// Blocks of a launch: enough threads on every SM, and no more blocks than rows.
int norm_grid(const Shape &s, int rows, int threads_per_sm)
{
    const int per_sm = threads_per_sm / (int)(s.block.x * s.block.y);
    const long long need = ((long long)rows + s.block.y - 1) / s.block.y;
    return (int)(need < (long long)NORM_SMS * (per_sm < 1 ? 1 : per_sm) ? need : NORM_SMS * (per_sm < 1 ? 1 : per_sm));
}

// Blocks of the backward pass, each of which leaves sums to be added up: at least four rows a block.
int backward_grid(int rows, int cols)
{
    const Shape s = norm_shape(cols, true);
    const int grid = norm_grid(s, rows, 1024), few = (rows + 4 * (int)s.block.y - 1) / (4 * (int)s.block.y);
    return grid < few ? grid : (few < 1 ? 1 : few);
}

template <int SRC, bool VEC>
void forward_launch(const NormForward &a, cudaStream_t s)
{
    const Shape sh = norm_shape(a.cols, VEC);
    const int grid = norm_grid(sh, a.rows, 1024);
    if (sh.chunks == 1) norm_forward_kernel<SRC, VEC, VEC ? 1 : 2, true><<<grid, sh.block, 0, s>>>(a);
    else if (sh.chunks == 2) norm_forward_kernel<SRC, VEC, VEC ? 2 : 4, false><<<grid, sh.block, 0, s>>>(a);
    else norm_forward_wide_kernel<SRC, VEC><<<grid, sh.block, 0, s>>>(a);
}

template <int DY, int SRC, bool VEC>
lrbi_status backward_launch(const NormBackward &a, int grid, cudaStream_t s)
{
    const Shape sh = norm_shape(a.cols, VEC);
    if (sh.chunks == 1) {
        const size_t smem = sh.block.y > 1 ? (size_t)sh.block.y * 2 * 256 * 4 : 0;
        norm_backward_kernel<DY, SRC, VEC, VEC ? 1 : 2, true><<<grid, sh.block, smem, s>>>(a);
    } else if (sh.chunks == 2) {
        const size_t smem = (size_t)2 * 16 * 4 * sh.block.x;
        auto kernel = norm_backward_kernel<DY, SRC, VEC, VEC ? 2 : 4, false>;
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) { note_cuda_error((int)e); return LRBI_ERR_CUDA; }
        kernel<<<grid, sh.block, smem, s>>>(a);
    } else norm_backward_wide_kernel<DY, SRC, VEC><<<grid, sh.block, 0, s>>>(a);
    return LRBI_OK;
}

lrbi_status launched(int n)
{
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) { note_cuda_error((int)e); return LRBI_ERR_CUDA; }
    count_launch(n);
    return LRBI_OK;
}

bool param16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace

size_t norm_backward_workspace(int rows, int cols) { return (size_t)backward_grid(rows < 1 ? 1 : rows, cols) * 2 * cols * 4; }

lrbi_status launch_layer_norm(const NormArgs &n, cudaStream_t s)
{
    const NormForward a = {{n.x, n.x_stride}, {n.gamma, n.beta, n.param_dtype}, {n.y, n.y_stride, n.y_dtype},
                           {n.q_out, n.scale_out, checkpoint_pitch(n.cols), checkpoint_groups(n.cols)}, n.mean_out, n.rstd_out, n.eps, n.rows, n.cols};
    const bool vec = n.cols % 8 == 0 && rows16(n.x, n.x_stride, n.x_dtype) && rows16(n.y, n.y_stride, n.y_dtype) && param16(n.gamma) && param16(n.beta);
    if (n.x_dtype == LRBI_Y_BF16) vec ? forward_launch<SRC_BF16, true>(a, s) : forward_launch<SRC_BF16, false>(a, s);
    else vec ? forward_launch<SRC_F32, true>(a, s) : forward_launch<SRC_F32, false>(a, s);
    return launched(1);
}

lrbi_status launch_layer_norm_backward(const NormArgs &n, float *workspace, cudaStream_t s)
{
    NormBackward a = {{n.dy, n.dy_stride}, {n.x, n.x_stride}, {n.dres, n.dres_stride}, {n.q, n.scale, checkpoint_pitch(n.cols), checkpoint_groups(n.cols)},
                      {n.gamma, n.beta, n.param_dtype}, n.mean, n.rstd, {n.dx, n.dx_stride, n.dx_dtype}, {n.y, n.y_stride, n.dy_dtype},
                      n.dx_dtype, workspace, n.rows, n.cols};
    const int grid = backward_grid(n.rows < 1 ? 1 : n.rows, n.cols);
    // rows of the workspace hold cols floats: vectors need cols % 8 == 0, which is asked for anyway
    const bool vec = n.cols % 8 == 0 && rows16(n.dy, n.dy_stride, n.dy_dtype) && (n.q || rows16(n.x, n.x_stride, n.x_dtype)) &&
                     (!n.dres || rows16(n.dres, n.dres_stride, n.dx_dtype)) && rows16(n.dx, n.dx_stride, n.dx_dtype) &&
                     (!n.y || rows16(n.y, n.y_stride, n.dy_dtype)) && param16(n.gamma) && param16(n.beta);
    const int src = n.q ? SRC_KEPT : n.x_dtype;
    lrbi_status st;
#define BACKWARD(DY, SRC) st = vec ? backward_launch<DY, SRC, true>(a, grid, s) : backward_launch<DY, SRC, false>(a, grid, s)
    if (n.dy_dtype == LRBI_Y_BF16) {
        if (src == SRC_BF16) BACKWARD(SRC_BF16, SRC_BF16);
        else if (src == SRC_F32) BACKWARD(SRC_BF16, SRC_F32);
        else BACKWARD(SRC_BF16, SRC_KEPT);
    } else {
        if (src == SRC_BF16) BACKWARD(SRC_F32, SRC_BF16);
        else if (src == SRC_F32) BACKWARD(SRC_F32, SRC_F32);
        else BACKWARD(SRC_F32, SRC_KEPT);
    }
#undef BACKWARD
    if (st != LRBI_OK) return st;
    if (n.dgamma || n.dbeta) norm_param_sum_kernel<<<(2 * n.cols + 31) / 32, dim3(32, 32), 0, s>>>(workspace, grid, n.cols, n.dgamma, n.dbeta);
    return launched(n.dgamma || n.dbeta ? 2 : 1);
}

}  // namespace lrbi
