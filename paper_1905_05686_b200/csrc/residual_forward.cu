// Between two blocks, forward (residual_common.cuh has the formulas).
#include "residual_common.cuh"

namespace lrbi {

// Sums over a row of two values a thread, in every thread.
__device__ __forceinline__ void row_two(float &p, float &q, Team &t, float *part)
{
    const bool up = t.lane & 16;
    float s = (up ? q : p) + __shfl_xor_sync(0xFFFFFFFFu, up ? p : q, 16);      // lower lanes have p, upper ones q
#pragma unroll
    for (int j = 8; j; j >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, j);
    if (t.alone()) {
        p = __shfl_sync(0xFFFFFFFFu, s, 0);
        q = __shfl_sync(0xFFFFFFFFu, s, 16);
        return;
    }
    float *all = t.board<2>(part);
    if ((t.lane & 15) == 0) t.tell(all + t.entry() * 2 + (t.lane >> 4), s);
    t.meet();
    p = q = 0.f;
    if (t.entries() <= 8) {
        for (int e = 0; e < t.entries(); ++e) {
            const float2 v = *reinterpret_cast<const float2 *>(all + 2 * e);
            p += v.x;
            q += v.y;
        }
    } else {
        for (int e = t.lane; e < t.entries(); e += 32) { p += all[2 * e]; q += all[2 * e + 1]; }
        p = warp_sum(p);
        q = warp_sum(q);
    }
}

// Mean and 1 / root over a row of the values v (zeros where there is no column).  Squares are summed beside the values, as long as
// the mean's square is at most the variance (the difference then loses one bit at most).  Else the mean is taken off the values, and
// what is left of them is summed once more with its squares: its mean corrects the first one, whose own error, roundings of a sum of
// large values, would be a part of the spread (values 1e5 times their spread from zero: 2e-2 of it).  centre: what is left to take off v.
// left: columns from the warp's first one on.
template <int K, bool STRIDED, bool RMS, bool FULL>
__device__ __forceinline__ void row_statistics(F2 (&v)[K][PAIRS], int left, const Join &j, Team &t, float *part, float &mean, float &centre, float &rstd)
{
    F2 s = f2(0.f), q = f2(0.f);
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            if (!RMS) s = s + v[k][i];
            q = fma2(v[k][i], v[k][i], q);
        }
    float sum = RMS ? 0.f : sum2(s), square = sum2(q);
    row_two(sum, square, t, part);
    mean = centre = RMS ? 0.f : sum * j.per;
    float variance = square * j.per;
    if (!RMS) {
        variance = fmaf(-mean, mean, variance);
        if (!(mean * mean <= variance)) {          // the same in all threads of the row
            s = q = f2(0.f);
#pragma unroll
            for (int k = 0; k < K; ++k) {
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) v[k][i] = v[k][i] + f2(-mean);
                keep_there<STRIDED, FULL>(v[k], left - k * SPAN, t.lane);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    s = s + v[k][i];
                    q = fma2(v[k][i], v[k][i], q);
                }
            }
            sum = sum2(s);
            square = sum2(q);
            row_two(sum, square, t, part);
            centre = sum * j.per;
            mean += centre;
            variance = fmaf(-centre, centre, square * j.per);
            if (variance < 0.f) variance = 0.f;    // (a NaN stays)
        }
    }
    rstd = inverse_root(variance + j.a.eps);
}

// blockDim = (threads of a row, rows of a block); clusters of `split` blocks share a row.  Shared memory: the vectors, the places to
// meet, and two rows for each team, one of them on its way.  DIRECT: the vectors are read where they are, by every row.
template <int X, int F, bool STRIDED, int K, bool RMS, bool DIRECT>
__global__ void __launch_bounds__(JOIN_THREADS, 1) join_forward_kernel(Join j)
{
    const JoinArgs &a = j.a;
    extern __shared__ __align__(16) float shared[];
    using XS = Stream<X, STRIDED, K>;
    using FS = Stream<F, STRIDED, K>;
    constexpr int SLOT = XS::SLOT + FS::SLOT, XSIZE = XS::SIZE, FSIZE = FS::SIZE;
    Team t(j.split);
    const int block0 = t.rank * j.width, w0 = t.warp * K * SPAN, c0 = block0 + w0, left = a.cols - c0;      // first columns of the block, of the warp
    float *vectors = shared;                                 // gate * post_gamma, gamma, beta, gate * post_beta, up to the last that there is
    float *part = vectors + (DIRECT ? 0 : join_vectors(a) * j.width);
    char *ring = reinterpret_cast<char *>(part + blockDim.y * 2 * t.entries() * 2) + (threadIdx.y * t.warps + t.warp) * 2 * SLOT;
    begin();
    const XS x(a.x, a.x_stride, c0, a.cols);
    const FS f(a.f, a.f_stride, c0, a.cols);
    const long long step = (long long)(gridDim.x / j.split) * blockDim.y;
    long long row = (long long)(blockIdx.x / j.split) * blockDim.y + threadIdx.y;
    if (row < a.rows) { f.template ask<false>(ring, row, t.lane); x.template ask<false>(ring + FS::SLOT, row, t.lane); }
    copies_asked();
    for (int c = (threadIdx.y * blockDim.x + threadIdx.x) * 4; !DIRECT && c < j.width; c += blockDim.x * blockDim.y * 4) {
        float4 *to = reinterpret_cast<float4 *>(vectors + vector_place<STRIDED>(c));
        const int from = block0 + c, pitch = j.width / 4;
        const float4 gate = four_of(a.gate, a.param_dtype, j.whole, from, a.cols, 1.f), pg = four_of(a.post_gamma, a.param_dtype, j.whole, from, a.cols, 1.f);
        const float4 pb = four_of(a.post_beta, a.param_dtype, j.whole, from, a.cols, 0.f), g = four_of(a.gamma, a.param_dtype, j.whole, from, a.cols, 0.f);
        const float4 b = four_of(a.beta, a.param_dtype, j.whole, from, a.cols, 0.f);
        to[0] = gate * pg;
        if (a.post_beta) to[3 * pitch] = gate * pb;
        if (a.gamma) to[pitch] = g;
        if (a.beta) to[2 * pitch] = b;
    }
    __syncthreads();
    if (j.split > 1) t.meet();       // blocks write to one another once all of them have begun
    const bool tells = a.stats && t.entry() == 0 && t.lane == 0;
    const int c = lane_column<STRIDED>(c0, t.lane);
    char *const out = static_cast<char *>(a.out) + (long long)c * XSIZE, *const u = static_cast<char *>(a.u) + (long long)c * FSIZE;
    const float *own = vectors + w0;
    const Params p = {nullptr, nullptr, a.param_dtype, j.whole};
    // Chunk k of a vector: gate * post_gamma, gamma, beta, gate * post_beta.
    auto vector = [&](int which, int k, F2 (&w)[PAIRS]) {
        if constexpr (!DIRECT) get_vector<STRIDED>(own + which * j.width, k, t.lane, w);
        else {
            const void *const all[4] = {a.post_gamma, a.gamma, a.beta, a.post_beta};
            load_param<STRIDED>(all[which], p, c + k * SPAN, a.cols, all[which] ? 0.f : 1.f, w);
            if ((which == 0 || which == 3) && a.gate) {
                F2 gate[PAIRS];
                load_param<STRIDED>(a.gate, p, c + k * SPAN, a.cols, 0.f, gate);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) w[i] = w[i] * gate[i];
            }
        }
    };
    auto rows = [&](auto full) {
    constexpr bool FULL = decltype(full)::value;         // the warp has all of its columns
    for (int stage = 0; row < a.rows; row += step, stage ^= 1) {
        const char *slot = ring + stage * SLOT;
        __syncwarp();
        if (row + step < a.rows) {
            f.template ask<FULL>(ring + (stage ^ 1) * SLOT, row + step, t.lane);
            x.template ask<FULL>(ring + (stage ^ 1) * SLOT + FS::SLOT, row + step, t.lane);
        }
        copies_asked();
        copies_wait<1>();
        __syncwarp();
        F2 v[K][PAIRS], w[PAIRS], b[PAIRS];
#pragma unroll
        for (int k = 0; k < K; ++k) f.template get<FULL>(slot, row, k, max(left - k * SPAN, 0), t.lane, v[k]);
        float mean = 0.f, centre = 0.f, rstd = 1.f;
        if (a.post_gamma) row_statistics<K, STRIDED, RMS, FULL>(v, left, j, t, part, mean, centre, rstd);
        if (tells) { a.stats[2ll * a.rows + row] = mean; a.stats[3ll * a.rows + row] = rstd; }
        F2 scale = f2(rstd), shift = f2(-centre * rstd);
        char *to = out + row * a.out_stride * XSIZE;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!FULL && left <= k * SPAN) break;
            vector(0, k, w);
            x.template get<FULL>(slot + FS::SLOT, row, k, left - k * SPAN, t.lane, b);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) v[k][i] = fma2(b[i], f2(a.residual_scale), fma2(v[k][i], scale, shift) * w[i]);
            if (a.post_beta) {
                vector(3, k, b);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) v[k][i] = v[k][i] + b[i];
            }
            if (X == SRC_BF16) {           // the stream as it is stored is what goes on
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    float lo, hi;
                    split(v[k][i], lo, hi);
                    const uint32_t r = pack_bf16(lo, hi);
                    v[k][i] = f2(bf16_lo(r), bf16_hi(r));
                }
            }
            store_at<XSIZE, STRIDED>(to + k * SPAN * XSIZE, FULL ? SPAN : a.cols - c - k * SPAN, v[k], STRIDED && (FULL || left >= (k + 1) * SPAN));
            keep_there<STRIDED, FULL>(v[k], left - k * SPAN, t.lane);
        }
        mean = centre = 0.f;
        rstd = 1.f;
        if (a.gamma) row_statistics<K, STRIDED, RMS, FULL>(v, left, j, t, part, mean, centre, rstd);
        if (tells) { a.stats[row] = mean; a.stats[a.rows + row] = rstd; }
        if (!a.gamma) continue;
        scale = f2(rstd);
        shift = f2(-centre * rstd);
        to = u + row * a.u_stride * FSIZE;
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!FULL && left <= k * SPAN) break;
            vector(1, k, w);
            if (a.beta) {
                vector(2, k, b);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) v[k][i] = fma2(fma2(v[k][i], scale, shift), w[i], b[i]);
            } else {
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) v[k][i] = fma2(v[k][i], scale, shift) * w[i];
            }
            if (a.u) store_at<FSIZE, STRIDED>(to + k * SPAN * FSIZE, FULL ? SPAN : a.cols - c - k * SPAN, v[k], STRIDED && (FULL || left >= (k + 1) * SPAN));
            if (a.q) {
                keep_there<STRIDED, FULL>(v[k], left - k * SPAN, t.lane);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    float lo, hi;
                    split(v[k][i], lo, hi);
                    top = max(top, max(__float_as_uint(lo) & 0x7FFFFFFFu, __float_as_uint(hi) & 0x7FFFFFFFu));
                }
            }
        }
        if (a.q) {
            top = __reduce_max_sync(0xFFFFFFFFu, top);
            if (!t.alone()) {
                float *all = t.board<2>(part);
                if (t.lane == 0) t.tell(all + t.entry() * 2, __uint_as_float(top));
                t.meet();
                top = 0;
                for (int e = t.lane; e < t.entries(); e += 32) top = max(top, __float_as_uint(all[2 * e]));
                top = __reduce_max_sync(0xFFFFFFFFu, top);
            }
            const TokenScale s(top);
            if (t.entry() == 0 && t.lane == 0) a.q_scale[row] = s.scale();
            const int pitch = (a.cols + 15) / 16 * 16;
#pragma unroll
            for (int k = 0; k < K; ++k) store_i8<STRIDED>(a.q + row * pitch + c + k * SPAN, pitch - c - k * SPAN, v[k], s.factor, s.fine, FULL);
        }
    }
    };
    if (left >= K * SPAN) rows(std::true_type());
    else rows(std::false_type());
    let_next();
    if (j.split > 1) t.meet();       // a block stays while others may still write to it
}

namespace {

template <int X, int F, bool STRIDED, bool RMS>
lrbi_status forward_rows(const JoinCut &k, cudaStream_t s, const Join &j)
{
    if (k.each == 1) return join_launch(join_forward_kernel<X, F, STRIDED, 1, RMS, false>, k, s, j);
    return k.direct ? join_launch(join_forward_kernel<X, F, STRIDED, 4, RMS, true>, k, s, j) : join_launch(join_forward_kernel<X, F, STRIDED, 4, RMS, false>, k, s, j);
}
template <int X, int F>
lrbi_status forward_types(const JoinCut &k, bool vector, cudaStream_t s, const Join &j)
{
    if (j.a.rms) return vector ? forward_rows<X, F, false, true>(k, s, j) : forward_rows<X, F, true, true>(k, s, j);
    return vector ? forward_rows<X, F, false, false>(k, s, j) : forward_rows<X, F, true, false>(k, s, j);
}
}  // namespace

lrbi_status launch_join(const JoinArgs &a, cudaStream_t s)
{
    const JoinCut k = forward_cut(a);
    const Join j = make_join(a, k, nullptr);
    const bool vector = join_vector(a);
    if (a.x_dtype == LRBI_Y_BF16) return forward_types<SRC_BF16, SRC_BF16>(k, vector, s, j);
    return a.f_dtype == LRBI_Y_BF16 ? forward_types<SRC_F32, SRC_BF16>(k, vector, s, j) : forward_types<SRC_F32, SRC_F32>(k, vector, s, j);
}

}  // namespace lrbi
