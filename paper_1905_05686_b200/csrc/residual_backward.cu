// Between two blocks, backward (residual_common.cuh has the formulas).
#include "residual_common.cuh"

namespace lrbi {

// The sums over a row of N = 8 values a thread, in every thread: within a warp they are folded into one another (norm_common.cuh).
__device__ __forceinline__ void row_eight(float (&v)[8], Team &t, float *part)
{
    float k[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) k[i] = v[i];
#pragma unroll
    for (int m = 8, at = 16; m > 1; m /= 2, at /= 2) {
        const bool up = t.lane & at;
#pragma unroll
        for (int i = 0; i < m / 2; ++i) {
            const float send = up ? k[i] : k[i + m / 2], stay = up ? k[i + m / 2] : k[i];
            k[i] = stay + __shfl_xor_sync(0xFFFFFFFFu, send, at);
        }
    }
    float s = k[0];
    s += __shfl_xor_sync(0xFFFFFFFFu, s, 2);
    s += __shfl_xor_sync(0xFFFFFFFFu, s, 1);
    const int mine = t.lane >> 2;        // the value that this lane has
    if (!t.alone()) {
        float *all = t.board<8>(part);
        if ((t.lane & 3) == 0) t.tell(all + t.entry() * 8 + mine, s);
        t.meet();
        s = 0.f;
        for (int e = t.lane & 3; e < t.entries(); e += 4) s += all[e * 8 + mine];
        s += __shfl_xor_sync(0xFFFFFFFFu, s, 2);
        s += __shfl_xor_sync(0xFFFFFFFFu, s, 1);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __shfl_sync(0xFFFFFFFFu, s, i * 4);
}

// As the forward kernel.  A row is read from shared memory twice, for its sums and for its results; a thread keeps the sums over
// rows of its columns; the rows of a block are added up at the end.  LEVEL: also those of ds and of du alone, for the betas.
template <int X, int F, bool STRIDED, int K, bool RMS, bool LEVEL>
__global__ void __launch_bounds__(JOIN_THREADS, 1) join_backward_kernel(Join j)
{
    const JoinArgs &a = j.a;
    extern __shared__ __align__(16) float shared[];
    using XS = Stream<X, STRIDED, K>;
    using FS = Stream<F, STRIDED, K>;
    constexpr int SLOT = 2 * XS::SLOT + 2 * FS::SLOT, XSIZE = XS::SIZE, FSIZE = FS::SIZE;      // f, du, dout, out
    Team t(j.split);
    const int block0 = t.rank * j.width, w0 = t.warp * K * SPAN, c0 = block0 + w0, left = a.cols - c0;
    float *vectors = shared;                                 // gamma, gate * post_gamma
    float *part = vectors + 2 * j.width;
    float *columns = part + blockDim.y * 2 * t.entries() * 8;
    char *ring = reinterpret_cast<char *>(columns) + (threadIdx.y * t.warps + t.warp) * 2 * SLOT;
    begin();
    const FS f(a.f, a.f_stride, c0, a.cols), du(a.du, a.du_stride, c0, a.cols);
    const XS dout(a.dout, a.dout_stride, c0, a.cols), out(a.out, a.out_stride, c0, a.cols);
    const bool post = a.post_gamma, pre = a.gamma;
    const long long step = (long long)(gridDim.x / j.split) * blockDim.y;
    long long row = (long long)(blockIdx.x / j.split) * blockDim.y + threadIdx.y;
    auto ask = [&](auto full, char *slot, long long r) {
        constexpr bool FULL = decltype(full)::value;
        if (r < a.rows) {
            f.template ask<FULL>(slot, r, t.lane);
            du.template ask<FULL>(slot + FS::SLOT, r, t.lane);
            dout.template ask<FULL>(slot + 2 * FS::SLOT, r, t.lane);
            out.template ask<FULL>(slot + 2 * FS::SLOT + XS::SLOT, r, t.lane);
        }
        copies_asked();
    };
    struct { float mean, rstd, f_mean, f_rstd; } now = {0.f, 0.f, 0.f, 1.f}, next = now;
    auto ask_statistics = [&](long long r) {
        if (r >= a.rows) return;
        if (pre) { next.rstd = __ldg(a.stats + a.rows + r); if (!RMS) next.mean = __ldg(a.stats + r); }
        if (post) { next.f_rstd = __ldg(a.stats + 3ll * a.rows + r); if (!RMS) next.f_mean = __ldg(a.stats + 2ll * a.rows + r); }
    };
    ask(std::false_type(), ring, row);
    ask_statistics(row);
    for (int c = (threadIdx.y * blockDim.x + threadIdx.x) * 4; c < j.width; c += blockDim.x * blockDim.y * 4) {
        float4 *to = reinterpret_cast<float4 *>(vectors + vector_place<STRIDED>(c));
        const int from = block0 + c;
        const float4 gate = four_of(a.gate, a.param_dtype, j.whole, from, a.cols, a.gate ? 0.f : 1.f), pg = four_of(a.post_gamma, a.param_dtype, j.whole, from, a.cols, post ? 0.f : 1.f);
        to[0] = four_of(a.gamma, a.param_dtype, j.whole, from, a.cols, 0.f);
        to[j.width / 4] = gate * pg;
    }
    __syncthreads();
    if (j.split > 1) t.meet();       // blocks write to one another once all of them have begun
    const float *own = vectors + w0;
    constexpr int SUMS = LEVEL ? 4 : 2;
    F2 sums[K][SUMS][PAIRS];         // ds nf, du n, ds, du
    float total_w = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int s = 0; s < SUMS; ++s)
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) sums[k][s][i] = f2(0.f);
        F2 w[PAIRS];
        if (RMS || left <= k * SPAN) continue;
        get_vector<STRIDED>(own + j.width, k, t.lane, w);
        keep_there<STRIDED>(w, left - k * SPAN, t.lane);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) total_w += sum2(w[i]);
    }
    const int c = lane_column<STRIDED>(c0, t.lane);
    char *const dx = static_cast<char *>(a.dx) + (long long)c * XSIZE, *const df = static_cast<char *>(a.df) + (long long)c * FSIZE;
    // full: the warp has all of its columns; all: there are a norm before and behind, and both gradients
    auto rows = [&](auto full, auto all) {
    constexpr bool FULL = decltype(full)::value, ALL = decltype(all)::value;
    const bool pre = ALL || a.gamma, post = ALL || a.post_gamma;
    for (int stage = 0; row < a.rows; row += step, stage ^= 1) {
        const char *slot = ring + stage * SLOT;
        __syncwarp();
        ask(full, ring + (stage ^ 1) * SLOT, row + step);
        now = next;
        ask_statistics(row + step);
        copies_wait<1>();
        __syncwarp();
        F2 acc[7];
#pragma unroll
        for (int i = 0; i < 7; ++i) acc[i] = f2(0.f);
        const F2 scale = f2(now.rstd), shift = f2(-now.mean * now.rstd), f_scale = f2(now.f_rstd), f_shift = f2(-now.f_mean * now.f_rstd);
        // n and nf where there is no column are not zero; what they are multiplied by is.
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!FULL && left <= k * SPAN) break;
            F2 p[PAIRS], n[PAIRS], g[PAIRS], w[PAIRS];
            dout.template get<FULL>(slot + 2 * FS::SLOT, row, k, left - k * SPAN, t.lane, p);
            if (pre) {
                du.template get<FULL>(slot + FS::SLOT, row, k, left - k * SPAN, t.lane, g);
                out.template get<FULL>(slot + 2 * FS::SLOT + XS::SLOT, row, k, left - k * SPAN, t.lane, n);
                get_vector<STRIDED>(own, k, t.lane, w);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    n[i] = fma2(n[i], scale, shift);
                    sums[k][1][i] = fma2(g[i], n[i], sums[k][1][i]);
                    if constexpr (LEVEL) sums[k][3][i] = sums[k][3][i] + g[i];
                    g[i] = g[i] * w[i];
                    if (!RMS) acc[0] = acc[0] + g[i];
                    acc[1] = fma2(g[i], n[i], acc[1]);
                    p[i] = fma2(g[i], scale, p[i]);
                }
            }
            if (post) {
                F2 nf[PAIRS];
                get_vector<STRIDED>(own + j.width, k, t.lane, w);
                f.template get<FULL>(slot, row, k, left - k * SPAN, t.lane, nf);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    nf[i] = w[i] * fma2(nf[i], f_scale, f_shift);
                    acc[4] = fma2(nf[i], p[i], acc[4]);
                    if (pre) acc[6] = fma2(nf[i], n[i], acc[6]);
                    if (!RMS) {
                        acc[2] = fma2(w[i], p[i], acc[2]);
                        if (pre) acc[3] = fma2(w[i], n[i], acc[3]);
                        acc[5] = acc[5] + nf[i];
                    }
                }
            }
        }
        float flat = 0.f, along = 0.f, f_flat = 0.f, f_along = 0.f;
        if (pre || post) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 7; ++i) v[i] = sum2(acc[i]);
            v[7] = total_w;
            row_eight(v, t, part);
            if (pre) {
                flat = v[0] * j.per * now.rstd;
                along = v[1] * j.per * now.rstd;
            }
            f_along = (v[4] - flat * v[5] - along * v[6]) * j.per;      // means of w ds nf and of w ds
            if (!RMS) f_flat = (v[2] - flat * v[7] - along * v[3]) * j.per;
        }
        const F2 minus_flat = f2(-flat), minus_along = f2(-along), f_across = f2(-f_along * now.f_rstd), f_level = f2(-f_flat * now.f_rstd);
        char *to_x = dx + row * a.dx_stride * XSIZE, *to_f = df + row * a.df_stride * FSIZE;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!FULL && left <= k * SPAN) break;
            F2 ds[PAIRS], n[PAIRS], g[PAIRS], w[PAIRS];
            dout.template get<FULL>(slot + 2 * FS::SLOT, row, k, left - k * SPAN, t.lane, ds);
            if (pre) {
                du.template get<FULL>(slot + FS::SLOT, row, k, left - k * SPAN, t.lane, g);
                out.template get<FULL>(slot + 2 * FS::SLOT + XS::SLOT, row, k, left - k * SPAN, t.lane, n);
                get_vector<STRIDED>(own, k, t.lane, w);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    ds[i] = fma2(g[i] * w[i], scale, ds[i]);
                    ds[i] = fma2(fma2(n[i], scale, shift), minus_along, ds[i]);
                    if (!RMS) ds[i] = ds[i] + minus_flat;
                }
            }
            f.template get<FULL>(slot, row, k, left - k * SPAN, t.lane, n);
            get_vector<STRIDED>(own + j.width, k, t.lane, w);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                n[i] = fma2(n[i], f_scale, f_shift);
                sums[k][0][i] = fma2(ds[i], n[i], sums[k][0][i]);
                if constexpr (LEVEL) sums[k][2][i] = sums[k][2][i] + ds[i];
                g[i] = ds[i] * f2(a.residual_scale);
                n[i] = post ? fma2(ds[i] * w[i], f_scale, fma2(n[i], f_across, f_level)) : ds[i] * w[i];
            }
            store_at<XSIZE, STRIDED>(to_x + k * SPAN * XSIZE, FULL ? SPAN : a.cols - c - k * SPAN, g, STRIDED && (FULL || left >= (k + 1) * SPAN));
            store_at<FSIZE, STRIDED>(to_f + k * SPAN * FSIZE, FULL ? SPAN : a.cols - c - k * SPAN, n, STRIDED && (FULL || left >= (k + 1) * SPAN));
        }
    }
    };
    if (left >= K * SPAN && pre && post && a.dout) rows(std::true_type(), std::true_type());
    else rows(std::false_type(), std::false_type());
    copies_wait<0>();
    if (j.parts) {
        // Every team leaves its sums where its rows were; they are added in the order of the teams, so that they have the same bits
        // every time.
        __syncthreads();
        float *mine = columns + threadIdx.y * SUMS * j.width;
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int s = 0; s < SUMS; ++s) {
                float v[CHUNK];
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) split(sums[k][s][i], v[2 * i], v[2 * i + 1]);
                float *at = mine + s * j.width + w0 + k * SPAN;
                if constexpr (STRIDED) {
#pragma unroll
                    for (int e = 0; e < CHUNK; ++e) at[t.lane + 32 * e] = v[e];
                } else {
                    *reinterpret_cast<float4 *>(at + t.lane * 4) = make_float4(v[0], v[1], v[2], v[3]);
                    *reinterpret_cast<float4 *>(at + 128 + t.lane * 4) = make_float4(v[4], v[5], v[6], v[7]);
                }
            }
        }
        __syncthreads();
        const int pitch = j.width * j.split;
        float *to = j.parts + (long long)(blockIdx.x / j.split) * 4 * pitch + block0;
        for (int q = threadIdx.y * blockDim.x + threadIdx.x; q < j.width / 4 * SUMS; q += blockDim.x * blockDim.y) {      // four columns of one sum
            const int s = q / (j.width / 4), at = (q - s * (j.width / 4)) * 4;
            const float *from = columns + s * j.width + vector_place<STRIDED>(at);
            float4 v = *reinterpret_cast<const float4 *>(from);
            for (int team = 1; team < (int)blockDim.y; ++team) {
                const float4 o = *reinterpret_cast<const float4 *>(from + team * SUMS * j.width);
                v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
            }
            *reinterpret_cast<float4 *>(to + s * pitch + at) = v;
        }
    }
    let_next();
    if (j.split > 1) t.meet();       // a block stays while others may still write to it
}

// Adds the groups' parts up: block (8 x 4 columns, 4 sums, 32 slices of the parts), a thread's loads all under way together.
constexpr int JOIN_SLICES = 32;
__global__ void __launch_bounds__(32 * JOIN_SLICES) join_sums_kernel(Join j, int groups, bool all)      // all: of the four, not the first two alone
{
    begin();
    let_next();
    const JoinArgs &a = j.a;
    __shared__ float4 part[JOIN_SLICES][4][8];
    __shared__ float sums[4][32];
    const int pitch = j.width * j.split, c0 = blockIdx.x * 32;      // the parts' rows are whole spans
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < (NORM_SMS + JOIN_SLICES - 1) / JOIN_SLICES; ++i) {
        const int g = i * JOIN_SLICES + threadIdx.z;
        if (g < groups && (all || threadIdx.y < 2)) {
            const float4 o = *reinterpret_cast<const float4 *>(j.parts + ((long long)g * 4 + threadIdx.y) * pitch + c0 + threadIdx.x * 4);
            v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        }
    }
    part[threadIdx.z][threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    const int at = (threadIdx.z * 4 + threadIdx.y) * 8 + threadIdx.x, s = at >> 5, lane = at & 31;
    if (s < 4) {
        float sum = 0.f;
#pragma unroll
        for (int z = 0; z < JOIN_SLICES; ++z) sum += reinterpret_cast<const float *>(part[z][s])[lane];
        sums[s][lane] = sum;
    }
    __syncthreads();
    const int c = c0 + at;
    if (at >= 32 || c >= a.cols) return;
    const float gate = a.gate ? one_param(a.gate, a.param_dtype, c) : 1.f, post = sums[0][at], level = sums[2][at];
    if (a.dgamma) a.dgamma[c] = sums[1][at];
    if (a.dbeta) a.dbeta[c] = sums[3][at];
    if (a.dpost_gamma) a.dpost_gamma[c] = gate * post;
    if (a.dpost_beta) a.dpost_beta[c] = gate * level;
    if (a.dgate) a.dgate[c] = fmaf(a.post_gamma ? one_param(a.post_gamma, a.param_dtype, c) : 1.f, post, a.post_beta ? one_param(a.post_beta, a.param_dtype, c) * level : 0.f);
}

namespace {

// Whether a gradient hangs on the sums of ds or of du alone.
bool join_level(const JoinArgs &a) { return a.beta || a.post_beta; }

template <int X, int F, bool STRIDED, bool RMS>
lrbi_status backward_rows(const JoinCut &k, cudaStream_t s, const Join &j)
{
    if (k.each == 1) return join_launch(join_backward_kernel<X, F, STRIDED, 1, RMS, true>, k, s, j);
    return join_level(j.a) ? join_launch(join_backward_kernel<X, F, STRIDED, 2, RMS, true>, k, s, j) : join_launch(join_backward_kernel<X, F, STRIDED, 2, RMS, false>, k, s, j);
}
template <int X, int F>
lrbi_status backward_types(const JoinCut &k, bool vector, cudaStream_t s, const Join &j)
{
    if (j.a.rms) return vector ? backward_rows<X, F, false, true>(k, s, j) : backward_rows<X, F, true, true>(k, s, j);
    return vector ? backward_rows<X, F, false, false>(k, s, j) : backward_rows<X, F, true, false>(k, s, j);
}

}  // namespace

// Enough for any types and vectors.
size_t join_backward_workspace(int rows, int cols)
{
    size_t most = 16;
    for (int f : {LRBI_Y_BF16, LRBI_Y_F32})
        for (int x : {f, (int)LRBI_Y_F32})
            for (bool level : {false, true}) {
                const JoinCut k = backward_cut(rows, cols, x, f, level);
                most = std::max(most, (size_t)k.groups * 16 * k.width() * k.split);
            }
    return most;
}

lrbi_status launch_join_backward(const JoinArgs &a, float *workspace, cudaStream_t s)
{
    const JoinCut k = backward_cut(a.rows, a.cols, a.x_dtype, a.f_dtype, join_level(a));
    const bool sums = a.dgamma || a.dbeta || a.dpost_gamma || a.dpost_beta || a.dgate, vector = join_vector(a);
    const Join j = make_join(a, k, sums ? workspace : nullptr);
    if (a.rows > 0) {
        lrbi_status rc;
        if (a.x_dtype == LRBI_Y_BF16) rc = backward_types<SRC_BF16, SRC_BF16>(k, vector, s, j);
        else rc = a.f_dtype == LRBI_Y_BF16 ? backward_types<SRC_F32, SRC_BF16>(k, vector, s, j) : backward_types<SRC_F32, SRC_F32>(k, vector, s, j);
        if (rc != LRBI_OK) return rc;
    }
    if (!sums) return LRBI_OK;
    return launch_kernel(join_sums_kernel, dim3((a.cols + 31) / 32), dim3(8, 4, JOIN_SLICES), 0, s, 1, j, a.rows > 0 ? k.groups : 0, k.each == 1 || join_level(a));
}

}  // namespace lrbi
