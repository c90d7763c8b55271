// Between two blocks, forward and backward: the norm behind a block, its gate and the residual scale, and the norm before the
// next block, in one pass.
//
//   z = norm(f) * post_gamma + post_beta           out = residual_scale * x + gate * z           u = norm(out) * gamma + beta
//
// (norm: about the mean, or of the root mean square alone.)  With n = (out - mean) rstd, g = du gamma, nf = (f - mean_f) rstd_f and
// w = gate post_gamma the backward pass is
//
//   ds = dout + rstd (g - mean(g) - n mean(g n)),   dx = residual_scale ds,   df = rstd_f (w ds - mean(w ds) - nf mean(w ds nf))
//   dgamma = sum du n, dbeta = sum du, and from A = sum ds nf, B = sum ds over the rows:
//   dpost_gamma = gate A,  dpost_beta = gate B,  dgate = post_gamma A + post_beta B
//
// so a gate that is the same for all rows costs no sum of its own.  The two means of df hang on those of ds, but only linearly:
// with p = dout + rstd g, ds = p - rstd (mean(g) + n mean(g n)), and mean(w ds), mean(w ds nf) follow from the sums of g, g n, w p,
// w n, w nf p, w nf and w nf n, which are taken together: the threads of a row meet once.
#include <algorithm>

#include "norm_common.cuh"

namespace lrbi {

constexpr int JOIN_THREADS = 512, JOIN_WARPS = JOIN_THREADS / 32;      // of a block
constexpr int JOIN_COLS = JOIN_THREADS * CHUNK;                         // columns that a block takes of a row: a chunk a thread
constexpr int JOIN_SPLIT = LRBI_MAX_RESIDUAL_COLS / JOIN_COLS;          // blocks of a cluster that share a row, at most
static_assert(JOIN_SPLIT <= 8, "larger clusters are not portable");

struct Join {
    JoinArgs a;
    bool whole;                // the vectors start on 16-byte boundaries
    int split;                 // blocks that share a row
    float *parts;              // backward: [groups][4][cols]
};

__device__ __forceinline__ uint32_t join_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void join_store(const float *mine, uint32_t rank, float v)     // to the same place in another block of the cluster
{
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there), "f"(v) : "memory");
}

constexpr int JOIN_ENTRIES = JOIN_WARPS * JOIN_SPLIT;      // warps that may share a row

// A bit for each column of a chunk that is there.
template <bool STRIDED> __device__ __forceinline__ uint32_t columns_there(int c, int cols)
{
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < CHUNK; ++e) m |= (uint32_t)(chunk_column<STRIDED>(c, e) < cols) << e;
    return m;
}
__device__ __forceinline__ void keep_there(F2 (&v)[PAIRS], uint32_t there)      // zeros elsewhere
{
    if (there == 0xFFu) return;
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
        float a, b;
        split(v[i], a, b);
        v[i] = f2(there >> (2 * i) & 1 ? a : 0.f, there >> (2 * i + 1) & 1 ? b : 0.f);
    }
}

// The threads that share a row: `warps` warps of this block, or of each of `split` blocks of a cluster.
struct Team {
    int lane, warp, warps, id, split, rank;
    int first;         // of its entries: a place for each warp that shares the row
    int phase;         // entries are there twice, so that a team meets once for each sum

    __device__ __forceinline__ Team(int split_)
    {
        lane = kept_lane();
        warp = threadIdx.x >> 5;
        warps = blockDim.x >> 5;
        id = 1 + threadIdx.y;
        split = split_;
        rank = split > 1 ? join_rank() : 0;
        first = threadIdx.y * warps;
        phase = 0;
    }
    __device__ __forceinline__ bool alone() const { return warps * split == 1; }
    __device__ __forceinline__ int entries() const { return warps * split; }
    __device__ __forceinline__ int entry() const { return rank * warps + warp; }       // in the order of the row's columns
    // Waits until all of them are here; what they wrote before is seen after.
    __device__ __forceinline__ void meet() const
    {
        if (split > 1) {
            __syncwarp();
            asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        } else row_barrier(id, warps * 32);
    }
    // Puts a value where every block of the team finds it; by one lane.
    __device__ __forceinline__ void tell(float *at, float v) const
    {
        if (split > 1) for (int r = 0; r < split; ++r) join_store(at, r, v);
        else *at = v;
    }
    template <int N> __device__ __forceinline__ float *board(float (&part)[2][JOIN_ENTRIES][N])
    {
        float *p = part[phase][first];
        phase ^= 1;
        return p;
    }
};

// Mean and 1 / root over a row of the values v (zeros where there is no column).  Squares are summed about the warp's own mean
// and joined by Chan's rule: no cancellation however far the values are from zero.  n: columns that the warp has.
__device__ __forceinline__ void row_statistics(const F2 (&v)[PAIRS], uint32_t there, int n, const JoinArgs &a, Team &t, float (&part)[2][JOIN_ENTRIES][2], float &mean, float &rstd)
{
    F2 s = f2(0.f);
    if (a.rms) {
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) s = fma2(v[i], v[i], s);
        float square = warp_sum(sum2(s));
        if (!t.alone()) {
            float *all = t.board(part);
            if (t.lane == 0) t.tell(all + t.entry() * 2, square);
            t.meet();
            square = 0.f;
            for (int e = t.lane; e < t.entries(); e += 32) square += all[2 * e];
            square = warp_sum(square);
        }
        mean = 0.f;
        rstd = inverse_root(square / (float)a.cols + a.eps);
        return;
    }
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) s = s + v[i];
    const float own = warp_sum(sum2(s)), own_mean = n > 0 ? own / (float)n : 0.f;
    F2 d[PAIRS], q = f2(0.f);
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) d[i] = v[i] + f2(-own_mean);
    keep_there(d, there);
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) q = fma2(d[i], d[i], q);
    float square = warp_sum(sum2(q));
    mean = own_mean;
    if (!t.alone()) {
        float *all = t.board(part);
        if (t.lane == 0) {
            t.tell(all + t.entry() * 2, own);
            t.tell(all + t.entry() * 2 + 1, square);
        }
        t.meet();
        float sum = 0.f;
        for (int e = t.lane; e < t.entries(); e += 32) sum += all[2 * e];
        mean = warp_sum(sum) / (float)a.cols;
        square = 0.f;
        for (int e = t.lane; e < t.entries(); e += 32) {
            const float count = (float)min(SPAN, a.cols - e * SPAN);      // of the entry's columns
            if (count > 0.f) {
                const float off = all[2 * e] / count - mean;
                square += fmaf(off * off, count, all[2 * e + 1]);
            }
        }
        square = warp_sum(square);
    }
    rstd = inverse_root(square / (float)a.cols + a.eps);
}

template <int TYPE> __device__ __forceinline__ char *chunk_at(const void *p, long long stride, long long row, int c)
{
    return static_cast<char *>(const_cast<void *>(p)) + (row * stride + c) * (TYPE == SRC_F32 ? 4 : 2);
}
template <int TYPE, bool STRIDED> __device__ __forceinline__ void read_chunk(const void *p, long long stride, long long row, int c, int cols, F2 (&v)[PAIRS])
{
    Raw<TYPE, STRIDED> raw;
    raw.clear();
    if (c < cols) raw.load_at(chunk_at<TYPE>(p, stride, row, c), cols - c);
    raw.get(v);
}
template <int TYPE, bool STRIDED> __device__ __forceinline__ void write_chunk(void *p, long long stride, long long row, int c, int cols, const F2 (&v)[PAIRS])
{
    store_at<TYPE == SRC_F32 ? 4 : 2, STRIDED>(chunk_at<TYPE>(p, stride, row, c), cols - c, v);
}

// blockDim = (threads of a row, rows of a block); clusters of `split` blocks share a row.
template <int X, int F, bool STRIDED>
__global__ void __launch_bounds__(JOIN_THREADS) join_forward_kernel(Join j)
{
    begin();
    const JoinArgs &a = j.a;
    __shared__ float part[2][JOIN_ENTRIES][2];
    Team t(j.split);
    const int c0 = t.entry() * SPAN, c = lane_column<STRIDED>(c0, t.lane), n = min(SPAN, max(0, a.cols - c0));
    const uint32_t there = columns_there<STRIDED>(c, a.cols);
    const Params p = {nullptr, nullptr, a.param_dtype, j.whole};
    const bool tells = a.stats && t.entry() == 0 && t.lane == 0;
    if (j.split > 1) t.meet();       // blocks write to one another once all of them have begun
    const long long step = (long long)(gridDim.x / j.split) * blockDim.y;
    for (long long row = (long long)(blockIdx.x / j.split) * blockDim.y + threadIdx.y; row < a.rows; row += step) {
        F2 z[PAIRS], v[PAIRS], w[PAIRS];
        read_chunk<F, STRIDED>(a.f, a.f_stride, row, c, a.cols, z);
        read_chunk<X, STRIDED>(a.x, a.x_stride, row, c, a.cols, v);
        float mean = 0.f, rstd = 1.f;
        if (a.post_gamma) {
            row_statistics(z, there, n, a, t, part, mean, rstd);
            load_param<STRIDED>(a.post_gamma, p, c, a.cols, 0.f, w);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) z[i] = (z[i] + f2(-mean)) * f2(rstd) * w[i];
            if (a.post_beta) {
                load_param<STRIDED>(a.post_beta, p, c, a.cols, 0.f, w);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) z[i] = z[i] + w[i];
            }
        }
        if (tells) { a.stats[2ll * a.rows + row] = mean; a.stats[3ll * a.rows + row] = rstd; }
        if (a.gate) {
            load_param<STRIDED>(a.gate, p, c, a.cols, 0.f, w);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) z[i] = z[i] * w[i];
        }
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) v[i] = fma2(v[i], f2(a.residual_scale), z[i]);
        if (X == SRC_BF16) {           // the stream as it is stored is what goes on
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                float lo, hi;
                split(v[i], lo, hi);
                const uint32_t r = pack_bf16(lo, hi);
                v[i] = f2(bf16_lo(r), bf16_hi(r));
            }
        }
        write_chunk<X, STRIDED>(a.out, a.out_stride, row, c, a.cols, v);
        mean = 0.f;
        rstd = 1.f;
        if (a.gamma) {
            keep_there(v, there);
            row_statistics(v, there, n, a, t, part, mean, rstd);
            load_param<STRIDED>(a.gamma, p, c, a.cols, 0.f, w);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) v[i] = (v[i] + f2(-mean)) * f2(rstd) * w[i];
            if (a.beta) {
                load_param<STRIDED>(a.beta, p, c, a.cols, 0.f, w);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) v[i] = v[i] + w[i];
            }
        }
        if (tells) { a.stats[row] = mean; a.stats[a.rows + row] = rstd; }
        if (a.u) write_chunk<F, STRIDED>(a.u, a.u_stride, row, c, a.cols, v);
        if (a.q) {
            keep_there(v, there);
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                float lo, hi;
                split(v[i], lo, hi);
                top = max(top, max(__float_as_uint(lo) & 0x7FFFFFFFu, __float_as_uint(hi) & 0x7FFFFFFFu));
            }
            top = __reduce_max_sync(0xFFFFFFFFu, top);
            if (!t.alone()) {
                float *all = t.board(part);
                if (t.lane == 0) t.tell(all + t.entry() * 2, __uint_as_float(top));
                t.meet();
                top = 0;
                for (int e = t.lane; e < t.entries(); e += 32) top = max(top, __float_as_uint(all[2 * e]));
                top = __reduce_max_sync(0xFFFFFFFFu, top);
            }
            const TokenScale s(top);
            if (t.entry() == 0 && t.lane == 0) a.q_scale[row] = s.scale();
            const int pitch = (a.cols + 15) / 16 * 16;
            store_i8<STRIDED>(a.q + row * pitch + c, pitch - c, v, s.factor, s.fine);
        }
    }
    let_next();
    if (j.split > 1) t.meet();       // a block stays while others may still write to it
}

// The sums over a row of N = 8 values a thread, in every thread: within a warp they are folded into one another (norm_common.cuh).
__device__ __forceinline__ void row_eight(float (&v)[8], Team &t, float (&part)[2][JOIN_ENTRIES][8])
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
        float *all = t.board(part);
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

__device__ __forceinline__ float dot(const F2 (&a)[PAIRS], const F2 (&b)[PAIRS])
{
    F2 s = a[0] * b[0];
#pragma unroll
    for (int i = 1; i < PAIRS; ++i) s = fma2(a[i], b[i], s);
    return sum2(s);
}
__device__ __forceinline__ float total(const F2 (&a)[PAIRS]) { return sum2((a[0] + a[1]) + (a[2] + a[3])); }

// As the forward kernel.  A thread keeps the four sums over rows of its columns; the rows of a block are added up at the end.
template <int X, int F, bool STRIDED>
__global__ void __launch_bounds__(JOIN_THREADS, 1) join_backward_kernel(Join j)
{
    begin();
    const JoinArgs &a = j.a;
    extern __shared__ float columns[];       // blocks of several rows: [4][columns]
    __shared__ float part[2][JOIN_ENTRIES][8];
    Team t(j.split);
    const int c0 = t.entry() * SPAN, c = lane_column<STRIDED>(c0, t.lane);
    const Params p = {nullptr, nullptr, a.param_dtype, j.whole};
    const bool post = a.post_gamma, pre = a.gamma;
    const float per = 1.f / (float)a.cols;
    F2 sums[4][PAIRS];       // ds nf, ds, du n, du
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) sums[k][i] = f2(0.f);
    F2 gamma[PAIRS], w[PAIRS];
    load_param<STRIDED>(a.gamma, p, c, a.cols, 0.f, gamma);
    load_param<STRIDED>(a.gate, p, c, a.cols, a.gate ? 0.f : 1.f, w);
    if (post) {
        F2 g[PAIRS];
        load_param<STRIDED>(a.post_gamma, p, c, a.cols, 0.f, g);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) w[i] = w[i] * g[i];
    }
    keep_there(w, columns_there<STRIDED>(c, a.cols));
    const float total_w = total(w);
    if (j.split > 1) t.meet();       // blocks write to one another once all of them have begun
    const long long step = (long long)(gridDim.x / j.split) * blockDim.y;
    for (long long row = (long long)(blockIdx.x / j.split) * blockDim.y + threadIdx.y; row < a.rows; row += step) {
        F2 ds[PAIRS], n[PAIRS], nf[PAIRS], g[PAIRS];
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, total_w};
        float mean = 0.f, rstd = 0.f, f_mean = 0.f, f_rstd = 1.f;
        if (post) { f_mean = __ldg(a.stats + 2ll * a.rows + row); f_rstd = __ldg(a.stats + 3ll * a.rows + row); }
        if (a.dout) read_chunk<X, STRIDED>(a.dout, a.dout_stride, row, c, a.cols, ds);
        else
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) ds[i] = f2(0.f);
        read_chunk<F, STRIDED>(a.f, a.f_stride, row, c, a.cols, nf);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) nf[i] = (nf[i] + f2(-f_mean)) * f2(f_rstd);
        if (pre) {
            mean = __ldg(a.stats + row);
            rstd = __ldg(a.stats + a.rows + row);
            read_chunk<F, STRIDED>(a.du, a.du_stride, row, c, a.cols, g);
            read_chunk<X, STRIDED>(a.out, a.out_stride, row, c, a.cols, n);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                n[i] = (n[i] + f2(-mean)) * f2(rstd);
                sums[2][i] = fma2(g[i], n[i], sums[2][i]);
                sums[3][i] = sums[3][i] + g[i];
                g[i] = g[i] * gamma[i];
                ds[i] = fma2(g[i], f2(rstd), ds[i]);       // p
            }
            v[0] = total(g);
            v[1] = dot(g, n);
        }
        if (post) {
            F2 wnf[PAIRS];
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) wnf[i] = w[i] * nf[i];
            v[2] = dot(w, ds);
            v[4] = dot(wnf, ds);
            v[5] = total(wnf);
            if (pre) { v[3] = dot(w, n); v[6] = dot(wnf, n); }
        }
        if (pre || post) row_eight(v, t, part);
        if (pre) {
            const float flat = a.rms ? 0.f : v[0] * per * rstd, along = v[1] * per * rstd;
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) ds[i] = fma2(n[i], f2(-along), ds[i] + f2(-flat));
            v[2] = v[2] - flat * v[7] - along * v[3];          // sums of w ds and of w ds nf
            v[4] = v[4] - flat * v[5] - along * v[6];
        }
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            sums[0][i] = fma2(ds[i], nf[i], sums[0][i]);
            sums[1][i] = sums[1][i] + ds[i];
            n[i] = ds[i] * f2(a.residual_scale);
        }
        write_chunk<X, STRIDED>(a.dx, a.dx_stride, row, c, a.cols, n);
        const float f_flat = a.rms ? 0.f : v[2] * per, f_along = v[4] * per;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            n[i] = ds[i] * w[i];
            if (post) n[i] = fma2(nf[i], f2(-f_along), n[i] + f2(-f_flat)) * f2(f_rstd);
        }
        write_chunk<F, STRIDED>(a.df, a.df_stride, row, c, a.cols, n);
    }
    if (j.parts) {
        // one after the other, so that the sums have the same bits every time
        const int width = t.warps * SPAN, own = lane_column<STRIDED>(t.warp * SPAN, t.lane);
        for (int k = 0; k < (int)blockDim.y; ++k) {
            if ((int)threadIdx.y == k) {
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) {
                        float lo, hi;
                        split(sums[s][i], lo, hi);
                        float *at = columns + s * width + chunk_column<STRIDED>(own, 2 * i), *next = columns + s * width + chunk_column<STRIDED>(own, 2 * i + 1);
                        *at = k ? *at + lo : lo;
                        *next = k ? *next + hi : hi;
                    }
            }
            __syncthreads();
        }
        const int base = t.rank * width, end = min(width, a.cols - base);
        float *to = j.parts + (long long)(blockIdx.x / j.split) * 4 * a.cols + base;
        for (int k = threadIdx.y * blockDim.x + threadIdx.x; k < end; k += blockDim.x * blockDim.y)
#pragma unroll
            for (int s = 0; s < 4; ++s) to[(long long)s * a.cols + k] = columns[s * width + k];
    }
    let_next();
    if (j.split > 1) t.meet();       // a block stays while others may still write to it
}

// Adds the blocks' parts up: block (32 columns, 16 slices of the parts).
constexpr int JOIN_SLICES = 16;
__global__ void __launch_bounds__(32 * JOIN_SLICES) join_sums_kernel(Join j, int groups)
{
    begin();
    const JoinArgs &a = j.a;
    __shared__ float part[JOIN_SLICES][4][32];
    const int c = blockIdx.x * 32 + threadIdx.x;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < a.cols)
        for (int g = threadIdx.y; g < groups; g += JOIN_SLICES)
#pragma unroll
            for (int k = 0; k < 4; ++k) s[k] += j.parts[((long long)g * 4 + k) * a.cols + c];
    let_next();
#pragma unroll
    for (int k = 0; k < 4; ++k) part[threadIdx.y][k][threadIdx.x] = s[k];
    __syncthreads();
    if (threadIdx.y || c >= a.cols) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        s[k] = 0.f;
#pragma unroll
        for (int y = 0; y < JOIN_SLICES; ++y) s[k] += part[y][k][threadIdx.x];
    }
    const float gate = a.gate ? one_param(a.gate, a.param_dtype, c) : 1.f;
    if (a.dgamma) a.dgamma[c] = s[2];
    if (a.dbeta) a.dbeta[c] = s[3];
    if (a.dpost_gamma) a.dpost_gamma[c] = gate * s[0];
    if (a.dpost_beta) a.dpost_beta[c] = gate * s[1];
    if (a.dgate) a.dgate[c] = fmaf(a.post_gamma ? one_param(a.post_gamma, a.param_dtype, c) : 1.f, s[0], a.post_beta ? one_param(a.post_beta, a.param_dtype, c) * s[1] : 0.f);
}

namespace {

// How rows are dealt out: threads of a row, rows of a block, blocks that share a row, groups of blocks.
struct JoinCut { int threads, teams, split, groups; };
JoinCut join_cut(int rows, int cols, int blocks)
{
    JoinCut k;
    const int spans = (cols + SPAN - 1) / SPAN;
    k.split = 1;
    while (k.split * JOIN_WARPS < spans) k.split *= 2;
    k.threads = 32 * ((spans + k.split - 1) / k.split);
    k.teams = k.split > 1 ? 1 : JOIN_THREADS / k.threads;
    k.groups = std::min((rows + k.teams - 1) / k.teams, std::max(1, blocks / k.split));
    return k;
}

template <class Kernel>
lrbi_status join_launch(Kernel kernel, const JoinCut &k, size_t smem, cudaStream_t s, const Join &j)
{
    return launch_kernel(kernel, dim3(k.groups * k.split), dim3(k.threads, k.teams), smem, s, k.split, j);
}

#define JOIN_TYPES(launch, kernel, ...)                                                                                                        \
    if (a.x_dtype == LRBI_Y_BF16) return vector ? launch(kernel<SRC_BF16, SRC_BF16, false>, __VA_ARGS__) : launch(kernel<SRC_BF16, SRC_BF16, true>, __VA_ARGS__);   \
    if (a.f_dtype == LRBI_Y_BF16) return vector ? launch(kernel<SRC_F32, SRC_BF16, false>, __VA_ARGS__) : launch(kernel<SRC_F32, SRC_BF16, true>, __VA_ARGS__);     \
    return vector ? launch(kernel<SRC_F32, SRC_F32, false>, __VA_ARGS__) : launch(kernel<SRC_F32, SRC_F32, true>, __VA_ARGS__)

bool join_vector(const JoinArgs &a)
{
    auto rows = [&](const void *p, long long stride, int dtype) { return !p || vector_rows(p, stride, dtype); };
    return a.cols % CHUNK == 0 && rows(a.x, a.x_stride, a.x_dtype) && rows(a.f, a.f_stride, a.f_dtype) && rows(a.out, a.out_stride, a.x_dtype) &&
           rows(a.u, a.u_stride, a.f_dtype) && rows(a.du, a.du_stride, a.f_dtype) && rows(a.dout, a.dout_stride, a.x_dtype) &&
           rows(a.dx, a.dx_stride, a.x_dtype) && rows(a.df, a.df_stride, a.f_dtype);
}

Join make_join(const JoinArgs &a, int split, float *parts)
{
    uintptr_t all = 0;
    for (const void *p : {a.gamma, a.beta, a.post_gamma, a.post_beta, a.gate}) all |= reinterpret_cast<uintptr_t>(p);
    return {a, (all & 15u) == 0, split, parts};
}

lrbi_status forward_rows(const JoinArgs &a, const JoinCut &k, cudaStream_t s)
{
    const Join j = make_join(a, k.split, nullptr);
    const bool vector = join_vector(a);
    JOIN_TYPES(join_launch, join_forward_kernel, k, 0, s, j);
}

lrbi_status backward_rows(const JoinArgs &a, const Join &j, const JoinCut &k, cudaStream_t s)
{
    const bool vector = join_vector(a);
    const size_t smem = j.parts ? (size_t)4 * 4 * (k.threads * CHUNK) : 0;
    JOIN_TYPES(join_launch, join_backward_kernel, k, smem, s, j);
}

}  // namespace

size_t join_backward_workspace(int rows, int cols)
{
    return std::max<size_t>(16, (size_t)join_cut(rows, cols, NORM_SMS).groups * 16 * cols);
}

lrbi_status launch_join(const JoinArgs &a, cudaStream_t s)
{
    return forward_rows(a, join_cut(a.rows, a.cols, 2 * NORM_SMS), s);
}

lrbi_status launch_join_backward(const JoinArgs &a, float *workspace, cudaStream_t s)
{
    const JoinCut k = join_cut(a.rows, a.cols, NORM_SMS);
    const bool sums = a.dgamma || a.dbeta || a.dpost_gamma || a.dpost_beta || a.dgate;
    const Join j = make_join(a, k.split, sums ? workspace : nullptr);
    if (a.rows > 0) {
        const lrbi_status rc = backward_rows(a, j, k, s);
        if (rc != LRBI_OK) return rc;
    }
    if (!sums) return LRBI_OK;
    return launch_kernel(join_sums_kernel, dim3((a.cols + 31) / 32), dim3(32, JOIN_SLICES), 0, s, 1, j, a.rows > 0 ? k.groups : 0);
}

}  // namespace lrbi
