// Layer norm, backward:  with n = (x - mean) * rstd and g = dy * gamma,
//     dx = dres + rstd * (g - mean(g) - n * mean(g * n)),   dgamma = sum over rows of dy * n,   dbeta = sum of dy;
// x as it was, or its 8-bit copy; optionally n * gamma + beta again, the forward result of that copy.
//
// A thread has the same columns in every row, so that the sums over rows stay in its registers; a group of threads has a
// whole row, and takes R rows at a time, so that the sums over columns share their shuffles and one barrier.  Rows come
// through a ring in shared memory, filled by asynchronous copies some rounds ahead, one block per SM.
// Rows go round the groups in a fixed order, a block's groups and then the blocks are summed in order: the parameters'
// gradients have the same bits in every run.
#include <algorithm>
#include <type_traits>

#include "norm_common.cuh"

namespace lrbi {

struct NormBackward {
    RowsIn dy, x, dres;    // dres.data null: nothing added; x unused when the copy is given
    KeptIn kept;
    Params p;
    const float *mean, *rstd;
    RowsOut dx, y;         // y.data null: the forward result is not restored
    int dres_dtype;
    float *part;           // [gridDim.x][2][pitch]: sums over the rows of a block
    int rows, cols, pitch; // pitch: cols rounded up to whole chunks
};

template <bool STRIDED>
__device__ __forceinline__ void add_residual(const NormBackward &a, long long row, int c, F2 (&v)[PAIRS])
{
    F2 r[PAIRS];
    if (a.dres_dtype == LRBI_Y_BF16) { Raw<SRC_BF16, STRIDED> w; w.load(a.dres, KeptIn{}, row, c, a.cols); w.get(r); }
    else { Raw<SRC_F32, STRIDED> w; w.load(a.dres, KeptIn{}, row, c, a.cols); w.get(r); }
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) v[i] = v[i] + r[i];
}

// A chunk's sums over the rows of this block: 0 of dgamma, 1 of dbeta.
template <bool STRIDED>
__device__ __forceinline__ void store_part(const NormBackward &a, int which, int c, const F2 (&v)[PAIRS])
{
    float *p = a.part + ((long long)blockIdx.x * 2 + which) * a.pitch + c;
    if constexpr (STRIDED) store_at<4, true>(reinterpret_cast<char *>(p), a.pitch - c, v);
    else if (c < a.pitch) {
        float f[CHUNK];
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) split(v[i], f[2 * i], f[2 * i + 1]);
        reinterpret_cast<float4 *>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
}

// Threads of a block: vector rows 16 warps of up to 128 registers; strided rows 20 of up to 96, without a ring to hide latency.
constexpr int BACK_THREADS = 512, BACK_THREADS_STRIDED = 640;

// blockDim = (threads of a row, rows side by side).  A thread has NV chunks of R rows at a time and keeps its columns' sums
// and their gamma in registers.  Vector rows come through a ring of STAGES rounds in shared memory, each thread copying what
// it reads itself; strided rows are loaded into registers a round ahead.
//
// Bound: memory on paper; half of the issue slots are taken (18 to 20 instructions a value, of which 7 are the sums and the
// result), and every round waits for its slowest warp once.  16384 x 4096: bf16 73 us (floor 61.5), from the 8-bit copy 80
// (51.6), with the residual and the restored forward result 116 (92.6); 8192 x 4096 fp32 66 (61.5); 8192 x 4097 bf16, where
// every access is of one value, 70 (30.8).  Addresses are one multiply-add each, and rounds that are whole check nothing.
template <int DY, int SRC, int OUT, bool STRIDED, bool EXTRA, int NV, int R>
__global__ void __launch_bounds__(STRIDED && NV == 1 ? BACK_THREADS_STRIDED : BACK_THREADS, 1) norm_backward_kernel(NormBackward a)
{
    begin();
    constexpr bool AHEAD = STRIDED && NV == 1;      // strided rows a round ahead in registers
    constexpr int STAGES = 3, WARPS = BACK_THREADS_STRIDED / 32;
    constexpr int DSIZE = DY == SRC_F32 ? 4 : 2, XSIZE = SRC == SRC_F32 ? 4 : SRC == SRC_BF16 ? 2 : 1, OSIZE = OUT == LRBI_Y_F32 ? 4 : 2;
    constexpr int DBYTES = CHUNK * DSIZE, XBYTES = CHUNK * XSIZE;     // of a chunk in the ring
    extern __shared__ float4 shared[];          // the ring: [STAGES][R][NV][dy, x][threads]
    __shared__ float part[2][2 * R * WARPS];
    const int lane = kept_lane(), warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), warps = blockDim.x >> 5;
    const int threads = blockDim.x * blockDim.y, me = threadIdx.y * blockDim.x + warp * 32 + lane, id = 1 + threadIdx.y;
    const float over = 1.f / (float)a.cols;
    const int c0 = lane_column<STRIDED>(warp * SPAN, lane), apart = warps * SPAN;
    const int left = a.cols - c0;               // columns from the thread's first one on
    const int warp_left = a.cols - warp * SPAN;  // from the warp's
    F2 dgamma[NV][PAIRS], dbeta[NV][PAIRS], gamma[NV][PAIRS];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        load_param<STRIDED>(a.p.gamma, a.p, c0 + j * apart, a.cols, 0.f, gamma[j]);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) { dgamma[j][i] = f2(0.f); dbeta[j][i] = f2(0.f); }
    }
    const char *dy0 = static_cast<const char *>(a.dy.data) + c0 * DSIZE;
    const char *x0 = SRC == SRC_KEPT ? reinterpret_cast<const char *>(a.kept.q + c0) : static_cast<const char *>(a.x.data) + c0 * XSIZE;
    char *dx0 = static_cast<char *>(a.dx.data) + c0 * OSIZE, *y0 = static_cast<char *>(a.y.data) + c0 * DSIZE;
    const char *res0 = static_cast<const char *>(a.dres.data) + c0 * OSIZE;
    const uint32_t dy_row = (uint32_t)(a.dy.stride * DSIZE), x_row = SRC == SRC_KEPT ? (uint32_t)a.kept.pitch : (uint32_t)(a.x.stride * XSIZE);
    const uint32_t dx_row = (uint32_t)(a.dx.stride * OSIZE), y_row = (uint32_t)(a.y.stride * DSIZE), res_row = (uint32_t)(a.dres.stride * OSIZE);
    const uint32_t step = gridDim.x * blockDim.y * R, rows = (uint32_t)a.rows;
    uint32_t row = (threadIdx.y * gridDim.x + blockIdx.x) * R;

    char *ring = reinterpret_cast<char *>(shared);
    const uint32_t ring0 = (uint32_t)__cvta_generic_to_shared(shared);
    const int chunk_bytes = (DBYTES + XBYTES) * threads, round_bytes = R * NV * chunk_bytes;
    auto ask = [&](uint32_t first, int at) {    // vector rows
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool there = first + r < rows;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const bool on = there && j * apart < left;
                const char *d = dy0 + (uint64_t)(first + r) * dy_row + j * apart * DSIZE, *x = x0 + (uint64_t)(first + r) * x_row + j * apart * XSIZE;
                const uint32_t to = ring0 + at * round_bytes + (r * NV + j) * chunk_bytes, to_x = to + DBYTES * threads;
                if (DSIZE == 2) copy_async_if(on, to + me * 16, d);
                if (SRC == SRC_BF16) copy_async_if(on, to_x + me * 16, x);
                if (SRC == SRC_KEPT) copy_async_if(on && (me & 1) == 0, to_x + me * 8, x);       // a vector for two threads; rows of the copy are whole vectors
                if constexpr (DSIZE == 4 || SRC == SRC_F32) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int c = warp * SPAN + j * apart + i * 128 + lane * 4;
                        const uint32_t mine = (me >> 5) * 1024 + i * 512 + fp32_copied(lane);
                        if (DSIZE == 4) copy_async_if(there && c < a.cols, to + mine, static_cast<const char *>(a.dy.data) + (uint64_t)(first + r) * dy_row + c * 4);
                        if (SRC == SRC_F32) copy_async_if(there && c < a.cols, to_x + mine, static_cast<const char *>(a.x.data) + (uint64_t)(first + r) * x_row + c * 4);
                    }
                }
            }
        }
        copies_asked();
    };
    float mean[R], rstd[R], scales[R][NV];      // of the round to come; a vector row's scales of its 8-bit copy
    auto statistics = [&](uint32_t first) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mean[r] = rstd[r] = 0.f;
            if (first + r < rows) { mean[r] = __ldg(a.mean + first + r); rstd[r] = __ldg(a.rstd + first + r); }
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (SRC == SRC_KEPT && !STRIDED)
                    scales[r][j] = first + r < rows && j * apart < left ? __ldg(a.kept.scale + (uint64_t)(first + r) * (uint32_t)a.kept.groups + (c0 + j * apart) / KEEP_GROUP) : 0.f;
        }
    };
    Raw<DY, STRIDED> raw_dy[R][NV];
    Raw<SRC, STRIDED> raw_x[R][NV];
    auto take = [&](int at) {
        if (SRC != SRC_BF16 || DSIZE == 4) __syncwarp();         // lanes read what others copied
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const char *from = ring + at * round_bytes + (r * NV + j) * chunk_bytes, *from_x = from + DBYTES * threads;
                raw_dy[r][j].clear();
                raw_x[r][j].clear();
                if (j * apart < left) {
#pragma unroll
                    for (int i = 0; i < DBYTES / 16; ++i) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(from + (DSIZE == 4 ? (me >> 5) * 1024 + fp32_read(lane, i) : me * 16));
                        uint32_t *w = raw_dy[r][j].w + (STRIDED ? 0 : 4 * i);
                        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
                    }
                    if constexpr (SRC == SRC_KEPT) {
                        const uint2 v = *reinterpret_cast<const uint2 *>(from_x + me * 8);
                        raw_x[r][j].w[0] = v.x;
                        raw_x[r][j].w[1] = v.y;
                        raw_x[r][j].scale[0] = scales[r][j];
                    } else {
#pragma unroll
                        for (int i = 0; i < XBYTES / 16; ++i) {
                            const uint4 v = *reinterpret_cast<const uint4 *>(from_x + (XSIZE == 4 ? (me >> 5) * 1024 + fp32_read(lane, i) : me * 16));
                            uint32_t *w = raw_x[r][j].w + (STRIDED ? 0 : 4 * i);
                            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
                        }
                    }
                }
            }
    };
    auto load = [&](uint32_t first) {           // strided rows
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int there = first + r < rows ? left - j * apart : 0;
                const bool whole = first + r < rows && warp_left - j * apart >= SPAN;
                raw_dy[r][j].load_at(dy0 + (uint64_t)(first + r) * dy_row + j * apart * DSIZE, there, whole);
                if constexpr (SRC == SRC_KEPT) raw_x[r][j].load(a.x, a.kept, first + r, c0 + j * apart, first + r < rows ? a.cols : 0);
                else raw_x[r][j].load_at(x0 + (uint64_t)(first + r) * x_row + j * apart * XSIZE, there, whole);
            }
    };
    int at = 0, turn = 0;
    // One round; `whole`: all R rows are there.
    auto round = [&](auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        if constexpr (!STRIDED) {
            ask(row + (STAGES - 1) * step, at == 0 ? STAGES - 1 : at - 1);      // the place that the last round was taken from
            copies_wait<STAGES - 1>();
            take(at);
            at = at + 1 == STAGES ? 0 : at + 1;
        } else if (!AHEAD) load(row);
        F2 g[R][NV][PAIRS], n[R][NV][PAIRS], scale[R];      // dy * gamma, and the normalised input
        float both[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const F2 less = f2(-mean[r]);
            scale[r] = f2(rstd[r]);
            F2 sg = f2(0.f), sgn = f2(0.f);
            if (!WHOLE && row + r >= rows) {
                both[2 * r] = both[2 * r + 1] = 0.f;
                continue;
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                F2 v[PAIRS], w[PAIRS];
                raw_dy[r][j].get(v);            // zeros past the last column, in dy and in gamma
                raw_x[r][j].get(w);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    w[i] = (w[i] + less) * scale[r];
                    dgamma[j][i] = fma2(v[i], w[i], dgamma[j][i]);
                    dbeta[j][i] = dbeta[j][i] + v[i];
                    v[i] = v[i] * gamma[j][i];
                    sg = sg + v[i];
                    sgn = fma2(v[i], w[i], sgn);
                    g[r][j][i] = v[i];
                    n[r][j][i] = w[i];
                }
            }
            both[2 * r] = sum2(sg);
            both[2 * r + 1] = sum2(sgn);
        }
        if constexpr (AHEAD) load(row + step);
        [[maybe_unused]] Raw<OUT, STRIDED> res[EXTRA && !STRIDED ? R * NV : 1];          // the residual's gradient, under way during the sums
        if constexpr (EXTRA && !STRIDED) {
            if (a.dres.data) {
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int j = 0; j < NV; ++j)
                        res[r * NV + j].load_at(res0 + (uint64_t)(row + r) * res_row + j * apart * OSIZE, WHOLE || row + r < rows ? left - j * apart : 0);
            }
        }
        statistics(row + step);                 // after a round's values are taken, within which scales are used
        row_sums<2 * R, WARPS>(both, part[turn] + threadIdx.y * warps, lane, warp, warps, id);
        turn ^= 1;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const F2 mg = f2(-both[2 * r] * over), mgn = f2(-both[2 * r + 1] * over);
            if (!WHOLE && row + r >= rows) continue;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                F2 d[PAIRS];
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) d[i] = fma2(n[r][j][i], mgn, g[r][j][i] + mg) * scale[r];
                if constexpr (EXTRA) {
                    if (a.dres.data) {
                        F2 w[PAIRS];
                        if (STRIDED) res[0].load_at(res0 + (uint64_t)(row + r) * res_row + j * apart * OSIZE, left - j * apart, warp_left - j * apart >= SPAN);
                        res[STRIDED ? 0 : r * NV + j].get(w);
#pragma unroll
                        for (int i = 0; i < PAIRS; ++i) d[i] = d[i] + w[i];
                    }
                }
                store_at<OSIZE, STRIDED>(dx0 + (uint64_t)(row + r) * dx_row + j * apart * OSIZE, left - j * apart, d, warp_left - j * apart >= SPAN);
                if constexpr (EXTRA) {
                    if (a.y.data) {
                        F2 beta[PAIRS];
                        load_param<STRIDED>(a.p.beta, a.p, c0 + j * apart, a.cols, 0.f, beta);
#pragma unroll
                        for (int i = 0; i < PAIRS; ++i) d[i] = fma2(n[r][j][i], gamma[j][i], beta[i]);
                        store_at<DSIZE, STRIDED>(y0 + (uint64_t)(row + r) * y_row + j * apart * DSIZE, left - j * apart, d, warp_left - j * apart >= SPAN);
                    }
                }
            }
        }
    };
    if constexpr (AHEAD) load(row);
    if constexpr (!STRIDED) {
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i) ask(row + i * step, i);
    }
    statistics(row);
    for (; row + R <= rows; row += step) round(std::true_type());
    let_next();
    if (R > 1 && row < rows) round(std::false_type());
    if constexpr (!STRIDED) copies_wait<0>();

    if (blockDim.y > 1) {           // rows side by side: add up their sums, in order
        __syncthreads();            // no copy of any thread is under way any more
        F2 *sums = reinterpret_cast<F2 *>(shared);     // [blockDim.y - 1][2][NV][PAIRS][blockDim.x]
        const int each = 2 * NV * PAIRS * blockDim.x;
        if (threadIdx.y > 0) {
            F2 *to = sums + (threadIdx.y - 1) * each + threadIdx.x;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    to[(j * PAIRS + i) * blockDim.x] = dgamma[j][i];
                    to[((NV + j) * PAIRS + i) * blockDim.x] = dbeta[j][i];
                }
        }
        __syncthreads();
        if (threadIdx.y > 0) return;
        for (int y = 1; y < (int)blockDim.y; ++y) {
            const F2 *from = sums + (y - 1) * each + threadIdx.x;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    dgamma[j][i] = dgamma[j][i] + from[(j * PAIRS + i) * blockDim.x];
                    dbeta[j][i] = dbeta[j][i] + from[((NV + j) * PAIRS + i) * blockDim.x];
                }
        }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        store_part<STRIDED>(a, 0, c0 + j * apart, dgamma[j]);
        store_part<STRIDED>(a, 1, c0 + j * apart, dbeta[j]);
    }
}

// Threads and shared memory of the kernel below.
template <int NV> constexpr int HELD_THREADS = NV == 2 ? 640 : 512;
template <int TYPE, bool STRIDED>
constexpr int HELD_BYTES = SPAN * (TYPE == SRC_F32 ? 4 : TYPE == SRC_BF16 ? 2 : 1) + (STRIDED && TYPE != SRC_KEPT ? 16 : 0);      // of a warp's chunk
template <int DY, int SRC, bool STRIDED>
constexpr int HELD_PLACE = HELD_BYTES<DY, STRIDED> + HELD_BYTES<SRC, STRIDED> + 16;      // of dy and x, and the two scales
template <int DY, int SRC>
constexpr int HELD_STAGES = DY == SRC_F32 || SRC == SRC_F32 ? 1 : 2;

// Rows of 8193 to 16384 columns: a thread has four chunks, whose sums over rows take half of its registers; it reads a row's
// values twice out of shared memory, where gamma is too.  A chunk's place is filled with the row after next (16 and 8 bits) or
// the next row (32 bits, which fill the memory) as soon as its second reading is through, so that copies are always under way.
// Warps have neighbouring chunks.  Strided: the 16-byte vectors of memory that hold a warp's chunk are copied, at the same
// distance from a boundary; vectors that begin before the row are not, and lanes hold the values in them until the row's turn.
// 4000 x 16384 bf16: 100 us (floor 60), with the values read twice from memory 139; 16383 columns: 176 and 374; 2000 x 16384
// fp32: 88 and 154.  What is left: with 16 warps of 128 registers, reading and unpacking each value twice.
template <int DY, int SRC, bool STRIDED, bool EXTRA, int NV>
__global__ void __launch_bounds__(HELD_THREADS<NV>, 1) norm_backward_held_kernel(NormBackward a)
{
    begin();
    constexpr int STAGES = HELD_STAGES<DY, SRC>, WARPS = HELD_THREADS<NV> / 32;
    constexpr int DSIZE = DY == SRC_F32 ? 4 : 2, XSIZE = SRC == SRC_F32 ? 4 : SRC == SRC_BF16 ? 2 : 1;
    constexpr bool SHARED = STRIDED || SRC != SRC_BF16 || DY == SRC_F32;     // lanes read what others copied
    constexpr int DBYTES = HELD_BYTES<DY, STRIDED>, XBYTES = HELD_BYTES<SRC, STRIDED>, PLACE = HELD_PLACE<DY, SRC, STRIDED>;
    extern __shared__ float4 shared[];          // gamma: [NV][2][threads]; then [STAGES][warps][NV][PLACE]
    __shared__ float part[2][2 * WARPS];
    const int lane = kept_lane(), warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), warps = blockDim.x >> 5;
    const int threads = blockDim.x, first = warp * NV * SPAN, c0 = lane_column<STRIDED>(first, lane);
    const float over = 1.f / (float)a.cols;
    F2 dgamma[NV][PAIRS], dbeta[NV][PAIRS];
    float4 *gammas = shared + warp * 32 + lane;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        F2 g[PAIRS];
        load_param<STRIDED>(a.p.gamma, a.p, c0 + j * SPAN, a.cols, 0.f, g);
        float f[CHUNK];
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            split(g[i], f[2 * i], f[2 * i + 1]);
            dgamma[j][i] = f2(0.f);
            dbeta[j][i] = f2(0.f);
        }
        gammas[2 * j * threads] = make_float4(f[0], f[1], f[2], f[3]);      // read by this thread alone
        gammas[(2 * j + 1) * threads] = make_float4(f[4], f[5], f[6], f[7]);
    }
    char *own = reinterpret_cast<char *>(shared + 2 * NV * threads) + warp * NV * PLACE;       // of this warp, in the first stage
    const uint32_t own_at = (uint32_t)__cvta_generic_to_shared(own);
    const int stage = warps * NV * PLACE;
    const uint32_t rows = (uint32_t)a.rows, step = gridDim.x;
    const char *dy_data = static_cast<const char *>(a.dy.data), *x_data = SRC == SRC_KEPT ? reinterpret_cast<const char *>(a.kept.q) : static_cast<const char *>(a.x.data);
    const uint32_t dy_row = (uint32_t)(a.dy.stride * DSIZE), x_row = SRC == SRC_KEPT ? (uint32_t)a.kept.pitch : (uint32_t)(a.x.stride * XSIZE);

    auto ask_vectors = [&](const char *p, int size, int c, uint32_t to) {      // p: the row; c: the span's first column; to: the place
#pragma unroll
        for (int i = 0; i < size / 2; ++i)
            if (c + (i * 32 + lane) * 16 / size < a.cols) copy_async(to + i * 512 + (size == 4 ? fp32_copied(lane) : lane * 16), p + c * size + i * 512 + lane * 16, 16);
    };
    // Values of a row that share their 16 bytes with what is before the row: held by the lanes of the first warp.
    uint32_t dy_edge = 0, x_edge = 0;
    auto ask_span = [&](const char *p, int size, int j, uint32_t to, uint32_t &edge) {      // p: the row; to: the place
        const int c = first + j * SPAN, bytes = min(SPAN, a.cols - c) * size;
        const char *from = p + c * size;
        const int move = (int)(reinterpret_cast<intptr_t>(from) & 15);
        from -= move;
        for (int i = lane * 16; i < move + bytes; i += 512)
            if (i > 0 || c > 0 || move == 0) copy_async_some(to + i, from + i, min(16, move + bytes - i));
        if (c == 0 && move && lane * size < min(16 - move, bytes)) edge = size == 4 ? __ldg(reinterpret_cast<const uint32_t *>(p) + lane) : (uint32_t)__ldg(reinterpret_cast<const uint16_t *>(p) + lane);
    };
    auto put_edge = [&](const char *p, int size, char *place, uint32_t edge) {
        const int move = (int)(reinterpret_cast<intptr_t>(p) & 15);
        if (move && lane * size < min(16 - move, a.cols * size)) {
            if (size == 4) *reinterpret_cast<uint32_t *>(place + move + lane * 4) = edge;
            else *reinterpret_cast<uint16_t *>(place + move + lane * 2) = (uint16_t)edge;
        }
    };
    auto put_edges = [&](uint32_t row, char *places) {
        if (row >= rows) return;
        put_edge(dy_data + (uint64_t)row * dy_row, DSIZE, places, dy_edge);
        if (SRC != SRC_KEPT) put_edge(x_data + (uint64_t)row * x_row, XSIZE, places + DBYTES, x_edge);
    };
    auto ask = [&](uint32_t row, int j, int at) {
        const int c = first + j * SPAN;
        if (STRIDED && STAGES == 2 && c == 0 && row != blockIdx.x) put_edges(row - step, own + (at ^ 1) * stage);      // those asked for last
        if (row < rows && c < a.cols) {
            const char *d = dy_data + (uint64_t)row * dy_row, *x = x_data + (uint64_t)row * x_row;
            const uint32_t to = own_at + at * stage + j * PLACE, to_x = to + DBYTES;
            if constexpr (STRIDED) ask_span(d, DSIZE, j, to, dy_edge);
            else ask_vectors(d, DSIZE, c, to);
            if constexpr (SRC == SRC_KEPT) {
                const int q = c + lane * 16;        // 16 columns a lane; rows of the copy are whole vectors
                if (lane < 16 && q < a.kept.pitch) copy_async(to_x + lane * 16, x + q, 16);
                if (lane < 2 && c + lane * KEEP_GROUP < a.cols) copy_async(to_x + XBYTES + lane * 4, a.kept.scale + (uint64_t)row * (uint32_t)a.kept.groups + c / KEEP_GROUP + lane, 4);
            } else if constexpr (STRIDED) ask_span(x, XSIZE, j, to_x, x_edge);
            else ask_vectors(x, XSIZE, c, to_x);
        }
        copies_asked();
    };
    // A chunk out of shared memory: `at` its place, `move` where its first value is (strided).
    auto chunk = [&](auto type, const char *at, int move, int left, int warp_left, F2 (&v)[PAIRS]) {
        constexpr int TYPE = decltype(type)::value;
        if constexpr (STRIDED && TYPE != SRC_KEPT) {
            constexpr int SIZE = TYPE == SRC_F32 ? 4 : 2;
            const char *p = at + move + lane * SIZE;
            float f[CHUNK];
#pragma unroll
            for (int e = 0; e < CHUNK; ++e) f[e] = SIZE == 4 ? reinterpret_cast<const float *>(p)[32 * e] : __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(p)[32 * e] << 16);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) v[i] = f2(f[2 * i], f[2 * i + 1]);
        } else if constexpr (TYPE == SRC_F32) {
            const float4 x = *reinterpret_cast<const float4 *>(at + fp32_read(lane, 0)), y = *reinterpret_cast<const float4 *>(at + fp32_read(lane, 1));
            v[0] = f2(x.x, x.y); v[1] = f2(x.z, x.w); v[2] = f2(y.x, y.y); v[3] = f2(y.z, y.w);
        } else if constexpr (TYPE == SRC_BF16) {
            const uint4 x = reinterpret_cast<const uint4 *>(at)[lane];
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) v[i] = f2(bf16_lo(w[i]), bf16_hi(w[i]));
        } else {
            const float *scale = reinterpret_cast<const float *>(at + XBYTES);
            if constexpr (STRIDED) {
                const int8_t *q = reinterpret_cast<const int8_t *>(at) + lane;
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) v[i] = f2((float)q[64 * i], (float)q[64 * i + 32]) * f2(scale[i / 2]);
            } else {
                const uint2 x = reinterpret_cast<const uint2 *>(at)[lane];
                const F2 s = f2(scale[lane >> 4]);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    const uint32_t q = (i < 2 ? x.x : x.y) >> (16 * (i & 1));
                    v[i] = f2((float)(int8_t)q, (float)(int8_t)(q >> 8)) * s;
                }
            }
        }
        if (warp_left < SPAN) {                 // zeros past the last column
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                float lo, hi;
                split(v[i], lo, hi);
                v[i] = f2(chunk_column<STRIDED>(0, 2 * i) < left ? lo : 0.f, chunk_column<STRIDED>(0, 2 * i + 1) < left ? hi : 0.f);
            }
        }
    };
    auto gamma = [&](int j, F2 (&g)[PAIRS]) {
        const float4 lo = gammas[2 * j * threads], hi = gammas[(2 * j + 1) * threads];
        g[0] = f2(lo.x, lo.y); g[1] = f2(lo.z, lo.w); g[2] = f2(hi.x, hi.y); g[3] = f2(hi.z, hi.w);
    };
    uint32_t row = blockIdx.x;
    int at = 0, turn = 0;
#pragma unroll
    for (int i = 0; i < STAGES * NV; ++i) ask(row + i / NV * step, i % NV, i / NV);
    float mean = 0.f, rstd = 0.f;
    auto statistics = [&](uint32_t r) { if (r < rows) { mean = __ldg(a.mean + r); rstd = __ldg(a.rstd + r); } };       // of the row to come
    statistics(row);
    for (; row < rows; row += step) {
        if (row + step >= rows) let_next();
        char *places = own + at * stage;
        const int dy_move = STRIDED ? (int)(reinterpret_cast<intptr_t>(dy_data + (uint64_t)row * dy_row) & 15) : 0;
        const int x_move = STRIDED ? (int)(reinterpret_cast<intptr_t>(x_data + (uint64_t)row * x_row) & 15) : 0;
        const F2 less = f2(-mean), scale = f2(rstd);
        // dy and the normalised input of chunk j
        auto values = [&](int j, F2 (&v)[PAIRS], F2 (&n)[PAIRS]) {
            const int left = a.cols - c0 - j * SPAN, warp_left = a.cols - first - j * SPAN;
            chunk(std::integral_constant<int, DY>(), places + j * PLACE, dy_move, left, warp_left, v);
            chunk(std::integral_constant<int, SRC>(), places + j * PLACE + DBYTES, x_move, left, warp_left, n);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) n[i] = (n[i] + less) * scale;
        };
        F2 sg = f2(0.f), sgn = f2(0.f);
        if (STRIDED && STAGES == 1 && warp == 0) put_edges(row, places);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (j == 0) copies_wait<STAGES * NV - 1>();
            if (j == 1) copies_wait<STAGES * NV - 2>();
            if (j == 2) copies_wait<STAGES * NV - 3>();
            if (j == 3) copies_wait<STAGES * NV - 4>();
            if (SHARED) __syncwarp();
            if (first + j * SPAN >= a.cols) continue;
            F2 v[PAIRS], n[PAIRS], g[PAIRS];
            gamma(j, g);
            values(j, v, n);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                dgamma[j][i] = fma2(v[i], n[i], dgamma[j][i]);
                dbeta[j][i] = dbeta[j][i] + v[i];
                v[i] = v[i] * g[i];
                sg = sg + v[i];
                sgn = fma2(v[i], n[i], sgn);
            }
        }
        float both[2] = {sum2(sg), sum2(sgn)};
        statistics(row + step);
        row_sums<2, WARPS>(both, part[turn], lane, warp, warps, 1);
        turn ^= 1;
        const F2 mg = f2(-both[0] * over), mgn = f2(-both[1] * over);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = c0 + j * SPAN;
            if (first + j * SPAN < a.cols) {
                F2 v[PAIRS], n[PAIRS], g[PAIRS];
                gamma(j, g);
                values(j, v, n);
                if (SHARED) __syncwarp();      // before another lane asks for the place again
                ask(row + STAGES * step, j, at);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) v[i] = fma2(n[i], mgn, fma2(v[i], g[i], mg)) * scale;
                if (EXTRA && a.dres.data) add_residual<STRIDED>(a, row, c, v);
                store_chunk<STRIDED>(a.dx, row, c, a.cols, v);
                if (EXTRA && a.y.data) {
                    F2 beta[PAIRS];
                    load_param<STRIDED>(a.p.beta, a.p, c, a.cols, 0.f, beta);
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) n[i] = fma2(n[i], g[i], beta[i]);
                    store_chunk<STRIDED>(a.y, row, c, a.cols, n);
                }
            } else copies_asked();
        }
        at = at + 1 == STAGES ? 0 : at + 1;
    }
    copies_wait<0>();
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        store_part<STRIDED>(a, 0, c0 + j * SPAN, dgamma[j]);
        store_part<STRIDED>(a, 1, c0 + j * SPAN, dbeta[j]);
    }
}

// Rows beyond the registers of a block: sums over rows in memory, a thread's own columns, read and written for every row; dy
// and x are read twice.  2000 x 20001 bf16 235 us (floor 37), 2000 x 32768 690 (60): the sums' traffic, 16 bytes a value.
template <int DY, int SRC, bool STRIDED>
__global__ void __launch_bounds__(1024) norm_backward_wide_kernel(NormBackward a)
{
    begin();
    __shared__ float part[2][2 * 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int span = warps * SPAN;
    const float over = 1.f / (float)a.cols;
    float *out = a.part + (long long)blockIdx.x * 2 * a.pitch;
    for (int k = threadIdx.x; k < 2 * a.pitch; k += blockDim.x) out[k] = 0.f;
    __syncthreads();
    int turn = 0;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const float mean = __ldg(a.mean + row), rstd = __ldg(a.rstd + row);
        Raw<DY, STRIDED> raw_dy;
        Raw<SRC, STRIDED> raw_x;
        F2 dy[PAIRS], n[PAIRS], gamma[PAIRS], sg = f2(0.f), sgn = f2(0.f);
        for (int c0 = warp * SPAN; c0 < a.cols; c0 += span) {
            const int c = lane_column<STRIDED>(c0, lane);
            raw_dy.load(a.dy, a.kept, row, c, a.cols);
            raw_x.load(a.x, a.kept, row, c, a.cols);
            load_param<STRIDED>(a.p.gamma, a.p, c, a.cols, 0.f, gamma);
            raw_dy.get(dy);
            raw_x.get(n);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) n[i] = (n[i] + f2(-mean)) * f2(rstd);
#pragma unroll
            for (int e = 0; e < CHUNK; ++e) {      // this thread's columns alone
                const int k = chunk_column<STRIDED>(c, e);
                float d[2], x[2];
                split(dy[e / 2], d[0], d[1]);
                split(n[e / 2], x[0], x[1]);
                if (k < a.cols) { out[k] = fmaf(d[e & 1], x[e & 1], out[k]); out[a.pitch + k] += d[e & 1]; }
            }
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                dy[i] = dy[i] * gamma[i];
                sg = sg + dy[i];
                sgn = fma2(dy[i], n[i], sgn);
            }
        }
        float both[2] = {sum2(sg), sum2(sgn)};
        row_sums<2, 32>(both, part[turn], lane, warp, warps, 1);
        const F2 mg = f2(-both[0] * over), mgn = f2(-both[1] * over);
        for (int c0 = warp * SPAN; c0 < a.cols; c0 += span) {
            const int c = lane_column<STRIDED>(c0, lane);
            F2 beta[PAIRS];
            raw_dy.load(a.dy, a.kept, row, c, a.cols);
            raw_x.load(a.x, a.kept, row, c, a.cols);
            load_param<STRIDED>(a.p.gamma, a.p, c, a.cols, 0.f, gamma);
            raw_dy.get(dy);
            raw_x.get(n);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                n[i] = (n[i] + f2(-mean)) * f2(rstd);
                dy[i] = fma2(n[i], mgn, fma2(dy[i], gamma[i], mg)) * f2(rstd);
            }
            if (a.dres.data) add_residual<STRIDED>(a, row, c, dy);
            store_chunk<STRIDED>(a.dx, row, c, a.cols, dy);
            if (a.y.data) {
                load_param<STRIDED>(a.p.beta, a.p, c, a.cols, 0.f, beta);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) n[i] = fma2(n[i], gamma[i], beta[i]);
                store_chunk<STRIDED>(a.y, row, c, a.cols, n);
            }
        }
    }
}

// Sums the blocks' parts in order: 32 columns a block, 32 threads along the parts of each, a thread's five loads (as many as
// 148 blocks need) all under way together: 4096 columns 0.35 us less than one after the other.
__global__ void __launch_bounds__(1024) norm_param_sum_kernel(const float *__restrict__ part, int parts, int pitch, int cols, float *dgamma, float *dbeta)
{
    begin();
    let_next();
    __shared__ float s[32][33];
    const int k = blockIdx.x * 32 + threadIdx.x;
    float v = 0.f;
    if (k < 2 * pitch)
        for (int p0 = threadIdx.y; p0 < parts; p0 += 160) {
            float w[5];
#pragma unroll
            for (int i = 0; i < 5; ++i) w[i] = p0 + 32 * i < parts ? __ldg(part + (long long)(p0 + 32 * i) * 2 * pitch + k) : 0.f;
#pragma unroll
            for (int i = 0; i < 5; ++i) v += w[i];
        }
    s[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    v = s[threadIdx.x][threadIdx.y];
#pragma unroll
    for (int j = 16; j; j >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, j);
    const int at = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0) {
        if (at < cols) { if (dgamma) dgamma[at] = v; }
        else if (at >= pitch && at < pitch + cols && dbeta) dbeta[at - pitch] = v;
    }
}

namespace {

struct Shape { int threads, side, chunks, at_a_time; };   // threads of a row, rows side by side, chunks of a thread (0: wide), R

// As few chunks a thread as 16 warps of 128 registers (20 of 96 with two chunks, or strided rows of one) have room for.
// 7000 x 9216: two chunks and 18 warps 103 us, four chunks and 9 warps 120.  Beyond 512 threads of two chunks, and from three
// on, the values stay in shared memory (norm_backward_held_kernel); strided rows of two chunks are faster out of registers:
// 8000 x 8191 bf16 152 us, through shared memory 177.
Shape backward_shape(int cols, bool strided)
{
    const int spans = (cols + SPAN - 1) / SPAN, most = BACK_THREADS / 32, most_strided = BACK_THREADS_STRIDED / 32;
    if (strided && spans <= most_strided) return {32 * spans, most_strided / spans, 1, 1};
    if (spans <= most) return {32 * spans, most / spans, 1, 2};
    if (spans <= 40) return {32 * ((spans + 1) / 2), 1, 2, 1};
    if (spans <= 48) return {32 * ((spans + 2) / 3), 1, 3, 1};
    if (spans <= 64) return {32 * ((spans + 3) / 4), 1, 4, 1};
    return {1024, 1, 0, 1};
}

// Blocks: one an SM, or fewer where that makes no round more and two thirds of the SMs keep one: there are fewer parts to
// write and to sum (1003 x 801 fp32, 101 blocks: 7.1 us, 148 7.25; 300 x 4096, where 75 would do: 8.1, 148 7.8).
int backward_grid(int rows, const Shape &s)
{
    const long long rounds = ((long long)rows + s.at_a_time - 1) / s.at_a_time, most = (rounds + NORM_SMS * s.side - 1) / (NORM_SMS * s.side);
    const long long fewer = most > 0 ? (rounds + most * s.side - 1) / (most * s.side) : 1;
    return (int)(fewer * 3 >= NORM_SMS * 2 ? fewer : std::max(1LL, std::min((long long)NORM_SMS, rounds)));
}
int backward_pitch(int cols) { return (cols + CHUNK - 1) / CHUNK * CHUNK; }

template <int DY, int SRC, int OUT, bool STRIDED, int NV, int R>
lrbi_status ring_launch(const NormBackward &a, const Shape &sh, int grid, cudaStream_t s)
{
    constexpr int bytes = CHUNK * ((DY == SRC_F32 ? 4 : 2) + (SRC == SRC_KEPT ? 1 : SRC == SRC_F32 ? 4 : 2));
    const size_t ring = STRIDED ? 0 : (size_t)3 * R * NV * bytes * sh.threads * sh.side, sums = (size_t)(sh.side - 1) * 2 * NV * CHUNK * 4 * sh.threads;
    const dim3 block(sh.threads, sh.side);
    if (a.dres.data || a.y.data) return norm_launch(norm_backward_kernel<DY, SRC, OUT, STRIDED, true, NV, R>, grid, block, std::max(ring, sums), s, a);
    return norm_launch(norm_backward_kernel<DY, SRC, OUT, STRIDED, false, NV, R>, grid, block, std::max(ring, sums), s, a);
}

template <int DY, int SRC, bool STRIDED, int NV>
lrbi_status held_launch(const NormBackward &a, const Shape &sh, int grid, cudaStream_t s)
{
    const size_t smem = (size_t)sh.threads * NV * 32 + (size_t)sh.threads / 32 * NV * HELD_STAGES<DY, SRC> * HELD_PLACE<DY, SRC, STRIDED>;
    if (a.dres.data || a.y.data) return norm_launch(norm_backward_held_kernel<DY, SRC, STRIDED, true, NV>, grid, dim3(sh.threads), smem, s, a);
    return norm_launch(norm_backward_held_kernel<DY, SRC, STRIDED, false, NV>, grid, dim3(sh.threads), smem, s, a);
}

template <int DY, int SRC, bool STRIDED>
lrbi_status backward_launch(const NormBackward &a, const Shape &sh, int grid, cudaStream_t s)
{
    const bool f32 = a.dx.dtype == LRBI_Y_F32;
    if (sh.chunks == 1) return f32 ? ring_launch<DY, SRC, LRBI_Y_F32, STRIDED, 1, STRIDED ? 1 : 2>(a, sh, grid, s) : ring_launch<DY, SRC, LRBI_Y_BF16, STRIDED, 1, STRIDED ? 1 : 2>(a, sh, grid, s);
    if (sh.chunks == 2 && sh.threads > BACK_THREADS) return held_launch<DY, SRC, STRIDED, 2>(a, sh, grid, s);
    if (sh.chunks == 3) return held_launch<DY, SRC, STRIDED, 3>(a, sh, grid, s);
    if (sh.chunks == 2) return f32 ? ring_launch<DY, SRC, LRBI_Y_F32, STRIDED, 2, 1>(a, sh, grid, s) : ring_launch<DY, SRC, LRBI_Y_BF16, STRIDED, 2, 1>(a, sh, grid, s);
    if (sh.chunks == 4) return held_launch<DY, SRC, STRIDED, 4>(a, sh, grid, s);
    return norm_launch(norm_backward_wide_kernel<DY, SRC, STRIDED>, grid, dim3(1024), 0, s, a);
}

}  // namespace

size_t norm_backward_workspace(int rows, int cols)      // for either way of taking the rows
{
    return (size_t)std::max(backward_grid(rows, backward_shape(cols, false)), backward_grid(rows, backward_shape(cols, true))) * 2 * backward_pitch(cols) * 4;
}

lrbi_status launch_layer_norm_backward(const NormArgs &n, float *workspace, cudaStream_t s)
{
    const int pitch = backward_pitch(n.cols);
    const NormBackward a = {{n.dy, n.dy_stride}, {n.x, n.x_stride}, {n.dres, n.dres_stride}, {n.q, n.scale, checkpoint_pitch(n.cols), checkpoint_groups(n.cols)},
                            make_params(n), n.mean, n.rstd, {n.dx, n.dx_stride, n.dx_dtype}, {n.y, n.y_stride, n.dy_dtype},
                            n.dx_dtype, workspace, n.rows, n.cols, pitch};
    const bool strided = n.cols % CHUNK != 0 || !vector_rows(n.dy, n.dy_stride, n.dy_dtype) || (!n.q && !vector_rows(n.x, n.x_stride, n.x_dtype)) ||
                       (n.dres && !vector_rows(n.dres, n.dres_stride, n.dx_dtype)) || !vector_rows(n.dx, n.dx_stride, n.dx_dtype) ||
                       (n.y && !vector_rows(n.y, n.y_stride, n.dy_dtype));
    const Shape sh = backward_shape(n.cols, strided);
    const int grid = backward_grid(n.rows, sh), src = n.q ? SRC_KEPT : n.x_dtype;
    lrbi_status st;
#define BACKWARD(DY, SRC) st = strided ? backward_launch<DY, SRC, true>(a, sh, grid, s) : backward_launch<DY, SRC, false>(a, sh, grid, s)
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
    if (st != LRBI_OK || (!n.dgamma && !n.dbeta)) return st;
    return launch_kernel(norm_param_sum_kernel, dim3((2 * pitch + 31) / 32), dim3(32, 32), 0, s, 1, (const float *)workspace, grid, pitch, n.cols, n.dgamma, n.dbeta);
}

}  // namespace lrbi
