// Layer norm over the columns of each row:  y = (x - mean) * rstd * gamma + beta, statistics in fp32, optionally an 8-bit
// copy of x on the way.
//
// Memory is read once and written once: a row's values stay in registers, as they were loaded, between the two sums and the
// result (the sum of squares is taken about the mean, from registers: no cancellation).  What bounds it then is the number
// of instructions per value as much as memory, which is why a lane holds as much of a row as it can:
//
//   tall  many rows.  A warp has a row, or `warps` of them share one; a lane holds up to 16 chunks (bf16; 8 in fp32), the
//         sums' shuffles are paid once per row, gamma and beta come from shared memory without bank conflicts, and warps
//         run apart from one another, so that loads, arithmetic and stores of different rows overlap.
//   row   few rows: latency counts, a block has a row, a lane one or two chunks.
//   wide  rows beyond the registers of a block: read three times, mostly from L2.  2000 x 32768 bf16 111 us (floor 40).
//
// Bound, tall: memory and issue about alike (12 instructions a value in bf16).  16384 x 4096 bf16 47.5 us (floor 41), with the
// copy 61 (51.6); 4096 x 4096 14.9 (10.3): three rounds of rows and 4 us to begin and to drain; 8192 x 4096 fp32 51 (41); 8192 x
// 4097 bf16, an access a value, 47.6 (20.5).  row: 2.3 us for one token of 4096, which is the launch, two waits for memory and
// two sums over a block.
#include <algorithm>

#include "norm_common.cuh"

namespace lrbi {

// How bf16 values are unpacked: by 16 bits and a mask of the upper half.  Each use in a kernel has its own copy, which the
// compiler takes for another one, and so unpacks the words anew: kept from one use to the next the values would take twice
// the registers of the words (and were spilled).
struct Unpack { uint32_t shift, mask; };      // 16, 0xFFFF0000

struct NormForward {
    RowsIn x;
    Params p;
    RowsOut y;
    KeptOut kept;          // q null: no copy
    float *mean, *rstd;    // both or neither
    float eps;
    int rows, cols;
    int warps, each;       // tall: warps that share a row, chunks of each
    Unpack use[4];
};

// The chunks of a lane of one row (or of the part of a row that a warp has: columns first .. end), chunk j in the span at
// first + j * SPAN.
template <int SRC, bool STRIDED, int K>
struct Part {
    static constexpr int SIZE = SRC == SRC_F32 ? 4 : 2;
    Raw<STRIDED ? SRC_F32 : SRC, STRIDED> chunk[K];      // strided: unpacked as they come from shared memory

    // Strided: element by element from shared memory, at: the lane's first column.  Spans that are whole are not checked.
    __device__ __forceinline__ void load(const char *at, int c, int first, int end)
    {
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const char *p = at + j * SPAN * SIZE;
            if (first + (j + 1) * SPAN <= end) {         // the whole warp
#pragma unroll
                for (int e = 0; e < CHUNK; ++e) chunk[j].w[e] = SIZE == 4 ? reinterpret_cast<const uint32_t *>(p)[32 * e] : (uint32_t)reinterpret_cast<const uint16_t *>(p)[32 * e] << 16;
            } else {
                const int left = end - c - j * SPAN;
#pragma unroll
                for (int e = 0; e < CHUNK; ++e) {
                    uint32_t v = 0;
                    if (32 * e < left) v = SIZE == 4 ? reinterpret_cast<const uint32_t *>(p)[32 * e] : (uint32_t)reinterpret_cast<const uint16_t *>(p)[32 * e] << 16;
                    chunk[j].w[e] = v;
                }
            }
        }
    }
    __device__ __forceinline__ void put(int j, int i, const uint4 &v) { uint32_t *w = chunk[j].w + 4 * i; w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
    __device__ __forceinline__ void get(int j, const Unpack &u, F2 (&v)[PAIRS]) const
    {
        const uint32_t *w = chunk[j].w;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            if constexpr (SIZE == 4 || STRIDED) v[i] = f2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
            else v[i] = f2(__uint_as_float(w[i] << u.shift), __uint_as_float(w[i] & u.mask));
        }
    }
};

// Warps of a block, and blocks of an SM: as many registers as K chunks need.  One block where the parameters are large: they
// are brought in once an SM (4096 x 4096 bf16: 24 warps 14.9 us, two blocks of 12 15.8; 900 rows: 6.7 and 8.2).
template <int SRC, bool STRIDED, int K>
struct Tall {
    static constexpr int WORDS = K * Raw<SRC, STRIDED>::WORDS;    // registers that hold a row's part
    static constexpr int WARPS = WORDS >= 64 ? 16 : WORDS >= 32 ? 24 : 16, BLOCKS = WORDS >= 32 ? 1 : 2;
};

// blockDim = (32, warps of a row, rows of a block).  The next row (whole vectors) is copied to shared memory meanwhile.
template <int SRC, int OUT, bool STRIDED, bool COPY, int K>
__global__ void __launch_bounds__(32 * Tall<SRC, STRIDED, K>::WARPS, Tall<SRC, STRIDED, K>::BLOCKS) norm_forward_tall_kernel(NormForward a)
{
    begin();
    constexpr int WARPS = Tall<SRC, STRIDED, K>::WARPS, SIZE = SRC == SRC_F32 ? 4 : 2, VECTORS = CHUNK * SIZE / 16;   // of a chunk
    extern __shared__ float4 params[];   // [chunks of a row][gamma, gamma, beta, beta][32]: a lane's 8 columns as 4 vectors
    __shared__ float part[WARPS][2][WARPS];
    const int lane = kept_lane(), warp = kept(threadIdx.y), warps = blockDim.y, side = kept(threadIdx.z);      // side: the row's place in the block
    const int first = warp * a.each * SPAN, end = min(first + a.each * SPAN, a.cols), c = lane_column<STRIDED>(first, lane);
    long long row = (long long)blockIdx.x * blockDim.z + side;
    const long long step = (long long)gridDim.x * blockDim.z;
    // then a place for each warp's part of the row to come.  Vector: [chunks][VECTORS][32] of 16 bytes.  Strided: the 16-byte vectors of
    // memory that lie in the part, at the same distance from a boundary; lanes hold the values before and after them until
    // the row's turn.
    const int place = a.each * VECTORS * 512 + (STRIDED ? 16 : 0);
    char *ahead = reinterpret_cast<char *>(params + (a.cols + SPAN - 1) / SPAN * 4 * 32) + (side * warps + warp) * place;
    const uint32_t ahead_at = (uint32_t)__cvta_generic_to_shared(ahead);
    uint32_t edge = 0;
    int edge_at = -1, move = 0;
    auto ask = [&](long long r) {
        if (r < a.rows && first < end) {
            if constexpr (!STRIDED) {
                const char *from = static_cast<const char *>(a.x.data) + (r * a.x.stride + first) * SIZE + lane * 16;
                const uint32_t to = ahead_at + (SIZE == 4 ? fp32_copied(lane) : lane * 16);
#pragma unroll
                for (int j = 0; j < K; ++j)
#pragma unroll
                    for (int i = 0; i < VECTORS; ++i)
                        if (first + j * SPAN + (i * 32 + lane) * 16 / SIZE < end) copy_async(to + (j * VECTORS + i) * 512, from + (j * VECTORS + i) * 512, 16);
            } else {
                const char *p = static_cast<const char *>(a.x.data) + (r * a.x.stride + first) * SIZE;
                const int bytes = (end - first) * SIZE, skip = (int)(-reinterpret_cast<intptr_t>(p) & 15), rest = skip + ((bytes - skip) & ~15);
                move = 16 - skip & 15;
                for (int i = skip + lane * 16; i + 16 <= bytes; i += 512) copy_async(ahead_at + move + i, p + i, 16);
                // lanes 0 .. 7: before the first vector; 16 .. 23: after the last (a part without one has only the former)
                const int e = lane < 16 ? lane * SIZE : (bytes > skip ? rest : skip) + (lane - 16) * SIZE;
                edge_at = lane < 16 ? (e < skip && e < bytes ? e : -1) : (e < bytes && bytes > skip ? e : -1);
                if (edge_at >= 0) edge = SIZE == 4 ? __ldg(reinterpret_cast<const uint32_t *>(p + edge_at)) : (uint32_t)__ldg(reinterpret_cast<const uint16_t *>(p + edge_at));
            }
        }
        copies_asked();
    };
    ask(row);
    for (int q = side * warps + warp; q * SPAN < a.cols; q += warps * blockDim.z) {
        F2 v[PAIRS];
        float f[CHUNK];
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            load_param<STRIDED>(which ? a.p.beta : a.p.gamma, a.p, lane_column<STRIDED>(q * SPAN, lane), a.cols, which ? 0.f : 1.f, v);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) split(v[i], f[2 * i], f[2 * i + 1]);
            params[(q * 4 + which * 2) * 32 + lane] = make_float4(f[0], f[1], f[2], f[3]);
            params[(q * 4 + which * 2 + 1) * 32 + lane] = make_float4(f[4], f[5], f[6], f[7]);
        }
    }
    bool set = false;       // the parameters are waited for when the first result needs them
    const float over = 1.f / (float)a.cols;
    const float4 *own = params + warp * a.each * 4 * 32;
    for (; row < a.rows; row += step) {
        if (row + step >= a.rows) let_next();
        Part<SRC, STRIDED, K> x;
        copies_wait<0>();
        if constexpr (STRIDED) {
            if (edge_at >= 0) {
                if (SIZE == 4) *reinterpret_cast<uint32_t *>(ahead + move + edge_at) = edge;
                else *reinterpret_cast<uint16_t *>(ahead + move + edge_at) = (uint16_t)edge;
            }
            __syncwarp();
            x.load(ahead + move + lane * SIZE, c, first, end);
        } else {
            if (SIZE == 4) __syncwarp();        // lanes read what others copied
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int i = 0; i < VECTORS; ++i)
                    x.put(j, i, c + j * SPAN < end ? *reinterpret_cast<const uint4 *>(ahead + j * VECTORS * 512 + (SIZE == 4 ? fp32_read(lane, i) : lane * 16)) : make_uint4(0, 0, 0, 0));
        }
        F2 v[PAIRS], t = f2(0.f);
#pragma unroll
        for (int j = 0; j < K; ++j) {
            if (STRIDED && first + j * SPAN >= end) break;       // the whole warp
            x.get(j, a.use[0], v);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) t = t + v[i];
        }
        float s[1] = {sum2(t)};       // all of the row is in registers
        if (STRIDED || SIZE == 4) __syncwarp();
        ask(row + step);
        row_sums<1, WARPS>(s, part[side][0], lane, warp, warps, 1 + side);
        const float mean = s[0] * over;
        t = f2(0.f);
#pragma unroll
        for (int j = 0; j < K; ++j) {
            if (STRIDED && first + j * SPAN >= end) break;
            x.get(j, a.use[1], v);
            const F2 less = f2(STRIDED || c + j * SPAN < end ? -mean : 0.f);      // zeros stay zeros past the last column
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) v[i] = v[i] + less;
            if (STRIDED && first + (j + 1) * SPAN > end) cut<STRIDED>(v, c + j * SPAN, end);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) t = fma2(v[i], v[i], t);
        }
        s[0] = sum2(t);
        row_sums<1, WARPS>(s, part[side][1], lane, warp, warps, 1 + side);
        const float rstd = inverse_root(fmaf(s[0], over, a.eps));
        if (a.mean && lane == 0 && warp == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
        if (!set) { __syncthreads(); set = true; }
        constexpr int YSIZE = OUT == LRBI_Y_F32 ? 4 : 2;
        char *y = static_cast<char *>(a.y.data) + (row * a.y.stride + c) * YSIZE;
        if constexpr (COPY) {
            int8_t *q = a.kept.q + row * a.kept.pitch + c;
            float *scale = a.kept.scale + row * a.kept.groups + first / KEEP_GROUP;
            using Keeper = Keep<STRIDED>;
            constexpr int TOGETHER = Keeper::CHUNKS;
#pragma unroll
            for (int j0 = 0; j0 < K; j0 += TOGETHER) {
                if (first + j0 * SPAN >= end) break;
                uint32_t tops[4] = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < TOGETHER; ++i) {
                    uint32_t t[STRIDED ? 2 : 1] = {};
                    if (j0 + i < K) x.chunk[j0 + i < K ? j0 + i : 0].tops(t);
                    tops[STRIDED ? 2 * i : i] = t[0];
                    if (STRIDED) tops[STRIDED ? 2 * i + 1 : 0] = t[STRIDED ? 1 : 0];
                }
                const Keeper keep(tops, lane);
#pragma unroll
                for (int i = 0; i < TOGETHER; ++i)
                    if (j0 + i < K) {
                        x.get(j0 + i, a.use[3], v);
                        keep.bytes(i, q + (j0 + i) * SPAN, (first + (j0 + i) * SPAN < end ? a.kept.pitch : 0) - c - (j0 + i) * SPAN, v);
                    }
                const int group = (j0 + Keeper::chunk(lane)) * (SPAN / KEEP_GROUP) + Keeper::group(lane);
                if (Keeper::stores(lane) && first + group * KEEP_GROUP < end) scale[group] = keep.quotient;
            }
        }
#pragma unroll
        for (int j = 0; j < K; ++j) {
            if (first + j * SPAN < end) {
                x.get(j, a.use[2], v);
                const float4 *g = own + j * 4 * 32 + lane;
                const float4 g0 = g[0], g1 = g[32], b0 = g[64], b1 = g[96];
                const F2 gamma[PAIRS] = {f2(g0.x, g0.y), f2(g0.z, g0.w), f2(g1.x, g1.y), f2(g1.z, g1.w)};
                const F2 beta[PAIRS] = {f2(b0.x, b0.y), f2(b0.z, b0.w), f2(b1.x, b1.y), f2(b1.z, b1.w)};
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) v[i] = fma2((v[i] + f2(-mean)) * f2(rstd), gamma[i], beta[i]);
                store_at<YSIZE, STRIDED>(y + j * SPAN * YSIZE, end - c - j * SPAN, v, first + (j + 1) * SPAN <= end);
            }
        }
    }
    if (!set) __syncthreads();
    copies_wait<0>();
}

// blockDim = 32 * warps of a row; one row a block.
template <int SRC, bool STRIDED, int NV>
__global__ void __launch_bounds__(1024) norm_forward_row_kernel(NormForward a)
{
    begin();
    let_next();
    __shared__ float part[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const long long row = blockIdx.x;
    const float over = 1.f / (float)a.cols;
    Raw<SRC, STRIDED> raw[NV];
    int c[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        c[j] = lane_column<STRIDED>((j * warps + warp) * SPAN, lane);
        raw[j].load(a.x, KeptIn{}, row, c[j], a.cols);
    }
    F2 gamma[PAIRS], beta[PAIRS], v[NV][PAIRS], t = f2(0.f);
    load_param<STRIDED>(a.p.gamma, a.p, c[0], a.cols, 1.f, gamma);
    load_param<STRIDED>(a.p.beta, a.p, c[0], a.cols, 0.f, beta);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        raw[j].get(v[j]);
        if (a.kept.q) keep_chunk(a.kept, row, (j * warps + warp) * SPAN, lane, v[j], raw[j]);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) t = t + v[j][i];
    }
    float s[1] = {sum2(t)};
    row_sums<1, 32>(s, part[0], lane, warp, warps, 1);
    const float mean = s[0] * over;
    t = f2(0.f);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) v[j][i] = v[j][i] + f2(-mean);
        cut<STRIDED>(v[j], c[j], a.cols);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) t = fma2(v[j][i], v[j][i], t);
    }
    s[0] = sum2(t);
    row_sums<1, 32>(s, part[1], lane, warp, warps, 1);
    const float rstd = inverse_root(fmaf(s[0], over, a.eps));
    if (a.mean && threadIdx.x == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (j > 0) {
            load_param<STRIDED>(a.p.gamma, a.p, c[j], a.cols, 1.f, gamma);
            load_param<STRIDED>(a.p.beta, a.p, c[j], a.cols, 0.f, beta);
        }
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) v[j][i] = fma2(v[j][i] * f2(rstd), gamma[i], beta[i]);
        store_chunk<STRIDED>(a.y, row, c[j], a.cols, v[j]);
    }
}

template <int SRC, bool STRIDED>
__global__ void __launch_bounds__(1024) norm_forward_wide_kernel(NormForward a)
{
    begin();
    __shared__ float part[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int span = warps * SPAN;
    const float over = 1.f / (float)a.cols;
    const long long row = blockIdx.x;
    Raw<SRC, STRIDED> raw;
    F2 v[PAIRS], t = f2(0.f);
    for (int c0 = warp * SPAN; c0 < a.cols; c0 += span) {
        raw.load(a.x, KeptIn{}, row, lane_column<STRIDED>(c0, lane), a.cols);
        raw.get(v);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) t = t + v[i];
    }
    float s[1] = {sum2(t)};
    row_sums<1, 32>(s, part[0], lane, warp, warps, 1);
    const float mean = s[0] * over;
    t = f2(0.f);
    for (int c0 = warp * SPAN; c0 < a.cols; c0 += span) {
        const int c = lane_column<STRIDED>(c0, lane);
        raw.load(a.x, KeptIn{}, row, c, a.cols);
        raw.get(v);
        if (a.kept.q) keep_chunk(a.kept, row, c0, lane, v, raw);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) v[i] = v[i] + f2(-mean);
        cut<STRIDED>(v, c, a.cols);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) t = fma2(v[i], v[i], t);
    }
    s[0] = sum2(t);
    row_sums<1, 32>(s, part[1], lane, warp, warps, 1);
    const float rstd = inverse_root(fmaf(s[0], over, a.eps));
    if (a.mean && threadIdx.x == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
    for (int c0 = warp * SPAN; c0 < a.cols; c0 += span) {
        const int c = lane_column<STRIDED>(c0, lane);
        F2 gamma[PAIRS], beta[PAIRS];
        load_param<STRIDED>(a.p.gamma, a.p, c, a.cols, 1.f, gamma);
        load_param<STRIDED>(a.p.beta, a.p, c, a.cols, 0.f, beta);
        raw.load(a.x, KeptIn{}, row, c, a.cols);
        raw.get(v);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) v[i] = fma2((v[i] + f2(-mean)) * f2(rstd), gamma[i], beta[i]);
        store_chunk<STRIDED>(a.y, row, c, a.cols, v);
    }
}

namespace {

template <int SRC, int OUT, bool STRIDED, bool COPY, int K>
lrbi_status tall_kernel_launch(const NormForward &a, cudaStream_t s)
{
    using T = Tall<SRC, STRIDED, K>;
    const size_t params = (size_t)((a.cols + SPAN - 1) / SPAN) * 4 * 512;
    const size_t ahead = (size_t)a.warps * (a.each * (CHUNK * (SRC == SRC_F32 ? 4 : 2) / 16) * 512 + (STRIDED ? 16 : 0));      // of a row
    int rows = T::WARPS / a.warps;
    rows = std::min<int>(rows, (int)((MOST_SHARED - params) / ahead));
    dim3 block(32, a.warps, std::max(1, rows));
    const size_t smem = params + ahead * block.z;
    auto kernel = norm_forward_tall_kernel<SRC, OUT, STRIDED, COPY, K>;
    const long long most = NORM_SMS * blocks_per_sm(kernel, 32 * block.y * block.z, smem);
    // Rows go in rounds over all blocks: the same number of rounds with the fewest rows a block, so that the last is not
    // nearly empty (4096 x 4096, two blocks an SM: 3 rounds of 6 rows a block, the last a third full, 18.0 us; of 5 rows, 16.8 us).
    const long long rounds = ((long long)a.rows + most * block.z - 1) / (most * block.z);
    block.z = (unsigned)std::max(1LL, ((long long)a.rows + most * rounds - 1) / (most * rounds));
    const long long need = ((long long)a.rows + block.z - 1) / block.z;
    return norm_launch(kernel, (int)std::min(need, most), block, params + ahead * block.z, s, a);
}

template <int SRC, int OUT, bool STRIDED, int K>
lrbi_status tall_launch(const NormForward &a, cudaStream_t s)
{
    return a.kept.q ? tall_kernel_launch<SRC, OUT, STRIDED, true, K>(a, s) : tall_kernel_launch<SRC, OUT, STRIDED, false, K>(a, s);
}

template <int SRC, int OUT, bool STRIDED>
lrbi_status forward_launch(NormForward a, cudaStream_t s)
{
    constexpr bool TWO = SRC == SRC_BF16 && !STRIDED;       // two values a register
    const int spans = (a.cols + SPAN - 1) / SPAN;
    // Chunks of a lane at most.  8: 24 warps an SM, 16384 x 4096 in 47 us (16 chunks, 16 warps: 49).  Rows beyond 8192 columns
    // share more of an SM's memory between fewer blocks, and there 16 are better: 4000 x 16384 in 55 us (8: 69).
    const int most = TWO && spans > 32 ? 16 : 8;
    a.warps = (spans + most - 1) / most;
    // Few rows leave most of the GPU idle with a warp each, and the parameters' way into shared memory is a good part of the
    // time: then a block takes a row.  Rows of two warps: 300 x 4096 3.9 us (two warps: 7.2), 700 6.5, 900 8.1 (6.7), 1300
    // 9.7 (7.3); of one: 590 x 1024 2.5 (2.8); at the change, 1183 and 1184 rows: x 1024 3.33 (3.01), x 1157 4.35 (4.22).
    const bool few = (long long)a.rows * a.warps < (a.warps > 1 ? 10 : 8) * NORM_SMS;
    if (spans > 64) return norm_launch(norm_forward_wide_kernel<SRC, STRIDED>, a.rows, dim3(1024), 0, s, a);
    if (few) {
        if (spans <= 32) return norm_launch(norm_forward_row_kernel<SRC, STRIDED, 1>, a.rows, dim3(32 * spans), 0, s, a);
        return norm_launch(norm_forward_row_kernel<SRC, STRIDED, 2>, a.rows, dim3(32 * ((spans + 1) / 2)), 0, s, a);
    }
    const int each = a.each = (spans + a.warps - 1) / a.warps;
    if (each <= 1) return tall_launch<SRC, OUT, STRIDED, 1>(a, s);
    if (each <= 2) return tall_launch<SRC, OUT, STRIDED, 2>(a, s);
    if (each <= 4) return tall_launch<SRC, OUT, STRIDED, 4>(a, s);
    if (each <= 8) return tall_launch<SRC, OUT, STRIDED, 8>(a, s);
    if constexpr (TWO) return tall_launch<SRC, OUT, STRIDED, 16>(a, s);
    return LRBI_ERR_UNSUPPORTED;
}

}  // namespace

lrbi_status launch_layer_norm(const NormArgs &n, cudaStream_t s)
{
    const NormForward a = {{n.x, n.x_stride}, make_params(n), {n.y, n.y_stride, n.y_dtype},
                           {n.q_out, n.scale_out, checkpoint_pitch(n.cols), checkpoint_groups(n.cols)}, n.mean_out, n.rstd_out, n.eps, n.rows, n.cols, 1, 1, {{16, 0xFFFF0000u}, {16, 0xFFFF0000u}, {16, 0xFFFF0000u}, {16, 0xFFFF0000u}}};
    const bool strided = n.cols % CHUNK != 0 || !vector_rows(n.x, n.x_stride, n.x_dtype) || !vector_rows(n.y, n.y_stride, n.y_dtype);
    if (n.x_dtype == LRBI_Y_BF16) {
        if (n.y_dtype == LRBI_Y_BF16) return strided ? forward_launch<SRC_BF16, LRBI_Y_BF16, true>(a, s) : forward_launch<SRC_BF16, LRBI_Y_BF16, false>(a, s);
        return strided ? forward_launch<SRC_BF16, LRBI_Y_F32, true>(a, s) : forward_launch<SRC_BF16, LRBI_Y_F32, false>(a, s);
    }
    if (n.y_dtype == LRBI_Y_BF16) return strided ? forward_launch<SRC_F32, LRBI_Y_BF16, true>(a, s) : forward_launch<SRC_F32, LRBI_Y_BF16, false>(a, s);
    return strided ? forward_launch<SRC_F32, LRBI_Y_F32, true>(a, s) : forward_launch<SRC_F32, LRBI_Y_F32, false>(a, s);
}

}  // namespace lrbi
