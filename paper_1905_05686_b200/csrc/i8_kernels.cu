// Rows in 8-bit integers with a scale each -- a layer's channels, a batch's tokens -- and their product for a few tokens.
//
//   a row v:   top = max |v|,   scale = top / 127,   q = rint(v * (127 / top))             (each step one fp32 operation)
//   product:   Y[b][o] = (sum over i of q_X[b][i] * q_W[o][i]) * scale_X[b] * scale_W[o]   (the sum is a whole number, exact)
//
// Rows of q start on 16-byte boundaries and hold zeros past the last column, so that a product takes them 16 bytes at a time.
#include <algorithm>

#include "activation.cuh"
#include "norm_common.cuh"

namespace lrbi {

// ---------------------------------------------------------------------------------------------------------------------
// Tokens
// ---------------------------------------------------------------------------------------------------------------------
struct TokenArgs {
    RowsIn x;
    int8_t *q;
    float *scale;
    int rows, cols, pitch;
};

__device__ __forceinline__ float not_below(float v, float least)      // a NaN stays
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(v), "f"(least));
    return r;
}

// The nonlinearity of values of a row, as for results in fp32; 0 stays 0 in all of them.  (gelu with a tail off by 2^-14, as results in
// bf16 allow, moved ten times the bytes to the other side of a tie that roundings in fp32 move.)
template <int ACT> __device__ __forceinline__ F2 token_act(F2 v)
{
    if constexpr (ACT == ACT_NONE) return v;
    else if constexpr (ACT == LRBI_ACT_RELU) {
        float a, b;
        split(v, a, b);
        return f2(not_below(a, 0.f), not_below(b, 0.f));
    } else {
        F2 slope;
        activate<ACT, false, true, false>(v, v, slope);
        return v;
    }
}

// Whether values are taken out of what was loaded twice, and relu again, rather than kept in fp32 between the maximum and the bytes:
// fewer registers, so twice the chunks a thread (4096 x 4096 of relu 9.6 us, kept 10.1).  Rows that are not whole vectors, and other
// nonlinearities, take longer again than the registers cost (a gelu of fewer steps than this one 21.4 and 14.7).
__host__ __device__ constexpr bool taken_again(int act, bool strided) { return !strided && (act == ACT_NONE || act == LRBI_ACT_RELU); }
// blockDim = (threads of a row, rows of a block).  A thread has up to K chunks of its row in registers between the maximum and the
// bytes: as they were loaded, or as results in fp32 (taken_again()).  Rows of more chunks are read, and activated, twice.
// 4096 x 4096 bf16 8.2 us (floor 7.8), fp32 12.6 (13.0); of gelu 15.7 and 17.8, of silu 16.5 and 14.0; 1000 x 16384 bf16 of gelu 17.0 (7.6): more
// than half of that is the arithmetic of gelu.
template <int SRC, int ACT, bool STRIDED, int K>
__global__ void __launch_bounds__(K == 8 ? 256 : 512, K == 8 ? 4 : 2) i8_tokens_kernel(TokenArgs a)
{
    begin();
    let_next();         // a product that follows is set up, and asks for its weights, meanwhile
    constexpr int SIZE = SRC == SRC_F32 ? 4 : 2;
    __shared__ uint32_t part[16];
    const int lane = kept_lane(), warp = threadIdx.x >> 5, warps = blockDim.x >> 5, team = threadIdx.y;
    const long long row = (long long)blockIdx.x * blockDim.y + team;
    const bool there = row < a.rows;
    const int rounds = (a.cols + warps * SPAN * K - 1) / (warps * SPAN * K);
    const char *x = static_cast<const char *>(a.x.data) + row * a.x.stride * SIZE;
    Raw<SRC, STRIDED> raw[K];
    constexpr bool AGAIN = taken_again(ACT, STRIDED);
    F2 results[AGAIN ? 1 : K][PAIRS];
    auto load = [&](int round) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c0 = ((round * K + k) * warps + warp) * SPAN, c = lane_column<STRIDED>(c0, lane);
            raw[k].clear();
            if (there && c < a.cols) raw[k].load_at(x + (long long)c * SIZE, a.cols - c, STRIDED && c0 + SPAN <= a.cols);
        }
        if constexpr (!AGAIN) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                raw[k].get(results[k]);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) results[k][i] = token_act<ACT>(results[k][i]);
            }
        }
    };
    auto get = [&](int k, F2 (&v)[PAIRS]) {
        if constexpr (AGAIN) raw[k].get(v);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) v[i] = AGAIN ? token_act<ACT>(v[i]) : results[AGAIN ? 0 : k][i];
    };
    float most = 0.f;
    for (int r = 0; r < rounds; ++r) {
        load(r);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            F2 v[PAIRS];
            get(k, v);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                float lo, hi;
                split(v[i], lo, hi);
                most = not_below(fabsf(hi), not_below(fabsf(lo), most));
            }
        }
    }
    uint32_t top = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most));      // a NaN is above infinity
    if (warps > 1) {
        if (lane == 0) part[team * warps + warp] = top;
        __syncthreads();
        top = __reduce_max_sync(0xFFFFFFFFu, part[team * warps + (lane < warps ? lane : 0)]);
    }
    if (!there) return;
    const TokenScale s(top);
    if (threadIdx.x == 0) a.scale[row] = s.scale();
    int8_t *q = a.q + row * a.pitch;
    for (int r = 0; r < rounds; ++r) {
        if (rounds > 1) load(r);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c0 = ((r * K + k) * warps + warp) * SPAN, c = lane_column<STRIDED>(c0, lane);
            F2 v[PAIRS];
            get(k, v);
            store_i8<STRIDED>(q + c, a.pitch - c, v, s.factor, s.fine, STRIDED && c0 + SPAN <= a.pitch);
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Weights
// ---------------------------------------------------------------------------------------------------------------------
// A block has a row.  The range is that of the kept weights; pruned ones are stored as zeros whatever the array holds there.
// A value an access, and the index of a weight decoded on its own, twice: a layer is quantised once, before it serves (4096 x 9216
// 134 us, with an index of rank 32 330; floor 17.5).
__global__ void __launch_bounds__(256) i8_quantize_kernel(Geo geo, const uint16_t *__restrict__ W, const uint32_t *__restrict__ ip,
                                                          const uint32_t *__restrict__ iz, int8_t *__restrict__ q, float *__restrict__ scale, int pitch)
{
    __shared__ uint32_t part[8];
    const int o = blockIdx.x, tr = o / geo.tm;
    const uint16_t *w = W + (long long)o * geo.cols;
    auto weight = [&](int c) {
        if (ip) {
            const int tc = c / geo.tn;
            const long long t = (long long)tr * geo.gc + tc;
            const uint32_t *a = ip + (t * geo.tm + (o - tr * geo.tm)) * geo.kw, *b = iz + (t * geo.tn + (c - tc * geo.tn)) * geo.kw;
            uint32_t any = 0;
            for (int i = 0; i < geo.kw; ++i) any |= __ldg(a + i) & __ldg(b + i) & (i == geo.kw - 1 ? tail_mask(geo.k) : 0xFFFFFFFFu);
            if (!any) return 0.f;
        }
        return __uint_as_float((uint32_t)__ldg(w + c) << 16);
    };
    uint32_t top = 0;
    for (int c = threadIdx.x; c < geo.cols; c += 256) top = max(top, __float_as_uint(weight(c)) & 0x7FFFFFFFu);
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
    __syncthreads();
    top = __reduce_max_sync(0xFFFFFFFFu, part[threadIdx.x & 7]);
    const TokenScale s(top);
    if (threadIdx.x == 0) scale[o] = s.scale();
    for (int c = threadIdx.x; c < pitch; c += 256) q[(long long)o * pitch + c] = s.fine && c < geo.cols ? (int8_t)(int)rintf(__fmul_rn(weight(c), s.factor)) : (int8_t)0;
}

// ---------------------------------------------------------------------------------------------------------------------
// Products of a few tokens
// ---------------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void mma_i8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A block has 16 rows of weights and 8 * NT tokens; its warps take 64 columns each in turn and add their sums up at the end.
// The column is a summation index: lane (g, t) takes 16 neighbouring bytes of rows g and g + 8, and of token g, as the four
// words that two steps of 32 columns want, both operands in the same order.
template <int NT, int I8_WARPS, int U>
__global__ void __launch_bounds__(32 * I8_WARPS) i8_few_kernel(I8Product p)
{
    __shared__ int sums[I8_WARPS][8 * NT][16];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int o0 = blockIdx.x * 16;
    const int8_t *w0 = p.w + (long long)min(o0 + g, p.rows - 1) * p.pitch, *w1 = p.w + (long long)min(o0 + g + 8, p.rows - 1) * p.pitch;
    // A hint that needs no order: the first weights come to L2 while the kernel before this one (the tokens') ends.  With the tokens,
    // 4096 x 9216, one of them: 10.3 us, without 11.3; all of the weights at once: 15.
    if (t < 2)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = (u * I8_WARPS + warp) * 64;
            if (c < p.pitch) asm volatile("prefetch.global.L2 [%0];" ::"l"((t ? w1 : w0) + c));
        }
    begin();
    const int8_t *x[NT];
    bool on[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        on[n] = 8 * n + g < p.batch;
        x[n] = p.x + (long long)(on[n] ? 8 * n + g : 0) * p.pitch;
    }
    int d[NT][4] = {};
    for (int c0 = warp * 64; c0 < p.pitch; c0 += I8_WARPS * 64 * U) {
        uint4 a[U][2], b[U][NT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * I8_WARPS * 64 + 16 * t;
            const bool in = c < p.pitch;
            a[u][0] = a[u][1] = make_uint4(0, 0, 0, 0);
            if (in) { a[u][0] = ld_once16(w0 + c); a[u][1] = ld_once16(w1 + c); }
#pragma unroll
            for (int n = 0; n < NT; ++n) b[u][n] = in && on[n] ? __ldg(reinterpret_cast<const uint4 *>(x[n] + c)) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                mma_i8(d[n], a[u][0].x, a[u][1].x, a[u][0].y, a[u][1].y, b[u][n].x, b[u][n].y);
                mma_i8(d[n], a[u][0].z, a[u][1].z, a[u][0].w, a[u][1].w, b[u][n].z, b[u][n].w);
            }
    }
    let_next();
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[warp][8 * n + 2 * t + (i & 1)][g + 8 * (i >> 1)] = d[n][i];
    __syncthreads();
    for (int k = threadIdx.x; k < 8 * NT * 16; k += 32 * I8_WARPS) {
        const int b = k / 16, o = o0 + k % 16;
        if (b >= p.batch || o >= p.rows) continue;
        int v = 0;
#pragma unroll
        for (int w = 0; w < I8_WARPS; ++w) v += sums[w][b][k % 16];
        const float y = ((float)v * __ldg(p.x_scale + b)) * __ldg(p.w_scale + o);
        const long long to = (long long)b * p.rows + o;
        if (p.y_dtype == LRBI_Y_F32) static_cast<float *>(p.y)[to] = y;
        else static_cast<uint16_t *>(p.y)[to] = (uint16_t)pack_bf16(y, 0.f);
    }
}

namespace {

template <int SRC, int ACT, bool STRIDED, int K>
lrbi_status tokens_launch(const TokenArgs &a, int threads, cudaStream_t s)
{
    const int teams = threads < 128 ? 128 / threads : 1;
    return launch_kernel(i8_tokens_kernel<SRC, ACT, STRIDED, K>, dim3((a.rows + teams - 1) / teams), dim3(threads, teams), 0, s, 1, a);
}

template <int SRC, int ACT, bool STRIDED>
lrbi_status tokens_chunks(const TokenArgs &a, cudaStream_t s)
{
    const int spans = (a.cols + SPAN - 1) / SPAN;
    // Many rows: a thread has more chunks of its row, all of them under way at once, and few others to wait for (4096 x 4096 bf16: one
    // 17.9 us, four 10.4, eight 9.2, all with a slower maximum than now).
    if (spans > 2 && (long long)a.rows * spans > 64 * NORM_SMS) {
        if constexpr (SRC == SRC_BF16 && taken_again(ACT, STRIDED)) return tokens_launch<SRC, ACT, STRIDED, 8>(a, 32 * std::min(8, (spans + 7) / 8), s);
        return tokens_launch<SRC, ACT, STRIDED, 4>(a, 32 * std::min(16, (spans + 3) / 4), s);
    }
    if (spans <= 16) return tokens_launch<SRC, ACT, STRIDED, 1>(a, 32 * (spans <= 1 ? 1 : spans <= 2 ? 2 : spans <= 4 ? 4 : spans <= 8 ? 8 : 16), s);
    if (spans <= 32) return tokens_launch<SRC, ACT, STRIDED, 2>(a, 512, s);
    return tokens_launch<SRC, ACT, STRIDED, 4>(a, 512, s);
}

template <int SRC, int ACT>
lrbi_status tokens_rows(const TokenArgs &a, cudaStream_t s)
{
    return a.cols % CHUNK == 0 && vector_rows(a.x.data, a.x.stride, SRC) ? tokens_chunks<SRC, ACT, false>(a, s) : tokens_chunks<SRC, ACT, true>(a, s);
}

template <int SRC>
lrbi_status tokens_act(const TokenArgs &a, int act, cudaStream_t s)
{
    if (act == LRBI_ACT_RELU) return tokens_rows<SRC, LRBI_ACT_RELU>(a, s);
    if (act == LRBI_ACT_GELU) return tokens_rows<SRC, LRBI_ACT_GELU>(a, s);
    if (act == LRBI_ACT_SILU) return tokens_rows<SRC, LRBI_ACT_SILU>(a, s);
    return tokens_rows<SRC, ACT_NONE>(a, s);
}

template <int NT, int W, int U>
lrbi_status few_launch(const I8Product &p, cudaStream_t s)
{
    return launch_kernel(i8_few_kernel<NT, W, U>, dim3((p.rows + 15) / 16), dim3(32 * W), 0, s, 1, p);
}

// One token, us: 4096 x 9216 with 8 warps 8.9, 16 11.1; 16384 x 4096 12.6 and 18.1; layers of fewer tiles than SMs: 64 x 16384 5.6 and
// 4.3, 1000 x 4096 2.9 and 2.5.  Short rows, two steps at a time: 16384 x 500 3.9, four 4.9.
lrbi_i8_plan few_plan(int rows, int cols, int batch)
{
    const int warps = batch > 8 || rows <= 16 * NORM_SMS ? 16 : 8;
    return {LRBI_I8_FEW, batch > 8 ? 16 : 8, 16, 1, warps == 8 && cols <= 1024 ? 2 : 4, 32 * warps, 1};
}
lrbi_status launch_few(const I8Product &p, const lrbi_i8_plan &plan, cudaStream_t s)
{
    if (plan.tokens > 8) return few_launch<2, 16, 4>(p, s);
    if (plan.threads == 512) return few_launch<1, 16, 4>(p, s);
    return plan.stages == 2 ? few_launch<1, 8, 2>(p, s) : few_launch<1, 8, 4>(p, s);
}

// Times in microseconds, as fitted to those measured (64 .. 16384 rows, 500 .. 16384 columns, 16 .. 4096 tokens).
struct Estimate {
    int rows, batch, blocks;      // blocks: of 128 columns
    double memory;                // what the arrays take

    Estimate(int rows_, int cols, int batch_, int y_dtype) : rows(rows_), batch(batch_), blocks((cols + 127) / 128)
    {
        memory = ((double)rows * cols + (double)batch * cols + (y_dtype == LRBI_Y_F32 ? 4. : 2.) * batch * rows) / 5.7e6;
    }
    static double rounds(long long units, int at_once) { return (double)((units + at_once - 1) / at_once); }
    // 9 to 16 tokens without tensor memory
    double few(int cols) const { return 1.5 + 0.0006 * cols + rows * (0.0004 + 1e-7 * cols); }
    // Pairs: a launch and the last tile's stores; 128 columns of a tile, in proportion to what a pair reads of both operands.  Tiles of
    // fewer channels where they fill the last round better (11049 x 7389, 1606 tokens: 256 channels 110 us, 224 101; 8192 x 8192, 700:
    // 256 43.8, 192 40.0; 4096 x 16384, 1000: 256 47, 224 82).
    double many(int channels) const
    {
        const double turns = rounds((long long)((batch + 255) / 256) * ((rows + channels - 1) / channels), NORM_SMS / 2);
        return 6. + std::max(turns * blocks * 0.28 * (256 + channels) / 512, memory);
    }
    // Clusters: a launch, 8 ns more for each CTA that has to start beside others, the sums and stores of a tile's tokens; 128 columns of a
    // CTA one after the other, or what all of them read of L2 (a block takes as long as 4000 bytes more would).
    double split(int tokens, int split) const
    {
        const long long ctas = (long long)((batch + tokens - 1) / tokens) * ((rows + 127) / 128) * split;
        const double turns = rounds(ctas, i8_at_once(split)), inner = rounds(ctas, (tokens <= 128 ? 2 : 1) * i8_at_once(split)) * (split == 8 && tokens > 128 ? 2. : 1.);
        const double tile = split == 1 ? 0.3 + 0.009 * tokens : 1. + 0.2 * (split > 2) + 0.35 * (split > 4) + 0.0145 * tokens;
        const double inside = std::max(inner * ((blocks + split - 1) / split) * (tokens <= 128 ? 0.22 : tokens <= 192 ? 0.25 : 0.34), (double)ctas * blocks / split * (20384 + 128 * tokens) / 16e6);
        return 2. + 0.008 * ctas + turns * tile + std::max(inside, memory);
    }
};

}  // namespace

lrbi_status launch_i8_tokens(const void *x, int dtype, long long stride, int rows, int cols, int act, int8_t *q, float *scale, cudaStream_t s)
{
    const TokenArgs a = {{x, stride}, q, scale, rows, cols, i8_pitch(cols)};
    return dtype == LRBI_Y_F32 ? tokens_act<SRC_F32>(a, act, s) : tokens_act<SRC_BF16>(a, act, s);
}

lrbi_status launch_i8_quantize(const Geo &g, const uint16_t *W, const uint32_t *ip, const uint32_t *iz, int8_t *q, float *scale, cudaStream_t s)
{
    i8_quantize_kernel<<<g.rows, 256, 0, s>>>(g, W, ip, iz, q, scale, i8_pitch(g.cols));
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) { note_cuda_error((int)e); return LRBI_ERR_CUDA; }
    count_launch();
    return LRBI_OK;
}

lrbi_i8_plan i8_gemm_plan(int rows, int cols, int batch, int y_dtype)
{
    // Up to 8 tokens, few blocks or many: over 12 .. 8192 rows and 512 .. 131072 columns warp-level products take as long as clusters that
    // share the columns or up to half of it (us, one token: 12 x 4096 2.0 and 4.1, 12 x 131072 29.6 and 30.8, 64 x 16384 4.9 and 6.7,
    // 4096 x 9216 8.4 and 10.3), but for rows of 65536 columns and more, where they take up to 14% longer (1000 x 131072 39.4 and 34.5).
    if (batch <= 8) return few_plan(rows, cols, batch);
    const Estimate e(rows, cols, batch, y_dtype);
    double best = e.many(256);
    int channels = 256, tokens = 0, split = 0;
    for (int n = 224; n >= 128; n -= 32)
        if (e.many(n) < best) { best = e.many(n); channels = n; }
    for (int n : {16, 32, 64, 128, 192, 256})
        for (int k = 1; k <= 8 && k <= e.blocks; k *= 2) {
            const int each = std::min(n, (batch + 15) / 16 * 16);
            const double t = e.split(each, k);
            if (t < best) { best = t; tokens = each; split = k; }
        }
    if (batch <= 16 && e.few(cols) < best) return few_plan(rows, cols, batch);
    return split ? i8_split_plan(rows, batch, tokens, split) : i8_long_plan(channels);
}

lrbi_status launch_i8_gemm(const I8Product &p, cudaStream_t s)
{
    const lrbi_i8_plan plan = i8_gemm_plan(p.rows, p.cols, p.batch, p.y_dtype);
    return plan.kernel == LRBI_I8_FEW ? launch_few(p, plan, s) : plan.kernel == LRBI_I8_SPLIT ? launch_i8_split(p, plan, s) : launch_i8_long(p, plan, s);
}

}  // namespace lrbi
