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
//
// Bound: memory where there are many rows (stream in fp32, f in bf16, root mean square, 16384 x 4096: forward 129 us of 125,
// backward 215 of 187; bf16 97 of 83 with layer norms, 89 without means).  Behind layer norms with betas the backward pass has four
// sums a column in the registers of its 512 threads and is bound by issue and what does not fit there (186 of 125).  Few rows: 5 us of
// launch, vectors and first rows.  Rows that are not whole vectors: an access a value (forward, 4096 x 4097 bf16 50 us of 21, 4096 x 801
// 13 of 4).  Means larger than the spread cost a row another sum (4096 x 4096 bf16 28 -> 36 us).  One span a thread and loads straight into registers, the first form, took 75 and 102 us for 4096 x 4096, now 28 and 56.
#pragma once
#include <algorithm>

#include "norm_common.cuh"

namespace lrbi {

constexpr int JOIN_THREADS = 512, JOIN_WARPS = JOIN_THREADS / 32;      // of a block, at most
constexpr int JOIN_SPLIT = 8;                                           // blocks of a cluster that share a row, at most
constexpr size_t JOIN_SHARED = 226 * 1024;                              // dynamic shared memory of a block, at most

struct Join {
    JoinArgs a;
    int split;                 // blocks that share a row
    int width;                 // columns of a block: whole spans
    bool whole;                // the vectors start on 16-byte boundaries
    float per;                 // 1 / cols
    float *parts;              // backward: [groups][4][split * width], or null
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

// ---------------------------------------------------------------------------------------------------------------------
// Rows on their way: a warp has K spans of a row, which come through shared memory
// ---------------------------------------------------------------------------------------------------------------------
// In whole vectors a lane copies 16 bytes at a time; fp32 ones are placed so that a lane's 32 bytes are read without bank conflicts
// (row_ops.cuh).  Other rows: the aligned 16-byte pieces of memory that hold the warp's columns are copied as they are, and lanes
// read single values out of them.  A piece may begin before the row, in the row before; the first row has none, and its first
// values are copied one by one.  Nothing past the row is read.
template <int SRC, bool STRIDED, int K>
struct Stream {
    static constexpr int SIZE = SRC == SRC_F32 ? 4 : 2, SLOT = K * SPAN * SIZE + (STRIDED ? 16 : 0);      // bytes of a warp and row
    const char *from;      // the warp's first column in row 0
    long long pitch;       // bytes from row to row
    int bytes;             // of the warp's columns
    bool lead;             // the warp has the first columns of the row

    __device__ __forceinline__ Stream(const void *p, long long stride, int c0, int cols)
    {
        from = static_cast<const char *>(p) + (long long)c0 * SIZE;
        pitch = stride * SIZE;
        bytes = p ? min(K * SPAN, cols - c0) * SIZE : 0;
        lead = c0 == 0;
    }
    // FULL: the warp has all of its columns; nothing is checked.
    template <bool FULL> __device__ __forceinline__ void ask(char *slot, long long row, int lane) const
    {
        if (bytes <= 0) return;
        const char *p = from + row * pitch;
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(slot);
        if constexpr (!STRIDED) {
            const char *mine = p + lane * 16;
            const uint32_t place = to + (SIZE == 4 ? fp32_copied(lane) : lane * 16);
#pragma unroll
            for (int i = 0; i < K * SPAN * SIZE / 512; ++i) {
                if (FULL) copy_async(place + i * 512, mine + i * 512, 16);
                else copy_async_if(i * 512 + lane * 16 < bytes, place + i * 512, mine + i * 512);
            }
        } else {
            const int before = (int)(reinterpret_cast<uintptr_t>(p) & 15u);
            const bool single = lead && before && row * pitch < before;       // the piece begins before the matrix
#pragma unroll
            for (int i = 0; i <= K * SPAN * SIZE / 512; ++i) {
                const int at = (i * 32 + lane) * 16, some = min(16, before + bytes - at);
                if (some > 0 && !(single && at == 0)) copy_async_some(to + at, p - before + at, some);
            }
            if (single && lane * SIZE < min(16 - before, bytes)) {
                if (SIZE == 4) *reinterpret_cast<uint32_t *>(slot + before + lane * 4) = __ldg(reinterpret_cast<const uint32_t *>(p) + lane);
                else *reinterpret_cast<uint16_t *>(slot + before + lane * 2) = __ldg(reinterpret_cast<const uint16_t *>(p) + lane);
            }
        }
    }
    // Chunk k of the lane: zeros where there is no column (left: columns from the span's first one on), or no matrix.
    template <bool FULL> __device__ __forceinline__ void get(const char *slot, long long row, int k, int left, int lane, F2 (&v)[PAIRS]) const
    {
        if constexpr (!STRIDED) {
            if (!FULL && (bytes <= 0 || lane * CHUNK >= left)) {
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) v[i] = f2(0.f);
            } else if (SIZE == 4) {
                const float4 a = *reinterpret_cast<const float4 *>(slot + k * 1024 + fp32_read(lane, 0)), b = *reinterpret_cast<const float4 *>(slot + k * 1024 + fp32_read(lane, 1));
                v[0] = f2(a.x, a.y); v[1] = f2(a.z, a.w); v[2] = f2(b.x, b.y); v[3] = f2(b.z, b.w);
            } else {
                const uint4 a = *reinterpret_cast<const uint4 *>(slot + k * 512 + lane * 16);
                v[0] = f2(bf16_lo(a.x), bf16_hi(a.x)); v[1] = f2(bf16_lo(a.y), bf16_hi(a.y));
                v[2] = f2(bf16_lo(a.z), bf16_hi(a.z)); v[3] = f2(bf16_lo(a.w), bf16_hi(a.w));
            }
        } else {
            const char *p = slot + (reinterpret_cast<uintptr_t>(from + row * pitch) & 15u) + (k * SPAN + lane) * SIZE;
            float f[CHUNK];
#pragma unroll
            for (int e = 0; e < CHUNK; ++e) {
                f[e] = 0.f;
                if (FULL || (bytes > 0 && lane + 32 * e < left)) f[e] = SIZE == 4 ? reinterpret_cast<const float *>(p)[32 * e] : __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(p)[32 * e] << 16);
            }
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) v[i] = f2(f[2 * i], f[2 * i + 1]);
        }
    }
};

// Zeros where there is no column.
template <bool STRIDED, bool FULL = false> __device__ __forceinline__ void keep_there(F2 (&v)[PAIRS], int left, int lane)
{
    if (FULL || left >= SPAN) return;
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
        float a, b;
        split(v[i], a, b);
        v[i] = f2(chunk_column<STRIDED>(lane_column<STRIDED>(0, lane), 2 * i) < left ? a : 0.f, chunk_column<STRIDED>(lane_column<STRIDED>(0, lane), 2 * i + 1) < left ? b : 0.f);
    }
}

// A vector of the call in fp32, in shared memory for a block's columns: a lane's eight as two pieces of 16 bytes half a span apart
// (strided: as they are), so that a warp reads without bank conflicts.  Four neighbouring columns stay together.
template <bool STRIDED> __device__ __forceinline__ int vector_place(int c) { return STRIDED ? c : (c & ~255) | (c & 4) << 5 | (c & 248) >> 1 | (c & 3); }
// Columns c .. c + 3 of a vector; `other` where there is none.
__device__ __forceinline__ float4 four_of(const void *p, int dtype, bool whole, int c, int cols, float other)
{
    float4 v = make_float4(other, other, other, other);
    if (!p) return v;
    if (whole && c + 4 <= cols) {
        if (dtype == LRBI_Y_F32) return __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(p) + c));
        const uint2 w = __ldg(reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p) + c));
        return make_float4(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y));
    }
    if (c < cols) v.x = one_param(p, dtype, c);
    if (c + 1 < cols) v.y = one_param(p, dtype, c + 1);
    if (c + 2 < cols) v.z = one_param(p, dtype, c + 2);
    if (c + 3 < cols) v.w = one_param(p, dtype, c + 3);
    return v;
}
__device__ __forceinline__ float4 operator*(float4 a, float4 b) { return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w); }
template <bool STRIDED> __device__ __forceinline__ void get_vector(const float *v, int span, int lane, F2 (&w)[PAIRS])
{
    if constexpr (STRIDED) {
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) w[i] = f2(v[span * SPAN + lane + 64 * i], v[span * SPAN + lane + 64 * i + 32]);
    } else {
        const float4 a = *reinterpret_cast<const float4 *>(v + span * SPAN + lane * 4), b = *reinterpret_cast<const float4 *>(v + span * SPAN + 128 + lane * 4);
        w[0] = f2(a.x, a.y); w[1] = f2(a.z, a.w); w[2] = f2(b.x, b.y); w[3] = f2(b.z, b.w);
    }
}

// The threads that share a row: `warps` warps of this block, or of each of `split` blocks of a cluster.
struct Team {
    int lane, warp, warps, id, split, rank;
    int phase;         // places to meet are there twice, so that a team meets once for each sum

    __device__ __forceinline__ Team(int split_)
    {
        lane = kept_lane();
        warp = kept(threadIdx.x >> 5);
        warps = blockDim.x >> 5;
        id = 1 + threadIdx.y;
        split = split_;
        rank = split > 1 ? join_rank() : 0;
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
    // The team's places of N values an entry, in turn.  part: for each team of the block twice the entries.
    template <int N> __device__ __forceinline__ float *board(float *part)
    {
        float *p = part + ((threadIdx.y * 2 + phase) * entries()) * N;
        phase ^= 1;
        return p;
    }
};

// How rows are dealt out: spans of a warp, threads of a row, rows of a block, blocks that share a row, groups of such blocks.
struct JoinCut {
    int each, threads, teams, split, groups;
    bool direct;       // the vectors stay in memory: a row fits a block, they beside it do not
    size_t smem;
    int width() const { return threads / 32 * each * SPAN; }
};

// most_each: spans of a warp where there are more rows than `few`.  A warp that has more of a row has fewer others to wait for, and
// more rows are under way side by side; few rows are better spread over many warps.
// row: bytes of a column of a row in shared memory; vectors: of the vectors' columns; meet: of the places to meet, an entry.
// may_direct: rows of a block may do without the vectors in shared memory (2048 x 16384, root mean square, forward: 96 us; as two
// blocks that share a row 118).
inline JoinCut join_cut(int rows, int cols, int most_each, int few, int row, int vectors, int meet, bool may_direct)
{
    JoinCut k = {};
    const int spans = (cols + SPAN - 1) / SPAN;
    k.each = spans > 1 && (rows > std::max(2 * NORM_SMS, few) || spans > JOIN_WARPS) ? most_each : 1;
    for (k.split = 1;; k.split *= 2) {
        const int warps = ((spans + k.split - 1) / k.split + k.each - 1) / k.each;
        k.threads = 32 * warps;
        auto need = [&](int teams) {
            return (size_t)(k.direct ? 0 : vectors) * k.width() + (size_t)teams * ((size_t)2 * (row * k.width() + warps * 64) + (size_t)2 * warps * k.split * meet);
        };
        k.direct = may_direct && k.split == 1 && warps <= JOIN_WARPS && need(1) > JOIN_SHARED;
        if (k.split < JOIN_SPLIT && (warps > JOIN_WARPS || need(1) > JOIN_SHARED)) continue;
        k.teams = 1;
        while (k.split == 1 && (k.teams + 1) * k.threads <= JOIN_THREADS && need(k.teams + 1) <= JOIN_SHARED) ++k.teams;
        k.smem = need(k.teams);
        break;
    }
    k.groups = std::min((rows + k.teams - 1) / k.teams, NORM_SMS / k.split);
    return k;
}
// Vectors of the forward pass in shared memory: gate * post_gamma, gamma, beta, gate * post_beta, up to the last that there is.
__host__ __device__ inline int join_vectors(const JoinArgs &a) { return a.post_beta ? 4 : a.beta ? 3 : a.gamma ? 2 : 1; }
inline int type_bytes(int dtype) { return dtype == LRBI_Y_F32 ? 4 : 2; }
// Rows that the blocks of all SMs take at a time, with `each` spans a warp.
inline int rows_at_once(int cols, int each) { return NORM_SMS * std::max(1, JOIN_WARPS / ((cols + SPAN * each - 1) / (SPAN * each))); }
// Forward.  Room for the vectors that there are (2000 x 12896 bf16, gamma alone: 54 us, with room for all four none fit, 90).  A row whose
// vectors have no room reads up to six: more than three, and two blocks that share the row, beside the vectors, are faster (2000 x 12891
// fp32: three 173 us and 160, six 263 and 161; in whole vectors, 12896, 117 and 124, 180 and 128; 100 rows 13 and 16, 20 and 17).
// 300 x 1000 3.9 us with one span a warp, 5.0 with four; 1003 x 801 6.7 and 6.4, 2000 x 1024 8.4 and 5.2.
inline JoinCut forward_cut(const JoinArgs &a)
{
    const int reads = (a.post_gamma != nullptr) + (a.gate != nullptr) * (a.post_beta ? 2 : 1) + (a.post_beta != nullptr) + (a.gamma != nullptr) + (a.beta != nullptr);
    return join_cut(a.rows, a.cols, 4, rows_at_once(a.cols, 4) / 4, type_bytes(a.x_dtype) + type_bytes(a.f_dtype), 4 * join_vectors(a), 8, reads <= 3);
}
// Backward: with one row for each team or less, 1003 x 801 12.0 us, with two spans a warp 13.9; 2000 x 1024 12.4 and 11.4, 700 x 1500
// (three rows a team with one span) 13.8 and 10.2.  level (the kernel that then runs is short of registers with two spans):
// 1000 x 4096 21.3 and 23.4, 5000 x 333 21.7 and 26.0, 2048 x 4096 alike.
inline JoinCut backward_cut(int rows, int cols, int x_dtype, int f_dtype, bool level)
{
    const int few = level ? 5 * rows_at_once(cols, 2) : std::min(rows_at_once(cols, 2), 2 * rows_at_once(cols, 1));
    return join_cut(rows, cols, 2, few, 2 * (type_bytes(x_dtype) + type_bytes(f_dtype)), 8, 32, false);
}

template <class Kernel>
lrbi_status join_launch(Kernel kernel, const JoinCut &k, cudaStream_t s, const Join &j)
{
    return launch_kernel(kernel, dim3(k.groups * k.split), dim3(k.threads, k.teams), k.smem, s, k.split, j);
}

inline bool join_vector(const JoinArgs &a)
{
    auto rows = [&](const void *p, long long stride, int dtype) { return !p || vector_rows(p, stride, dtype); };
    return a.cols % CHUNK == 0 && rows(a.x, a.x_stride, a.x_dtype) && rows(a.f, a.f_stride, a.f_dtype) && rows(a.out, a.out_stride, a.x_dtype) &&
           rows(a.u, a.u_stride, a.f_dtype) && rows(a.du, a.du_stride, a.f_dtype) && rows(a.dout, a.dout_stride, a.x_dtype) &&
           rows(a.dx, a.dx_stride, a.x_dtype) && rows(a.df, a.df_stride, a.f_dtype);
}

inline Join make_join(const JoinArgs &a, const JoinCut &k, float *parts)
{
    uintptr_t all = 0;
    for (const void *p : {a.gamma, a.beta, a.post_gamma, a.post_beta, a.gate}) all |= reinterpret_cast<uintptr_t>(p);
    return {a, k.split, k.width(), (all & 15u) == 0, 1.f / (float)a.cols, parts};
}

}  // namespace lrbi
