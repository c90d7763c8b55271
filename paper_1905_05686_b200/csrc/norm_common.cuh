// Shared by the forward and the backward pass of the layer norm.
#pragma once
#include "row_ops.cuh"

namespace lrbi {

constexpr int NORM_SMS = 148;
constexpr size_t MOST_SHARED = 224 * 1024;   // dynamic shared memory of a block, beside its static arrays

struct Params {            // gamma and beta, fp32 or bf16; beta may be null
    const void *gamma, *beta;
    int dtype;
    bool whole;            // in vectors: the arrays start on 16-byte boundaries
};

inline Params make_params(const NormArgs &n)
{
    return {n.gamma, n.beta, n.param_dtype, ((reinterpret_cast<uintptr_t>(n.gamma) | reinterpret_cast<uintptr_t>(n.beta)) & 15u) == 0};
}

__device__ __forceinline__ float one_param(const void *p, int dtype, int c)
{
    return dtype == LRBI_Y_F32 ? __ldg(static_cast<const float *>(p) + c) : __uint_as_float((uint32_t)__ldg(static_cast<const uint16_t *>(p) + c) << 16);
}

// The parameters of a chunk; `other` where there is none.
template <bool STRIDED>
__device__ __forceinline__ void load_param(const void *p, const Params &how, int c, int cols, float other, F2 (&v)[PAIRS])
{
    if (!STRIDED && p && how.whole && c + CHUNK <= cols) {
        if (how.dtype == LRBI_Y_F32) {
            const float4 *f = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + c);
            const float4 a = __ldg(f), b = __ldg(f + 1);
            v[0] = f2(a.x, a.y); v[1] = f2(a.z, a.w); v[2] = f2(b.x, b.y); v[3] = f2(b.z, b.w);
        } else {
            const uint4 a = __ldg(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + c));
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) v[i] = f2(bf16_lo(w[i]), bf16_hi(w[i]));
        }
        return;
    }
    float f[CHUNK];
#pragma unroll
    for (int e = 0; e < CHUNK; ++e) f[e] = p && chunk_column<STRIDED>(c, e) < cols ? one_param(p, how.dtype, chunk_column<STRIDED>(c, e)) : other;
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) v[i] = f2(f[2 * i], f[2 * i + 1]);
}

// Sets what lies past the last column to zero.
template <bool STRIDED>
__device__ __forceinline__ void cut(F2 (&v)[PAIRS], int c, int cols)
{
    if (chunk_column<STRIDED>(c, CHUNK - 1) < cols) return;
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
        float lo, hi;
        split(v[i], lo, hi);
        v[i] = f2(chunk_column<STRIDED>(c, 2 * i) < cols ? lo : 0.f, chunk_column<STRIDED>(c, 2 * i + 1) < cols ? hi : 0.f);
    }
}

// 1 / sqrt(a): one Newton step on the hardware's estimate r, where r and a r are normal numbers (a may be a denormal one, whose
// half need not be representable).  0 gives infinity, infinity 0.
__device__ __forceinline__ float inverse_root(float a)
{
    const float r = rsqrtf(a);
    return a > 0.f && a < 3e38f ? r * fmaf(-0.5f * (a * r), r, 1.5f) : r;
}

// Waits for the warps that share a row: `threads` of the block, barrier `id` (1 .. 15).
__device__ __forceinline__ void row_barrier(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// Sums over a row's threads of N values at a time, in every thread.  Within a warp the values are folded into one another
// (lanes of each half keep half of the values, and so on), so N values cost N + 3 shuffles or so instead of 5 N; the warps'
// sums meet in `part`, [N][WARPS] with room for the most warps that there are; it may be written again after the next barrier.
template <int N, int WARPS>
__device__ __forceinline__ void row_sums(float (&v)[N], float *part, int lane, int warp, int warps, int id)
{
    static_assert(N == 1 || N == 2 || N == 4 || N == 8, "");
    constexpr int G = 32 / N;          // lanes that share a value in the end
    float k[N];
#pragma unroll
    for (int i = 0; i < N; ++i) k[i] = v[i];
#pragma unroll
    for (int n = N, j = 16; n > 1; n /= 2, j /= 2) {
        const bool up = lane & j;
#pragma unroll
        for (int i = 0; i < n / 2; ++i) {
            const float send = up ? k[i] : k[i + n / 2], stay = up ? k[i + n / 2] : k[i];
            k[i] = stay + __shfl_xor_sync(0xFFFFFFFFu, send, j);
        }
    }
    float s = k[0];
#pragma unroll
    for (int j = G / 2; j; j >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, j);
    const int mine = lane / G;         // the value that this lane has: the upper lanes have the upper values
    if (warps > 1) {
        if ((lane & (G - 1)) == 0) part[mine * WARPS + warp] = s;
        row_barrier(id, warps * 32);
        s = 0.f;
#pragma unroll
        for (int i = 0; i < (WARPS + G - 1) / G; ++i) {
            const int w = (lane & (G - 1)) + i * G;
            if (w < warps) s += part[mine * WARPS + w];
        }
#pragma unroll
        for (int j = G / 2; j; j >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, j);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = N == 1 ? s : __shfl_sync(0xFFFFFFFFu, s, i * G);
}

template <class K, class A>
lrbi_status norm_launch(K kernel, int grid, dim3 block, size_t smem, cudaStream_t s, const A &a)
{
    return launch_kernel(kernel, dim3(grid), block, smem, s, 1, a);
}

}  // namespace lrbi
