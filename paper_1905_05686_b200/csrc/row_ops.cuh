// Row-wise building blocks of the layer norm, the 8-bit copies and the activations: how a warp takes columns of a
// row, loads and stores them in 16 or 32 bits, and keeps a group of them in 8 bits.
//
// A warp takes columns in chunks, in one of two ways:
//   vector   a lane has 8 neighbouring columns (a chunk is 256 columns).  Needs rows that start on 16-byte boundaries
//            and a multiple of 8 columns.
//   strided  a lane has columns lane, lane + 32, lane + 64, lane + 96 (a chunk is 128 columns).  Any alignment; every
//            access of the warp is still one run of memory.
// Either way a group of 128 columns (what shares a scale in 8 bits) lies in one warp: 16 neighbouring lanes, or all.
#pragma once
#include "lrbi_common.cuh"

namespace lrbi {

constexpr int KEEP_GROUP = LRBI_CHECKPOINT_GROUP;
// A group whose largest magnitude is below this is kept as zeros: 127 / top would leave the range of fp32.
constexpr float KEEP_TINY = 0x1p-118f;

enum { SRC_BF16 = LRBI_Y_BF16, SRC_F32 = LRBI_Y_F32, SRC_KEPT = 2 };

// Rows of a matrix in device memory: element (r, c) is at data[r * stride + c].
struct RowsIn { const void *data; long long stride; };
struct RowsOut { void *data; long long stride; int dtype; };
// The 8-bit copy: q[r * pitch + c], one scale per group of columns of a row.
struct KeptIn { const int8_t *q; const float *scale; int pitch, groups; };
struct KeptOut { int8_t *q; float *scale; int pitch, groups; };

__device__ __forceinline__ uint4 ld_once16(const void *p)   // read once: does not displace what is read again from L1
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint2 ld_once8(const void *p)
{
    uint2 v;
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)   // round to nearest even, lo in the low half
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// How a lane's chunk maps to columns.
template <bool VEC>
struct Chunk {
    static constexpr int E = VEC ? 8 : 4;            // columns of a lane
    static constexpr int SPAN = VEC ? 256 : 128;     // columns of a warp
    // first column of this lane in the chunk that starts at column c0
    static __device__ __forceinline__ int first(int c0, int lane) { return VEC ? c0 + lane * 8 : c0 + lane; }
    static __device__ __forceinline__ int column(int first, int e) { return VEC ? first + e : first + 32 * e; }
};

// Raw contents of a lane's chunk, as loaded; unpacked when they are used, so that several loads can be under way.
template <int SRC, bool VEC>
struct Raw;

template <bool VEC>
struct Raw<SRC_BF16, VEC> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const RowsIn &x, const KeptIn &, long long row, int c, int cols)
    {
        const uint16_t *p = static_cast<const uint16_t *>(x.data) + row * x.stride;
        if (VEC) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (c < cols) v = ld_once16(p + c);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = c + 32 * e < cols ? (uint32_t)__ldg(p + c + 32 * e) << 16 : 0u;
        }
    }
    __device__ __forceinline__ void get(float (&v)[Chunk<VEC>::E]) const
    {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_lo(w[i]); v[2 * i + 1] = bf16_hi(w[i]); }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(w[e]);
        }
    }
};

template <bool VEC>
struct Raw<SRC_F32, VEC> {
    float w[Chunk<VEC>::E];
    __device__ __forceinline__ void load(const RowsIn &x, const KeptIn &, long long row, int c, int cols)
    {
        const float *p = static_cast<const float *>(x.data) + row * x.stride;
        if constexpr (VEC) {
            uint4 a = make_uint4(0, 0, 0, 0), b = a;
            if (c < cols) { a = ld_once16(p + c); b = ld_once16(p + c + 4); }
            w[0] = __uint_as_float(a.x); w[1] = __uint_as_float(a.y); w[2] = __uint_as_float(a.z); w[3] = __uint_as_float(a.w);
            w[4] = __uint_as_float(b.x); w[5] = __uint_as_float(b.y); w[6] = __uint_as_float(b.z); w[7] = __uint_as_float(b.w);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = c + 32 * e < cols ? __ldg(p + c + 32 * e) : 0.f;
        }
    }
    __device__ __forceinline__ void get(float (&v)[Chunk<VEC>::E]) const
    {
#pragma unroll
        for (int e = 0; e < Chunk<VEC>::E; ++e) v[e] = w[e];
    }
};

// The 8-bit copy stands for q * scale; rows of q start on 16-byte boundaries and end in zeros.
template <bool VEC>
struct Raw<SRC_KEPT, VEC> {
    uint32_t w[VEC ? 2 : 1];
    float scale;
    __device__ __forceinline__ void load(const RowsIn &, const KeptIn &k, long long row, int c, int cols)
    {
        const int8_t *p = k.q + row * k.pitch;
        w[0] = 0; scale = 0.f;
        if constexpr (VEC) {
            w[1] = 0;
            if (c < cols) { const uint2 v = ld_once8(p + c); w[0] = v.x; w[1] = v.y; }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) if (c + 32 * e < cols) w[0] |= (uint32_t)(uint8_t)__ldg(p + c + 32 * e) << (8 * e);
        }
        if (c / KEEP_GROUP < k.groups) scale = __ldg(k.scale + row * k.groups + c / KEEP_GROUP);
    }
    __device__ __forceinline__ void get(float (&v)[Chunk<VEC>::E]) const
    {
#pragma unroll
        for (int e = 0; e < Chunk<VEC>::E; ++e) v[e] = (float)(int8_t)(w[VEC ? e / 4 : 0] >> (8 * (e & 3))) * scale;
    }
};

// Stores a lane's chunk, rounding once (to nearest even) to the output's type.
template <bool VEC>
__device__ __forceinline__ void store_chunk(const RowsOut &y, long long row, int c, int cols, const float (&v)[Chunk<VEC>::E])
{
    if (y.dtype == LRBI_Y_BF16) {
        uint16_t *p = static_cast<uint16_t *>(y.data) + row * y.stride;
        if constexpr (VEC) {
            if (c < cols)
                *reinterpret_cast<uint4 *>(p + c) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) if (c + 32 * e < cols) p[c + 32 * e] = (uint16_t)pack_bf16(v[e], 0.f);
        }
    } else {
        float *p = static_cast<float *>(y.data) + row * y.stride;
        if constexpr (VEC) {
            if (c < cols) {
                *reinterpret_cast<float4 *>(p + c) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4 *>(p + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) if (c + 32 * e < cols) p[c + 32 * e] = v[e];
        }
    }
}

// Keeps a lane's chunk in 8 bits: q = rint(v * (127 / top)), scale = top / 127, top = max |v| over the group.  The
// quotients and the product are single IEEE operations, so the bytes are a function of the values alone.  Magnitudes are
// compared as bit patterns, where a NaN is above infinity and cannot be lost; a group that holds either is kept with the
// scale NaN.  Columns past the last one hold v = 0 here.  Every lane of the warp calls this.
template <bool VEC>
__device__ __forceinline__ void keep_chunk(const KeptOut &k, long long row, int c, const float (&v)[Chunk<VEC>::E])
{
    constexpr int E = Chunk<VEC>::E;
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
#pragma unroll
    for (int j = VEC ? 8 : 16; j; j >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, j));
    const float t = __uint_as_float(top);
    const bool fine = top < 0x7F800000u, low = t < KEEP_TINY;
    const float factor = fine && !low ? __fdiv_rn(127.f, t) : 0.f;
    const float scale = fine ? (low ? 0.f : __fdiv_rn(t, 127.f)) : __uint_as_float(0x7FC00000u);
    uint32_t b[E];
    // adding 1.5 * 2^23 leaves the integer nearest to the product (ties to even) in the low bits
#pragma unroll
    for (int e = 0; e < E; ++e) b[e] = fine ? __float_as_uint(__fadd_rn(__fmul_rn(v[e], factor), 12582912.f)) : 0u;
    int8_t *p = k.q + row * k.pitch;
    if constexpr (VEC) {
        uint2 w;
        w.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
        w.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
        if (c < k.pitch) *reinterpret_cast<uint2 *>(p + c) = w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) if (c + 32 * e < k.pitch) p[c + 32 * e] = (int8_t)b[e];
    }
    if ((c & (KEEP_GROUP - 1)) == 0 && c / KEEP_GROUP < k.groups) k.scale[row * k.groups + c / KEEP_GROUP] = scale;
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int j = 16; j; j >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, j);
    return v;
}

// Host side: whether rows can be taken in vectors of 8 columns.
inline bool rows16(const void *p, long long stride, int dtype)
{
    const long long bytes = dtype == LRBI_Y_F32 ? 4 : 2;
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (stride * bytes & 15) == 0;
}

}  // namespace lrbi
