// Row-wise building blocks of the layer norm, the 8-bit copies and the activations: how lanes take columns of a row,
// load and store them in 16 or 32 bits, and keep them in 8 bits.
//
// A warp takes 256 columns at a time (a span), 8 a lane (a chunk), in one of two ways:
//   vector    a lane has 8 neighbouring columns: one access of 16 bytes in bf16, of 32 in fp32.  For rows that start on
//             boundaries of that many bytes and hold a multiple of 8 columns.
//   strided   a lane has columns lane, lane + 32, ..: any alignment and any width; an access of the warp is 64 or 128
//             neighbouring bytes.  (Aligned vectors moved into place by shuffles and funnel shifts a value were built too: 35
//             instructions a value in the layer norm against 9.  A leaner form, which settles the shift once for a whole row,
//             was not built.)
// Either way a group of 128 columns (what shares a scale in 8 bits) lies within a span.
#pragma once
#include <type_traits>

#include "lrbi_common.cuh"

namespace lrbi {

constexpr int KEEP_GROUP = LRBI_CHECKPOINT_GROUP;
// A group whose largest magnitude is below this is kept as zeros: 127 / top would leave the range of fp32.
constexpr float KEEP_TINY = 0x1p-118f;

enum { SRC_BF16 = LRBI_Y_BF16, SRC_F32 = LRBI_Y_F32, SRC_KEPT = 2 };
constexpr int CHUNK = 8, SPAN = 32 * CHUNK;   // columns of a lane, of a warp

// First column of a lane in the span that starts at c0, and column e of a chunk that starts at c.
template <bool STRIDED> __device__ __forceinline__ int lane_column(int c0, int lane) { return STRIDED ? c0 + lane : c0 + lane * CHUNK; }
template <bool STRIDED> __device__ __forceinline__ constexpr int chunk_column(int c, int e) { return STRIDED ? c + 32 * e : c + e; }

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
// 32 bytes at once: in two accesses of 16 every 32-byte sector is asked for twice (fp32, 8192 x 4096, with the rings below:
// layer norm 70 us, now 51; its backward 116, now 66).
__device__ __forceinline__ void ld_once32(const void *p, uint32_t (&w)[8])
{
    asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
}
__device__ __forceinline__ void st32(void *p, const float (&f)[8])
{
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]) : "memory");
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

// Two fp32 values that go through the pipeline together: each operation is the IEEE one on both halves, at half the issue
// slots.  The kernels here stream at rates where arithmetic and memory take about the same time.
struct F2 { unsigned long long v; };
__device__ __forceinline__ F2 f2(float a, float b)
{
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ F2 f2(float a) { return f2(a, a); }
__device__ __forceinline__ void split(F2 p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.v)); }
__device__ __forceinline__ F2 operator+(F2 a, F2 b)
{
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 operator*(F2 a, F2 b)
{
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c)
{
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ float sum2(F2 p)
{
    float a, b;
    split(p, a, b);
    return a + b;
}
constexpr int PAIRS = CHUNK / 2;

// Contents of a lane's chunk, as loaded; unpacked when they are used, so that several loads can be under way.  Zeros where
// there is no column.
template <int SRC, bool STRIDED>
struct Raw {
    static constexpr int SIZE = SRC == SRC_F32 ? 4 : 2, WORDS = STRIDED ? CHUNK : CHUNK * SIZE / 4;
    uint32_t w[WORDS];

    static __device__ __forceinline__ uint32_t one(const char *p)     // strided: the value at p
    {
        return SIZE == 4 ? __ldg(reinterpret_cast<const uint32_t *>(p)) : (uint32_t)__ldg(reinterpret_cast<const uint16_t *>(p));
    }

    __device__ __forceinline__ void load(const RowsIn &x, const KeptIn &, long long row, int c, int cols)
    {
        load_at(static_cast<const char *>(x.data) + (row * x.stride + c) * SIZE, cols - c, STRIDED && (c | 31) + 7 * 32 < cols);
    }
    // p: the place of the chunk's first column; `left` columns are there from that one on.  whole: strided, the warp's whole
    // span is there (nothing is checked).
    __device__ __forceinline__ void load_at(const char *p, int left, bool whole = false)
    {
        if constexpr (!STRIDED && SIZE == 4) {
            clear();
            if (left > 0) ld_once32(p, w);
        } else if constexpr (!STRIDED) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (left > 0) v = ld_once16(p);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
            if (whole) {
#pragma unroll
                for (int e = 0; e < CHUNK; ++e) w[e] = one(p + 32 * e * SIZE);
            } else {
#pragma unroll
                for (int e = 0; e < CHUNK; ++e) {
                    w[e] = 0;
                    if (32 * e < left) w[e] = one(p + 32 * e * SIZE);
                }
            }
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void get(F2 (&v)[PAIRS]) const
    {
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            if constexpr (SIZE == 4) v[i] = f2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
            else if constexpr (STRIDED) v[i] = f2(__uint_as_float(w[2 * i] << 16), __uint_as_float(w[2 * i + 1] << 16));
            else v[i] = f2(bf16_lo(w[i]), bf16_hi(w[i]));
        }
    }
    // Largest magnitude as a bit pattern of fp32 (a NaN is above infinity): of the chunk, or of each half of it (its two groups).
    __device__ __forceinline__ void tops(uint32_t (&top)[STRIDED ? 2 : 1]) const
    {
        if constexpr (SIZE == 2 && !STRIDED) {   // both halves of a word at once
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < WORDS; ++i) m = __vmaxu2(m, w[i] & 0x7FFF7FFFu);
            top[0] = max(m << 16, m & 0xFFFF0000u);
        } else {
#pragma unroll
            for (int h = 0; h < (STRIDED ? 2 : 1); ++h) {
                uint32_t m = 0;
#pragma unroll
                for (int i = 0; i < WORDS / (STRIDED ? 2 : 1); ++i) m = max(m, w[h * WORDS / 2 + i] & (SIZE == 4 ? 0x7FFFFFFFu : 0x7FFFu));
                top[h] = SIZE == 4 ? m : m << 16;
            }
        }
    }
};

// The 8-bit copy stands for q * scale; its rows start on 16-byte boundaries, and q is 0 past the last column.
template <bool STRIDED>
struct Raw<SRC_KEPT, STRIDED> {
    uint32_t w[STRIDED ? CHUNK : 2];
    float scale[STRIDED ? 2 : 1];
    __device__ __forceinline__ void load(const RowsIn &, const KeptIn &k, long long row, int c, int cols)
    {
        clear();
        if constexpr (!STRIDED) {
            if (c < cols) {
                const uint2 v = ld_once8(k.q + row * k.pitch + c);
                w[0] = v.x;
                w[1] = v.y;
                scale[0] = __ldg(k.scale + row * k.groups + c / KEEP_GROUP);
            }
        } else {
            const int8_t *p = k.q + row * k.pitch + c;
            const float *s = k.scale + row * k.groups + c / KEEP_GROUP;
            if ((c | 31) + 7 * 32 < cols) {
#pragma unroll
                for (int e = 0; e < CHUNK; ++e) w[e] = (uint32_t)(int)__ldg(p + 32 * e);
                scale[0] = __ldg(s);
                scale[1] = __ldg(s + 1);
            } else {
#pragma unroll
                for (int e = 0; e < CHUNK; ++e) if (c + 32 * e < cols) w[e] = (uint32_t)(int)__ldg(p + 32 * e);
#pragma unroll
                for (int h = 0; h < 2; ++h) if ((c | 31) - 31 + h * KEEP_GROUP < cols) scale[h] = __ldg(s + h);
            }
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < (STRIDED ? CHUNK : 2); ++i) w[i] = 0;
#pragma unroll
        for (int h = 0; h < (STRIDED ? 2 : 1); ++h) scale[h] = 0.f;
    }
    __device__ __forceinline__ void get(F2 (&v)[PAIRS]) const
    {
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            if constexpr (STRIDED) v[i] = f2((float)(int)w[2 * i], (float)(int)w[2 * i + 1]) * f2(scale[i / 2]);
            else {
                const uint32_t q = w[i / 2] >> (16 * (i & 1));
                v[i] = f2((float)(int8_t)q, (float)(int8_t)(q >> 8)) * f2(scale[0]);
            }
        }
    }
};

// Kernels here are launched so that their blocks may be set up while the kernel before them in the stream drains: every
// thread calls begin() first, which waits until that kernel is through with memory, and let_next() where the next kernel's
// blocks may come (early in short kernels, towards the end of long ones: blocks that come while others still run fill the
// SMs unevenly).  On calls of a few microseconds the gap between two kernels is a good part of the time.
__device__ __forceinline__ void begin() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// The lane, as a value that stays in a register: out of threadIdx.x the compiler reads it from its special register again and
// again where registers are short (60 times a row in the layer norm), and spills more for it.
__device__ __forceinline__ int kept_lane() { return __shfl_sync(0xFFFFFFFFu, threadIdx.x & 31, threadIdx.x & 31); }
__device__ __forceinline__ int kept(int v) { return __shfl_sync(0xFFFFFFFFu, v, 0); }      // what is the same in all lanes

// Asynchronous copies into shared memory: later rows are under way without registers to wait for them.
__device__ __forceinline__ void copy_async(uint32_t to, const void *from, int bytes)   // bytes: 4 or 16
{
    if (bytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_async_if(bool on, uint32_t to, const void *from)      // 16 bytes; a predicate, not a branch
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}" ::"r"(to), "l"(from), "r"((uint32_t)on) : "memory");
}
__device__ __forceinline__ void copy_async_some(uint32_t to, const void *from, int bytes)   // 1 to 16, and zeros up to 16
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
// A span of fp32 vectors goes over in two accesses of 512 neighbouring bytes: a lane copies 16 bytes of either (from its byte
// 512 i + 16 lane) and reads its own 32 bytes after the warp's copies are there.  Vectors are placed so that neither has bank
// conflicts: copies at fp32_copied(lane) + 512 i, read at fp32_read(lane, i).
__device__ __forceinline__ int fp32_copied(int lane) { return (lane ^ (lane >> 3 & 1)) * 16; }
__device__ __forceinline__ int fp32_read(int lane, int i) { return lane * 32 + (i ^ (lane >> 2 & 1)) * 16; }
__device__ __forceinline__ void copies_asked() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>   // all but the last LEFT groups are there
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// Stores a lane's chunk at p, the place of its first column; `left` columns are there from that one on (none: 0 or less).
template <int SIZE, bool STRIDED>
__device__ __forceinline__ void store_at(char *p, int left, const F2 (&v)[PAIRS], bool whole = false)
{
    if constexpr (STRIDED) {
        auto put = [&](auto all) {
            constexpr bool ALL = decltype(all)::value;
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                float lo, hi;
                split(v[i], lo, hi);
                if (SIZE == 4) {
                    if (ALL || 64 * i < left) *(reinterpret_cast<float *>(p) + 64 * i) = lo;
                    if (ALL || 64 * i + 32 < left) *(reinterpret_cast<float *>(p) + 64 * i + 32) = hi;
                } else {
                    const uint32_t w = pack_bf16(lo, hi);
                    if (ALL || 64 * i < left) *(reinterpret_cast<uint16_t *>(p) + 64 * i) = (uint16_t)w;
                    if (ALL || 64 * i + 32 < left) *(reinterpret_cast<uint16_t *>(p) + 64 * i + 32) = (uint16_t)(w >> 16);
                }
            }
        };
        if (whole) put(std::true_type());
        else put(std::false_type());
    } else if (left > 0) {
        float f[CHUNK];
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) split(v[i], f[2 * i], f[2 * i + 1]);
        if (SIZE == 4) st32(p, f);
        else
            *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    }
}

// Stores a lane's chunk, rounding once (to nearest even) to the output's type.
template <bool STRIDED>
__device__ __forceinline__ void store_chunk(const RowsOut &y, long long row, int c, int cols, const F2 (&v)[PAIRS])
{
    const bool whole = STRIDED && (c | 31) + 7 * 32 < cols;
    if (y.dtype == LRBI_Y_BF16) store_at<2, STRIDED>(static_cast<char *>(y.data) + (row * y.stride + c) * 2, cols - c, v, whole);
    else store_at<4, STRIDED>(static_cast<char *>(y.data) + (row * y.stride + c) * 4, cols - c, v, whole);
}

// Keeping chunks in 8 bits: q = rint(v * (127 / top)), scale = top / 127, top = max |v| over the group.  Four groups go
// together, so that their maxima share shuffles and all their divisions are one: vector, the groups of four chunks in either
// half warp; strided, the two groups of two chunks over the warp.  The quotients and the product are single IEEE operations,
// so the bytes are a function of the values alone.  Magnitudes are compared as bit patterns, where a NaN is above infinity
// and cannot be lost; a group that holds either is kept with the scale NaN.  Columns past the last one hold 0.
template <bool STRIDED>
struct Keep {
    static constexpr int L = STRIDED ? 32 : 16, EACH = L / 4, CHUNKS = STRIDED ? 2 : 4;   // lanes of four groups, of one in the end; chunks at a time
    float quotient;      // even lanes of a group 127 / top, odd ones the scale

    // tops: of the chunks in turn (strided: of each chunk's two groups); by every lane of the warp
    __device__ __forceinline__ Keep(const uint32_t (&tops)[4], int lane)
    {
        const bool up = lane & (L / 2), up2 = lane & (L / 4);
        const uint32_t a = max(up ? tops[2] : tops[0], __shfl_xor_sync(0xFFFFFFFFu, up ? tops[0] : tops[2], L / 2));
        const uint32_t b = max(up ? tops[3] : tops[1], __shfl_xor_sync(0xFFFFFFFFu, up ? tops[1] : tops[3], L / 2));
        uint32_t top = max(up2 ? b : a, __shfl_xor_sync(0xFFFFFFFFu, up2 ? a : b, L / 4));
#pragma unroll
        for (int j = EACH / 2; j; j >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, j));
        const float t = __uint_as_float(top);
        const bool fine = top < 0x7F800000u && t >= KEEP_TINY, odd = lane & 1;
        quotient = fine ? __fdiv_rn(odd ? t : 127.f, odd ? 127.f : t) : top < 0x7F800000u ? 0.f : __uint_as_float(0x7FC00000u);
    }
    // The scale that this lane stores, if any: of chunk `chunk`, group `group` of the chunk's span.
    static __device__ __forceinline__ bool stores(int lane) { return lane % EACH == 1; }
    static __device__ __forceinline__ int chunk(int lane) { return STRIDED ? lane / EACH / 2 : lane % L / EACH; }
    static __device__ __forceinline__ int group(int lane) { return STRIDED ? lane / EACH & 1 : lane / L; }

    // The bytes of chunk `i`: at `to`, the place of its first column, `left` bytes from there on.
    __device__ __forceinline__ void bytes(int i, int8_t *to, int left, const F2 (&v)[PAIRS]) const
    {
        float factors[2];
        factors[0] = __shfl_sync(0xFFFFFFFFu, quotient, (STRIDED ? 2 * i : i) * EACH, L);
        factors[1] = STRIDED ? __shfl_sync(0xFFFFFFFFu, quotient, (2 * i + 1) * EACH, L) : factors[0];
        uint32_t b[CHUNK];
        // Adding 1.5 * 2^23 leaves the integer nearest to the product (ties to even) in the low bits.  The product is rounded
        // first: the sum is a scalar one, since a packed product and a packed sum came out as one fused step.
#pragma unroll
        for (int j = 0; j < PAIRS; ++j) {
            float lo, hi;
            split(v[j] * f2(factors[STRIDED ? j / 2 : 0]), lo, hi);
            b[2 * j] = __float_as_uint(__fadd_rn(lo, 12582912.f));
            b[2 * j + 1] = __float_as_uint(__fadd_rn(hi, 12582912.f));
        }
        if constexpr (STRIDED) {
#pragma unroll
            for (int e = 0; e < CHUNK; ++e)
                if (32 * e < left) to[32 * e] = factors[e / 4] == factors[e / 4] ? (int8_t)b[e] : (int8_t)0;
        } else {
            uint2 w;
            w.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
            w.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
            if (!(factors[0] == factors[0])) w = make_uint2(0, 0);
            if (left > 0) *reinterpret_cast<uint2 *>(to) = w;
        }
    }
};

// One chunk by itself, in the span at c0.
template <int SRC, bool STRIDED>
__device__ __forceinline__ void keep_chunk(const KeptOut &k, long long row, int c0, int lane, const F2 (&v)[PAIRS], const Raw<SRC, STRIDED> &raw)
{
    uint32_t own[STRIDED ? 2 : 1], tops[4] = {0, 0, 0, 0};
    raw.tops(own);
    tops[0] = own[0];
    if (STRIDED) tops[1] = own[STRIDED ? 1 : 0];
    const Keep<STRIDED> keep(tops, lane);
    const int c = lane_column<STRIDED>(c0, lane), group = c0 / KEEP_GROUP + Keep<STRIDED>::group(lane);
    keep.bytes(0, k.q + row * k.pitch + c, k.pitch - c, v);
    if (Keep<STRIDED>::stores(lane) && Keep<STRIDED>::chunk(lane) == 0 && group < k.groups) k.scale[row * k.groups + group] = keep.quotient;
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int j = 16; j; j >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, j);
    return v;
}

// Host side: lets a kernel have `smem` bytes of dynamic shared memory on the current device; asked once for what is enough.
// (The most that was allowed is kept by kernel and device: pointers of kernels are few.)
cudaError_t allow_shared(const void *kernel, size_t smem);
template <class... A>
cudaError_t allow_shared(void (*kernel)(A...), size_t smem) { return allow_shared(reinterpret_cast<const void *>(kernel), smem); }

// Host side: blocks of a kernel that an SM of the current device takes at once, 1 where it does not say.
int blocks_per_sm(const void *kernel, int threads, size_t smem);
template <class... A>
int blocks_per_sm(void (*kernel)(A...), int threads, size_t smem) { return blocks_per_sm(reinterpret_cast<const void *>(kernel), threads, smem); }

// Host side: launches a kernel that calls begin(), with `smem` bytes of dynamic shared memory and clusters of `cluster` blocks.
template <class K, class... A>
lrbi_status launch_kernel(K kernel, dim3 grid, dim3 block, size_t smem, cudaStream_t s, unsigned cluster, const A &...a)
{
    cudaError_t e = cudaSuccess;
    if (smem > 32 * 1024) e = allow_shared(kernel, smem);      // 48 KB are free, with static arrays
    cudaLaunchConfig_t c = {};
    c.gridDim = grid;
    c.blockDim = block;
    c.dynamicSmemBytes = smem;
    c.stream = s;
    cudaLaunchAttribute attribute[2] = {};
    attribute[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attribute[0].val.programmaticStreamSerializationAllowed = 1;
    attribute[1].id = cudaLaunchAttributeClusterDimension;
    attribute[1].val.clusterDim.x = cluster;
    attribute[1].val.clusterDim.y = attribute[1].val.clusterDim.z = 1;
    c.attrs = attribute;
    c.numAttrs = cluster > 1 ? 2 : 1;
    if (e == cudaSuccess) e = cudaLaunchKernelEx(&c, kernel, a...);
    if (e != cudaSuccess) { note_cuda_error((int)e); return LRBI_ERR_CUDA; }
    count_launch();
    return LRBI_OK;
}

// Host side: whether rows are whole vectors.
inline bool vector_rows(const void *p, long long stride, int dtype)
{
    const long long size = dtype == LRBI_Y_F32 ? 4 : 2, vector = CHUNK * size;
    return reinterpret_cast<uintptr_t>(p) % vector == 0 && stride * size % vector == 0;
}

}  // namespace lrbi
