// Products of a few rows of activations with 4-bit weights, and the quantiser that lays such weights out.
//
//   Y[b][o] = sum over groups g of columns  s[o][g] * sum over i in g of (q[o][i] - z[o][g]) * X[b][i]
//
// The weights are streamed once in the order in which a warp consumes them: a unit is 16 rows x 64 columns = 512 bytes,
// 16 bytes a lane, four words for four m16n8k16 tensor-core steps.  A word's nibbles j and j + 4 sit 16 bits apart, so
// (w >> 4j) & 0x000F000F with the exponent of 128 set gives the pair (128 + q, 128 + q') in bf16 with a shift and one
// logic operation, and subtracting (128 + z) gives q - z exactly: weights and activations enter the product unrounded,
// sums and scales are fp32.
#include "row_ops.cuh"

namespace lrbi {

struct W4 {
    const uint32_t *packed, *meta;
    int rows, cols;
    int units, groups;     // units of 64 columns, groups of columns, per row
};

__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

__device__ __forceinline__ void mma_m16n8k16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Activations of a batch row that a lane needs for a unit: columns c .. c + 7 and c + 32 .. c + 39 (zeros past the last
// column and for rows past the batch).
template <bool VEC>
__device__ __forceinline__ void load_x16(const uint16_t *X, int batch, int cols, int n, int c, uint32_t (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0;
    if (n >= batch) return;
    const uint16_t *p = X + (long long)n * cols;
#pragma unroll
    for (int h = 0; h < 2; ++h, c += 32) {
        if (VEC) {
            if (c < cols) { const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p + c)); x[4 * h] = v.x; x[4 * h + 1] = v.y; x[4 * h + 2] = v.z; x[4 * h + 3] = v.w; }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (c + 2 * i < cols) x[4 * h + i] = __ldg(p + c + 2 * i);
                if (c + 2 * i + 1 < cols) x[4 * h + i] |= (uint32_t)__ldg(p + c + 2 * i + 1) << 16;
            }
        }
    }
}

constexpr int W4_WARPS = 8;

// A block takes 16 rows; its warps split the columns in steps of 128 and add up in shared memory.  NT: tiles of 8 batch rows.
template <int GROUP, int NT, bool VEC>
__global__ void __launch_bounds__(32 * W4_WARPS) w4_gemv_kernel(W4 w, const uint16_t *__restrict__ X, int batch, void *__restrict__ Y, int y_dtype)
{
    __shared__ float4 part[W4_WARPS][NT][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int tile = blockIdx.x, batch0 = blockIdx.y * 8 * NT;
    X += (long long)batch0 * w.cols;
    const int left = batch - batch0;
    const uint4 *packed = reinterpret_cast<const uint4 *>(w.packed) + (long long)tile * w.units * 32 + lane;
    const uint32_t *meta = w.meta + (long long)tile * w.groups * 16 + g;
    float acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = 0.f;
    constexpr int PER = GROUP >= 64 ? 1 : 64 / GROUP;     // groups in a unit
    constexpr int STEPS = 4 / PER;                         // tensor-core steps of a group within a unit
    for (int u0 = warp * 2; u0 < w.units; u0 += W4_WARPS * 2) {
        uint4 q[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) q[h] = u0 + h < w.units ? ld_once16(packed + (long long)(u0 + h) * 32) : make_uint4(0, 0, 0, 0);
        float part_acc[NT][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int u = u0 + h;
            if (u >= w.units) break;
            uint32_t x[NT][8];
#pragma unroll
            for (int n = 0; n < NT; ++n) load_x16<VEC>(X, left, w.cols, n * 8 + g, u * 64 + t * 8, x[n]);
            const uint32_t word[4] = {q[h].x, q[h].y, q[h].z, q[h].w};
#pragma unroll
            for (int p = 0; p < PER; ++p) {
                const int group = min(GROUP == 128 ? u >> 1 : u * PER + p, w.groups - 1);
                const uint32_t lo = __ldg(meta + group * 16), hi = __ldg(meta + group * 16 + 8);
                const uint32_t z_lo = ((lo & 15u) | 0x4300u) * 0x10001u, z_hi = ((hi & 15u) | 0x4300u) * 0x10001u;
                if (GROUP != 128 || h == 0) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) part_acc[n][i] = 0.f;
                }
#pragma unroll
                for (int s = p * STEPS; s < (p + 1) * STEPS; ++s) {
                    uint32_t a[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) a[j] = sub_bf16x2(((word[s] >> (4 * j)) & 0x000F000Fu) | 0x43004300u, j & 1 ? z_hi : z_lo);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma_m16n8k16(part_acc[n], a[0], a[1], a[2], a[3], x[n][2 * s], x[n][2 * s + 1]);
                }
                if (GROUP != 128 || h == 1 || u + 1 == w.units) {
                    const float s_lo = bf16_hi(lo), s_hi = bf16_hi(hi);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        acc[n][0] = fmaf(s_lo, part_acc[n][0], acc[n][0]);
                        acc[n][1] = fmaf(s_lo, part_acc[n][1], acc[n][1]);
                        acc[n][2] = fmaf(s_hi, part_acc[n][2], acc[n][2]);
                        acc[n][3] = fmaf(s_hi, part_acc[n][3], acc[n][3]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) part[warp][n][lane] = make_float4(acc[n][0], acc[n][1], acc[n][2], acc[n][3]);
    __syncthreads();
    // thread -> (batch row, output row): neighbouring threads have neighbouring output rows
    const float *sums = reinterpret_cast<const float *>(part);
    for (int k = threadIdx.x; k < NT * 128; k += 32 * W4_WARPS) {
        const int row = k & 15, b = k >> 4, n = b >> 3, in = b & 7;
        // the sum of (row, column in) is value (row >> 3) * 2 + (in & 1) of lane (row & 7) * 4 + in / 2
        const int at = n * 128 + ((row & 7) * 4 + (in >> 1)) * 4 + (row >> 3) * 2 + (in & 1);
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < W4_WARPS; ++i) v += sums[i * NT * 128 + at];
        const int o = tile * 16 + row;
        if (o < w.rows && b < left) {
            const long long to = (long long)(batch0 + b) * w.rows + o;
            if (y_dtype == LRBI_Y_F32) static_cast<float *>(Y)[to] = v;
            else static_cast<uint16_t *>(Y)[to] = (uint16_t)pack_bf16(v, 0.f);
        }
    }
}

// Quantises a block of 16 rows x 128 columns (bf16) and lays it out.  A group's range is that of its kept weights and
// zero; a pruned weight takes the zero point, so it is exactly zero whatever the array holds at its place.
__global__ void __launch_bounds__(256) w4_quantize_kernel(Geo geo, const uint16_t *__restrict__ W, const uint32_t *__restrict__ ip,
                                                          const uint32_t *__restrict__ iz, int group, uint32_t *__restrict__ packed,
                                                          uint32_t *__restrict__ meta)
{
    __shared__ float value[16][128];
    __shared__ uint8_t kept[16][128], nibble[16][128];
    const int tile = blockIdx.x, c0 = blockIdx.y * 128;
    for (int k = threadIdx.x; k < 16 * 128; k += 256) {
        const int r = k >> 7, j = k & 127, o = tile * 16 + r, c = c0 + j;
        bool keep = o < geo.rows && c < geo.cols;
        float v = 0.f;
        if (keep && ip) {
            const int tr = o / geo.tm, tc = c / geo.tn;
            const long long t = (long long)tr * geo.gc + tc;
            const uint32_t *a = ip + (t * geo.tm + (o - tr * geo.tm)) * geo.kw, *b = iz + (t * geo.tn + (c - tc * geo.tn)) * geo.kw;
            uint32_t any = 0;
            for (int i = 0; i < geo.kw; ++i) any |= a[i] & b[i] & (i == geo.kw - 1 ? tail_mask(geo.k) : 0xFFFFFFFFu);
            keep = any != 0;
        }
        if (keep) v = __uint_as_float((uint32_t)W[(long long)o * geo.cols + c] << 16);
        value[r][j] = v;
        kept[r][j] = keep;
    }
    __syncthreads();
    const int lane = threadIdx.x & 31, groups = (geo.cols + group - 1) / group, per = 128 / group;
    for (int k = threadIdx.x >> 5; k < 16 * per; k += 8) {
        const int r = k / per, p = k - r * per, at = c0 / group + p;
        if (at >= groups) continue;     // the whole warp
        float lo = 0.f, hi = 0.f;
        bool bad = false;
        for (int j = lane; j < group; j += 32) {
            const float v = value[r][p * group + j];
            bad |= !(fabsf(v) <= 3.4e38f);
            lo = fminf(lo, v);
            hi = fmaxf(hi, v);
        }
        for (int j = 16; j; j >>= 1) {
            lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, j));
            hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, j));
        }
        bad = __any_sync(0xFFFFFFFFu, bad);
        const float range = __fsub_rn(hi, lo);
        uint32_t bits = f32_to_bf16_rne(__fdiv_rn(range, 15.f));
        if (bad || !(range <= 3.4e38f)) bits = 0x7FC0u;      // a weight that is not finite, or a range beyond fp32
        const float s = __uint_as_float(bits << 16);
        const bool fine = bits != 0x7FC0u && s > 0.f;
        const int z = fine ? (int)fminf(fmaxf(rintf(__fdiv_rn(-lo, s)), 0.f), 15.f) : 8;
        for (int j = lane; j < group; j += 32) {
            int q = z;
            if (fine && kept[r][p * group + j]) q = (int)fminf(fmaxf(rintf(__fdiv_rn(value[r][p * group + j], s)) + (float)z, 0.f), 15.f);
            nibble[r][p * group + j] = (uint8_t)q;
        }
        if (lane == 0) meta[((long long)tile * groups + at) * 16 + r] = bits << 16 | (uint32_t)z;
    }
    // columns of the last unit that belong to no group
    for (int k = threadIdx.x; k < 16 * 128; k += 256) if (c0 + (k & 127) >= groups * group) nibble[k >> 7][k & 127] = 0;
    __syncthreads();
    const int units = (geo.cols + 63) / 64;
    const int unit = threadIdx.x >> 7, l = (threadIdx.x >> 2) & 31, step = threadIdx.x & 3;
    const int u = blockIdx.y * 2 + unit;
    if (u >= units) return;
    const int g = l >> 2, t = l & 3;
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int r = g + (j & 1) * 8, i = (j >> 1 & 1) * 2 + (j >> 2);
        word |= (uint32_t)nibble[r][unit * 64 + (step >> 1) * 32 + t * 8 + (step & 1) * 4 + i] << (4 * j);
    }
    packed[((long long)tile * units + u) * 128 + threadIdx.x % 128] = word;
}

namespace {

template <int GROUP, int NT>
void gemv_launch(const W4 &w, const uint16_t *X, int batch, void *Y, int y_dtype, bool vec, cudaStream_t s)
{
    const dim3 grid((w.rows + 15) / 16, (batch + 8 * NT - 1) / (8 * NT));
    if (vec) w4_gemv_kernel<GROUP, NT, true><<<grid, 32 * W4_WARPS, 0, s>>>(w, X, batch, Y, y_dtype);
    else w4_gemv_kernel<GROUP, NT, false><<<grid, 32 * W4_WARPS, 0, s>>>(w, X, batch, Y, y_dtype);
}

template <int GROUP>
void gemv_group(const W4 &w, const uint16_t *X, int batch, void *Y, int y_dtype, bool vec, cudaStream_t s)
{
    if (batch <= 8) gemv_launch<GROUP, 1>(w, X, batch, Y, y_dtype, vec, s);
    else gemv_launch<GROUP, 2>(w, X, batch, Y, y_dtype, vec, s);
}

lrbi_status launched()
{
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) { note_cuda_error((int)e); return LRBI_ERR_CUDA; }
    count_launch(1);
    return LRBI_OK;
}

}  // namespace

lrbi_status launch_w4_gemv(const uint32_t *packed, const uint32_t *meta, int rows, int cols, int group, const uint16_t *X, int batch, void *Y,
                           int y_dtype, cudaStream_t s)
{
    const W4 w = {packed, meta, rows, cols, (cols + 63) / 64, (cols + group - 1) / group};
    if ((batch + 15) / 16 > 65535) return LRBI_ERR_UNSUPPORTED;
    const bool vec = cols % 8 == 0 && (reinterpret_cast<uintptr_t>(X) & 15u) == 0;
    if (group == 32) gemv_group<32>(w, X, batch, Y, y_dtype, vec, s);
    else if (group == 64) gemv_group<64>(w, X, batch, Y, y_dtype, vec, s);
    else gemv_group<128>(w, X, batch, Y, y_dtype, vec, s);
    return launched();
}

lrbi_status launch_w4_quantize(const Geo &g, const uint16_t *W, const uint32_t *ip, const uint32_t *iz, int group, uint32_t *packed, uint32_t *meta,
                               cudaStream_t s)
{
    const dim3 grid((g.rows + 15) / 16, (g.cols + 127) / 128);
    if (grid.y > 65535) return LRBI_ERR_UNSUPPORTED;
    w4_quantize_kernel<<<grid, 256, 0, s>>>(g, W, ip, iz, group, packed, meta);
    return launched();
}

}  // namespace lrbi
