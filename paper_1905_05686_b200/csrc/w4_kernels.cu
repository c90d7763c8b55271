// Products of a few rows of activations with 4-bit weights, and the quantiser that lays such weights out.
//
//   Y[b][o] = sum over groups g of columns  s[o][g] * sum over i in g of (q[o][i] - z[o][g]) * X[b][i]
//
// The weights are streamed once in the order in which a warp consumes them: a unit is 16 rows x 64 columns = 512 bytes,
// 16 bytes a lane, four words for four m16n8k16 tensor-core steps.  A word's nibbles j and j + 4 sit 16 bits apart, so
// (w >> 4j) & 0x000F000F with the exponent of 128 set gives the pair (128 + q, 128 + q') in bf16 with a shift and one
// logic operation, and subtracting (128 + z) gives q - z exactly: weights and activations enter the product unrounded,
// sums and scales are fp32.
#include <cfloat>
#include <type_traits>

#include "row_ops.cuh"

namespace lrbi {

struct W4 {
    const uint32_t *packed, *meta;
    int rows, cols;
    int units, groups;     // units of 64 columns, groups of columns, per row
};

// (128 + nibble j, 128 + nibble j + 4) in bf16, less (z, z): z holds 128 + zero point twice.
__device__ __forceinline__ uint32_t nibbles(uint32_t word, int j, uint32_t z)
{
    uint32_t r;
    asm("{\n\t.reg .b32 s, t;\n\tshr.b32 s, %1, %2;\n\tlop3.b32 t, s, %3, %4, 0xEA;\n\tsub.rn.bf16x2 %0, t, %5;\n\t}"     // 0xEA: (a & b) | c
        : "=r"(r) : "r"(word), "r"(4 * j), "r"(0x000F000Fu), "r"(0x43004300u), "r"(z));
    return r;
}

__device__ __forceinline__ void mma_m16n8k16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bool first)
{
    if (first)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                     : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Two 16-byte loads, 64 bytes apart, where `on`; the registers stay as they are elsewhere.  (As one predicate, not a branch.)
__device__ __forceinline__ void load_pair(const uint16_t *p, bool on, uint32_t (&x)[8])
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %9, 0;\n\t@q ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%8];\n\t@q ld.global.nc.v4.u32 {%4, %5, %6, %7}, [%8+64];\n\t}"
                 : "+r"(x[0]), "+r"(x[1]), "+r"(x[2]), "+r"(x[3]), "+r"(x[4]), "+r"(x[5]), "+r"(x[6]), "+r"(x[7]) : "l"(p), "r"((uint32_t)on));
}
__device__ __forceinline__ void copy_async16(uint32_t to, const void *from, bool on)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t@q cp.async.cg.shared.global [%0], [%1], 16;\n\t}" ::"r"(to), "l"(from), "r"((uint32_t)on) : "memory");
}
__device__ __forceinline__ void copy_async32(uint32_t to, const void *from, bool on)     // and 512 bytes on
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t@q cp.async.cg.shared.global [%0], [%1], 16;\n\t@q cp.async.cg.shared.global [%0+512], [%1+512], 16;\n\t}"
                 ::"r"(to), "l"(from), "r"((uint32_t)on) : "memory");
}

__device__ __forceinline__ void copy_activations(uint32_t to, const uint16_t *from, bool on)     // four pieces, 64 bytes apart, to places 512 bytes apart
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t@q cp.async.cg.shared.global [%0], [%1], 16;\n\t@q cp.async.cg.shared.global [%0+512], [%1+64], 16;\n\t"
                 "@q cp.async.cg.shared.global [%0+1024], [%1+128], 16;\n\t@q cp.async.cg.shared.global [%0+1536], [%1+192], 16;\n\t}"
                 ::"r"(to), "l"(from), "r"((uint32_t)on) : "memory");
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

constexpr int W4_WARPS = 8, W4_STEP = 128;                       // warps of a block; columns that a warp takes at a time

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ float cluster_load(const float *mine, uint32_t rank)   // the same place in another block of the cluster
{
    uint32_t at = (uint32_t)__cvta_generic_to_shared(mine), there;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(there) : "memory");
    return v;
}

__device__ __forceinline__ void store(const W4 &w, void *Y, int y_dtype, int o, int b, int batch, float v)
{
    if (o >= w.rows || b >= batch) return;
    const long long to = (long long)b * w.rows + o;
    if (y_dtype == LRBI_Y_F32) static_cast<float *>(Y)[to] = v;
    else static_cast<uint16_t *>(Y)[to] = (uint16_t)pack_bf16(v, 0.f);
}

// Whether the activations go through the ring too (one tile a warp: 4096 x 9216 7.7 -> 7.4 us; two tiles hide the loads of
// registers themselves and lose by it: 16384 x 4096, eight rows, 11.9 -> 13.1), how many steps it has room for, and the bytes of one.
template <int NT, int TILES, bool VEC> constexpr bool W4_X_RING = VEC && NT == 1 && TILES == 1;
template <int NT, int TILES, bool VEC> constexpr int W4_DEPTH = TILES == 1 && !W4_X_RING<NT, TILES, VEC> ? 4 : 3;
template <int GROUP, int NT, int TILES, bool VEC> constexpr int W4_SLOT = TILES * (1024 + W4_STEP / GROUP * 64) + (W4_X_RING<NT, TILES, VEC> ? 2048 : 0);

// `sharing` warps of a block (and of each block of a cluster) take TILES * 16 rows: the columns in turn, in steps of 128, and
// add up in shared memory, block by block and then over the cluster, in a fixed order that depends on the layer alone.  A step's
// weights come through a ring of asynchronous copies, the activations too or a step ahead in registers.  NT: tiles of 8 batch rows.
//
// Bound: on paper the weights' bytes (16384 x 16384, one row: 21.5 us).  Measured 33.7 us, and 30.0 with every load taken out.
// No one unit is full: the kernel issues in half of the slots and waits for memory longest.  What is known to cost time:
// turning four bits into bf16 (a shift, a logic operation and a subtraction for two weights; leaving the 128 + z in and taking
// it out of the sums would save the subtraction, and pruned weights would no longer be exact zeros), and the cut in whole
// tiles: 256 blocks, as the common sizes have, give 108 SMs two and 40 one, so that the busiest has 1 / 0.865 of the mean, in
// the 30.0 us too.  The smaller layers add about 2 us of launch and first latency.  Activations that are not whole vectors
// (columns not a multiple of 8, or X not on a 16-byte boundary) are loaded a value at a time: 4096 x 9216, one row, 16.3 us
// (7.4), 16384 x 4096, eight rows, 26.6 (12.1).
template <int GROUP, int NT, int TILES, bool VEC>
__global__ void __launch_bounds__(32 * W4_WARPS, NT > 1 || TILES > 1 ? 2 : VEC ? 3 : 4) w4_gemv_kernel(W4 w, const uint16_t *__restrict__ X, int batch, void *__restrict__ Y, int y_dtype, int sharing)
{
    begin();
    constexpr int PER = W4_STEP / GROUP, IN_UNIT = GROUP >= 64 ? 1 : 64 / GROUP, MMAS = 4 / IN_UNIT;   // groups of a step, of a unit; products of a group in a unit
    constexpr bool X_RING = W4_X_RING<NT, TILES, VEC>;
    constexpr int DEPTH = W4_DEPTH<NT, TILES, VEC>;                   // steps under way, with the one that is worked on
    constexpr int TILE = 1024 + PER * 64, SLOT = W4_SLOT<GROUP, NT, TILES, VEC>;     // bytes of a step: weights, then scales and zero points, of each tile; activations
    extern __shared__ __align__(16) char ring[];                      // [W4_WARPS][DEPTH][SLOT]
    __shared__ float4 part[W4_WARPS][TILES][NT][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int ranks = cluster_size(), rank = cluster_rank(), side = W4_WARPS / sharing;
    const int all_tiles = (w.rows + 15) / 16, tile0 = blockIdx.x / ranks * side * TILES, tile = tile0 + warp / sharing * TILES;   // of the block, of this warp
    const bool two = TILES == 1 || tile + 1 < all_tiles;      // the second tile is there
    const int batch0 = blockIdx.y * 8 * NT, left = batch - batch0;
    const int steps = tile < all_tiles ? (w.units + 1) / 2 : 0, stride = sharing * ranks, whole = min(steps, w.cols / W4_STEP);      // steps of 128 columns that are all there
    X += (long long)batch0 * w.cols;
    int step = rank * sharing + warp % sharing;
    const char *packed = reinterpret_cast<const char *>(w.packed) + ((long long)tile * w.units * 512 + (long long)step * 1024 + lane * 16);
    const char *meta = reinterpret_cast<const char *>(w.meta) + ((long long)tile * w.groups * 64 + (long long)step * PER * 64 + lane * 16);
    const uint16_t *from = X + (long long)g * w.cols + step * W4_STEP + t * 8;
    char *slots = ring + warp * DEPTH * SLOT;
    const uint32_t slots_lane = (uint32_t)__cvta_generic_to_shared(slots) + lane * 16;
    const long long packed_tile = (long long)w.units * 512, meta_tile = (long long)w.groups * 64;
    int asked = step;
    // Whole steps go through the ring.
    auto ask = [&](int at) {
        const bool on = asked < whole;
#pragma unroll
        for (int r = 0; r < TILES; ++r) {
            const uint32_t to = slots_lane + at * SLOT + r * TILE;
            copy_async32(to, packed + r * packed_tile, on && (r == 0 || two));
            copy_async16(to + 1024, meta + r * meta_tile, on && (r == 0 || two) && lane < PER * 4);
        }
        if (X_RING) {
            copy_activations(slots_lane + at * SLOT + TILES * TILE, from, on && g < left);
            from += stride * W4_STEP;
        }
        copies_asked();
        asked += stride;
        packed += stride * 1024;
        meta += stride * PER * 64;
    };
    float acc[TILES][NT][4];
    uint32_t x[2][NT][8];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int i = 0; i < 4 * TILES; ++i) acc[i / 4][n][i & 3] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[0][n][i] = x[1][n][i] = 0;      // rows past the batch stay zero
    }
    // Activations of a step: for each half of 64 columns the lane's 8 columns of either 32.
    auto activations = [&](int s) {
        if (VEC) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) load_pair(from + (long long)n * 8 * w.cols + h * 64, s < whole && n * 8 + g < left, x[h][n]);
        } else if (s < whole) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int n = 0; n < NT; ++n) load_x16<VEC>(X, left, w.cols, n * 8 + g, s * W4_STEP + h * 64 + t * 8, x[h][n]);
        }
        from += stride * W4_STEP;
    };
    // The products of a step; all: both of its units and all of its groups are there.
    auto products = [&](const char *places, auto all) {
        constexpr bool ALL = decltype(all)::value;
#pragma unroll
        for (int r = 0; r < TILES; ++r) {
        const char *slot = places + r * TILE;
        const uint32_t *own = reinterpret_cast<const uint32_t *>(slot + 1024) + g;
        float sum[NT][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (!ALL && step * 2 + h >= w.units) break;
            const uint4 q = *reinterpret_cast<const uint4 *>(slot + h * 512 + lane * 16);
            const uint32_t word[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int p = 0; p < IN_UNIT; ++p) {
                const int group = GROUP == 128 ? 0 : h * IN_UNIT + p;
                const bool there = ALL || step * PER + group < w.groups;
                const uint32_t lo = there ? own[group * 16] : 0u, hi = there ? own[group * 16 + 8] : 0u;
                const uint32_t z_lo = ((lo & 15u) | 0x4300u) * 0x10001u, z_hi = ((hi & 15u) | 0x4300u) * 0x10001u;
#pragma unroll
                for (int m = p * MMAS; m < (p + 1) * MMAS; ++m) {
                    uint32_t a[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) a[j] = nibbles(word[m], j, j & 1 ? z_hi : z_lo);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma_m16n8k16(sum[n], a, x[h][n][2 * m], x[h][n][2 * m + 1], m == p * MMAS && (GROUP != 128 || h == 0));
                }
                if (GROUP != 128 || h == 1 || (!ALL && step * 2 + 1 == w.units)) {
                    const float s_lo = bf16_hi(lo), s_hi = bf16_hi(hi);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        acc[r][n][0] = fmaf(s_lo, sum[n][0], acc[r][n][0]);
                        acc[r][n][1] = fmaf(s_lo, sum[n][1], acc[r][n][1]);
                        acc[r][n][2] = fmaf(s_hi, sum[n][2], acc[r][n][2]);
                        acc[r][n][3] = fmaf(s_hi, sum[n][3], acc[r][n][3]);
                    }
                }
            }
        }
        }
    };
    if (X_RING && g >= left) {              // rows past the batch
#pragma unroll
        for (int i = 0; i < DEPTH * 4; ++i) *reinterpret_cast<uint4 *>(slots + i / 4 * SLOT + TILES * TILE + i % 4 * 512 + lane * 16) = make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < DEPTH - 1; ++i) ask(i);
    if (!X_RING) activations(step);
    while (step < whole) {
#pragma unroll
        for (int at = 0; at < DEPTH; ++at) {
            if (step >= whole) break;
            ask((at + DEPTH - 1) % DEPTH);
            copies_wait<DEPTH - 1>();
            __syncwarp();                   // scales and zero points were copied by other lanes
            if (X_RING) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 v = *reinterpret_cast<const uint4 *>(slots + at * SLOT + TILES * TILE + i * 512 + lane * 16);
                    uint32_t *to = x[i / 2][0] + i % 2 * 4;
                    to[0] = v.x; to[1] = v.y; to[2] = v.z; to[3] = v.w;
                }
            }
            products(slots + at * SLOT, std::true_type());
            step += stride;
            if (!X_RING) activations(step);
            __syncwarp();                   // before the place is asked for again
        }
    }
    let_next();
    copies_wait<0>();
    if (step < steps) {                     // the last step, where it is not whole: units and groups that are there
        __syncwarp();
        const char *p = reinterpret_cast<const char *>(w.packed) + (long long)tile * packed_tile + (long long)step * 1024 + lane * 16;
        const char *m = reinterpret_cast<const char *>(w.meta) + (long long)tile * meta_tile + (long long)step * PER * 64 + lane * 16;
#pragma unroll
        for (int r = 0; r < TILES; ++r) {
            const bool on = r == 0 || two;
            copy_async16(slots_lane + r * TILE, p + r * packed_tile, on);
            copy_async16(slots_lane + r * TILE + 512, p + r * packed_tile + 512, on && step * 2 + 1 < w.units);
            copy_async16(slots_lane + r * TILE + 1024, m + r * meta_tile, on && lane < PER * 4 && step * PER + lane / 4 < w.groups);
        }
        copies_asked();
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int n = 0; n < NT; ++n) load_x16<VEC>(X, left, w.cols, n * 8 + g, step * W4_STEP + h * 64 + t * 8, x[h][n]);
        copies_wait<0>();
        __syncwarp();
        products(slots, std::false_type());
    }
    __syncthreads();                        // the ring may be written anew
#pragma unroll
    for (int r = 0; r < TILES; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) part[warp][r][n][lane] = make_float4(acc[r][n][0], acc[r][n][1], acc[r][n][2], acc[r][n][3]);
    __syncthreads();
    // thread -> (batch row, output row): neighbouring threads have neighbouring output rows
    const float *sums = reinterpret_cast<const float *>(part);
    constexpr int ALL = TILES * NT * 128;
    const int rows = side * TILES * 16, outputs = rows * NT * 8;
    float *block = reinterpret_cast<float *>(ring);             // the ring is through
    for (int k = threadIdx.x; k < outputs; k += 32 * W4_WARPS) {
        // the sum of (row, batch row b) is value (row >> 3) * 2 + (b & 1) of lane (row & 7) * 4 + (b & 7) / 2 of tile b >> 3
        const int row = k % rows, b = k / rows, in = b & 7, r = row >> 4;
        const int value = ((r % TILES) * NT + (b >> 3)) * 128 + ((row & 7) * 4 + (in >> 1)) * 4 + (row >> 3 & 1) * 2 + (in & 1);
        float v = 0.f;
        for (int i = 0; i < sharing; ++i) v += sums[(r / TILES * sharing + i) * ALL + value];
        if (ranks > 1) block[k] = v;
        else store(w, Y, y_dtype, tile0 * 16 + row, batch0 + b, batch, v);
    }
    if (ranks == 1) return;
    cluster_barrier();
    if (rank == 0)
        for (int k = threadIdx.x; k < outputs; k += 32 * W4_WARPS) {
            float v = block[k];
            for (int r = 1; r < ranks; ++r) v += cluster_load(block + k, r);
            store(w, Y, y_dtype, tile0 * 16 + k % rows, batch0 + k / rows, batch, v);
        }
    cluster_barrier();                      // the other blocks' sums are read before they end
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
            bad |= !(fabsf(v) <= FLT_MAX);
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
        if (bad || !(range <= FLT_MAX)) bits = 0x7FC0u;      // a weight that is not finite, or a range beyond fp32
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

// How a layer is cut: warps of a block that share a tile, and blocks (of a cluster) that do.
struct Cut { int sharing, split; };
Cut gemv_cut(const W4 &w, int at_once)      // at_once: tiles of a warp
{
    constexpr int SMS = 148;
    const int tiles = (w.rows + 15) / 16, steps = (w.units + 1) / 2;
    auto blocks = [&](int sharing) { const int each = at_once * (W4_WARPS / sharing); return (tiles + each - 1) / each; };
    auto most = [&](int sharing) { return (blocks(sharing) + SMS - 1) / SMS * at_once * (W4_WARPS / sharing); };      // tiles of the SM that has the most
    Cut c = {W4_WARPS, 1};
    // Fewer warps share a tile, and each has more steps of it, as long as the SMs have two blocks or more and the one that has
    // the most tiles hardly more of them.  16384 x 4096: 4 warps 11.1 us, 8 or 2 12.8; 12000 x 9216 (with 4, a few SMs have two
    // blocks and most one): 8 warps 17.1, 4 19.7; 8192 x 8192, eight rows: 8 warps 11.5, 4 16.8.
    while (c.sharing > 1 && blocks(c.sharing / 2) > SMS && most(c.sharing / 2) * 7 <= most(c.sharing) * 8) c.sharing /= 2;
    // Layers of few tiles: blocks share one, while a warp has four steps or more.  64 x 16384: 8 blocks 3.3 us, 4 3.8, 2 4.9;
    // 1024 x 4096: 1 block 3.1, 2 3.3, 4 3.8; 1024 x 8192: 1 4.7, 2 4.4, 4 4.4.
    while (c.split < 8 && tiles * c.split < SMS && steps >= 4 * c.split * W4_WARPS) c.split *= 2;
    return c;
}

template <int GROUP, int NT, int TILES, bool VEC>
lrbi_status gemv_launch(const W4 &w, const uint16_t *X, int batch, void *Y, int y_dtype, cudaStream_t s)
{
    const Cut cut = gemv_cut(w, TILES);
    const int rows = 16 * TILES * (W4_WARPS / cut.sharing), split = cut.split;      // of a block
    constexpr size_t smem = (size_t)W4_WARPS * W4_DEPTH<NT, TILES, VEC> * W4_SLOT<GROUP, NT, TILES, VEC>;
    return launch_kernel(w4_gemv_kernel<GROUP, NT, TILES, VEC>, dim3((w.rows + rows - 1) / rows * split, (batch + 8 * NT - 1) / (8 * NT)), dim3(32 * W4_WARPS), smem, s,
                         split, w, X, batch, Y, y_dtype, cut.sharing);
}

template <int GROUP, int NT>
lrbi_status gemv_tiles(const W4 &w, const uint16_t *X, int batch, void *Y, int y_dtype, bool vec, cudaStream_t s)
{
    // Two tiles a warp share what is loaded of the activations, where every SM still has a block.  6000 x 4096, eight rows:
    // 7.6 us, one tile 8.3; 5000 x 9216, sixteen rows: 16.1 and 18.4; with 4500 rows there are 141 blocks: 6.0 and 4.9.
    if ((w.rows + 15) / 16 >= 2 * 148)
        return vec ? gemv_launch<GROUP, NT, 2, true>(w, X, batch, Y, y_dtype, s) : gemv_launch<GROUP, NT, 2, false>(w, X, batch, Y, y_dtype, s);
    return vec ? gemv_launch<GROUP, NT, 1, true>(w, X, batch, Y, y_dtype, s) : gemv_launch<GROUP, NT, 1, false>(w, X, batch, Y, y_dtype, s);
}

template <int GROUP>
lrbi_status gemv_group(const W4 &w, const uint16_t *X, int batch, void *Y, int y_dtype, bool vec, cudaStream_t s)
{
    return batch <= 8 ? gemv_tiles<GROUP, 1>(w, X, batch, Y, y_dtype, vec, s) : gemv_tiles<GROUP, 2>(w, X, batch, Y, y_dtype, vec, s);
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
    if (group == 32) return gemv_group<32>(w, X, batch, Y, y_dtype, vec, s);
    if (group == 64) return gemv_group<64>(w, X, batch, Y, y_dtype, vec, s);
    return gemv_group<128>(w, X, batch, Y, y_dtype, vec, s);
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
