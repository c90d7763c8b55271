// Products of 8-bit rows on the tensor cores:  Y[b][o] = (sum over i of q_X[b][i] * q_W[o][i]) * scale_X[b] * scale_W[o].
//
// tcgen05.mma kind::i8, K-major operands with the 128-byte swizzle (a stage is 128 columns of both), sums in tensor memory as
// 32-bit whole numbers: exact, in any order.  Two kernels:
//
//   long   many tokens.  CTA pairs (cta_group::2) of 256 tokens x 128 to 256 channels walk the output tiles; two accumulators, so that
//          eight warps scale and store one tile while the next one is computed.  Bound: the tensor cores (pipe 94% busy; 4096
//          tokens, 16384 x 4096: 167 us by itself, 3.3 Pop/s, twice what bf16 products of that size reach; call after call, each
//          with its tokens, the power cap: 195 us for both, 2.8 Pop/s), at smaller sizes the last round of tiles (1000 tokens,
//          4096 x 16384: 64 tiles on 74 pairs, 47 us of 40).
//   split  fewer.  128 channels x up to 256 tokens a CTA; the CTAs of a cluster share the columns and add their sums to one another
//          by bulk copies that add (whole numbers: the same bits however they are cut), so that all SMs stream the weights.
//          Bound: memory, with 2 us of set-up before and 2 to 5 us of sums and stores behind it (4096 x 9216: 16 tokens 10.6 us,
//          128 12.4, 256 17.4; floor 5.9 to 6.5).
//
// Every wait is bounded; a wait that runs out leaves a code in the device status word, and the CTA ends early.
#include <algorithm>

#include "norm_common.cuh"
#include "tcgen05_ptx.cuh"

namespace lrbi {

constexpr int I8_KB = 128;                               // columns (and bytes of a row) of a stage
constexpr int I8_A_BYTES = 128 * I8_KB;                  // 128 rows of the M operand
constexpr int I8_EPI_WARPS = 8;                          // long: warps 2-9 scale and store (warp 0 copies, warp 1 multiplies)
constexpr int I8_LONG_THREADS = 32 * (2 + I8_EPI_WARPS);
constexpr int I8_SPLIT_WARPS = 10;                       // split: warps 2-9 empty tensor memory, all of them scale and store
constexpr size_t I8_SHARED = 226 * 1024;                 // dynamic shared memory of a CTA that has an SM to itself

struct I8Ctl {
    uint64_t full[8], empty[8];      // of the stages
    uint64_t accum[2], drained[2];   // of the accumulators
    uint64_t added;                  // split: the other CTAs' sums have been added to this one's
    alignas(16) float token[256];    // split: the tile's scales
    uint32_t tmem;
    int abort_flag;
};

struct I8Tc {
    const float *x_scale, *w_scale;
    void *y;
    int y_dtype;
    int rows, batch;                 // channels, tokens
    int blocks;                      // of columns: stages of a tile
    int stages;
    int channels;                    // long: of a tile, a multiple of 32 from 128 to 256
    int tokens;                      // split: of a tile
    int split;
    int vector;                      // bytes that an access to Y may have: 16, 8, 4 or 2
    int *status;
};

__device__ __forceinline__ void umma_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma2_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// Signed 8-bit operands, 32-bit sums.
__host__ __device__ constexpr uint32_t i8_idesc(int m, int n) { return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

// A copy of a CTA of a pair into its own shared memory that signals a barrier of the pair's first CTA (`bar`: its address there).
__device__ __forceinline__ void tma_load_2d_pair(void *dst, const CUtensorMap *map, uint32_t bar, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ uint32_t in_cta(uint32_t mine, uint32_t rank)      // the same place in the shared memory of another CTA of the cluster
{
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(rank));
    return there;
}
// Adds `bytes` of whole numbers of this CTA's shared memory to those at `to` in another CTA of the cluster, whose barrier `bar` counts them.
__device__ __forceinline__ void add_to_cta(uint32_t to, uint32_t from, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.reduce.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes.add.s32 [%0], [%1], %2, [%3];"
                 ::"r"(to), "r"(from), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void l2_prefetch_2d(const CUtensorMap *map, int x, int y)
{
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(map), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t at, int (&v)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]),
                   "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
                   "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
                 : "r"(at) : "memory");
}

// Copies that are under way must land before shared memory is given up: about 2 ms, far beyond any of them.
__device__ __forceinline__ void let_copies_land()
{
    const long long t0 = clock64();
    while (clock64() - t0 < 4000000ll) { }
}

// ---------------------------------------------------------------------------------------------------------------------
// Many tokens
// ---------------------------------------------------------------------------------------------------------------------
// The tile's M is the token (a lane of tensor memory), its N the channel: a thread has neighbouring outputs of one row of Y.
// They go through 2 KB a warp, 32 rows x 64 bytes with the pieces of a row in an order that keeps the banks apart, and out as
// whole sectors.
constexpr int I8_LONG_STAGES = 6, I8_LONG_STAGE = 2 * I8_A_BYTES, I8_EPI_BYTES = 32 * 64 + 128 * 4;
__global__ void __launch_bounds__(I8_LONG_THREADS, 1) i8_long_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map, I8Tc p)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t *epi = smem + (size_t)p.stages * I8_LONG_STAGE;
    I8Ctl *ctl = reinterpret_cast<I8Ctl *>(epi + I8_EPI_WARPS * I8_EPI_BYTES);
    volatile int *abort_flag = &ctl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    if ((smem_u32(smem) & 1023u) != 0) {         // never expected; refuse rather than compute garbage
        if (threadIdx.x == 0) atomicCAS(p.status, 0, DEV_BAD_SMEM_ALIGN);
        return;
    }
    if (warp == 0) {
        if (lane < p.stages) {
            mbar_init(&ctl->full[lane], 1);
            mbar_init(&ctl->empty[lane], 1);
        } else if (lane == 8 || lane == 9) {
            mbar_init(&ctl->accum[lane - 8], 1);
            mbar_init(&ctl->drained[lane - 8], 2 * I8_EPI_WARPS);
        } else if (lane == 10) ctl->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc2(&ctl->tmem, 512);
    tc_fence_before();
    __syncthreads();
    __syncwarp();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = ctl->tmem;
    begin();

    // Tiles run fastest along the smaller operand: the pairs at work at any time share all of it, and the larger one streams
    // from memory once.
    const int token_tiles = (p.batch + 255) / 256, channel_tiles = (p.rows + p.channels - 1) / p.channels, tiles = token_tiles * channel_tiles;
    const int first = blockIdx.x >> 1, step = gridDim.x >> 1;
    const bool tokens_fast = p.batch <= p.rows;
    auto tile_at = [&](int t, int &b0, int &o0) {
        b0 = (tokens_fast ? t % token_tiles : t / channel_tiles) * 256;
        o0 = (tokens_fast ? t / token_tiles : t % channel_tiles) * p.channels;
    };

    if (warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t parity = 1;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += step) {
                int b0, o0;
                tile_at(t, b0, o0);
                for (int k = 0; k < p.blocks; ++k) {
                    ok = mbar_wait(&ctl->empty[s], parity, abort_flag, p.status, DEV_TIMEOUT_EMPTY);
                    if (!ok) break;
                    if (rank == 0) mbar_arrive_expect_tx(&ctl->full[s], 2 * I8_A_BYTES + p.channels * I8_KB);       // of both CTAs
                    const uint32_t bar = in_cta(smem_u32(&ctl->full[s]), 0);
                    uint8_t *a = smem + (size_t)s * I8_LONG_STAGE;
                    tma_load_2d_pair(a, &x_map, bar, k * I8_KB, b0 + (int)rank * 128);
                    tma_load_2d_pair(a + I8_A_BYTES, &w_map, bar, k * I8_KB, o0 + (int)rank * (p.channels / 2));
                    if (++s == p.stages) { s = 0; parity ^= 1; }
                }
            }
            if (!ok) let_copies_land();
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t idesc = i8_idesc(256, p.channels);
            int s = 0, n = 0;
            uint32_t parity = 0;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += step, ++n) {
                ok = mbar_wait(&ctl->drained[n & 1], (n >> 1 & 1) ^ 1, abort_flag, p.status, DEV_TIMEOUT_ACCUM);
                if (!ok) break;
                tc_fence_after();
                const uint32_t d = tmem + (n & 1) * 256;
                for (int k = 0; k < p.blocks; ++k) {
                    ok = mbar_wait(&ctl->full[s], parity, abort_flag, p.status, DEV_TIMEOUT_FULL);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t a = make_sw128_desc(smem_u32(smem + (size_t)s * I8_LONG_STAGE)), b = make_sw128_desc(smem_u32(smem + (size_t)s * I8_LONG_STAGE + I8_A_BYTES));
#pragma unroll
                    for (int q = 0; q < I8_KB / 32; ++q) umma2_i8(d, a + (uint64_t)(2 * q), b + (uint64_t)(2 * q), idesc, (k | q) ? 1u : 0u);
                    umma2_commit_both(&ctl->empty[s]);
                    if (++s == p.stages) { s = 0; parity ^= 1; }
                }
                if (ok) umma2_commit_both(&ctl->accum[n & 1]);
            }
        }
    } else {
        // a warp has the tokens of its quarter of tensor memory and half of the channels
        const int quad = warp & 3, half = (warp - 2) >> 2;
        uint8_t *stage = epi + (warp - 2) * I8_EPI_BYTES;
        float *scale = reinterpret_cast<float *>(stage + 32 * 64);
        const int mine0 = (p.channels + 32) / 64 * 32, mine = half ? p.channels - mine0 : mine0;      // channels of the warp
        const bool f32 = p.y_dtype == LRBI_Y_F32;
        const int size = f32 ? 4 : 2;
        bool ok = true;
        int n = 0;
        for (int t = first; t < tiles; t += step, ++n) {
            int b0, o0;
            tile_at(t, b0, o0);
            b0 += (int)rank * 128 + quad * 32;
            const int end = min(o0 + p.channels, p.rows);
            o0 += half * mine0;
            const int left = min(32, p.batch - b0);      // rows of Y that the warp has
            const float token = lane < left ? __ldg(p.x_scale + b0 + lane) : 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) scale[i * 32 + lane] = o0 + i * 32 + lane < end ? __ldg(p.w_scale + o0 + i * 32 + lane) : 0.f;
            ok = mbar_wait(&ctl->accum[n & 1], n >> 1 & 1, abort_flag, p.status, DEV_TIMEOUT_ACCUM);
            __syncwarp();                                // the loads below are the whole warp's: one verdict for all lanes
            if (!ok || *abort_flag) break;
            tc_fence_after();
            const uint32_t from = tmem + ((uint32_t)(quad * 32) << 16) + (n & 1) * 256 + half * mine0;
            uint4 *own = reinterpret_cast<uint4 *>(stage + lane * 64);
            const int swap = lane >> 1 & 3;
            for (int c = 0; c < mine; c += 32) {
                int v[32];
                tmem_ld32(from + c, v);
                tmem_ld_wait();
                if (c == mine - 32) {                    // read: the accumulator may be overwritten
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        if (rank == 0) mbar_arrive(&ctl->drained[n & 1]);
                        else mbar_arrive_remote(&ctl->drained[n & 1], 0);
                    }
                }
                const float4 *w = reinterpret_cast<const float4 *>(scale + c);
                float y[32];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float4 s = w[i];
                    y[4 * i] = ((float)v[4 * i] * token) * s.x;
                    y[4 * i + 1] = ((float)v[4 * i + 1] * token) * s.y;
                    y[4 * i + 2] = ((float)v[4 * i + 2] * token) * s.z;
                    y[4 * i + 3] = ((float)v[4 * i + 3] * token) * s.w;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {            // fp32: 16 columns at a time
                    if (h == 1 && !f32) break;
                    if (f32) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            own[i ^ swap] = make_uint4(__float_as_uint(y[16 * h + 4 * i]), __float_as_uint(y[16 * h + 4 * i + 1]), __float_as_uint(y[16 * h + 4 * i + 2]), __float_as_uint(y[16 * h + 4 * i + 3]));
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            own[i ^ swap] = make_uint4(pack_bf16(y[8 * i], y[8 * i + 1]), pack_bf16(y[8 * i + 2], y[8 * i + 3]), pack_bf16(y[8 * i + 4], y[8 * i + 5]), pack_bf16(y[8 * i + 6], y[8 * i + 7]));
                    }
                    __syncwarp();
                    const int at = o0 + c + h * 16;      // first channel of the 64 bytes
                    char *const to = static_cast<char *>(p.y) + ((long long)b0 * p.rows + at) * size;
                    const long long pitch = (long long)p.rows * size;
                    const int width = min(64 / size, end - at) * size;      // bytes that are there
                    if (p.vector == 16) {                // eight rows at a time
                        const int piece = lane & 3;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int r = i * 8 + (lane >> 2);
                            if (r < left && piece * 16 < width) *reinterpret_cast<uint4 *>(to + r * pitch + piece * 16) = *reinterpret_cast<const uint4 *>(stage + r * 64 + ((piece ^ (r >> 1 & 3)) << 4));
                        }
                    } else if (p.vector >= 4) {          // two rows at a time, so that a warp still writes whole stretches
                        const int word = lane & 15;
#pragma unroll 8
                        for (int i = 0; i < 16; ++i) {
                            const int r = i * 2 + (lane >> 4);
                            if (r < left && word * 4 < width) *reinterpret_cast<uint32_t *>(to + r * pitch + word * 4) = *reinterpret_cast<const uint32_t *>(stage + r * 64 + (((word >> 2) ^ (r >> 1 & 3)) << 4) + (word & 3) * 4);
                        }
                    } else {
#pragma unroll 8
                        for (int r = 0; r < 32; ++r)
                            if (r < left && lane * 2 < width) *reinterpret_cast<uint16_t *>(to + r * pitch + lane * 2) = *reinterpret_cast<const uint16_t *>(stage + r * 64 + (((lane >> 3) ^ (r >> 1 & 3)) << 4) + (lane & 7) * 2);
                    }
                    __syncwarp();
                }
            }
        }
    }
    let_next();
    tc_fence_before();
    __syncthreads();
    __syncwarp();
    cluster_sync_all();              // neither CTA frees tensor memory or leaves while the other may still touch it
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc2(tmem, 512);
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Fewer tokens
// ---------------------------------------------------------------------------------------------------------------------
// The tile's M is the channel, its N the token (a multiple of 16 up to 256, as many as there are).  TWO: two CTAs fit an SM, so
// that one is set up, and asks for its first weights, while another ends.
template <bool TWO>
__global__ void __launch_bounds__(32 * I8_SPLIT_WARPS, TWO ? 2 : 1) i8_split_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map, I8Tc p)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    const int stage_bytes = I8_A_BYTES + p.tokens * I8_KB;
    I8Ctl *ctl = reinterpret_cast<I8Ctl *>(smem + (size_t)p.stages * stage_bytes);
    volatile int *abort_flag = &ctl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t columns = p.tokens <= 32 ? 32 : p.tokens <= 64 ? 64 : p.tokens <= 128 ? 128 : 256;
    const int rank = p.split > 1 ? (int)cluster_ctarank() : 0;
    if ((smem_u32(smem) & 1023u) != 0) {         // never expected; refuse rather than compute garbage
        if (threadIdx.x == 0) atomicCAS(p.status, 0, DEV_BAD_SMEM_ALIGN);
        return;
    }
    const int token_tiles = (p.batch + p.tokens - 1) / p.tokens, tile = blockIdx.x / p.split;
    const int b0 = (tile % token_tiles) * p.tokens, o0 = (tile / token_tiles) * 128;
    const int k0 = (int)((long long)p.blocks * rank / p.split), k1 = (int)((long long)p.blocks * (rank + 1) / p.split);      // at least one block: blocks >= split
    const int used = min(p.tokens, p.batch - b0);
    if (warp == 0) {
        if (lane < p.stages) {
            mbar_init(&ctl->full[lane], 1);
            mbar_init(&ctl->empty[lane], 1);
        } else if (lane == 8) mbar_init(&ctl->accum[0], 1);
        else if (lane == 9) mbar_init(&ctl->added, 1);
        else if (lane == 10) ctl->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(&ctl->tmem, columns);
    // A hint that needs no order: the first weights come to L2 while the kernel before this one (the tokens') ends.
    if (warp == 2 && lane < p.stages && k0 + lane < k1) l2_prefetch_2d(&w_map, (k0 + lane) * I8_KB, o0);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctl->tmem;
    begin();
    // In the end the CTAs of the cluster take the tokens in equal parts, a warp one at a time: four neighbouring channels a lane where rows of
    // Y are whole vectors of four, else channels 32 apart.
    const bool f32 = p.y_dtype == LRBI_Y_F32, four = p.vector >= (f32 ? 16 : 8);
    const int gap = four ? 1 : 32, o = o0 + lane * (four ? 4 : 1);
    float channel[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) channel[i] = o + i * gap < p.rows ? __ldg(p.w_scale + o + i * gap) : 0.f;

    if (warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t parity = 1;
            bool ok = true;
            for (int k = k0; k < k1; ++k) {
                ok = mbar_wait(&ctl->empty[s], parity, abort_flag, p.status, DEV_TIMEOUT_EMPTY);
                if (!ok) break;
                mbar_arrive_expect_tx(&ctl->full[s], stage_bytes);
                tma_load_2d(smem + (size_t)s * stage_bytes, &w_map, &ctl->full[s], k * I8_KB, o0);
                tma_load_2d(smem + (size_t)s * stage_bytes + I8_A_BYTES, &x_map, &ctl->full[s], k * I8_KB, b0);
                if (++s == p.stages) { s = 0; parity ^= 1; }
            }
            if (!ok) let_copies_land();
        }
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = i8_idesc(128, p.tokens);
            int s = 0;
            uint32_t parity = 0;
            bool ok = true;
            for (int k = k0; k < k1; ++k) {
                ok = mbar_wait(&ctl->full[s], parity, abort_flag, p.status, DEV_TIMEOUT_FULL);
                if (!ok) break;
                tc_fence_after();
                const uint64_t a = make_sw128_desc(smem_u32(smem + (size_t)s * stage_bytes)), b = make_sw128_desc(smem_u32(smem + (size_t)s * stage_bytes + I8_A_BYTES));
#pragma unroll
                for (int q = 0; q < I8_KB / 32; ++q) umma_i8(tmem, a + (uint64_t)(2 * q), b + (uint64_t)(2 * q), idesc, (k != k0 || q) ? 1u : 0u);
                umma_commit(&ctl->empty[s]);
                if (++s == p.stages) { s = 0; parity ^= 1; }
            }
            if (ok) umma_commit(&ctl->accum[0]);
        }
    } else {
        const int quad = warp & 3, half = (warp - 2) >> 2;
        for (int j = threadIdx.x - 64; j < used; j += 256) ctl->token[j] = __ldg(p.x_scale + b0 + j);
        asm volatile("bar.sync 1, 256;" ::: "memory");           // these eight warps
        bool ok = mbar_wait(&ctl->accum[0], 0, abort_flag, p.status, DEV_TIMEOUT_ACCUM);
        __syncwarp();
        ok = ok && *abort_flag == 0;
        if (ok) {
            tc_fence_after();
            const uint32_t from = tmem + ((uint32_t)(quad * 32) << 16);
            const int own = o0 + quad * 32 + lane;
            const float scale = own < p.rows ? __ldg(p.w_scale + own) : 0.f;
            // Alone, straight from tensor memory: the warp has 32 neighbouring channels of a token.  Else (all products are through,
            // and so are the copies that they waited for) the sums, [token][channel], take the stages' place.
            int *part = reinterpret_cast<int *>(smem) + quad * 32 + lane;
            for (int c = half * 32; c < used; c += 64) {
                int v[32];
                tmem_ld32(from + c, v);
                tmem_ld_wait();
                if (p.split > 1) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) part[(c + j) * 128] = v[j];
                    if (c + 16 < p.tokens) {         // (else they are beyond the tile, not beyond what was allocated of tensor memory)
#pragma unroll
                        for (int j = 16; j < 32; ++j) part[(c + j) * 128] = v[j];
                    }
                } else if (own < p.rows) {
                    char *to = static_cast<char *>(p.y) + ((long long)(b0 + c) * p.rows + own) * (f32 ? 4 : 2);
                    const long long pitch = (long long)p.rows * (f32 ? 4 : 2);
                    const int left = used - c;
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 token = *reinterpret_cast<const float4 *>(&ctl->token[c + j]);
                        const float y[4] = {((float)v[j] * token.x) * scale, ((float)v[j + 1] * token.y) * scale, ((float)v[j + 2] * token.z) * scale, ((float)v[j + 3] * token.w) * scale};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (j + i < left) {
                                if (f32) *reinterpret_cast<float *>(to) = y[i];
                                else *reinterpret_cast<uint16_t *>(to) = (uint16_t)pack_bf16(y[i], 0.f);
                            }
                            to += pitch;
                        }
                    }
                }
            }
            if (p.split > 1) fence_async_proxy();    // the sums are read by bulk copies
        }
        tc_fence_before();
    }
    let_next();
    __syncwarp();
    if (p.split > 1) {
        // Every CTA takes an equal part of the tokens: the others add theirs to its sums, and it scales and stores them.
        const int j0 = used * rank / p.split, j1 = used * (rank + 1) / p.split;
        cluster_sync_all();
        if (*abort_flag == 0 && threadIdx.x == 0) {
            mbar_arrive_expect_tx(&ctl->added, (uint32_t)((p.split - 1) * (j1 - j0) * 512));
            for (int r = 1; r < p.split; ++r) {
                const int to = (rank + r) % p.split, first = used * to / p.split, bytes = (used * (to + 1) / p.split - first) * 512;
                const uint32_t at = smem_u32(smem) + first * 512;
                if (bytes) add_to_cta(in_cta(at, to), at, bytes, in_cta(smem_u32(&ctl->added), to));
            }
        }
        const bool ok = *abort_flag == 0 && mbar_wait(&ctl->added, 0, abort_flag, p.status, DEV_TIMEOUT_ACCUM);
        if (!ok) let_copies_land();
        __syncwarp();
        if (ok && *abort_flag == 0) {
            constexpr int T = 4;                     // tokens of a warp at a time
            const uint8_t *mine = smem + lane * (four ? 16 : 4);
            for (int j = j0 + warp; j < j1; j += I8_SPLIT_WARPS * T) {
                int4 sum[T];
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    const int *at = reinterpret_cast<const int *>(mine + min(j + t * I8_SPLIT_WARPS, j1 - 1) * 512);
                    sum[t] = four ? *reinterpret_cast<const int4 *>(at) : make_int4(at[0], at[32], at[64], at[96]);
                }
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    const int own = j + t * I8_SPLIT_WARPS;
                    if (own >= j1) break;
                    const float token = ctl->token[own];
                    const float y[4] = {((float)sum[t].x * token) * channel[0], ((float)sum[t].y * token) * channel[1], ((float)sum[t].z * token) * channel[2],
                                        ((float)sum[t].w * token) * channel[3]};
                    const long long to = (long long)(b0 + own) * p.rows + o;
                    if (four && o < p.rows) {        // rows is a multiple of four: all of them are there
                        if (f32) *reinterpret_cast<float4 *>(static_cast<float *>(p.y) + to) = make_float4(y[0], y[1], y[2], y[3]);
                        else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.y) + to) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
                    } else if (!four) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (o + 32 * i >= p.rows) continue;
                            if (f32) static_cast<float *>(p.y)[to + 32 * i] = y[i];
                            else static_cast<uint16_t *>(p.y)[to + 32 * i] = (uint16_t)pack_bf16(y[i], 0.f);
                        }
                    }
                }
            }
        }
    } else __syncthreads();
    __syncwarp();
    if (p.split > 1) cluster_sync_all();         // a CTA stays while its sums are under way to others
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, columns);
    }
}

namespace {

lrbi_status i8_map(CUtensorMap *map, const int8_t *q, int rows, int cols, int pitch, int box_rows)
{
    const EncodeTiledFn encode = get_encode_fn();
    if (!encode) { note_cuda_error(-1); return LRBI_ERR_CUDA; }
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {I8_KB, (cuuint32_t)box_rows}, each[2] = {1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t *>(q), dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) { note_cuda_error((int)r); return LRBI_ERR_CUDA; }
    return LRBI_OK;
}

I8Tc i8_args(const I8Product &p)
{
    I8Tc t = {};
    t.x_scale = p.x_scale; t.w_scale = p.w_scale;
    t.y = p.y; t.y_dtype = p.y_dtype;
    t.rows = p.rows; t.batch = p.batch;
    t.blocks = (p.cols + I8_KB - 1) / I8_KB;
    const uintptr_t at = reinterpret_cast<uintptr_t>(p.y) | (uintptr_t)((long long)p.rows * (p.y_dtype == LRBI_Y_F32 ? 4 : 2));
    t.vector = at % 16 == 0 ? 16 : at % 8 == 0 ? 8 : at % 4 == 0 ? 4 : 2;
    t.status = device_status_ptr();
    return t;
}

}  // namespace

lrbi_i8_plan i8_long_plan(int channels) { return {LRBI_I8_LONG, 256, channels, 1, I8_LONG_STAGES, I8_LONG_THREADS, 1}; }

lrbi_status launch_i8_long(const I8Product &p, const lrbi_i8_plan &plan, cudaStream_t s)
{
    I8Tc t = i8_args(p);
    const int channels = t.channels = plan.channels;
    t.stages = plan.stages;
    const size_t smem = (size_t)t.stages * I8_LONG_STAGE + I8_EPI_WARPS * I8_EPI_BYTES + sizeof(I8Ctl);
    static_assert((size_t)I8_LONG_STAGES * I8_LONG_STAGE + I8_EPI_WARPS * I8_EPI_BYTES + sizeof(I8Ctl) <= I8_SHARED, "");
    CUtensorMap x_map, w_map;
    lrbi_status rc = i8_map(&x_map, p.x, p.batch, p.cols, p.pitch, 128);
    if (rc == LRBI_OK) rc = i8_map(&w_map, p.w, p.rows, p.cols, p.pitch, channels / 2);
    if (rc != LRBI_OK) return rc;
    const long long tiles = (long long)((p.batch + 255) / 256) * ((p.rows + channels - 1) / channels);
    if (tiles > INT32_MAX) return LRBI_ERR_UNSUPPORTED;
    const int pairs = (int)(tiles < NORM_SMS / 2 ? tiles : NORM_SMS / 2);
    return launch_kernel(i8_long_kernel, dim3(2 * pairs), dim3(I8_LONG_THREADS), smem, s, 2, x_map, w_map, t);
}

namespace {
long long split_tiles(int rows, int batch, int tokens) { return (long long)((batch + tokens - 1) / tokens) * ((rows + 127) / 128); }
}  // namespace

lrbi_i8_plan i8_split_plan(int rows, int batch, int tokens, int split)
{
    const bool two = tokens <= 128 && split_tiles(rows, batch, tokens) * split > i8_at_once(split);      // three stages or more in half of an SM's shared memory
    const int stages = std::min(8, (int)(((two ? I8_SHARED / 2 : I8_SHARED) - sizeof(I8Ctl)) / (I8_A_BYTES + tokens * I8_KB)));
    return {LRBI_I8_SPLIT, tokens, 128, split, stages, 32 * I8_SPLIT_WARPS, two ? 2 : 1};
}

lrbi_status launch_i8_split(const I8Product &p, const lrbi_i8_plan &plan, cudaStream_t s)
{
    I8Tc t = i8_args(p);
    t.tokens = plan.tokens;
    const int split = t.split = plan.split;
    t.stages = plan.stages;
    const int stage = I8_A_BYTES + t.tokens * I8_KB;
    const long long tiles = split_tiles(p.rows, p.batch, t.tokens);
    if (tiles * split > INT32_MAX) return LRBI_ERR_UNSUPPORTED;
    const bool two = plan.per_sm == 2;
    const size_t smem = (size_t)t.stages * stage + sizeof(I8Ctl);      // in all cases more than the 512 bytes a token that the sums take
    CUtensorMap x_map, w_map;
    lrbi_status rc = i8_map(&x_map, p.x, p.batch, p.cols, p.pitch, t.tokens);
    if (rc == LRBI_OK) rc = i8_map(&w_map, p.w, p.rows, p.cols, p.pitch, 128);
    if (rc != LRBI_OK) return rc;
    const dim3 grid((unsigned)(tiles * split)), block(32 * I8_SPLIT_WARPS);
    return two ? launch_kernel(i8_split_kernel<true>, grid, block, smem, s, split, x_map, w_map, t) : launch_kernel(i8_split_kernel<false>, grid, block, smem, s, split, x_map, w_map, t);
}

}  // namespace lrbi
