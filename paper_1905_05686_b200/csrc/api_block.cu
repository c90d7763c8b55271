// C ABI of the operators around the masked layers: argument checks and calls of the launchers.
#include <unordered_map>

#include "occupancy_cache.cuh"
#include "row_ops.cuh"

namespace lrbi {

cudaError_t allow_shared(const void *kernel, size_t smem)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || dev < 0 || dev >= LRBI_MAX_DEVICES) return e != cudaSuccess ? e : cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(lib_mutex());
    static std::unordered_map<const void *, size_t> allowed[LRBI_MAX_DEVICES];
    try {
        size_t &most = allowed[dev][kernel];
        if (most >= smem) return cudaSuccess;
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e == cudaSuccess) most = smem;
    } catch (...) {      // no room to remember it
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    }
    return e;
}

int blocks_per_sm(const void *kernel, int threads, size_t smem)
{
    static OccupancyCache cache;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 1;
    return cache.get(kernel, dev, threads, smem, [&] {
        int n = 0;
        if ((smem > 32 * 1024 && allow_shared(kernel, smem) != cudaSuccess) || cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem) != cudaSuccess) return 0;
        return n;
    });
}

}  // namespace lrbi

using namespace lrbi;

namespace {

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool dtype_ok(int t) { return t == LRBI_Y_BF16 || t == LRBI_Y_F32; }
bool cols_ok(int cols) { return cols >= 1 && cols <= LRBI_MAX_ROW_COLS; }

// A matrix of a call: present where rows > 0, its element's alignment, rows that do not overlap and whose distance in bytes is a
// 32-bit number (kernels take a row's place as one multiply-add of 32-bit factors).
bool matrix_ok(const void *p, int dtype, int64_t stride, int rows, int cols)
{
    const int size = dtype == LRBI_Y_F32 ? 4 : 2;
    if (!dtype_ok(dtype) || stride < cols || stride > UINT32_MAX / size) return false;
    return rows == 0 || (p && aligned(p, size));
}
bool floats_ok(const void *p, int n) { return n == 0 || (p && aligned(p, 4)); }
bool copy_ok(const void *q, const void *scale, int rows) { return rows == 0 || (q && scale && aligned(q, 16) && aligned(scale, 4)); }
bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }

}  // namespace

extern "C" {

int32_t lrbi_checkpoint_pitch(int32_t cols) { return cols_ok(cols) ? checkpoint_pitch(cols) : 0; }
int32_t lrbi_checkpoint_groups(int32_t cols) { return cols_ok(cols) ? checkpoint_groups(cols) : 0; }

lrbi_status lrbi_checkpoint_store(const void *x, int32_t x_dtype, int64_t x_stride, int32_t rows, int32_t cols, int8_t *q, float *scale,
                                  void *stream)
{
    if (rows < 0 || !cols_ok(cols) || !matrix_ok(x, x_dtype, x_stride, rows, cols) || !copy_ok(q, scale, rows)) return LRBI_ERR_INVALID_ARG;
    if (device_timeout_seen()) return LRBI_ERR_TIMEOUT;
    if (rows == 0) return LRBI_OK;
    return launch_checkpoint_store(x, x_dtype, x_stride, rows, cols, q, scale, static_cast<cudaStream_t>(stream));
}

lrbi_status lrbi_checkpoint_load(const int8_t *q, const float *scale, int32_t rows, int32_t cols, void *x, int32_t x_dtype, int64_t x_stride,
                                 void *stream)
{
    if (rows < 0 || !cols_ok(cols) || !matrix_ok(x, x_dtype, x_stride, rows, cols) || !copy_ok(q, scale, rows)) return LRBI_ERR_INVALID_ARG;
    if (device_timeout_seen()) return LRBI_ERR_TIMEOUT;
    if (rows == 0) return LRBI_OK;
    return launch_checkpoint_load(q, scale, rows, cols, x, x_dtype, x_stride, static_cast<cudaStream_t>(stream));
}

lrbi_status lrbi_layer_norm(const void *x, int32_t x_dtype, int64_t x_stride, int32_t rows, int32_t cols, const void *gamma, const void *beta,
                            int32_t param_dtype, float eps, void *y, int32_t y_dtype, int64_t y_stride, float *mean, float *rstd, int8_t *q,
                            float *scale, void *stream)
{
    if (rows < 0 || !cols_ok(cols) || !matrix_ok(x, x_dtype, x_stride, rows, cols) || !matrix_ok(y, y_dtype, y_stride, rows, cols)) return LRBI_ERR_INVALID_ARG;
    if (!matrix_ok(gamma, param_dtype, cols, 1, cols) || (beta && !matrix_ok(beta, param_dtype, cols, 1, cols)) || !(eps >= 0.f)) return LRBI_ERR_INVALID_ARG;
    if (!mean != !rstd || (mean && (!floats_ok(mean, rows) || !floats_ok(rstd, rows)))) return LRBI_ERR_INVALID_ARG;
    if (!q != !scale || (q && !copy_ok(q, scale, rows))) return LRBI_ERR_INVALID_ARG;
    if (device_timeout_seen()) return LRBI_ERR_TIMEOUT;
    if (rows == 0) return LRBI_OK;
    NormArgs n = {};
    n.x = x; n.x_stride = x_stride; n.x_dtype = x_dtype;
    n.gamma = gamma; n.beta = beta; n.param_dtype = param_dtype; n.eps = eps;
    n.y = y; n.y_stride = y_stride; n.y_dtype = y_dtype;
    n.mean_out = mean; n.rstd_out = rstd;
    n.q_out = q; n.scale_out = scale;
    n.rows = rows; n.cols = cols;
    return launch_layer_norm(n, static_cast<cudaStream_t>(stream));
}

size_t lrbi_layer_norm_backward_workspace(int32_t rows, int32_t cols)
{
    return rows >= 0 && cols_ok(cols) ? norm_backward_workspace(rows, cols) : 0;
}

lrbi_status lrbi_layer_norm_backward(const void *dy, int32_t dy_dtype, int64_t dy_stride, const void *x, int32_t x_dtype, int64_t x_stride,
                                     const int8_t *q, const float *scale, int32_t rows, int32_t cols, const void *gamma, const void *beta,
                                     int32_t param_dtype, const float *mean, const float *rstd, const void *dres, int64_t dres_stride, void *dx,
                                     int32_t dx_dtype, int64_t dx_stride, void *y, int64_t y_stride, float *dgamma, float *dbeta,
                                     void *workspace, size_t workspace_bytes, void *stream)
{
    if (rows < 0 || !cols_ok(cols) || !matrix_ok(dy, dy_dtype, dy_stride, rows, cols) || !matrix_ok(dx, dx_dtype, dx_stride, rows, cols)) return LRBI_ERR_INVALID_ARG;
    const bool copy = q || scale;
    if (copy && x) return LRBI_ERR_INVALID_ARG;            // one of the two
    if (copy ? !copy_ok(q, scale, rows) : !matrix_ok(x, x_dtype, x_stride, rows, cols)) return LRBI_ERR_INVALID_ARG;
    if (!matrix_ok(gamma, param_dtype, cols, 1, cols) || (beta && !matrix_ok(beta, param_dtype, cols, 1, cols))) return LRBI_ERR_INVALID_ARG;
    if (!floats_ok(mean, rows) || !floats_ok(rstd, rows)) return LRBI_ERR_INVALID_ARG;
    if (dres && !matrix_ok(dres, dx_dtype, dres_stride, rows, cols)) return LRBI_ERR_INVALID_ARG;
    if (y && !matrix_ok(y, dy_dtype, y_stride, rows, cols)) return LRBI_ERR_INVALID_ARG;
    if ((dgamma && !aligned(dgamma, 4)) || (dbeta && !aligned(dbeta, 4))) return LRBI_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < norm_backward_workspace(rows, cols)) return LRBI_ERR_INVALID_ARG;
    if (device_timeout_seen()) return LRBI_ERR_TIMEOUT;
    NormArgs n = {};
    n.x = x; n.x_stride = x_stride; n.x_dtype = x_dtype;
    n.q = q; n.scale = scale;
    n.gamma = gamma; n.beta = beta; n.param_dtype = param_dtype;
    n.y = y; n.y_stride = y_stride;
    n.dy = dy; n.dy_stride = dy_stride; n.dy_dtype = dy_dtype;
    n.mean = mean; n.rstd = rstd;
    n.dres = dres; n.dres_stride = dres_stride;
    n.dx = dx; n.dx_stride = dx_stride; n.dx_dtype = dx_dtype;
    n.dgamma = dgamma; n.dbeta = dbeta;
    n.rows = rows; n.cols = cols;
    return launch_layer_norm_backward(n, static_cast<float *>(workspace), static_cast<cudaStream_t>(stream));
}

lrbi_status lrbi_activation(const void *h, int32_t h_dtype, int64_t h_stride, int32_t rows, int32_t cols, int32_t act, void *a, int32_t a_dtype,
                            int64_t a_stride, int8_t *q, float *scale, void *stream)
{
    if (rows < 0 || !cols_ok(cols) || act < LRBI_ACT_RELU || act > LRBI_ACT_SILU) return LRBI_ERR_INVALID_ARG;
    if (!matrix_ok(h, h_dtype, h_stride, rows, cols) || !matrix_ok(a, a_dtype, a_stride, rows, cols)) return LRBI_ERR_INVALID_ARG;
    if (!q != !scale || (q && !copy_ok(q, scale, rows))) return LRBI_ERR_INVALID_ARG;
    if (device_timeout_seen()) return LRBI_ERR_TIMEOUT;
    if (rows == 0) return LRBI_OK;
    ActArgs n = {};
    n.h = h; n.h_stride = h_stride; n.h_dtype = h_dtype;
    n.act = act;
    n.a = a; n.a_stride = a_stride; n.a_dtype = a_dtype;
    n.q_out = q; n.scale_out = scale;
    n.rows = rows; n.cols = cols;
    return launch_activation(n, static_cast<cudaStream_t>(stream));
}

lrbi_status lrbi_activation_backward(const void *da, int32_t da_dtype, int64_t da_stride, const void *h, int32_t h_dtype, int64_t h_stride,
                                     const int8_t *q, const float *scale, int32_t rows, int32_t cols, int32_t act, void *dh, int32_t dh_dtype,
                                     int64_t dh_stride, void *a, int64_t a_stride, void *stream)
{
    if (rows < 0 || !cols_ok(cols) || act < LRBI_ACT_RELU || act > LRBI_ACT_SILU) return LRBI_ERR_INVALID_ARG;
    if (!matrix_ok(da, da_dtype, da_stride, rows, cols) || !matrix_ok(dh, dh_dtype, dh_stride, rows, cols)) return LRBI_ERR_INVALID_ARG;
    const bool copy = q || scale;
    if (copy && h) return LRBI_ERR_INVALID_ARG;            // one of the two
    if (copy ? !copy_ok(q, scale, rows) : !matrix_ok(h, h_dtype, h_stride, rows, cols)) return LRBI_ERR_INVALID_ARG;
    if (a && !matrix_ok(a, da_dtype, a_stride, rows, cols)) return LRBI_ERR_INVALID_ARG;
    if (device_timeout_seen()) return LRBI_ERR_TIMEOUT;
    if (rows == 0) return LRBI_OK;
    ActArgs n = {};
    n.h = h; n.h_stride = h_stride; n.h_dtype = h_dtype;
    n.q = q; n.scale = scale;
    n.act = act;
    n.a = a; n.a_stride = a_stride; n.a_dtype = da_dtype;
    n.da = da; n.da_stride = da_stride; n.da_dtype = da_dtype;
    n.dh = dh; n.dh_stride = dh_stride; n.dh_dtype = dh_dtype;
    n.rows = rows; n.cols = cols;
    return launch_activation_backward(n, static_cast<cudaStream_t>(stream));
}

size_t lrbi_w4_packed_words(int32_t rows, int32_t cols)
{
    return rows >= 1 && cols_ok(cols) ? ((size_t)(rows - 1) / 16 + 1) * ((size_t)(cols - 1) / 64 + 1) * 128 : 0;
}
size_t lrbi_w4_meta_words(int32_t rows, int32_t cols, int32_t group)
{
    return rows >= 1 && cols_ok(cols) && group_ok(group) ? ((size_t)(rows - 1) / 16 + 1) * ((size_t)(cols - 1) / group + 1) * 16 : 0;
}

lrbi_status lrbi_w4_quantize(const lrbi_layout *layout, const uint16_t *W, const uint32_t *ip, const uint32_t *iz, int32_t group,
                             uint32_t *packed, uint32_t *meta, void *stream)
{
    if (!layout || layout->rows < 1 || !cols_ok(layout->cols) || !group_ok(group) || !W || !packed || !meta) return LRBI_ERR_INVALID_ARG;
    if (!aligned(W, 2) || !aligned(packed, 16) || !aligned(meta, 16) || !ip != !iz) return LRBI_ERR_INVALID_ARG;
    if (ip && (!aligned(ip, 4) || !aligned(iz, 4) || layout->tile_rows < 1 || layout->tile_cols < 1 || layout->rank < 1)) return LRBI_ERR_INVALID_ARG;
    if (device_timeout_seen()) return LRBI_ERR_TIMEOUT;
    lrbi_layout l = *layout;
    if (!ip) { l.tile_rows = l.rows; l.tile_cols = l.cols; l.rank = 1; }
    return launch_w4_quantize(make_geo(l), W, ip, iz, group, packed, meta, static_cast<cudaStream_t>(stream));
}

lrbi_status lrbi_w4_gemv(const uint32_t *packed, const uint32_t *meta, int32_t rows, int32_t cols, int32_t group, const uint16_t *X, int32_t batch,
                         void *Y, int32_t y_dtype, void *stream)
{
    if (rows < 1 || !cols_ok(cols) || !group_ok(group) || batch < 0 || !packed || !meta || !dtype_ok(y_dtype)) return LRBI_ERR_INVALID_ARG;
    if (!aligned(packed, 16) || !aligned(meta, 16)) return LRBI_ERR_INVALID_ARG;      // both are copied 16 bytes at a time
    if (batch > 0 && (!X || !Y || !aligned(X, 2) || !aligned(Y, y_dtype == LRBI_Y_F32 ? 4 : 2))) return LRBI_ERR_INVALID_ARG;
    if (device_timeout_seen()) return LRBI_ERR_TIMEOUT;
    if (batch == 0) return LRBI_OK;
    return launch_w4_gemv(packed, meta, rows, cols, group, X, batch, Y, y_dtype, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
