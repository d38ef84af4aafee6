// Layer norm, forward and backward, with the reduction of the gradients of its
// weight and bias.
//
//   forward   mean = sum(x) / n, var = sum((x - mean)^2) / n,
//             y = (x - mean) / sqrt(var + eps) * w + b
//   backward  xhat = (x - mean) rstd, g = dy w,
//             dx = rstd (g - mean(g) - xhat mean(g xhat)),
//             dw = sum over rows of dy xhat, db = sum over rows of dy
#include "so_ops.cuh"

using namespace so_ops;

namespace {

struct NormArgs {
    const void *x, *dy, *weight, *bias;
    void *y;                              // y, or dx in the backward pass
    float *mean, *rstd;
    float *partials;                      // [blocks][2][cols]: sums of dy xhat, of dy
    int64_t x_stride, dy_stride, y_stride, rows, cols;
    int32_t param_dtype;
    float eps, inv_cols;
};

// Sum over the block, returned to every thread.  `s` holds one float per warp;
// the caller alternates between two of them so that one barrier is enough.
__device__ __forceinline__ float block_sum(float x, float *s)
{
    x = warp_sum(x);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
    __syncthreads();
    const int warps = blockDim.x >> 5;
    float v = 0.0f;
    for (int i = 0; i < warps; ++i) v += s[i];
    return v;
}

constexpr int kLoopThreads = 512;

template <typename T>
__global__ void __launch_bounds__(kLoopThreads) norm_forward_loop_kernel(NormArgs a)
{
    __shared__ float s_red[2][32];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        T *y = static_cast<T *>(a.y) + row * a.y_stride;
        float sum = 0.0f;
        for (int64_t c = threadIdx.x; c < a.cols; c += kLoopThreads) sum += to_f32(x[c]);
        const float mean = block_sum(sum, s_red[0]) * a.inv_cols;
        float sq = 0.0f;
        for (int64_t c = threadIdx.x; c < a.cols; c += kLoopThreads) {
            const float d = to_f32(x[c]) - mean;
            sq = fmaf(d, d, sq);
        }
        const float rstd = 1.0f / sqrtf(block_sum(sq, s_red[1]) * a.inv_cols + a.eps);
        for (int64_t c = threadIdx.x; c < a.cols; c += kLoopThreads) {
            const float w = a.weight ? load_any(a.weight, c, a.param_dtype) : 1.0f;
            const float b = a.bias ? load_any(a.bias, c, a.param_dtype) : 0.0f;
            y[c] = from_f32<T>(fmaf((to_f32(x[c]) - mean) * rstd, w, b));
        }
        if (a.mean && threadIdx.x == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kLoopThreads) norm_backward_loop_kernel(NormArgs a)
{
    __shared__ float s_red[2][32];
    float *dw = a.partials ? a.partials + (int64_t)blockIdx.x * 2 * a.cols : nullptr;
    float *db = dw ? dw + a.cols : nullptr;
    if (dw)
        for (int64_t c = threadIdx.x; c < a.cols; c += kLoopThreads) dw[c] = db[c] = 0.0f;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
        T *dx = static_cast<T *>(a.y) + row * a.y_stride;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float sg = 0.0f, sgx = 0.0f;
        for (int64_t c = threadIdx.x; c < a.cols; c += kLoopThreads) {
            const float w = a.weight ? load_any(a.weight, c, a.param_dtype) : 1.0f;
            const float g = to_f32(dy[c]) * w;
            const float xh = (to_f32(x[c]) - mean) * rstd;
            sg += g;
            sgx = fmaf(g, xh, sgx);
        }
        const float mg = block_sum(sg, s_red[0]) * a.inv_cols;
        const float mgx = block_sum(sgx, s_red[1]) * a.inv_cols;
        for (int64_t c = threadIdx.x; c < a.cols; c += kLoopThreads) {
            const float w = a.weight ? load_any(a.weight, c, a.param_dtype) : 1.0f;
            const float d = to_f32(dy[c]);
            const float xh = (to_f32(x[c]) - mean) * rstd;
            if (dw) {
                dw[c] = fmaf(d, xh, dw[c]);
                db[c] += d;
            }
            dx[c] = from_f32<T>(rstd * (fmaf(d, w, -mg) - xh * mgx));
        }
    }
}

// Sums the blocks' partial rows: 32 columns a block, 8 threads down each
// column, in a fixed order.
constexpr int kReduceRows = 8;

__global__ void __launch_bounds__(32 * kReduceRows)
norm_reduce_kernel(const float *partials, int n_blocks, int64_t cols, void *dweight, void *dbias,
                   int32_t grad_dtype, int32_t accumulate)
{
    __shared__ float s[kReduceRows][33];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t at = (int64_t)blockIdx.x * 32 + lane;      // column of [dweight | dbias]
    grid_dependency_wait();
    float sum = 0.0f;
    if (at < 2 * cols)
        for (int i = part; i < n_blocks; i += kReduceRows) sum += partials[(int64_t)i * 2 * cols + at];
    s[part][lane] = sum;
    __syncthreads();
    if (part != 0 || at >= 2 * cols) return;
    for (int i = 1; i < kReduceRows; ++i) sum += s[i][lane];
    void *out = at < cols ? dweight : dbias;
    if (!out) return;
    const int64_t c = at < cols ? at : at - cols;
    if (accumulate) sum += load_any(out, c, grad_dtype);
    store_any(out, c, grad_dtype, sum);
}

constexpr int kMaxPartials = 512;         // blocks that may leave a partial row

}  // namespace

extern "C" {

so_status so_layer_norm_forward(const void *x, int64_t x_stride, const void *weight,
                                const void *bias, void *y, int64_t y_stride, float *mean,
                                float *rstd, int64_t rows, int64_t cols, int32_t dtype,
                                int32_t param_dtype, double eps, void *stream)
{
    if (!valid_dtype(dtype) || (param_dtype != dtype && param_dtype != SO_DTYPE_FP32)) return SO_ERR_INVALID_ARG;
    if (rows < 0 || cols < 1 || cols > INT32_MAX || !(eps >= 0.0) || !std::isfinite(eps)) return SO_ERR_INVALID_ARG;
    const int es = elem_size(dtype), ps = elem_size(param_dtype);
    if ((weight && !aligned(weight, ps)) || (bias && !aligned(bias, ps))) return SO_ERR_INVALID_ARG;
    if ((mean == nullptr) != (rstd == nullptr)) return SO_ERR_INVALID_ARG;
    if (!aligned(mean, 4) || !aligned(rstd, 4)) return SO_ERR_INVALID_ARG;
    if (rows == 0) return SO_OK;
    if (!x || !y || !aligned(x, es) || !aligned(y, es)) return SO_ERR_INVALID_ARG;
    if (!valid_in_stride(rows, x_stride, cols) || !valid_out_stride(rows, y_stride, cols)) return SO_ERR_INVALID_ARG;
    if (!valid_extent(rows, x_stride) || !valid_extent(rows, y_stride)) return SO_ERR_INVALID_ARG;
    if (x == y && rows > 1 && x_stride != y_stride) return SO_ERR_INVALID_ARG;

    NormArgs a = {};
    a.x = x; a.weight = weight; a.bias = bias; a.y = y; a.mean = mean; a.rstd = rstd;
    a.x_stride = x_stride; a.y_stride = y_stride; a.rows = rows; a.cols = cols;
    a.param_dtype = param_dtype; a.eps = (float)eps; a.inv_cols = (float)(1.0 / (double)cols);
    int sms = 0;
    const so_status s = device_sms(&sms);
    if (s != SO_OK) return s;
    const unsigned grid = (unsigned)(rows < 4 * sms ? rows : 4 * sms);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == SO_DTYPE_BF16) return launch(norm_forward_loop_kernel<bf16_t>, grid, kLoopThreads, 0, st, false, a);
    if (dtype == SO_DTYPE_FP16) return launch(norm_forward_loop_kernel<f16_t>, grid, kLoopThreads, 0, st, false, a);
    return launch(norm_forward_loop_kernel<float>, grid, kLoopThreads, 0, st, false, a);
}

so_status so_layer_norm_backward_scratch(int64_t rows, int64_t cols, uint64_t *bytes)
{
    if (!bytes || rows < 0 || cols < 1 || cols > INT32_MAX) return SO_ERR_INVALID_ARG;
    const uint64_t blocks = (uint64_t)(rows < kMaxPartials ? (rows > 0 ? rows : 1) : kMaxPartials);
    *bytes = blocks * 2u * (uint64_t)cols * sizeof(float);
    return SO_OK;
}

so_status so_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x,
                                 int64_t x_stride, const void *weight, const float *mean,
                                 const float *rstd, void *dx, int64_t dx_stride, void *dweight,
                                 void *dbias, int64_t rows, int64_t cols, int32_t dtype,
                                 int32_t param_dtype, int32_t grad_dtype, int32_t accumulate,
                                 void *scratch, uint64_t scratch_bytes, void *stream)
{
    if (!valid_dtype(dtype) || (param_dtype != dtype && param_dtype != SO_DTYPE_FP32)) return SO_ERR_INVALID_ARG;
    if (!valid_dtype(grad_dtype) || (accumulate != 0 && accumulate != 1)) return SO_ERR_INVALID_ARG;
    if (rows < 0 || cols < 1 || cols > INT32_MAX) return SO_ERR_INVALID_ARG;
    const int es = elem_size(dtype), gs = elem_size(grad_dtype);
    if (weight && !aligned(weight, elem_size(param_dtype))) return SO_ERR_INVALID_ARG;
    if (!aligned(dweight, gs) || !aligned(dbias, gs)) return SO_ERR_INVALID_ARG;
    const bool reduce = dweight || dbias;
    uint64_t need = 0;
    so_layer_norm_backward_scratch(rows, cols, &need);
    if (reduce && (!scratch || !aligned(scratch, 16) || scratch_bytes < need)) return SO_ERR_INVALID_ARG;
    if (rows > 0) {
        if (!dy || !x || !dx || !mean || !rstd) return SO_ERR_INVALID_ARG;
        if (!aligned(dy, es) || !aligned(x, es) || !aligned(dx, es) || !aligned(mean, 4) || !aligned(rstd, 4))
            return SO_ERR_INVALID_ARG;
        if (!valid_in_stride(rows, x_stride, cols) || !valid_in_stride(rows, dy_stride, cols) ||
            !valid_out_stride(rows, dx_stride, cols))
            return SO_ERR_INVALID_ARG;
        if (!valid_extent(rows, x_stride) || !valid_extent(rows, dy_stride) || !valid_extent(rows, dx_stride))
            return SO_ERR_INVALID_ARG;
        if (rows > 1 && ((dx == dy && dx_stride != dy_stride) || (dx == x && dx_stride != x_stride)))
            return SO_ERR_INVALID_ARG;
    }

    NormArgs a = {};
    a.x = x; a.dy = dy; a.weight = weight; a.y = dx;
    a.mean = const_cast<float *>(mean); a.rstd = const_cast<float *>(rstd);
    a.partials = reduce ? static_cast<float *>(scratch) : nullptr;
    a.x_stride = x_stride; a.dy_stride = dy_stride; a.y_stride = dx_stride; a.rows = rows; a.cols = cols;
    a.param_dtype = param_dtype; a.inv_cols = (float)(1.0 / (double)cols);
    int sms = 0;
    so_status s = device_sms(&sms);
    if (s != SO_OK) return s;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    int64_t blocks = 2 * sms < kMaxPartials ? 2 * sms : kMaxPartials;
    if (blocks > rows) blocks = rows;
    if (rows > 0) {
        const unsigned grid = (unsigned)blocks;
        if (dtype == SO_DTYPE_BF16) s = launch(norm_backward_loop_kernel<bf16_t>, grid, kLoopThreads, 0, st, false, a);
        else if (dtype == SO_DTYPE_FP16) s = launch(norm_backward_loop_kernel<f16_t>, grid, kLoopThreads, 0, st, false, a);
        else s = launch(norm_backward_loop_kernel<float>, grid, kLoopThreads, 0, st, false, a);
        if (s != SO_OK) return s;
    }
    if (!reduce) return SO_OK;
    const unsigned grid = (unsigned)((2 * cols + 31) / 32);
    return launch(norm_reduce_kernel, grid, 32 * kReduceRows, 0, st, true, a.partials, (int)blocks, cols, dweight,
                  dbias, grad_dtype, accumulate);
}

}  // extern "C"
