// The norm after a block, its gate, the scaled residual and the norm before the next
// block, forward and backward.
//
//   forward   u = N(block) pw + pb        (or u = block),  N: layer or RMS norm of a row
//             h = scale x + gate u        rounded to its type: what the next norm sees
//             y = N(h) w + b
//   backward  hat = (h - mean) rstd,  e = dy w,
//             t = dh + rstd (e - [mean(e)] - hat mean(e hat))      [layer norm only]
//             dx = scale t
//             bhat = (block - pmean) prstd,  q = t gate pw
//             dblock = prstd (q - [mean(q)] - bhat mean(q bhat))   (or t gate)
//             S1 = sum t bhat, S2 = sum t   over the rows of a gate's group
//             dgate = pw S1 + pb S2,  dpw = sum over groups of gate S1,  dpb = .. gate S2
//             dw = sum dy hat,  db = sum dy
#include "so_ops.cuh"

using namespace so_ops;

namespace {

struct Args {
    const void *x, *block, *dy, *dh, *hin;
    void *h, *y, *dx, *dblock;
    const void *gate, *pw, *pb, *w, *b;
    float *stats;                         // [4][rows]: mean and rstd of block, of h
    float *moments;                       // backward: [2][rows]: mean(e), mean(e hat)
    int64_t x_stride, block_stride, dy_stride, dh_stride, h_stride, y_stride, dx_stride, dblock_stride;
    int64_t rows, cols, group_rows;       // rows that share a gate
    int32_t param_dtype, post;
    float scale, eps, inv_cols;
};

// E elements of a row from element c
template <typename T, int E>
__device__ __forceinline__ void load_row(const void *p, int64_t at, float (&f)[E])
{
    if constexpr (E == 1) f[0] = to_f32(static_cast<const T *>(p)[at]);
    else unpack<T>(*reinterpret_cast<const uint4 *>(static_cast<const T *>(p) + at), f);
}
template <typename T, int E>
__device__ __forceinline__ void store_row(void *p, int64_t at, const float (&f)[E])
{
    if constexpr (E == 1) static_cast<T *>(p)[at] = from_f32<T>(f[0]);
    else *reinterpret_cast<uint4 *>(static_cast<T *>(p) + at) = pack<T>(f);
}
// E parameters (`fill` where there are none); aligned like the rows
template <int E>
__device__ __forceinline__ void load_params(const void *p, int64_t at, int32_t dtype, float fill, float (&f)[E])
{
    if (!p) {
#pragma unroll
        for (int i = 0; i < E; ++i) f[i] = fill;
    } else if constexpr (E == 1) {
        f[0] = load_any(p, at, dtype);
    } else if (dtype == SO_DTYPE_FP32) {
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            const float4 q = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + at + i);
            f[i] = q.x, f[i + 1] = q.y, f[i + 2] = q.z, f[i + 3] = q.w;
        }
    } else if constexpr (E == 8) {
        const uint4 q = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + at);
        if (dtype == SO_DTYPE_BF16) unpack<bf16_t>(q, f);
        else unpack<f16_t>(q, f);
    }
}

constexpr int kLoopThreads = 256;

// Sums over the block of two values, returned to every thread; the caller alternates between
// two places for them so that one barrier is enough.
__device__ __forceinline__ void block_sum2(float &a, float &b, float (*s)[2])
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    a = warp_sum(a);
    b = warp_sum(b);
    if (lane == 0) s[warp][0] = a, s[warp][1] = b;
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int i = 0; i < kLoopThreads / 32; ++i) a += s[i][0], b += s[i][1];
}

// A block per row, which comes from L1 or L2 after its first reading.
template <typename T, int E, bool kLayer>
__global__ void __launch_bounds__(kLoopThreads) forward_loop_kernel(const __grid_constant__ Args a)
{
    __shared__ float s_red[4][kLoopThreads / 32][2];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride, *block = static_cast<const T *>(a.block) + row * a.block_stride;
        T *h = static_cast<T *>(a.h) + row * a.h_stride, *y = static_cast<T *>(a.y) + row * a.y_stride;
        float pmean = 0.0f, prstd = 1.0f, none = 0.0f;
        if (a.post) {
            float sum = 0.0f, sq = 0.0f;
            if (kLayer) {
                for (int64_t c = threadIdx.x * E; c < a.cols; c += kLoopThreads * E) {
                    float f[E];
                    load_row<T, E>(block, c, f);
#pragma unroll
                    for (int i = 0; i < E; ++i) sum += f[i];
                }
                block_sum2(sum, none, s_red[0]);
                pmean = sum * a.inv_cols;
            }
            for (int64_t c = threadIdx.x * E; c < a.cols; c += kLoopThreads * E) {
                float f[E];
                load_row<T, E>(block, c, f);
#pragma unroll
                for (int i = 0; i < E; ++i) sq = fmaf(f[i] - pmean, f[i] - pmean, sq);
            }
            block_sum2(sq, none, s_red[1]);
            prstd = 1.0f / sqrtf(sq * a.inv_cols + a.eps);
        }
        const int64_t gate = row / a.group_rows * a.cols;
        float sum = 0.0f, sq = 0.0f;
        for (int64_t c = threadIdx.x * E; c < a.cols; c += kLoopThreads * E) {
            float u[E], r[E], g[E];
            load_row<T, E>(block, c, u);
            load_row<T, E>(x, c, r);
            load_params<E>(a.gate, gate + c, a.param_dtype, 1.0f, g);
            if (a.post) {
                float pw[E], pb[E];
                load_params<E>(a.pw, c, a.param_dtype, 1.0f, pw);
                load_params<E>(a.pb, c, a.param_dtype, 0.0f, pb);
#pragma unroll
                for (int i = 0; i < E; ++i) u[i] = fmaf((u[i] - pmean) * prstd, pw[i], pb[i]);
            }
#pragma unroll
            for (int i = 0; i < E; ++i) r[i] = to_f32(from_f32<T>(fmaf(g[i], u[i], r[i] * a.scale)));
            store_row<T, E>(h, c, r);
#pragma unroll
            for (int i = 0; i < E; ++i) sum += r[i];
        }
        float mean = 0.0f;
        if (kLayer) {
            block_sum2(sum, none, s_red[2]);
            mean = sum * a.inv_cols;
        }
        for (int64_t c = threadIdx.x * E; c < a.cols; c += kLoopThreads * E) {
            float f[E];
            load_row<T, E>(h, c, f);
#pragma unroll
            for (int i = 0; i < E; ++i) sq = fmaf(f[i] - mean, f[i] - mean, sq);
        }
        block_sum2(sq, none, s_red[3]);
        const float rstd = 1.0f / sqrtf(sq * a.inv_cols + a.eps);
        for (int64_t c = threadIdx.x * E; c < a.cols; c += kLoopThreads * E) {
            float f[E], w[E], b[E];
            load_row<T, E>(h, c, f);
            load_params<E>(a.w, c, a.param_dtype, 1.0f, w);
            load_params<E>(a.b, c, a.param_dtype, 0.0f, b);
#pragma unroll
            for (int i = 0; i < E; ++i) f[i] = fmaf((f[i] - mean) * rstd, w[i], b[i]);
            store_row<T, E>(y, c, f);
        }
        if (a.stats && threadIdx.x == 0) {
            a.stats[row] = pmean;
            a.stats[a.rows + row] = prstd;
            a.stats[2 * a.rows + row] = mean;
            a.stats[3 * a.rows + row] = rstd;
        }
        __syncthreads();
    }
}

// What the gradients of a row have in common.
struct RowStats { float pmean, prstd, mean, rstd; };
__device__ __forceinline__ RowStats row_stats(const Args &a, int64_t row)
{
    return RowStats{a.stats[row], a.stats[a.rows + row], a.stats[2 * a.rows + row], a.stats[3 * a.rows + row]};
}

// t of E elements, given the row's mean(e) and mean(e hat)
template <typename T, int E>
__device__ __forceinline__ void total_gradient(const Args &a, int64_t row, int64_t c, const RowStats &s, float me, float meh, float (&t)[E])
{
    float dy[E], h[E], w[E];
    load_row<T, E>(a.dy, row * a.dy_stride + c, dy);
    load_row<T, E>(a.hin, row * a.h_stride + c, h);
    load_params<E>(a.w, c, a.param_dtype, 1.0f, w);
    if (a.dh) load_row<T, E>(a.dh, row * a.dh_stride + c, t);
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const float hat = (h[i] - s.mean) * s.rstd;
        t[i] = (a.dh ? t[i] : 0.0f) + s.rstd * (fmaf(dy[i], w[i], -me) - hat * meh);
    }
}

template <typename T, int E, bool kLayer>
__global__ void __launch_bounds__(kLoopThreads) backward_loop_kernel(const __grid_constant__ Args a)
{
    __shared__ float s_red[2][kLoopThreads / 32][2];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const RowStats s = row_stats(a, row);
        const int64_t gate = row / a.group_rows * a.cols;
        float me = 0.0f, meh = 0.0f;
        for (int64_t c = threadIdx.x * E; c < a.cols; c += kLoopThreads * E) {
            float dy[E], h[E], w[E];
            load_row<T, E>(a.dy, row * a.dy_stride + c, dy);
            load_row<T, E>(a.hin, row * a.h_stride + c, h);
            load_params<E>(a.w, c, a.param_dtype, 1.0f, w);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float e = dy[i] * w[i];
                me += e;
                meh = fmaf(e, (h[i] - s.mean) * s.rstd, meh);
            }
        }
        block_sum2(me, meh, s_red[0]);
        me = kLayer ? me * a.inv_cols : 0.0f;
        meh *= a.inv_cols;
        if (a.moments && threadIdx.x == 0) {
            a.moments[row] = me;
            a.moments[a.rows + row] = meh;
        }
        float mq = 0.0f, mqb = 0.0f;
        if (a.post) {
            for (int64_t c = threadIdx.x * E; c < a.cols; c += kLoopThreads * E) {
                float t[E], u[E], g[E], pw[E];
                total_gradient<T, E>(a, row, c, s, me, meh, t);
                load_row<T, E>(a.block, row * a.block_stride + c, u);
                load_params<E>(a.gate, gate + c, a.param_dtype, 1.0f, g);
                load_params<E>(a.pw, c, a.param_dtype, 1.0f, pw);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float q = t[i] * g[i] * pw[i];
                    mq += q;
                    mqb = fmaf(q, (u[i] - s.pmean) * s.prstd, mqb);
                }
            }
            block_sum2(mq, mqb, s_red[1]);
            mq = kLayer ? mq * a.inv_cols : 0.0f;
            mqb *= a.inv_cols;
        }
        for (int64_t c = threadIdx.x * E; c < a.cols; c += kLoopThreads * E) {
            float t[E], d[E], g[E];
            total_gradient<T, E>(a, row, c, s, me, meh, t);
            load_params<E>(a.gate, gate + c, a.param_dtype, 1.0f, g);
            if (a.post) {
                float u[E], pw[E];
                load_row<T, E>(a.block, row * a.block_stride + c, u);
                load_params<E>(a.pw, c, a.param_dtype, 1.0f, pw);
#pragma unroll
                for (int i = 0; i < E; ++i)
                    d[i] = s.prstd * (fmaf(t[i] * g[i], pw[i], -mq) - (u[i] - s.pmean) * s.prstd * mqb);
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i) d[i] = t[i] * g[i];
            }
#pragma unroll
            for (int i = 0; i < E; ++i) t[i] *= a.scale;
            store_row<T, E>(a.dx, row * a.dx_stride + c, t);
            store_row<T, E>(a.dblock, row * a.dblock_stride + c, d);
        }
        __syncthreads();
    }
}

// Column sums of the rows of a part: S1, S2, sum dy hat, sum dy, each thread E columns.
// Parts never cross from one gate's rows to the next's.
template <typename T, int E>
__global__ void __launch_bounds__(kLoopThreads) columns_kernel(const __grid_constant__ Args a, float *partials, int parts_per_group, bool gates)
{
    const int64_t c = ((int64_t)blockIdx.x * kLoopThreads + threadIdx.x) * E;
    const int64_t part = blockIdx.y, group = part / parts_per_group;
    const int64_t each = (a.group_rows + parts_per_group - 1) / parts_per_group;
    int64_t row = part % parts_per_group * each, end = row + each;
    if (end > a.group_rows) end = a.group_rows;
    row += group * a.group_rows;
    end += group * a.group_rows;
    if (end > a.rows) end = a.rows;
    if (c >= a.cols) return;
    float s1[E] = {}, s2[E] = {}, t1[E] = {}, t2[E] = {};
    for (; row < end; ++row) {
        const RowStats s = row_stats(a, row);
        float dy[E], h[E];
        load_row<T, E>(a.dy, row * a.dy_stride + c, dy);
        load_row<T, E>(a.hin, row * a.h_stride + c, h);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            t1[i] = fmaf(dy[i], (h[i] - s.mean) * s.rstd, t1[i]);
            t2[i] += dy[i];
        }
        if (gates) {
            float t[E], u[E];
            total_gradient<T, E>(a, row, c, s, a.moments[row], a.moments[a.rows + row], t);
            load_row<T, E>(a.block, row * a.block_stride + c, u);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                s1[i] = fmaf(t[i], (u[i] - s.pmean) * s.prstd, s1[i]);
                s2[i] += t[i];
            }
        }
    }
    float *out = partials + part * 4 * a.cols + c;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        out[i] = s1[i];
        out[a.cols + i] = s2[i];
        out[2 * a.cols + i] = t1[i];
        out[3 * a.cols + i] = t2[i];
    }
}

struct Grads {
    const float *partials;
    void *dgate, *dpw, *dpb, *dw, *db;
    int32_t dtype, accumulate, groups, parts_per_group;
};

__device__ __forceinline__ void put(const Grads &g, void *p, int64_t at, float x)
{
    if (!p) return;
    if (g.accumulate) x += load_any(p, at, g.dtype);
    store_any(p, at, g.dtype, x);
}

// Sums the parts, 32 columns a block and a warp to every eighth part, in a fixed order.
constexpr int kSumWarps = 8;
__global__ void __launch_bounds__(32 * kSumWarps) sum_kernel(const __grid_constant__ Args a, const __grid_constant__ Grads g)
{
    __shared__ float s[4][kSumWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    const bool in = c < a.cols;
    float dpw = 0.0f, dpb = 0.0f, dw = 0.0f, db = 0.0f;
    grid_dependency_wait();
    for (int group = 0; group < g.groups; ++group) {
        float sum[4] = {};
        if (in)
            for (int p = warp; p < g.parts_per_group; p += kSumWarps) {
                const float *at = g.partials + ((int64_t)group * g.parts_per_group + p) * 4 * a.cols + c;
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[k] += at[k * a.cols];
            }
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k][warp][lane] = sum[k];
        __syncthreads();
        if (warp == 0 && in) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                sum[k] = 0.0f;
                for (int i = 0; i < kSumWarps; ++i) sum[k] += s[k][i][lane];
            }
            const float gate = a.gate ? load_any(a.gate, group * a.cols + c, a.param_dtype) : 1.0f;
            const float pw = a.pw ? load_any(a.pw, c, a.param_dtype) : 1.0f, pb = a.pb ? load_any(a.pb, c, a.param_dtype) : 0.0f;
            put(g, g.dgate, group * a.cols + c, fmaf(pw, sum[0], pb * sum[1]));
            dpw = fmaf(gate, sum[0], dpw);
            dpb = fmaf(gate, sum[1], dpb);
            dw += sum[2];
            db += sum[3];
        }
        __syncthreads();
    }
    if (warp != 0 || !in) return;
    put(g, g.dpw, c, dpw);
    put(g, g.dpb, c, dpb);
    put(g, g.dw, c, dw);
    put(g, g.db, c, db);
}

// ---- host ------------------------------------------------------------------------

constexpr int kMaxParts = 1024;           // per gate's rows, at most

// Parts a gate's rows are cut into, by the sizes alone: about 600 over all, of 16 rows at least.
int parts_of(int64_t rows, int64_t groups)
{
    const int64_t group_rows = groups > 0 ? rows / groups : 0;
    int64_t n = (600 + groups - 1) / (groups > 0 ? groups : 1);
    if (n > (group_rows + 15) / 16) n = (group_rows + 15) / 16;
    return n < 1 ? 1 : n > kMaxParts ? kMaxParts : (int)n;
}

bool row_ok(const void *p, int64_t stride, int64_t rows, int64_t cols, int size, bool out)
{
    return p && aligned(p, size) && valid_extent(rows, stride) && (out ? valid_out_stride(rows, stride, cols) : valid_in_stride(rows, stride, cols));
}
bool on16(const void *p, int64_t stride, int64_t rows, int size) { return aligned(p, 16) && (rows <= 1 || stride * size % 16 == 0); }

// Parameters: addresses that fit their type; `vec` is cleared where 16-byte loads would not do.
bool params_ok(const Args &a, int32_t param_dtype, bool *vec)
{
    for (const void *p : {a.gate, a.pw, a.pb, a.w, a.b}) {
        if (!aligned(p, elem_size(param_dtype))) return false;
        if (!aligned(p, 16)) *vec = false;
    }
    return true;
}

so_status common(int64_t rows, int64_t cols, int64_t groups, int32_t dtype, int32_t param_dtype, int32_t kind, int32_t post, double scale)
{
    if (!valid_dtype(dtype) || (param_dtype != dtype && param_dtype != SO_DTYPE_FP32)) return SO_ERR_INVALID_ARG;
    if (rows < 0 || rows > (int64_t(1) << 40) || cols < 1 || cols > (int64_t(1) << 30)) return SO_ERR_INVALID_ARG;
    if (groups < 1 || groups > 65535 || rows % groups != 0) return SO_ERR_INVALID_ARG;
    if ((kind != SO_NORM_LAYER && kind != SO_NORM_RMS) || (post != 0 && post != 1)) return SO_ERR_INVALID_ARG;
    if (!std::isfinite(scale) || !std::isfinite((float)scale)) return SO_ERR_INVALID_ARG;
    return SO_OK;
}

template <typename T>
so_status forward(const Args &a, bool vec, bool layer, int sms, cudaStream_t st)
{
    constexpr int E = Vec<T>::kElems;
    const unsigned grid = (unsigned)(a.rows < 8 * sms ? a.rows : 8 * sms);
    const auto kernel = vec ? (layer ? forward_loop_kernel<T, E, true> : forward_loop_kernel<T, E, false>)
                            : (layer ? forward_loop_kernel<T, 1, true> : forward_loop_kernel<T, 1, false>);
    return launch(kernel, grid, kLoopThreads, 0, st, false, a);
}

template <typename T>
so_status backward(const Args &a, const Grads &g, bool sums, bool vec, bool layer, int sms, cudaStream_t st)
{
    constexpr int E = Vec<T>::kElems;
    so_status s = SO_OK;
    if (a.rows > 0) {
        const unsigned grid = (unsigned)(a.rows < 8 * sms ? a.rows : 8 * sms);
        const auto kernel = vec ? (layer ? backward_loop_kernel<T, E, true> : backward_loop_kernel<T, E, false>)
                                : (layer ? backward_loop_kernel<T, 1, true> : backward_loop_kernel<T, 1, false>);
        s = launch(kernel, grid, kLoopThreads, 0, st, false, a);
        if (s != SO_OK || !sums) return s;
    }
    if (!sums) return SO_OK;
    const bool gates = g.dgate || g.dpw || g.dpb;
    const int e = vec ? E : 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.cols + (int64_t)kLoopThreads * e - 1) / ((int64_t)kLoopThreads * e)), (unsigned)(g.groups * g.parts_per_group));
    cfg.blockDim = dim3(kLoopThreads);
    cfg.stream = st;
    const auto columns = vec ? columns_kernel<T, E> : columns_kernel<T, 1>;
    if (cudaLaunchKernelEx(&cfg, columns, a, const_cast<float *>(g.partials), g.parts_per_group, gates) != cudaSuccess) return SO_ERR_CUDA;
    return launch(sum_kernel, (unsigned)((a.cols + 31) / 32), 32 * kSumWarps, 0, st, false, a, g);
}

}  // namespace

extern "C" {

so_status so_residual_norm_forward(const void *x, int64_t x_stride, const void *block, int64_t block_stride,
                                   const void *gate, int64_t groups, const void *post_weight, const void *post_bias,
                                   const void *weight, const void *bias, void *h, int64_t h_stride, void *y,
                                   int64_t y_stride, float *stats, int64_t rows, int64_t cols, int32_t dtype,
                                   int32_t param_dtype, int32_t kind, int32_t post, double scale, double eps,
                                   void *stream)
{
    const so_status c = common(rows, cols, groups, dtype, param_dtype, kind, post, scale);
    if (c != SO_OK) return c;
    if (!(eps >= 0.0) || !std::isfinite((float)eps) || (!post && (post_weight || post_bias)) || !aligned(stats, 4)) return SO_ERR_INVALID_ARG;
    const int size = elem_size(dtype);
    if (rows == 0) return SO_OK;
    if (!row_ok(x, x_stride, rows, cols, size, false) || !row_ok(block, block_stride, rows, cols, size, false) ||
        !row_ok(h, h_stride, rows, cols, size, true) || !row_ok(y, y_stride, rows, cols, size, true))
        return SO_ERR_INVALID_ARG;
    // h may take x's or the block's place, row for row; y is apart
    if (h == y || y == x || y == block || (h == x && h_stride != x_stride) || (h == block && h_stride != block_stride)) return SO_ERR_INVALID_ARG;
    Args a = {};
    a.x = x, a.block = block, a.h = h, a.y = y, a.gate = gate, a.pw = post_weight, a.pb = post_bias, a.w = weight, a.b = bias;
    a.stats = stats;
    a.x_stride = x_stride, a.block_stride = block_stride, a.h_stride = h_stride, a.y_stride = y_stride;
    a.rows = rows, a.cols = cols, a.group_rows = rows / groups, a.param_dtype = param_dtype, a.post = post;
    a.scale = (float)scale, a.eps = (float)eps, a.inv_cols = 1.0f / (float)cols;
    bool vec = cols * size % 16 == 0 && on16(x, x_stride, rows, size) && on16(block, block_stride, rows, size) &&
               on16(h, h_stride, rows, size) && on16(y, y_stride, rows, size);
    if (!params_ok(a, param_dtype, &vec)) return SO_ERR_INVALID_ARG;
    int sms;
    const so_status d = device_sms(&sms);
    if (d != SO_OK) return d;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool layer = kind == SO_NORM_LAYER;
    if (dtype == SO_DTYPE_BF16) return forward<bf16_t>(a, vec, layer, sms, st);
    if (dtype == SO_DTYPE_FP16) return forward<f16_t>(a, vec, layer, sms, st);
    return forward<float>(a, vec, layer, sms, st);
}

so_status so_residual_norm_backward_scratch(int64_t rows, int64_t cols, int64_t groups, uint64_t *bytes)
{
    if (!bytes || common(rows, cols, groups, SO_DTYPE_FP32, SO_DTYPE_FP32, SO_NORM_RMS, 0, 1.0) != SO_OK) return SO_ERR_INVALID_ARG;
    // the sums of the parts, and two means per row
    *bytes = ((uint64_t)parts_of(rows, groups) * groups * 4 * cols + 2 * (uint64_t)rows) * sizeof(float);
    return SO_OK;
}

so_status so_residual_norm_backward(const void *dy, int64_t dy_stride, const void *dh, int64_t dh_stride,
                                    const void *h, int64_t h_stride, const void *block, int64_t block_stride,
                                    const float *stats, const void *gate, int64_t groups, const void *post_weight,
                                    const void *post_bias, const void *weight, void *dx, int64_t dx_stride,
                                    void *dblock, int64_t dblock_stride, void *dgate, void *dpost_weight,
                                    void *dpost_bias, void *dweight, void *dbias, int64_t rows, int64_t cols,
                                    int32_t dtype, int32_t param_dtype, int32_t grad_dtype, int32_t kind, int32_t post,
                                    int32_t accumulate, double scale, void *scratch, uint64_t scratch_bytes, void *stream)
{
    const so_status c = common(rows, cols, groups, dtype, param_dtype, kind, post, scale);
    if (c != SO_OK) return c;
    if (!valid_dtype(grad_dtype) || (accumulate != 0 && accumulate != 1)) return SO_ERR_INVALID_ARG;
    if (!post && (post_weight || post_bias || dpost_weight || dpost_bias)) return SO_ERR_INVALID_ARG;
    for (const void *p : {dgate, dpost_weight, dpost_bias, dweight, dbias})
        if (!aligned(p, elem_size(grad_dtype))) return SO_ERR_INVALID_ARG;
    const bool sums = dgate || dpost_weight || dpost_bias || dweight || dbias;
    uint64_t need = 0;
    so_residual_norm_backward_scratch(rows, cols, groups, &need);
    if (sums && (!scratch || !aligned(scratch, 16) || scratch_bytes < need)) return SO_ERR_INVALID_ARG;
    const int size = elem_size(dtype);
    if (rows > 0) {
        if (!row_ok(dy, dy_stride, rows, cols, size, false) || (dh && !row_ok(dh, dh_stride, rows, cols, size, false)) ||
            !row_ok(h, h_stride, rows, cols, size, false) || !row_ok(block, block_stride, rows, cols, size, false) ||
            !row_ok(dx, dx_stride, rows, cols, size, true) || !row_ok(dblock, dblock_stride, rows, cols, size, true) ||
            !stats || !aligned(stats, 4))
            return SO_ERR_INVALID_ARG;
        if (dx == dblock) return SO_ERR_INVALID_ARG;
        for (const void *p : {dy, dh, h, block})
            if (p == dx || p == dblock) return SO_ERR_INVALID_ARG;
    }
    Args a = {};
    a.dy = dy, a.dh = dh, a.hin = h, a.block = block, a.dx = dx, a.dblock = dblock;
    a.gate = gate, a.pw = post_weight, a.pb = post_bias, a.w = weight;
    a.stats = const_cast<float *>(stats);
    a.dy_stride = dy_stride, a.dh_stride = dh_stride, a.h_stride = h_stride, a.block_stride = block_stride;
    a.dx_stride = dx_stride, a.dblock_stride = dblock_stride;
    a.rows = rows, a.cols = cols, a.group_rows = rows / groups, a.param_dtype = param_dtype, a.post = post;
    a.scale = (float)scale, a.inv_cols = 1.0f / (float)cols;
    bool vec = cols * size % 16 == 0 && on16(dy, dy_stride, rows, size) && (!dh || on16(dh, dh_stride, rows, size)) &&
               on16(h, h_stride, rows, size) && on16(block, block_stride, rows, size) && on16(dx, dx_stride, rows, size) &&
               on16(dblock, dblock_stride, rows, size);
    if (!params_ok(a, param_dtype, &vec)) return SO_ERR_INVALID_ARG;
    int sms;
    const so_status d = device_sms(&sms);
    if (d != SO_OK) return d;
    const int parts = parts_of(rows, groups);
    float *partials = static_cast<float *>(scratch);
    a.moments = sums ? partials + (int64_t)parts * groups * 4 * cols : nullptr;
    const Grads g = {partials, dgate, dpost_weight, dpost_bias, dweight, dbias, grad_dtype, accumulate, (int32_t)groups, parts};
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool layer = kind == SO_NORM_LAYER;
    if (dtype == SO_DTYPE_BF16) return backward<bf16_t>(a, g, sums, vec, layer, sms, st);
    if (dtype == SO_DTYPE_FP16) return backward<f16_t>(a, g, sums, vec, layer, sms, st);
    return backward<float>(a, g, sums, vec, layer, sms, st);
}

}  // extern "C"
