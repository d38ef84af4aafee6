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

// ---- rows held in registers ------------------------------------------------------
//
// A group of threads takes a row: a warp, or a whole block if the row is
// longer.  A thread holds kNV vectors of E elements (16 bytes, or one element
// where rows are not aligned) of the row it works on, and the next row's are on
// their way meanwhile; groups walk the rows with a stride of the grid, so weight
// and bias are read once per thread and stay in registers.
//
// Statistics: each warp has the mean of its elements and the sum of squares
// around it (two passes over registers); warps are joined by
//   M2 = sum M2_w + sum n_w (mean_w - mean)^2
// which needs one barrier a row and loses nothing when the mean is large.

template <typename T, int E> struct Raw;
template <typename T> struct Raw<T, 1> { T v; };
template <> struct Raw<float, 4> { uint4 v; };
template <> struct Raw<bf16_t, 8> { uint4 v; };
template <> struct Raw<f16_t, 8> { uint4 v; };

template <typename T, int E>
__device__ __forceinline__ void load_raw(Raw<T, E> &r, const T *p)
{
    if constexpr (E == 1) r.v = *p;
    else r.v = __ldcs(reinterpret_cast<const uint4 *>(p));
}

template <typename T, int E>
__device__ __forceinline__ void widen(const Raw<T, E> &r, float (&f)[E])
{
    if constexpr (E == 1) f[0] = to_f32(r.v);
    else unpack<T>(r.v, f);
}

template <typename T, int E>
__device__ __forceinline__ void store_vec(T *p, const float (&f)[E])
{
    if constexpr (E == 1) *p = from_f32<T>(f[0]);
    else *reinterpret_cast<uint4 *>(p) = pack<T>(f);
}

// E parameters from element c, as fp32 (`fill` where the array is absent)
template <int E>
__device__ __forceinline__ void load_params(const void *p, int64_t c, int32_t dtype, float fill, float (&f)[E])
{
    if (!p) {
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = fill;
    } else if constexpr (E == 1) {
        f[0] = load_any(p, c, dtype);
    } else if (dtype == SO_DTYPE_FP32) {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            const float4 q = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + c + e);
            f[e] = q.x; f[e + 1] = q.y; f[e + 2] = q.z; f[e + 3] = q.w;
        }
    } else if constexpr (E == 8) {
        const uint4 q = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + c);
        if (dtype == SO_DTYPE_BF16) unpack<bf16_t>(q, f);
        else unpack<f16_t>(q, f);
    }
}

// How the threads of a block are dealt to rows.
struct Group {
    int threads, index, thread, warps, warp, per_block;
    __device__ explicit Group(int per_row)
    {
        threads = per_row;
        per_block = blockDim.x / per_row;
        index = threadIdx.x / per_row;
        thread = threadIdx.x - index * per_row;
        warps = per_row >> 5;
        warp = thread >> 5;
    }
    __device__ __forceinline__ void sync() const
    {
        asm volatile("bar.sync %0, %1;" ::"r"(index + 1), "r"(threads) : "memory");
    }
};

constexpr int kRowThreads = 256;          // a block: one long row's threads, or several short rows'
constexpr int kMaxRowThreads = 1024;

template <typename T, int E, int kNV, int kMaxThreads>
__global__ void __launch_bounds__(kMaxThreads) norm_forward_kernel(NormArgs a, int per_row)
{
    // weight and bias stay in registers, unless 1024 threads leave 64 registers each
    constexpr bool kHold = kNV * E <= 32 && kMaxThreads <= kRowThreads;
    __shared__ float2 s_part[2][32];      // (mean, M2) of each warp, two rows in turn
    const Group g(per_row);
    const int cols = (int)a.cols;         // rows held in registers are short
    const int64_t step = (int64_t)gridDim.x * g.per_block;
    int64_t row = (int64_t)blockIdx.x * g.per_block + g.index;
    if (g.index >= g.per_block || row >= a.rows) return;

    float w[kHold ? kNV : 1][E], b[kHold ? kNV : 1][E];
    Raw<T, E> cur[kNV], next[kNV];
    int mine = 0;                         // elements of this thread
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        const int c = (g.thread + i * g.threads) * E;
        if (c < cols) {
            load_raw<T, E>(cur[i], static_cast<const T *>(a.x) + row * a.x_stride + c);
            mine += E;
        }
    }
    if constexpr (kHold) {
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            const int c = (g.thread + i * g.threads) * E;
            if (c < cols) {
                load_params<E>(a.weight, c, a.param_dtype, 1.0f, w[i]);
                load_params<E>(a.bias, c, a.param_dtype, 0.0f, b[i]);
            }
        }
    }
    const float warp_count = warp_sum((float)mine);
    const float warp_inv = warp_count > 0.0f ? 1.0f / warp_count : 0.0f;

    for (int turn = 0; row < a.rows; row += step, turn ^= 1) {
        const bool more = row + step < a.rows;
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            const int c = (g.thread + i * g.threads) * E;
            if (more && c < cols) load_raw<T, E>(next[i], static_cast<const T *>(a.x) + (row + step) * a.x_stride + c);
        }
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            if ((g.thread + i * g.threads) * E >= cols) break;
            float f[E];
            widen<T, E>(cur[i], f);
#pragma unroll
            for (int e = 0; e < E; ++e) sum += f[e];
        }
        float mean = warp_sum(sum) * warp_inv, m2 = 0.0f;
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            if ((g.thread + i * g.threads) * E >= cols) break;
            float f[E];
            widen<T, E>(cur[i], f);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float d = f[e] - mean;
                m2 = fmaf(d, d, m2);
            }
        }
        m2 = warp_sum(m2);
        if (g.warps > 1) {
            float2 *part = s_part[turn] + g.index * g.warps;
            if ((threadIdx.x & 31) == 0) part[g.warp] = make_float2(mean, m2);
            g.sync();
            // every warp but the last has 32 kNV E elements, or as the columns end
            float total = 0.0f;
            const float first = part[0].x;
            for (int i = 0; i < g.warps; ++i) {
                int n = 0;
#pragma unroll
                for (int j = 0; j < kNV; ++j) {
                    const int left = cols - (i * 32 + j * g.threads) * E;
                    n += left <= 0 ? 0 : left < 32 * E ? left : 32 * E;
                }
                total = fmaf((float)n, part[i].x - first, total);
            }
            mean = fmaf(total, a.inv_cols, first);
            m2 = 0.0f;
            for (int i = 0; i < g.warps; ++i) {
                int n = 0;
#pragma unroll
                for (int j = 0; j < kNV; ++j) {
                    const int left = cols - (i * 32 + j * g.threads) * E;
                    n += left <= 0 ? 0 : left < 32 * E ? left : 32 * E;
                }
                const float d = part[i].x - mean;
                m2 += n > 0 ? fmaf((float)n * d, d, part[i].y) : 0.0f;
            }
        }
        const float rstd = 1.0f / sqrtf(fmaf(m2, a.inv_cols, a.eps));
        if (a.mean && g.thread == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
        T *y = static_cast<T *>(a.y) + row * a.y_stride;
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            const int c = (g.thread + i * g.threads) * E;
            if (c >= cols) break;
            float f[E], wi[E], bi[E];
            widen<T, E>(cur[i], f);
            if constexpr (!kHold) {
                load_params<E>(a.weight, c, a.param_dtype, 1.0f, wi);
                load_params<E>(a.bias, c, a.param_dtype, 0.0f, bi);
            }
#pragma unroll
            for (int e = 0; e < E; ++e)
                f[e] = fmaf((f[e] - mean) * rstd, kHold ? w[i][e] : wi[e], kHold ? b[i][e] : bi[e]);
            store_vec<T, E>(y + c, f);
            cur[i] = next[i];
        }
    }
}

// Backward: as above with both x and dy in registers, and each thread's part of
// dweight and dbias, which it keeps for all its rows.  Groups of a block are
// joined in shared memory in their order, blocks by norm_reduce_kernel.
template <typename T, int E, int kNV, int kMaxThreads>
__global__ void __launch_bounds__(kMaxThreads) norm_backward_kernel(NormArgs a, int per_row)
{
    extern __shared__ float s_sums[];     // [2][cols], if a block has several groups
    __shared__ float2 s_part[2][32];
    const Group g(per_row);
    const int cols = (int)a.cols;         // rows held in registers are short
    const int64_t step = (int64_t)gridDim.x * g.per_block;
    int64_t row = (int64_t)blockIdx.x * g.per_block + g.index;
    const bool working = g.index < g.per_block && row < a.rows;

    float w[kNV][E], dw[kNV][E], db[kNV][E];
    Raw<T, E> xc[kNV], yc[kNV], xn[kNV], yn[kNV];
    float mean = 0.0f, rstd = 0.0f;
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        const int c = (g.thread + i * g.threads) * E;
        if (working && c < cols) {
            load_raw<T, E>(xc[i], static_cast<const T *>(a.x) + row * a.x_stride + c);
            load_raw<T, E>(yc[i], static_cast<const T *>(a.dy) + row * a.dy_stride + c);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) dw[i][e] = db[i][e] = 0.0f;
    }
    if (working) {
        mean = a.mean[row];
        rstd = a.rstd[row];
    }
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        const int c = (g.thread + i * g.threads) * E;
        if (working && c < cols) load_params<E>(a.weight, c, a.param_dtype, 1.0f, w[i]);
    }

    for (int turn = 0; working && row < a.rows; row += step, turn ^= 1) {
        const bool more = row + step < a.rows;
        float mean_n = 0.0f, rstd_n = 0.0f;
        if (more) {
            mean_n = a.mean[row + step];
            rstd_n = a.rstd[row + step];
        }
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            const int c = (g.thread + i * g.threads) * E;
            if (more && c < cols) {
                load_raw<T, E>(xn[i], static_cast<const T *>(a.x) + (row + step) * a.x_stride + c);
                load_raw<T, E>(yn[i], static_cast<const T *>(a.dy) + (row + step) * a.dy_stride + c);
            }
        }
        float sg = 0.0f, sgx = 0.0f;
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            if ((g.thread + i * g.threads) * E >= cols) break;
            float x[E], d[E];
            widen<T, E>(xc[i], x);
            widen<T, E>(yc[i], d);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float xh = (x[e] - mean) * rstd, gw = d[e] * w[i][e];
                sg += gw;
                sgx = fmaf(gw, xh, sgx);
                dw[i][e] = fmaf(d[e], xh, dw[i][e]);
                db[i][e] += d[e];
            }
        }
        sg = warp_sum(sg);
        sgx = warp_sum(sgx);
        if (g.warps > 1) {
            float2 *part = s_part[turn] + g.index * g.warps;
            if ((threadIdx.x & 31) == 0) part[g.warp] = make_float2(sg, sgx);
            g.sync();
            sg = sgx = 0.0f;
            for (int i = 0; i < g.warps; ++i) {
                sg += part[i].x;
                sgx += part[i].y;
            }
        }
        const float mg = sg * a.inv_cols, mgx = sgx * a.inv_cols;
        T *dx = static_cast<T *>(a.y) + row * a.y_stride;
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            const int c = (g.thread + i * g.threads) * E;
            if (c >= cols) break;
            float x[E], d[E];
            widen<T, E>(xc[i], x);
            widen<T, E>(yc[i], d);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float xh = (x[e] - mean) * rstd;
                d[e] = rstd * fmaf(-xh, mgx, fmaf(d[e], w[i][e], -mg));
            }
            store_vec<T, E>(dx + c, d);
            xc[i] = xn[i];
            yc[i] = yn[i];
        }
        mean = mean_n;
        rstd = rstd_n;
    }

    if (!a.partials) return;
    float *out = a.partials + (int64_t)blockIdx.x * 2 * a.cols;
    float *sums = g.per_block > 1 ? s_sums : out;
    for (int turn = 0; turn < g.per_block; ++turn) {
        if (turn > 0) __syncthreads();
        if (g.index != turn) continue;
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            const int c = (g.thread + i * g.threads) * E;
            if (c >= cols) break;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float pw = turn > 0 ? sums[c + e] + dw[i][e] : dw[i][e];
                const float pb = turn > 0 ? sums[a.cols + c + e] + db[i][e] : db[i][e];
                float *to = turn == g.per_block - 1 ? out : sums;
                to[c + e] = pw;
                to[a.cols + c + e] = pb;
            }
        }
    }
}

// ---- rows too long for that ------------------------------------------------------

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

// Sums the blocks' partial rows: 32 columns a block, kReduceRows threads down each
// column, in a fixed order.
constexpr int kReduceRows = 32;

__global__ void __launch_bounds__(32 * kReduceRows)
norm_reduce_kernel(const float *partials, int n_blocks, int64_t cols, void *dweight, void *dbias,
                   int32_t grad_dtype, int32_t accumulate)
{
    __shared__ float s[kReduceRows][33];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t at = (int64_t)blockIdx.x * 32 + lane;      // column of [dweight | dbias]
    grid_dependency_wait();
    float sum = 0.0f;
    if (at < 2 * cols) {
#pragma unroll 8
        for (int i = part; i < n_blocks; i += kReduceRows) sum += partials[(int64_t)i * 2 * cols + at];
    }
    s[part][lane] = sum;
    __syncthreads();
    sum = warp_sum(s[lane][part]);                           // warp p: column p of the block
    if (lane != 0) return;
    const int64_t mine = (int64_t)blockIdx.x * 32 + part;
    if (mine >= 2 * cols) return;
    void *out = mine < cols ? dweight : dbias;
    if (!out) return;
    const int64_t c = mine < cols ? mine : mine - cols;
    if (accumulate) sum += load_any(out, c, grad_dtype);
    store_any(out, c, grad_dtype, sum);
}

constexpr int kMaxPartials = 512;         // blocks that may leave a partial row

// ---- which kernel ----------------------------------------------------------------

// How a row is dealt out: `per_row` threads with `nv` vectors of E elements each,
// blocks of `block` threads; per_row = 0: the row does not fit, use the loop.
struct Plan { int per_row, nv, block; };

// A warp takes a row of up to `warp_nv` vectors a lane, then a block of at most
// `max_threads`, with the fewest vectors a thread that are compiled.
inline Plan plan_row(int64_t vectors, int warp_nv, const int *nvs, int n_nvs, int max_threads)
{
    Plan p = {0, 0, 0};
    for (int i = 0; i < n_nvs && p.per_row == 0; ++i) {
        const int64_t threads = (vectors + nvs[i] - 1) / nvs[i];
        if (nvs[i] <= warp_nv && threads <= 32) p.per_row = 32, p.nv = nvs[i];
    }
    for (int i = 0; i < n_nvs && p.per_row == 0; ++i) {
        const int64_t threads = (vectors + nvs[i] - 1) / nvs[i];
        const int64_t most = i + 1 < n_nvs ? kRowThreads : max_threads;
        if (threads <= most) p.per_row = (int)((threads + 31) / 32 * 32), p.nv = nvs[i];
    }
    p.block = p.per_row >= kRowThreads || p.per_row == 0 ? p.per_row : kRowThreads / p.per_row * p.per_row;
    return p;
}

// Resident blocks per SM of a kernel, asked for once per device.
template <typename K>
so_status resident(K kernel, int block, size_t smem, std::atomic<int> (&cache)[kMaxDevices], int *out)
{
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return SO_ERR_CUDA;
    if (dev < 0 || dev >= kMaxDevices) return SO_ERR_UNSUPPORTED;
    // one word: the block size and shared memory it was asked for, and the answer
    const int tag = (int)((block / 32) * 4096 + (int)(smem >> 10) * 32);
    int v = cache[dev].load(std::memory_order_relaxed);
    if (v == 0 || (v & ~31) != tag) {
        int n = 0;
        if (smem > 48 * 1024 &&
            cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
            return SO_ERR_CUDA;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, block, smem) != cudaSuccess || n < 1)
            return SO_ERR_CUDA;
        v = tag | (n < 31 ? n : 31);
        cache[dev].store(v, std::memory_order_relaxed);
    }
    *out = v & 31;
    return SO_OK;
}

template <typename T, int E, int kNV, int kMaxThreads>
so_status launch_forward(const NormArgs &a, const Plan &p, int sms, cudaStream_t st)
{
    static std::atomic<int> cache[kMaxDevices];
    int per_sm = 0;
    const so_status s = resident(norm_forward_kernel<T, E, kNV, kMaxThreads>, p.block, 0, cache, &per_sm);
    if (s != SO_OK) return s;
    const int groups = p.block / p.per_row;
    const int64_t want = (a.rows + groups - 1) / groups, most = (int64_t)per_sm * sms;
    return launch(norm_forward_kernel<T, E, kNV, kMaxThreads>, (unsigned)(want < most ? want : most), p.block, 0, st,
                  false, a, p.per_row);
}

template <typename T, int E, int kNV, int kMaxThreads>
so_status launch_backward(const NormArgs &a, const Plan &p, int sms, cudaStream_t st, int *blocks)
{
    static std::atomic<int> cache[kMaxDevices];
    const int groups = p.block / p.per_row;
    const size_t smem = groups > 1 ? (size_t)a.cols * 2 * sizeof(float) : 0;
    int per_sm = 0;
    const so_status s = resident(norm_backward_kernel<T, E, kNV, kMaxThreads>, p.block, smem, cache, &per_sm);
    if (s != SO_OK) return s;
    const int64_t want = (a.rows + groups - 1) / groups;
    int64_t most = (int64_t)per_sm * sms;
    if (most > kMaxPartials) most = kMaxPartials;
    *blocks = (int)(want < most ? want : most);
    return launch(norm_backward_kernel<T, E, kNV, kMaxThreads>, (unsigned)*blocks, p.block, smem, st, false, a, p.per_row);
}

template <typename T>
so_status forward(const NormArgs &a, bool vec, int sms, cudaStream_t st)
{
    constexpr int E = Vec<T>::kElems;
    static const int vec_nv[] = {1, 2, 3, 4}, one_nv[] = {4, 8, 16};
    const Plan p = vec ? plan_row(a.cols / E, 4, vec_nv, 4, kMaxRowThreads) : plan_row(a.cols, 16, one_nv, 3, kMaxRowThreads);
    if (p.per_row == 0) {
        const unsigned grid = (unsigned)(a.rows < 4 * sms ? a.rows : 4 * sms);
        return launch(norm_forward_loop_kernel<T>, grid, kLoopThreads, 0, st, false, a);
    }
    const bool wide = p.block > kRowThreads;
    if (vec) {
        if (p.nv == 1) return launch_forward<T, E, 1, kRowThreads>(a, p, sms, st);
        if (p.nv == 2) return launch_forward<T, E, 2, kRowThreads>(a, p, sms, st);
        if (p.nv == 3) return launch_forward<T, E, 3, kRowThreads>(a, p, sms, st);
        if (!wide) return launch_forward<T, E, 4, kRowThreads>(a, p, sms, st);
        return launch_forward<T, E, 4, kMaxRowThreads>(a, p, sms, st);
    }
    if (p.nv == 4) return launch_forward<T, 1, 4, kRowThreads>(a, p, sms, st);
    if (p.nv == 8) return launch_forward<T, 1, 8, kRowThreads>(a, p, sms, st);
    return launch_forward<T, 1, 16, kMaxRowThreads>(a, p, sms, st);
}

// The backward pass keeps three values per element besides the rows, so it
// takes fewer elements a thread.
template <typename T>
so_status backward(const NormArgs &a, bool vec, int sms, cudaStream_t st, int *blocks)
{
    constexpr int E = Vec<T>::kElems;
    static const int vec_nv[] = {1, 2}, one_nv[] = {4, 8};
    constexpr int kMost = 512;
    const Plan p = vec ? plan_row(a.cols / E, 1, vec_nv, 2, kMost) : plan_row(a.cols, 8, one_nv, 2, kMost);
    if (p.per_row == 0) {
        int64_t most = 2 * sms < kMaxPartials ? 2 * sms : kMaxPartials;
        *blocks = (int)(a.rows < most ? a.rows : most);
        return launch(norm_backward_loop_kernel<T>, (unsigned)*blocks, kLoopThreads, 0, st, false, a);
    }
    const bool wide = p.block > kRowThreads;
    if (vec) {
        if (p.nv == 1) return launch_backward<T, E, 1, kRowThreads>(a, p, sms, st, blocks);
        if (!wide) return launch_backward<T, E, 2, kRowThreads>(a, p, sms, st, blocks);
        return launch_backward<T, E, 2, kMost>(a, p, sms, st, blocks);
    }
    if (p.nv == 4) return launch_backward<T, 1, 4, kRowThreads>(a, p, sms, st, blocks);
    if (!wide) return launch_backward<T, 1, 8, kRowThreads>(a, p, sms, st, blocks);
    return launch_backward<T, 1, 8, kMost>(a, p, sms, st, blocks);
}

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
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const auto fits = [&](const void *p, int64_t stride, int size) {
        return aligned(p, 16) && (rows == 1 || (stride * size) % 16 == 0);
    };
    const bool vec = (cols * es) % 16 == 0 && fits(x, x_stride, es) && fits(y, y_stride, es) && aligned(weight, 16) &&
                     aligned(bias, 16);
    if (dtype == SO_DTYPE_BF16) return forward<bf16_t>(a, vec, sms, st);
    if (dtype == SO_DTYPE_FP16) return forward<f16_t>(a, vec, sms, st);
    return forward<float>(a, vec, sms, st);
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
    int blocks = 0;
    if (rows > 0) {
        const auto fits = [&](const void *p, int64_t stride) {
            return aligned(p, 16) && (rows == 1 || (stride * es) % 16 == 0);
        };
        const bool vec = (cols * es) % 16 == 0 && fits(x, x_stride) && fits(dy, dy_stride) && fits(dx, dx_stride) &&
                         aligned(weight, 16);
        if (dtype == SO_DTYPE_BF16) s = backward<bf16_t>(a, vec, sms, st, &blocks);
        else if (dtype == SO_DTYPE_FP16) s = backward<f16_t>(a, vec, sms, st, &blocks);
        else s = backward<float>(a, vec, sms, st, &blocks);
        if (s != SO_OK) return s;
    }
    if (!reduce) return SO_OK;
    const unsigned grid = (unsigned)((2 * cols + 31) / 32);
    return launch(norm_reduce_kernel, grid, 32 * kReduceRows, 0, st, true, a.partials, blocks, cols, dweight,
                  dbias, grad_dtype, accumulate);
}

}  // extern "C"
