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
#include "so_rows.cuh"

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
    int32_t combine;                      // backward: one gate, and several groups of threads to a block
    int32_t needs_block;                  // backward: the first norm, or a sum, goes by the block
    float scale, eps, inv_cols;
    int64_t each;                         // consecutive rows of a group of threads (or of a part of the column sums)
    float *partials;                      // backward: [groups of threads + gates - 1][4][cols]
    Patience patience;
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
__device__ __forceinline__ void params_at(const void *p, int64_t at, int32_t dtype, float fill, float (&f)[E])
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
            params_at<E>(a.gate, gate + c, a.param_dtype, 1.0f, g);
            if (a.post) {
                float pw[E], pb[E];
                params_at<E>(a.pw, c, a.param_dtype, 1.0f, pw);
                params_at<E>(a.pb, c, a.param_dtype, 0.0f, pb);
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
            params_at<E>(a.w, c, a.param_dtype, 1.0f, w);
            params_at<E>(a.b, c, a.param_dtype, 0.0f, b);
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
    params_at<E>(a.w, c, a.param_dtype, 1.0f, w);
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
            params_at<E>(a.w, c, a.param_dtype, 1.0f, w);
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
                params_at<E>(a.gate, gate + c, a.param_dtype, 1.0f, g);
                params_at<E>(a.pw, c, a.param_dtype, 1.0f, pw);
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
            params_at<E>(a.gate, gate + c, a.param_dtype, 1.0f, g);
            if (a.post) {
                float u[E], pw[E];
                load_row<T, E>(a.block, row * a.block_stride + c, u);
                params_at<E>(a.pw, c, a.param_dtype, 1.0f, pw);
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


// ---- aligned rows through a ring of bulk copies ----------------------------------------
//
// A group of threads, a warp or several, takes consecutive rows: a thread holds its columns'
// parameters in registers for all of them (the gate's until the next one's rows begin), the
// rows come through a ring of bulk copies in shared memory.  A row is read from there once for
// each of its two norms, whose sums the group exchanges; the second exchange also tells the
// group's first thread that everyone is done with the row's place, which it refills.
//
// A copy that does not arrive in time turns the rows that the group has not written into NaN,
// statistics and gradients of parameters included.

// E values one by one.  Pairs (Vals) halve the arithmetic's instructions, but a row's scalars have to be
// paired with themselves and registers come in twos: 32768 x 4096 bf16 forward takes 195 us with
// pairs and 173 us without, backward with sums 186 us with pairs and 195 us without.
template <int E> struct Floats {
    float f[E];
    __device__ __forceinline__ void set(float x)
    {
#pragma unroll
        for (int i = 0; i < E; ++i) f[i] = x;
    }
    __device__ __forceinline__ void get(float (&o)[E]) const
    {
#pragma unroll
        for (int i = 0; i < E; ++i) o[i] = f[i];
    }
    __device__ __forceinline__ void put(const float (&o)[E])
    {
#pragma unroll
        for (int i = 0; i < E; ++i) f[i] = o[i];
    }
};
#define SO_EACH(expr) do { _Pragma("unroll") for (int i = 0; i < E; ++i) r.f[i] = (expr); return r; } while (0)
template <int E> __device__ __forceinline__ Floats<E> operator+(const Floats<E> &a, const Floats<E> &b) { Floats<E> r; SO_EACH(a.f[i] + b.f[i]); }
template <int E> __device__ __forceinline__ Floats<E> operator+(const Floats<E> &a, float b) { Floats<E> r; SO_EACH(a.f[i] + b); }
template <int E> __device__ __forceinline__ Floats<E> operator*(const Floats<E> &a, const Floats<E> &b) { Floats<E> r; SO_EACH(a.f[i] * b.f[i]); }
template <int E> __device__ __forceinline__ Floats<E> operator*(const Floats<E> &a, float b) { Floats<E> r; SO_EACH(a.f[i] * b); }
template <int E> __device__ __forceinline__ Floats<E> fma(const Floats<E> &a, const Floats<E> &b, const Floats<E> &c) { Floats<E> r; SO_EACH(fmaf(a.f[i], b.f[i], c.f[i])); }
template <int E> __device__ __forceinline__ Floats<E> fma(const Floats<E> &a, float b, const Floats<E> &c) { Floats<E> r; SO_EACH(fmaf(a.f[i], b, c.f[i])); }
template <int E> __device__ __forceinline__ Floats<E> fma(const Floats<E> &a, float b, float c) { Floats<E> r; SO_EACH(fmaf(a.f[i], b, c)); }
#undef SO_EACH
template <int E> __device__ __forceinline__ float total(const Floats<E> &a)
{
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < E; ++i) s += a.f[i];
    return s;
}

// V: Vals<E> or Floats<E>, E elements of 16 bytes of T
template <typename V, typename T> __device__ __forceinline__ V widen_as(const uint4 &bits)
{
    V v;
    if constexpr (std::is_same<V, Vals<Vec<T>::kElems>>::value) {
        v = widen16<T>(bits);
    } else {
        float f[Vec<T>::kElems];
        unpack<T>(bits, f);
        v.put(f);
    }
    return v;
}
template <typename T, typename V> __device__ __forceinline__ uint4 narrow(const V &v)
{
    float f[Vec<T>::kElems];
    v.get(f);
    return pack<T>(f);
}
template <typename V> __device__ __forceinline__ V all(float x)
{
    V v;
    v.set(x);
    return v;
}
template <typename V, int E> __device__ __forceinline__ V params_as(const void *p, int64_t at, int32_t dtype, float fill)
{
    float f[E];
    params_at<E>(p, at, dtype, fill, f);
    V v;
    v.put(f);
    return v;
}

constexpr int kRingBars = 64;             // groups x stages of a block, at most
constexpr int kMaxWarps = 16;             // of a group

struct RingShared {
    uint64_t full[kRingBars];
    float part[2][4][kMaxWarps];          // of an exchange and the one before: up to four values of every warp
    float count[kMaxWarps];               // elements of a warp
    int gave_up[8], issued[8];
};

// What a kernel leaves out: biases and their gradients with the RMS norm; the mean with either.
enum Form { kPlainRms, kBiasedRms, kLayerNorm };

// One row in `kNV` vectors a thread; kFull: every thread has all of them.
template <typename T, int E, int kNV, bool kFull>
struct Columns {
    const Group &g;
    int cols;
    float mine, warp_n;                   // elements of this thread, of its warp
    __device__ Columns(const Group &g_, int cols_) : g(g_), cols(cols_)
    {
        mine = 0.0f;
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (has(i)) mine += E;
        warp_n = warp_sum(mine);
    }
    __device__ __forceinline__ int at(int i) const { return (g.thread + i * g.threads) * E; }
    __device__ __forceinline__ bool has(int i) const { return kFull || at(i) < cols; }
};

// The exchanges of a row.  A warp sums N values at once (its lanes end with one each, in groups of
// 32 / N) and leaves them in shared memory; behind the barrier a lane takes what some of the warps left
// of its value, and 32 / N lanes add up.
struct Exchange {
    const Group &g;
    float (*part)[4][kMaxWarps];          // from the group's first warp on
    __device__ Exchange(const Group &g_, RingShared &s) : g(g_), part(reinterpret_cast<float (*)[4][kMaxWarps]>(&s.part[0][0][g_.index * g_.warps])) {}

    static __device__ __forceinline__ float add16(float x)
    {
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
        return x;
    }
    // what the lanes' warps hold of the k-th exchange
    __device__ __forceinline__ float take(int k) const
    {
        const int lane = threadIdx.x & 31, w = lane & 15;
        return w < g.warps ? part[k][lane >> 4][w] : 0.0f;
    }
    __device__ __forceinline__ void leave(int k, float one) const
    {
        const int lane = threadIdx.x & 31;
        if ((lane & 15) == 0) part[k][lane >> 4][g.warp] = one;
        g.sync();
    }
    static __device__ __forceinline__ float2 both(float one)
    {
        return make_float2(__shfl_sync(0xFFFFFFFFu, one, 0), __shfl_sync(0xFFFFFFFFu, one, 16));
    }
    // N sums over the group (2 or 4)
    template <int N>
    __device__ __forceinline__ void sums(int k, float (&v)[N]) const
    {
        constexpr int kLanes = 32 / N;
        float one = warp_sum_many<N>(v);
        if (g.warps > 1) {
            const int lane = threadIdx.x & 31, value = lane / kLanes, at = lane % kLanes;
            if (at == 0) part[k][value][g.warp] = one;
            g.sync();
            one = 0.0f;
#pragma unroll
            for (int w = 0; w < kMaxWarps; w += kLanes)
                if (w + at < g.warps) one += part[k][value][w + at];
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) one += __shfl_xor_sync(0xFFFFFFFFu, one, o);
        } else {
            __syncwarp();
        }
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xFFFFFFFFu, one, i * kLanes);
    }
    __device__ __forceinline__ float sum(int k, float a) const
    {
        a = warp_sum(a);
        if (g.warps > 1) {
            if ((threadIdx.x & 31) == 0) part[k][0][g.warp] = a;
            g.sync();
            const int w = threadIdx.x & 15;
            a = add16(w < g.warps ? part[k][0][w] : 0.0f);
        } else {
            __syncwarp();
        }
        return a;
    }
    // mean and squares around it of the group, from each warp's
    __device__ __forceinline__ float2 join(int k, float mean, float m2, const float *count, float inv_cols) const
    {
        if (g.warps == 1) {
            __syncwarp();
            return make_float2(mean, m2);
        }
        const int lane = threadIdx.x & 31, w = lane & 15;
        leave(k, lane < 16 ? mean : m2);
        const float one = take(k), n = w < g.warps && lane < 16 ? count[w] : 0.0f;
        mean = __shfl_sync(0xFFFFFFFFu, add16(one * n), 0) * inv_cols;
        return make_float2(mean, warp_sum(lane < 16 ? (one - mean) * (one - mean) * n : one));
    }
};

// Mean (0 with the RMS norm) and 1 / sqrt(variance + eps) of a row.  Layer norm in one exchange:
// a warp has the mean of its first lane's elements as its centre c, and with n_t, m_t, Q_t each
// thread's number, mean and squares around that mean,
//   D = sum n_t (m_t - c),  Q = sum (Q_t + n_t (m_t - c)^2),
// so that its mean is c + D / n, and its squares around that Q - D^2 / n; warps are joined by
// M2 = sum (M2_w + n_w (mean_w - mean)^2).
template <bool kLayer, typename V, typename T, int E, int kNV, bool kFull>
__device__ __forceinline__ float2 row_statistics(const Columns<T, E, kNV, kFull> &c, const Exchange &x, int k, const float *count, const V (&f)[kNV],
                                                 float inv_mine, float inv_warp, float inv_cols, float eps)
{
    V acc;
    acc.set(0.0f);
    if constexpr (!kLayer) {
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (c.has(i)) acc = fma(f[i], f[i], acc);
        return make_float2(0.0f, 1.0f / sqrtf(x.sum(k, total(acc)) * inv_cols + eps));
    } else {
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (c.has(i)) acc = acc + f[i];
        const float m = total(acc) * inv_mine;
        acc.set(0.0f);
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (c.has(i)) {
                const V d = f[i] + -m;
                acc = fma(d, d, acc);
            }
        const float centre = __shfl_sync(0xFFFFFFFFu, m, 0), d = kFull || c.mine > 0.0f ? m - centre : 0.0f;
        float v[2] = {d * c.mine, fmaf(d * c.mine, d, total(acc))};
        const float2 w = Exchange::both(warp_sum_many<2>(v));
        const float2 r = x.join(k, centre + w.x * inv_warp, w.y - w.x * w.x * inv_warp, count, inv_cols);
        return make_float2(r.x, 1.0f / sqrtf(r.y * inv_cols + eps));
    }
}

// What the two kernels share: the ring of `kMats` rows a stage, and who waits for what.
template <int kMats>
struct Ring {
    const Group &g;
    RingShared &s;
    uint32_t base, bars, row_bytes, stage_bytes;
    int stages, stage, turn;
    uint32_t phase, polls;
    __device__ Ring(const Group &g_, RingShared &s_, uint8_t *room, uint32_t row_bytes_, int stages_, uint32_t polls_)
        : g(g_), s(s_), row_bytes(row_bytes_), stages(stages_), stage(0), turn(1), phase(0), polls(polls_)
    {
        stage_bytes = row_bytes * kMats;
        base = smem_addr(room) + (uint32_t)(g.index * stages) * stage_bytes;
        bars = smem_addr(s.full) + (uint32_t)(g.index * stages) * 8;
        if (threadIdx.x < (unsigned)(g.per_block * stages)) {
            mbar_init(smem_addr(s.full + threadIdx.x), 1);
            mbar_init_fence();            // before any group's first thread issues a copy
        }
        if (g.thread == 0) {
            s.gave_up[g.index] = polls == 0;
            s.issued[g.index] = 0;
        }
    }
    // by the group's first thread: row copies into stage `at`
    __device__ __forceinline__ void fill(int at, const char *const (&src)[kMats]) const
    {
        uint32_t n = 0;
#pragma unroll
        for (int k = 0; k < kMats; ++k) n += src[k] ? row_bytes : 0;
        mbar_expect(bars + at * 8, n);
#pragma unroll
        for (int k = 0; k < kMats; ++k)
            if (src[k]) bulk_load(base + at * stage_bytes + k * row_bytes, src[k], row_bytes, bars + at * 8);
        ++s.issued[g.index];
    }
    // The turn (from 1 on) whose wait ran out is in shared memory; a thread that is a turn behind the
    // one that ran out goes by the number, so that all of the group stop at the same row.
    __device__ __forceinline__ bool gave_up() const
    {
        const int at = *const_cast<const volatile int *>(&s.gave_up[g.index]);
        return at != 0 && at <= turn;
    }
    __device__ __forceinline__ void wait() const
    {
        if (!mbar_test(bars + stage * 8, phase) && !gave_up() && !mbar_wait(bars + stage * 8, phase, polls))
            *const_cast<volatile int *>(&s.gave_up[g.index]) = turn;
    }
    __device__ __forceinline__ uint32_t row(int k) const { return base + stage * stage_bytes + k * row_bytes; }
    __device__ __forceinline__ void next()
    {
        ++turn;
        if (++stage == stages) stage = 0, phase ^= 1;
    }
};

// Bound: memory (two reads, two writes).  32768 x 4096 bf16: 173 us in a short run, 6.2 TB/s, 95 % of a copy's rate
// (186 to 207 us in long ones); 8192 x 8192 94 us for 82 of bytes; 65536 x 768 92 us for 61 (a warp to a row,
// 24 elements a lane; with three warps to a row 139 us).  One row of 4096: 5 us on the device.  Rows read once
// for each pass from L2, without the ring: 32768 x 4096 290 us.
template <typename T, Form kForm, int kNV, bool kFull, int kMaxThreads>
__global__ void __launch_bounds__(kMaxThreads, kMaxThreads <= 256 && kNV * Vec<T>::kElems <= 16 ? 2 : 1) forward_ring_kernel(const __grid_constant__ Args a, int per_row, int stages)
{
    constexpr int E = Vec<T>::kElems;
    using V = Floats<E>;
    constexpr bool kLayer = kForm == kLayerNorm, kBias = kForm != kPlainRms;
    extern __shared__ __align__(128) uint8_t s_room[];
    __shared__ __align__(8) RingShared s;
    const Group g(per_row);
    Ring<2> ring(g, s, s_room, (uint32_t)a.cols * sizeof(T), stages, a.patience.of((int)blockIdx.x));
    const Columns<T, E, kNV, kFull> c(g, (int)a.cols);
    const Exchange x(g, s);
    const float *count = s.count + g.index * g.warps;
    if ((threadIdx.x & 31) == 0) s.count[threadIdx.x >> 5] = c.warp_n;
    const float inv_mine = c.mine > 0.0f ? 1.0f / c.mine : 0.0f, inv_warp = 1.0f / c.warp_n;
    __syncthreads();
    int64_t row = ((int64_t)blockIdx.x * g.per_block + g.index) * a.each, end = row + a.each;
    if (end > a.rows) end = a.rows;
    const auto fill = [&](int at, int64_t r) {
        const char *const src[2] = {reinterpret_cast<const char *>(static_cast<const T *>(a.x) + r * a.x_stride),
                                    reinterpret_cast<const char *>(static_cast<const T *>(a.block) + r * a.block_stride)};
        ring.fill(at, src);
    };
    if (g.thread == 0)
        for (int n = 0; n < stages && row + n < end; ++n) fill(n, row + n);
    V w[kNV], b[kNV], gw[kNV], gb[kNV];                // gw, gb: gate times the first norm's
#pragma unroll
    for (int i = 0; i < kNV; ++i)
        if (c.has(i)) {
            w[i] = params_as<V, E>(a.w, c.at(i), a.param_dtype, 1.0f);
            if (kBias) b[i] = params_as<V, E>(a.b, c.at(i), a.param_dtype, 0.0f);
        }
    int64_t gate_end = 0;
    T *h = static_cast<T *>(a.h) + row * a.h_stride, *y = static_cast<T *>(a.y) + row * a.y_stride;
    for (; row < end; ++row, h += a.h_stride, y += a.y_stride) {
        if (row >= gate_end) {
            const int64_t gate = row / a.group_rows;
            gate_end = (gate + 1) * a.group_rows;
#pragma unroll
            for (int i = 0; i < kNV; ++i)
                if (c.has(i)) {
                    gw[i] = a.gate ? params_as<V, E>(static_cast<const char *>(a.gate) + gate * a.cols * (a.param_dtype == SO_DTYPE_FP32 ? 4 : 2), c.at(i), a.param_dtype, 1.0f)
                                   : all<V>(1.0f);
                    if (kBias) gb[i] = a.pb ? gw[i] * params_as<V, E>(a.pb, c.at(i), a.param_dtype, 0.0f) : all<V>(0.0f);
                    if (a.pw) gw[i] = gw[i] * params_as<V, E>(a.pw, c.at(i), a.param_dtype, 1.0f);
                }
        }
        ring.wait();
        float2 post = make_float2(0.0f, 1.0f);
        V f[kNV];
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (c.has(i)) f[i] = widen_as<V, T>(lds16(ring.row(1) + c.at(i) * sizeof(T)));
        if (a.post) post = row_statistics<kLayer>(c, x, 0, count, f, inv_mine, inv_warp, a.inv_cols, a.eps);
        const float shift = -post.x * post.y;
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (c.has(i)) {
                const V from = widen_as<V, T>(lds16(ring.row(0) + c.at(i) * sizeof(T)));
                // in fp32 the mean is taken off first: rows far from zero keep their digits
                const V hat = !kLayer ? f[i] * post.y : sizeof(T) == 4 ? (f[i] + -post.x) * post.y : fma(f[i], post.y, shift);
                const uint4 bits = narrow<T>(fma(gw[i], hat, kBias ? fma(from, a.scale, gb[i]) : from * a.scale));
                *reinterpret_cast<uint4 *>(h + c.at(i)) = bits;
                f[i] = widen_as<V, T>(bits);
            }
        const float2 st = row_statistics<kLayer>(c, x, 1, count, f, inv_mine, inv_warp, a.inv_cols, a.eps);
        if (ring.gave_up()) break;
        if (g.thread == 0) {
            if (row + stages < end) fill(ring.stage, row + stages);
            if (a.stats) {
                a.stats[row] = post.x;
                a.stats[a.rows + row] = post.y;
                a.stats[2 * a.rows + row] = st.x;
                a.stats[3 * a.rows + row] = st.y;
            }
        }
        const float back = -st.x * st.y;
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (c.has(i)) {
                const V hat = !kLayer ? f[i] * st.y : sizeof(T) == 4 ? (f[i] + -st.x) * st.y : fma(f[i], st.y, back);
                *reinterpret_cast<uint4 *>(y + c.at(i)) = narrow<T>(kBias ? fma(hat, w[i], b[i]) : hat * w[i]);
            }
        ring.next();
        // one exchange a row: its place must not be written again before all have read it
        if (!a.post && g.warps > 1) g.sync();
    }
    if (row >= end) return;
    if (g.thread == 0) land(ring.bars, s.issued[g.index], stages);
    const uint4 nan = narrow<T>(all<V>(kNan));
    for (; row < end; ++row, h += a.h_stride, y += a.y_stride) {
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (c.has(i)) {
                *reinterpret_cast<uint4 *>(h + c.at(i)) = nan;
                *reinterpret_cast<uint4 *>(y + c.at(i)) = nan;
            }
        if (a.stats && g.thread == 0)
            for (int k = 0; k < 4; ++k) a.stats[k * a.rows + row] = kNan;
    }
}

// kSums: the thread keeps its columns' S1, S2, sum dy hat and sum dy, and leaves them as a part
// of its own where a gate's rows or its own end: part t + i for the t-th group of threads in the
// rows of gate i.  Without kSums the rows' means are left for the sums to be taken from.
//
// The second half of a row and the first half of the next one share an exchange and its barrier.
//
// Bound: what a row costs the few warps that the registers leave room for, then memory (four reads, two writes).
// 16384 x 4096 layer norm: 220 registers, eight warps an SM, 570 instructions a row and warp of 16 elements a lane
// with its exchange, at 36 % of the issue slots and 54 % of DRAM's peak rate.  32768 x 2048 bf16 with 16 gates 184 us
// for 123 of bytes, 16384 x 4096 187 us with layer norm and 166 us in the plain form, 32768 x 1024 fp32 145 us for 123, 65536 x 768 bf16 147 us for 92.
// Two exchanges a row instead of one: 224 us for the first of these; two rows a turn: 257 us; 8 elements a thread
// instead of 16: 206 us.  The loop, with rows and columns' sums in passes of their own: 579 us.
template <typename T, Form kForm, bool kSums, int kNV, bool kFull, int kMaxThreads>
__global__ void __launch_bounds__(kMaxThreads, kMaxThreads <= 256 && kNV * Vec<T>::kElems <= 8 ? 2 : 1) backward_ring_kernel(const __grid_constant__ Args a, int per_row, int stages)
{
    constexpr int E = Vec<T>::kElems;
    using V = typename std::conditional<kMaxThreads == 512, Floats<E>, Vals<E>>::type;   // (pairs spill at 128 registers)
    constexpr bool kLayer = kForm == kLayerNorm, kBias = kForm != kPlainRms;
    constexpr int kEach = kLayer ? 2 : 1;                    // sums of half a row
    extern __shared__ __align__(128) uint8_t s_room[];
    __shared__ __align__(8) RingShared s;
    const Group g(per_row);
    Ring<4> ring(g, s, s_room, (uint32_t)a.cols * sizeof(T), stages, a.patience.of((int)blockIdx.x));
    const Columns<T, E, kNV, kFull> c(g, (int)a.cols);
    const Exchange x(g, s);
    __syncthreads();
    const int64_t me = (int64_t)blockIdx.x * g.per_block + g.index;
    int64_t row = me * a.each, end = row + a.each;
    if (end > a.rows) end = a.rows;
    const auto fill = [&](int at, int64_t r) {
        const char *const src[4] = {reinterpret_cast<const char *>(static_cast<const T *>(a.dy) + r * a.dy_stride),
                                    reinterpret_cast<const char *>(static_cast<const T *>(a.hin) + r * a.h_stride),
                                    a.dh ? reinterpret_cast<const char *>(static_cast<const T *>(a.dh) + r * a.dh_stride) : nullptr,
                                    a.needs_block ? reinterpret_cast<const char *>(static_cast<const T *>(a.block) + r * a.block_stride) : nullptr};
        ring.fill(at, src);
    };
    if (g.thread == 0)
        for (int n = 0; n < stages && row + n < end; ++n) fill(n, row + n);
    V w[kNV], gw[kNV], s1[kNV], s2[kNV], t1[kNV], t2[kNV];   // gw: gate times the first norm's weight
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        if (c.has(i)) w[i] = params_as<V, E>(a.w, c.at(i), a.param_dtype, 1.0f);
        if (kSums) s1[i].set(0.0f), s2[i].set(0.0f), t1[i].set(0.0f), t2[i].set(0.0f);
    }
    const auto leave = [&](int64_t gate) {
        float *out = a.partials + (me + gate) * 4 * a.cols;
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (c.has(i)) {
                V *const v[4] = {&s1[i], &s2[i], &t1[i], &t2[i]};
#pragma unroll
                for (int k = 0; k < 4; k += kBias ? 1 : 2) {
                    float f[E];
                    v[k]->get(f);
#pragma unroll
                    for (int j = 0; j < E; j += 4)
                        *reinterpret_cast<float4 *>(out + k * a.cols + c.at(i) + j) = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
                    v[k]->set(0.0f);
                }
            }
    };
    const auto norm = [&](const V &v, float mean, float rstd) {
        return !kLayer ? v * rstd : sizeof(T) == 4 ? (v + -mean) * rstd : fma(v, rstd, -mean * rstd);
    };
    // first half of a row: e and hat, their sums into v[0] (and v[1])
    const auto first_half = [&](uint32_t at, const RowStats &st, float *v) {
        V sum, dot;
        sum.set(0.0f), dot.set(0.0f);
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (c.has(i)) {
                const V dy = widen_as<V, T>(lds16(at + c.at(i) * sizeof(T))), q = dy * w[i];
                const V u = norm(widen_as<V, T>(lds16(at + ring.row_bytes + c.at(i) * sizeof(T))), st.mean, st.rstd);
                if (kLayer) sum = sum + q;
                dot = fma(q, u, dot);
                if (kSums) t1[i] = fma(dy, u, t1[i]);
                if (kSums && kBias) t2[i] = t2[i] + dy;
            }
        v[0] = total(dot);
        if (kLayer) v[1] = total(sum);
    };
    const bool any = row < end;           // (the last blocks may have groups without rows)
    if (!any && !a.combine) return;
    int64_t gate = row / a.group_rows, gate_end = (gate + 1) * a.group_rows;
    const auto load_gate = [&]() {
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (c.has(i)) {
                gw[i] = a.gate ? params_as<V, E>(static_cast<const char *>(a.gate) + gate * a.cols * (a.param_dtype == SO_DTYPE_FP32 ? 4 : 2), c.at(i), a.param_dtype, 1.0f)
                               : all<V>(1.0f);
                if (a.pw) gw[i] = gw[i] * params_as<V, E>(a.pw, c.at(i), a.param_dtype, 1.0f);
            }
    };
    if (any) load_gate();
    T *dx = static_cast<T *>(a.dx) + row * a.dx_stride, *dblock = static_cast<T *>(a.dblock) + row * a.dblock_stride;
    RowStats st = {}, next = {};
    float v[2 * kEach];                   // sums of a second half, and of the next row's first
    if (any) {
        st = row_stats(a, row);
        if (row + 1 < end) next = row_stats(a, row + 1);
        ring.wait();
        float first[2] = {0.0f, 0.0f};
        first_half(ring.row(0), st, first);
        x.template sums<2>(0, first);
        v[kEach] = first[0];
        if (kLayer) v[2 * kEach - 1] = first[1];
    }
    bool lost = false;
    int turn = 1;                         // exchanges so far
    for (; row < end; ++row, dx += a.dx_stride, dblock += a.dblock_stride) {
        const float meh = v[kEach] * a.inv_cols, me_ = kLayer ? v[2 * kEach - 1] * a.inv_cols : 0.0f;
        if (!kSums && a.moments && g.thread == 0) {
            a.moments[row] = me_;
            a.moments[a.rows + row] = meh;
        }
        // second half: t = dh + rstd (e - me) - rstd meh hat
        const float c0 = -st.rstd * me_, c1 = -st.rstd * meh;
        const uint32_t at = ring.row(0);
        V t[kNV], bhat[kNV], sum, dot;
        sum.set(0.0f), dot.set(0.0f);
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (c.has(i)) {
                const auto from = [&](int k) { return widen_as<V, T>(lds16(at + k * ring.row_bytes + c.at(i) * sizeof(T))); };
                const V u = norm(from(1), st.mean, st.rstd), q = from(0) * w[i];
                t[i] = fma(u, c1, kLayer ? fma(q, st.rstd, c0) : q * st.rstd);
                if (a.dh) t[i] = t[i] + from(2);
                if (a.needs_block) {
                    const V d = t[i] * gw[i];
                    bhat[i] = norm(from(3), st.pmean, st.prstd);
                    if (kLayer) sum = sum + d;
                    dot = fma(d, bhat[i], dot);
                    if (kSums) s1[i] = fma(t[i], bhat[i], s1[i]);
                }
                if (kSums && kBias) s2[i] = s2[i] + t[i];
            }
        v[0] = total(dot);
        if (kLayer) v[1] = total(sum);
        const int stage = ring.stage;
        const RowStats now = st;
        if (row + 1 < end) {
            ring.next();
            st = next;
            if (row + 2 < end) next = row_stats(a, row + 2);
            ring.wait();
            first_half(ring.row(0), st, v + kEach);
        }
        x.template sums<2 * kEach>(turn++ & 1, v);
        if (ring.gave_up()) {
            lost = true;
            break;
        }
        if (g.thread == 0 && row + stages < end) fill(stage, row + stages);
        const float c2 = kLayer ? -now.prstd * v[1] * a.inv_cols : 0.0f, c3 = -now.prstd * v[0] * a.inv_cols;
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (c.has(i)) {
                *reinterpret_cast<uint4 *>(dx + c.at(i)) = narrow<T>(t[i] * a.scale);
                V d = t[i] * gw[i];
                if (a.post) d = fma(bhat[i], c3, kLayer ? fma(d, now.prstd, c2) : d * now.prstd);
                *reinterpret_cast<uint4 *>(dblock + c.at(i)) = narrow<T>(d);
            }
        if (row + 1 >= gate_end && row + 1 < end) {
            // (the sums of dy go by no gate: that of the row ahead may be in this part)
            if (kSums) leave(gate);
            gate = (row + 1) / a.group_rows;
            gate_end = (gate + 1) * a.group_rows;
            load_gate();
        }
    }
    if (lost) {
        if (g.thread == 0) land(ring.bars, s.issued[g.index], stages);
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (kSums) s1[i].set(kNan), s2[i].set(kNan), t1[i].set(kNan), t2[i].set(kNan);
    }
    if (kSums && !a.combine) {
        leave(gate);
        if (lost)
            for (const int64_t last = (end - 1) / a.group_rows; gate < last;) {
#pragma unroll
                for (int i = 0; i < kNV; ++i) s1[i].set(kNan), s2[i].set(kNan), t1[i].set(kNan), t2[i].set(kNan);
                leave(++gate);
            }
    } else if (kSums) {
        // one gate: the block's groups add up in shared memory, one after the other, and leave one part
        float *room = reinterpret_cast<float *>(s_room);
        for (int k = 0; k < g.per_block; ++k) {
            __syncthreads();              // (first of all: nobody reads a row there any more)
            if (k != g.index) continue;
            float *out = a.partials + (int64_t)blockIdx.x * 4 * a.cols;
#pragma unroll
            for (int i = 0; i < kNV; ++i)
                if (c.has(i)) {
                    V *const sums[4] = {&s1[i], &s2[i], &t1[i], &t2[i]};
#pragma unroll
                    for (int n = 0; n < 4; n += kBias ? 1 : 2) {
                        float f[E];
                        sums[n]->get(f);
#pragma unroll
                        for (int j = 0; j < E; j += 4) {
                            const int64_t at = n * a.cols + c.at(i) + j;
                            float4 q = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
                            if (k > 0) {
                                const float4 o = *reinterpret_cast<const float4 *>(room + at);
                                q.x += o.x, q.y += o.y, q.z += o.z, q.w += o.w;
                            }
                            *reinterpret_cast<float4 *>((k + 1 == g.per_block ? out : room) + at) = q;
                        }
                    }
                }
        }
    }
    if (!lost) return;
    const uint4 nan = narrow<T>(all<V>(kNan));
    for (; row < end; ++row) {
#pragma unroll
        for (int i = 0; i < kNV; ++i)
            if (c.has(i)) {
                *reinterpret_cast<uint4 *>(static_cast<T *>(a.dx) + row * a.dx_stride + c.at(i)) = nan;
                *reinterpret_cast<uint4 *>(static_cast<T *>(a.dblock) + row * a.dblock_stride + c.at(i)) = nan;
            }
        if (!kSums && a.moments && g.thread == 0) a.moments[row] = a.moments[a.rows + row] = kNan;
    }
}

// ---- sums over rows ------------------------------------------------------------------

// Column sums of the rows of a part: S1, S2, sum dy hat, sum dy, each thread E columns.  A part that
// crosses from one gate's rows to the next's leaves two sums, as above.
template <typename T, int E>
__global__ void __launch_bounds__(kLoopThreads) columns_kernel(const __grid_constant__ Args a, bool gates)
{
    grid_dependency_wait();
    const int64_t c = ((int64_t)blockIdx.x * kLoopThreads + threadIdx.x) * E;
    int64_t row = (int64_t)blockIdx.y * a.each, end = row + a.each;
    if (end > a.rows) end = a.rows;
    if (c >= a.cols) return;
    while (row < end) {
        const int64_t gate = row / a.group_rows;
        const int64_t stop = end < (gate + 1) * a.group_rows ? end : (gate + 1) * a.group_rows;
        float s1[E] = {}, s2[E] = {}, t1[E] = {}, t2[E] = {};
        for (; row < stop; ++row) {
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
        float *out = a.partials + ((int64_t)blockIdx.y + gate) * 4 * a.cols + c;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            out[i] = s1[i];
            out[a.cols + i] = s2[i];
            out[2 * a.cols + i] = t1[i];
            out[3 * a.cols + i] = t2[i];
        }
    }
}

struct Grads {
    void *dgate, *dpw, *dpb, *dw, *db;
    int32_t dtype, accumulate, groups;
    int32_t biased;                       // the parts hold S2 and sum dy too
};

__device__ __forceinline__ void put(const Grads &g, void *p, int64_t at, float x)
{
    if (!p) return;
    if (g.accumulate) x += load_any(p, at, g.dtype);
    store_any(p, at, g.dtype, x);
}

// Sums the parts, 32 columns a block, in a fixed order.  kByGate: a warp to every gate in turn,
// else all warps to the parts of one gate after the other.
constexpr int kSumWarps = 16;
template <bool kByGate>
__global__ void __launch_bounds__(32 * kSumWarps) sum_kernel(const __grid_constant__ Args a, const __grid_constant__ Grads g)
{
    __shared__ float s[4][kSumWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    const bool in = c < a.cols, gates = g.dgate || g.dpw || g.dpb;
    const float pw = in && a.pw ? load_any(a.pw, c, a.param_dtype) : 1.0f, pb = in && a.pb ? load_any(a.pb, c, a.param_dtype) : 0.0f;
    float dpw = 0.0f, dpb = 0.0f, dw = 0.0f, db = 0.0f;
    grid_dependency_wait();
    for (int gate = kByGate ? warp : 0; gate < g.groups; gate += kByGate ? kSumWarps : 1) {
        float sum[4] = {};
        if (in && a.rows > 0) {
            // the parts whose rows reach into this gate's
            const int64_t first = gate * a.group_rows / a.each, last = ((gate + 1) * a.group_rows - 1) / a.each;
#pragma unroll 4
            for (int64_t t = first + (kByGate ? 0 : warp); t <= last; t += kByGate ? 1 : kSumWarps) {
                const float *at = a.partials + (t + gate) * 4 * a.cols + c;
                if (gates) sum[0] += at[0];
                if (gates && g.biased) sum[1] += at[a.cols];
                sum[2] += at[2 * a.cols];
                if (g.biased) sum[3] += at[3 * a.cols];
            }
        }
        if (!kByGate) {
#pragma unroll
            for (int k = 0; k < 4; ++k) s[k][warp][lane] = sum[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                sum[k] = 0.0f;
                if (warp == 0)
                    for (int i = 0; i < kSumWarps; ++i) sum[k] += s[k][i][lane];
            }
            __syncthreads();
        }
        if (in && (kByGate || warp == 0)) {
            const float weight = a.gate ? load_any(a.gate, gate * a.cols + c, a.param_dtype) : 1.0f;
            put(g, g.dgate, gate * a.cols + c, fmaf(pw, sum[0], pb * sum[1]));
            dpw = fmaf(weight, sum[0], dpw);
            dpb = fmaf(weight, sum[1], dpb);
            dw += sum[2];
            db += sum[3];
        }
    }
    if (kByGate) {
        s[0][warp][lane] = dpw, s[1][warp][lane] = dpb, s[2][warp][lane] = dw, s[3][warp][lane] = db;
        __syncthreads();
        if (warp == 0) {
            dpw = dpb = dw = db = 0.0f;
            for (int i = 0; i < kSumWarps; ++i) dpw += s[0][i][lane], dpb += s[1][i][lane], dw += s[2][i][lane], db += s[3][i][lane];
        }
    }
    if (warp != 0 || !in) return;
    put(g, g.dpw, c, dpw);
    put(g, g.dpb, c, dpb);
    put(g, g.dw, c, dw);
    put(g, g.db, c, db);
}

// ---- host ------------------------------------------------------------------------

// Groups of threads (or parts of the column sums) whose sums there is room for: about 16 MB of them.
int64_t most_parts(int64_t rows, int64_t cols)
{
    int64_t n = (int64_t(1) << 24) / (16 * cols);
    if (n > 1184) n = 1184;
    if (n < 148) n = 148;
    return n < rows ? n : rows > 0 ? rows : 1;
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

// How a row is dealt out: `per_row` threads with `nv` vectors each, blocks of `block`; 0: by the loop.
struct Plan { int per_row, nv, block; };

// The choice that leaves the fewest lanes idle, and the most vectors a thread of equals (fewer warps
// share a row): `least`, twice or three times that many vectors, the latter two for blocks of 256 and 512.
Plan plan_rows(int64_t vectors, int least, int most = 0, bool wide = true)
{
    Plan best = {0, 0, 0};
    int64_t waste = INT64_MAX;
    for (int nv = most ? most : 3 * least; nv >= least; nv -= least) {
        const int64_t threads = ((vectors + nv - 1) / nv + 31) / 32 * 32, idle = threads * nv - vectors;
        if (threads > (wide && (nv == 2 * least || most) ? 32 * kMaxWarps : 256) || idle >= waste) continue;
        waste = idle;
        best = {(int)threads, nv, threads >= 256 ? (int)threads : (int)(256 / threads * threads)};
    }
    return best;
}

constexpr int kRingBytes = 100 * 1024;    // of a block's ring, or twice that where only one block of threads fits an SM
constexpr int kMostShared = 220 * 1024;

int ring_stages(size_t stage_bytes, int groups, int block)
{
    int stages = (int)((block > 256 ? 2 : 1) * kRingBytes / stage_bytes);
    stages = stages > 4 ? 4 : stages < 2 ? 2 : stages;
    return stages < kRingBars / groups ? stages : kRingBars / groups;
}

// Launches a ring kernel on as many groups of threads as the device has room for (at most `most`),
// each with its share of consecutive rows; a.each is set to it.
template <typename K>
so_status launch_ring(K kernel, std::atomic<uint64_t> (&cache)[kMaxDevices], Args &a, const Plan &p, int mats, int size, int64_t most, int sms, cudaStream_t st)
{
    const int groups = p.block / p.per_row;
    const size_t stage = (size_t)a.cols * size * mats * groups;
    const int stages = ring_stages(stage, groups, p.block);
    const size_t smem = stage * stages;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return SO_ERR_CUDA;
    if (dev < 0 || dev >= kMaxDevices) return SO_ERR_UNSUPPORTED;
    // resident blocks per SM, asked for again only when block or shared memory change (the key is exact)
    const uint64_t tag = (uint64_t)smem << 24 | (uint64_t)p.block << 8;
    uint64_t v = cache[dev].load(std::memory_order_relaxed);
    if ((v & ~uint64_t(255)) != tag) {
        int n = 0;
        if (smem > 40 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared) != cudaSuccess) return SO_ERR_CUDA;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, p.block, smem) != cudaSuccess || n < 1) return SO_ERR_CUDA;
        v = tag | (uint64_t)(n < 255 ? n : 255);
        cache[dev].store(v, std::memory_order_relaxed);
    }
    int64_t units = (int64_t)(v & 255) * sms * groups;
    if (units > most) units = most / groups * groups;
    if (units < groups) units = groups;
    a.each = (a.rows + units - 1) / units;
    const int64_t used = (a.rows + a.each - 1) / a.each;
    a.combine = a.combine && groups > 1;
    const so_status done = launch(kernel, (unsigned)((used + groups - 1) / groups), p.block, smem, st, false, a, p.per_row, stages);
    if (a.combine) a.each *= groups;      // of a part
    return done;
}

template <typename T, Form kForm, int kNV>
so_status forward_ring(Args &a, const Plan &p, int sms, cudaStream_t st)
{
    static std::atomic<uint64_t> cache[4][kMaxDevices];
    const bool full = (int64_t)p.per_row * p.nv * Vec<T>::kElems == a.cols;
    if (p.block <= 256 && full) return launch_ring(forward_ring_kernel<T, kForm, kNV, true, 256>, cache[0], a, p, 2, sizeof(T), INT64_MAX, sms, st);
    if (p.block <= 256) return launch_ring(forward_ring_kernel<T, kForm, kNV, false, 256>, cache[1], a, p, 2, sizeof(T), INT64_MAX, sms, st);
    if constexpr (kNV * Vec<T>::kElems == 16) {
        if (full) return launch_ring(forward_ring_kernel<T, kForm, kNV, true, 512>, cache[2], a, p, 2, sizeof(T), INT64_MAX, sms, st);
        return launch_ring(forward_ring_kernel<T, kForm, kNV, false, 512>, cache[3], a, p, 2, sizeof(T), INT64_MAX, sms, st);
    }
    return SO_ERR_INVALID_ARG;            // no plan has long rows of other vectors
}

template <typename T, Form kForm>
so_status forward(Args &a, bool vec, int sms, cudaStream_t st)
{
    constexpr int E = Vec<T>::kElems;
    constexpr bool kLayer = kForm == kLayerNorm;
    if (vec && a.cols * (int64_t)sizeof(T) * 2 * 2 <= kMostShared) {
        const Plan p = plan_rows(a.cols / E, 8 / E);
        if (p.nv == 24 / E) return forward_ring<T, kForm, 24 / E>(a, p, sms, st);
        if (p.nv == 16 / E) return forward_ring<T, kForm, 16 / E>(a, p, sms, st);
        if (p.nv == 8 / E) return forward_ring<T, kForm, 8 / E>(a, p, sms, st);
    }
    const unsigned grid = (unsigned)(a.rows < 8 * sms ? a.rows : 8 * sms);
    return launch(vec ? forward_loop_kernel<T, E, kLayer> : forward_loop_kernel<T, 1, kLayer>, grid, kLoopThreads, 0, st, false, a);
}

template <typename T, Form kForm, int kNV>
so_status backward_ring(Args &a, const Plan &p, int64_t most, int sms, cudaStream_t st)
{
    static std::atomic<uint64_t> cache[4][kMaxDevices];
    const bool full = (int64_t)p.per_row * p.nv * Vec<T>::kElems == a.cols;
    if (p.block <= 256 && full) return launch_ring(backward_ring_kernel<T, kForm, true, kNV, true, 256>, cache[0], a, p, 4, sizeof(T), most, sms, st);
    if (p.block <= 256) return launch_ring(backward_ring_kernel<T, kForm, true, kNV, false, 256>, cache[1], a, p, 4, sizeof(T), most, sms, st);
    if constexpr (kNV * Vec<T>::kElems == 16 && kForm == kPlainRms) {
        if (full) return launch_ring(backward_ring_kernel<T, kForm, true, kNV, true, 512>, cache[2], a, p, 4, sizeof(T), most, sms, st);
        return launch_ring(backward_ring_kernel<T, kForm, true, kNV, false, 512>, cache[3], a, p, 4, sizeof(T), most, sms, st);
    }
    return SO_ERR_INVALID_ARG;            // no plan has long rows of other vectors
}

// Without sums: 16 elements a thread.
template <typename T, Form kForm>
so_status backward_rows(Args &a, const Plan &p, int sms, cudaStream_t st)
{
    constexpr int kNV = 16 / Vec<T>::kElems;
    static std::atomic<uint64_t> cache[2][kMaxDevices];
    if (p.block <= 256) return launch_ring(backward_ring_kernel<T, kForm, false, kNV, false, 256>, cache[0], a, p, 4, sizeof(T), INT64_MAX, sms, st);
    return launch_ring(backward_ring_kernel<T, kForm, false, kNV, false, 512>, cache[1], a, p, 4, sizeof(T), INT64_MAX, sms, st);
}

template <typename T, Form kForm>
so_status backward(Args &a, const Grads &g, bool sums, bool vec, int sms, cudaStream_t st)
{
    constexpr int E = Vec<T>::kElems;
    constexpr bool kLayer = kForm == kLayerNorm;
    const int64_t most = most_parts(a.rows, a.cols);
    a.each = 1;
    a.combine = a.group_rows == a.rows;
    a.needs_block = a.post || (sums && (g.dgate || g.dpw || g.dpb));
    bool taken = false;                   // the rows' kernel has left the parts of the sums
    if (a.rows > 0) {
        const bool ring = vec && a.cols * (int64_t)sizeof(T) * 4 * 2 <= kMostShared;
        // with sums 512 threads have registers for those of the plain form alone (8192 x 8192 bf16: 220 us;
        // layer norm 559 us, against 383 us with sums of their own)
        const Plan with = ring && sums ? plan_rows(a.cols / E, 8 / E, 0, kForm == kPlainRms) : Plan{0, 0, 0};
        const Plan without = ring ? plan_rows(a.cols / E, 16 / E, 16 / E) : Plan{0, 0, 0};
        so_status s;
        if (with.nv) {
            taken = true;
            s = with.nv == 24 / E   ? backward_ring<T, kForm, 24 / E>(a, with, most, sms, st)
                : with.nv == 16 / E ? backward_ring<T, kForm, 16 / E>(a, with, most, sms, st)
                                    : backward_ring<T, kForm, 8 / E>(a, with, most, sms, st);
        } else if (without.nv) {
            a.combine = 0;
            s = backward_rows<T, kForm>(a, without, sms, st);
        } else {
            const unsigned grid = (unsigned)(a.rows < 8 * sms ? a.rows : 8 * sms);
            s = launch(vec ? backward_loop_kernel<T, E, kLayer> : backward_loop_kernel<T, 1, kLayer>, grid, kLoopThreads, 0, st, false, a);
        }
        if (s != SO_OK || !sums) return s;
    }
    if (!sums) return SO_OK;
    if (!taken && a.rows > 0) {
        const bool gates = g.dgate || g.dpw || g.dpb;
        const int64_t across = (a.cols + (int64_t)kLoopThreads * (vec ? E : 1) - 1) / ((int64_t)kLoopThreads * (vec ? E : 1));
        // some thousand blocks in all, of 16 rows at least
        int64_t parts = (4096 + across - 1) / across;
        if (parts > (a.rows + 15) / 16) parts = (a.rows + 15) / 16;
        if (parts > most) parts = most;
        a.each = (a.rows + parts - 1) / parts;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)across, (unsigned)((a.rows + a.each - 1) / a.each));
        cfg.blockDim = dim3(kLoopThreads);
        cfg.stream = st;
        if (cudaLaunchKernelEx(&cfg, vec ? columns_kernel<T, E> : columns_kernel<T, 1>, a, gates) != cudaSuccess) return SO_ERR_CUDA;
    }
    const auto kernel = g.groups >= kSumWarps ? sum_kernel<true> : sum_kernel<false>;
    return launch(kernel, (unsigned)((a.cols + 31) / 32), 32 * kSumWarps, 0, st, true, a, g);
}

template <typename F>
so_status by_form(Form form, F fn)
{
    if (form == kLayerNorm) return fn(std::integral_constant<Form, kLayerNorm>());
    if (form == kBiasedRms) return fn(std::integral_constant<Form, kBiasedRms>());
    return fn(std::integral_constant<Form, kPlainRms>());
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
    const Span at_x(x, rows, x_stride, cols, size), at_block(block, rows, block_stride, cols, size), at_h(h, rows, h_stride, cols, size),
        at_y(y, rows, y_stride, cols, size);
    if ((!at_h.same(at_x) && overlap(at_h, at_x)) || (!at_h.same(at_block) && overlap(at_h, at_block)) || overlap(at_y, at_x) ||
        overlap(at_y, at_block) || overlap(at_y, at_h))
        return SO_ERR_INVALID_ARG;
    Args a = {};
    a.x = x, a.block = block, a.h = h, a.y = y, a.gate = gate, a.pw = post_weight, a.pb = post_bias, a.w = weight, a.b = bias;
    a.stats = stats;
    a.x_stride = x_stride, a.block_stride = block_stride, a.h_stride = h_stride, a.y_stride = y_stride;
    a.rows = rows, a.cols = cols, a.group_rows = rows / groups, a.param_dtype = param_dtype, a.post = post;
    a.scale = (float)scale, a.eps = (float)eps, a.inv_cols = 1.0f / (float)cols;
    a.patience = patience();
    bool vec = cols * size % 16 == 0 && on16(x, x_stride, rows, size) && on16(block, block_stride, rows, size) &&
               on16(h, h_stride, rows, size) && on16(y, y_stride, rows, size);
    if (!params_ok(a, param_dtype, &vec)) return SO_ERR_INVALID_ARG;
    int sms;
    const so_status d = device_sms(&sms);
    if (d != SO_OK) return d;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const Form form = kind == SO_NORM_LAYER ? kLayerNorm : post_bias || bias ? kBiasedRms : kPlainRms;
    if (dtype == SO_DTYPE_BF16) return by_form(form, [&](auto f) { return forward<bf16_t, decltype(f)::value>(a, vec, sms, st); });
    if (dtype == SO_DTYPE_FP16) return by_form(form, [&](auto f) { return forward<f16_t, decltype(f)::value>(a, vec, sms, st); });
    return by_form(form, [&](auto f) { return forward<float, decltype(f)::value>(a, vec, sms, st); });
}

so_status so_residual_norm_backward_scratch(int64_t rows, int64_t cols, int64_t groups, uint64_t *bytes)
{
    if (!bytes || common(rows, cols, groups, SO_DTYPE_FP32, SO_DTYPE_FP32, SO_NORM_RMS, 0, 1.0) != SO_OK) return SO_ERR_INVALID_ARG;
    // the sums of the parts, and two means per row
    *bytes = ((uint64_t)(most_parts(rows, cols) + groups - 1) * 4 * cols + 2 * (uint64_t)rows) * sizeof(float);
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
        const Span at_dx(dx, rows, dx_stride, cols, size), at_dblock(dblock, rows, dblock_stride, cols, size);
        if (overlap(at_dx, at_dblock)) return SO_ERR_INVALID_ARG;
        for (const Span &in : {Span(dy, rows, dy_stride, cols, size), Span(dh, dh ? rows : 0, dh_stride, cols, size),
                               Span(h, rows, h_stride, cols, size), Span(block, rows, block_stride, cols, size)})
            if (overlap(at_dx, in) || overlap(at_dblock, in)) return SO_ERR_INVALID_ARG;
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
    a.partials = static_cast<float *>(scratch);
    a.moments = sums ? a.partials + (most_parts(rows, cols) + groups - 1) * 4 * cols : nullptr;
    a.patience = patience();
    const Form form = kind == SO_NORM_LAYER ? kLayerNorm : post_bias || dpost_bias || dbias ? kBiasedRms : kPlainRms;
    const Grads g = {dgate, dpost_weight, dpost_bias, dweight, dbias, grad_dtype, accumulate, (int32_t)groups, form != kPlainRms};
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == SO_DTYPE_BF16) return by_form(form, [&](auto f) { return backward<bf16_t, decltype(f)::value>(a, g, sums, vec, sms, st); });
    if (dtype == SO_DTYPE_FP16) return by_form(form, [&](auto f) { return backward<f16_t, decltype(f)::value>(a, g, sums, vec, sms, st); });
    return by_form(form, [&](auto f) { return backward<float, decltype(f)::value>(a, g, sums, vec, sms, st); });
}

}  // extern "C"
