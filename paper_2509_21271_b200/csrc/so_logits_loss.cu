// Losses on the logits with their gradient: distillation from a teacher's top
// logits, and the clipped policy loss with a KL term.
//
// Both are one softmax per row and a few entries of that row:
//
//   M = max z, S = sum exp((z - M) / T), q_j = exp((z_j - M) / T) / S
//   distillation  loss = T^2 sum_k p_k (log p_k - log q[id_k])
//                 grad_j = w s T (q_j - P_j),   P_j = sum of p_k with id_k = j
//   policy        loss from logp = log q[token];  grad_j = -w s slope / T (q_j - [j = token])
//
// so the gradient is coef * (q_j - P_j) with P zero but for the targets of the row.
#include "so_ops.cuh"

using namespace so_ops;

namespace {

enum Mode { kDistill = 0, kPolicy = 1 };

struct LossArgs {
    const void *logits;
    void *grad;                           // nullptr: the loss alone
    const float *weight;                  // nullptr: 1
    float *row_loss, *logp;
    int64_t stride, grad_stride, rows, vocab;
    float temperature, inv_temperature, log2e_over_t, grad_scale;
    int32_t ids_dtype;
    // distillation
    const void *ids, *teacher;
    int64_t ids_stride, teacher_stride;
    int32_t top_k, teacher_dtype;
    // policy (ids: the tokens)
    const float *advantage, *old_logp, *ref_logp;
    float clip_lo, clip_hi, kl_coef;      // clip_lo = 1 - clip_low, clip_hi = 1 + clip_high
};

// The targets of a row, in shared memory.  id < 0 marks an empty entry.
struct Targets {
    int32_t id[SO_DISTILL_MAX_TOP_K];
    float p[SO_DISTILL_MAX_TOP_K];        // the teacher's probability
    float logp[SO_DISTILL_MAX_TOP_K];     // and its logarithm
    float z[SO_DISTILL_MAX_TOP_K];        // the student's logit there
    int32_t live;                         // 0: no entry, the row counts as masked
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Running maximum m and sum s of exp((z - m) / T) over the elements seen.  A sum
// stays 0 while everything was -inf; NaN reaches the sum, not the maximum.
struct MaxSum { float m, s; };

__device__ __forceinline__ void add_element(MaxSum &a, float z, float c)
{
    if (z > a.m) {
        a.s = a.m == -CUDART_INF_F ? a.s : a.s * exp2_fast((a.m - z) * c);
        a.m = z;
    }
    a.s += exp2_fast((z - (a.m == -CUDART_INF_F ? 0.0f : a.m)) * c);
}

__device__ __forceinline__ MaxSum merge(const MaxSum &a, const MaxSum &b, float c)
{
    const float m = fmaxf(a.m, b.m);
    MaxSum r;
    r.m = m;
    r.s = (a.m == m || a.m == -CUDART_INF_F ? a.s : a.s * exp2_fast((a.m - m) * c)) +
          (b.m == m || b.m == -CUDART_INF_F ? b.s : b.s * exp2_fast((b.m - m) * c));
    return r;
}

__device__ __forceinline__ MaxSum warp_merge(MaxSum a, float c)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        MaxSum b;
        b.m = __shfl_xor_sync(0xFFFFFFFFu, a.m, o);
        b.s = __shfl_xor_sync(0xFFFFFFFFu, a.s, o);
        a = merge(a, b, c);
    }
    return a;
}

// One warp fills the targets of a distillation row: the teacher's softmax over
// the entries that are there.
template <typename T>
__device__ void load_teacher(const LossArgs &a, int64_t row, Targets &t)
{
    const int lane = threadIdx.x & 31;
    const T *z = static_cast<const T *>(a.logits) + row * a.stride;
    MaxSum ms{-CUDART_INF_F, 0.0f};
    bool any = false;
    for (int k = lane; k < a.top_k; k += 32) {
        const int64_t id = load_id(a.ids, row * a.ids_stride + k, a.ids_dtype);
        const float x = load_any(a.teacher, row * a.teacher_stride + k, a.teacher_dtype);
        const bool ok = id >= 0 && id < a.vocab && x != -CUDART_INF_F;
        t.id[k] = ok ? (int32_t)id : -1;
        t.logp[k] = x;
        t.z[k] = ok ? to_f32(z[id]) : 0.0f;
        if (ok) {
            any = true;
            if (x > ms.m) {
                ms.s = ms.m == -CUDART_INF_F ? ms.s : ms.s * expf((ms.m - x) * a.inv_temperature);
                ms.m = x;
            }
            ms.s += expf((x - (ms.m == -CUDART_INF_F ? 0.0f : ms.m)) * a.inv_temperature);
        }
    }
    for (int o = 16; o > 0; o >>= 1) {
        MaxSum b;
        b.m = __shfl_xor_sync(0xFFFFFFFFu, ms.m, o);
        b.s = __shfl_xor_sync(0xFFFFFFFFu, ms.s, o);
        const float m = fmaxf(ms.m, b.m);
        const float sa = ms.m == m || ms.m == -CUDART_INF_F ? ms.s : ms.s * expf((ms.m - m) * a.inv_temperature);
        const float sb = b.m == m || b.m == -CUDART_INF_F ? b.s : b.s * expf((b.m - m) * a.inv_temperature);
        ms.m = m;
        ms.s = sa + sb;
    }
    const float inv = 1.0f / ms.s, log_s = logf(ms.s);
    for (int k = lane; k < a.top_k; k += 32) {
        const float d = (t.logp[k] - ms.m) * a.inv_temperature;
        t.p[k] = t.id[k] >= 0 ? expf(d) * inv : 0.0f;
        t.logp[k] = d - log_s;
    }
    any = __any_sync(0xFFFFFFFFu, any);
    if (lane == 0) t.live = any;
    __syncwarp();
}

// sum_k p_k (log p_k - log q[id_k]) by one warp; log q = (z - m) / T - log_s.
__device__ float distill_row_loss(const LossArgs &a, const Targets &t, float m, float log_s)
{
    float sum = 0.0f;
    for (int k = threadIdx.x & 31; k < a.top_k; k += 32)
        if (t.id[k] >= 0 && t.p[k] != 0.0f)
            sum = fmaf(t.p[k], t.logp[k] - ((t.z[k] - m) * a.inv_temperature - log_s), sum);
    return warp_sum(sum) * a.temperature * a.temperature;
}

// Loss and slope d loss / d logp of a policy row.
__device__ __forceinline__ void policy_row(const LossArgs &a, int64_t row, float logp, float &loss, float &slope)
{
    const float adv = a.advantage[row];
    const float ratio = a.old_logp ? expf(logp - a.old_logp[row]) : 1.0f;
    const float free_gain = ratio * adv;
    const float held_gain = fminf(fmaxf(ratio, a.clip_lo), a.clip_hi) * adv;
    // written so that a NaN ratio or advantage stays NaN in both
    const bool held = held_gain < free_gain;
    loss = -(held ? held_gain : free_gain);
    slope = held ? 0.0f : -free_gain;
    if (a.ref_logp) {
        const float d = a.ref_logp[row] - logp;
        const float e = expm1f(d);
        loss = fmaf(a.kl_coef, e - d, loss);
        slope = fmaf(-a.kl_coef, e, slope);
    }
}

// ---- a block per row, the row read twice -----------------------------------------

constexpr int kRowThreads = 512;

template <typename T, int kMode>
__global__ void __launch_bounds__(kRowThreads) loss_two_pass_kernel(LossArgs a)
{
    __shared__ Targets t;
    __shared__ MaxSum s_ms[kRowThreads / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *z = static_cast<const T *>(a.logits) + row * a.stride;
        T *g = a.grad ? static_cast<T *>(a.grad) + row * a.grad_stride : nullptr;
        const float w = a.weight ? a.weight[row] : 1.0f;
        int64_t token = -1;
        if (kMode == kPolicy) token = load_id(a.ids, row, a.ids_dtype);
        bool live = w != 0.0f && (kMode == kDistill || (token >= 0 && token < a.vocab));
        if (live && warp == 0) {
            if (kMode == kDistill) load_teacher<T>(a, row, t);
            else if (lane == 0) {
                t.id[0] = (int32_t)token;
                t.p[0] = 1.0f;
                t.z[0] = to_f32(z[token]);
                t.live = 1;
            }
        }
        __syncthreads();
        live = live && t.live;
        if (!live) {
            if (g)
                for (int64_t j = threadIdx.x; j < a.vocab; j += kRowThreads) g[j] = from_f32<T>(0.0f);
            if (threadIdx.x == 0) {
                a.row_loss[row] = 0.0f;
                if (kMode == kPolicy && a.logp) a.logp[row] = 0.0f;
            }
            __syncthreads();
            continue;
        }
        MaxSum ms{-CUDART_INF_F, 0.0f};
        for (int64_t j = threadIdx.x; j < a.vocab; j += kRowThreads) add_element(ms, to_f32(z[j]), a.log2e_over_t);
        ms = warp_merge(ms, a.log2e_over_t);
        if (lane == 0) s_ms[warp] = ms;
        __syncthreads();
        ms = s_ms[0];
        for (int i = 1; i < kRowThreads / 32; ++i) ms = merge(ms, s_ms[i], a.log2e_over_t);
        const float log_s = logf(ms.s);
        float coef;
        if (kMode == kDistill) {
            if (warp == 0) {
                const float loss = distill_row_loss(a, t, ms.m, log_s);
                if (lane == 0) a.row_loss[row] = loss;
            }
            coef = a.grad_scale * w * a.temperature;
        } else {
            const float logp = (t.z[0] - ms.m) * a.inv_temperature - log_s;
            float loss, slope;
            policy_row(a, row, logp, loss, slope);
            if (threadIdx.x == 0) {
                a.row_loss[row] = loss;
                if (a.logp) a.logp[row] = logp;
            }
            coef = -a.grad_scale * w * slope * a.inv_temperature;
        }
        if (g) {
            const float inv_s = 1.0f / ms.s, scaled = coef * inv_s;
            for (int64_t j = threadIdx.x; j < a.vocab; j += kRowThreads)
                g[j] = from_f32<T>(exp2_fast((to_f32(z[j]) - ms.m) * a.log2e_over_t) * scaled);
            __syncthreads();
            const int n = kMode == kDistill ? a.top_k : 1;
            for (int k = threadIdx.x; k < n; k += kRowThreads) {
                const int32_t id = t.id[k];
                if (id < 0) continue;
                float p = 0.0f;
                for (int i = 0; i < n; ++i)
                    if (t.id[i] == id) p += t.p[i];
                g[id] = from_f32<T>(coef * (exp2_fast((t.z[k] - ms.m) * a.log2e_over_t) * inv_s - p));
            }
        }
        __syncthreads();
    }
}

// loss = sum of weight * row_loss, in fp64 and in a fixed order
constexpr int kTotalThreads = 1024;

__global__ void __launch_bounds__(kTotalThreads)
loss_total_kernel(const float *row_loss, const float *weight, int64_t rows, float *loss)
{
    __shared__ double s[32];
    grid_dependency_wait();
    double sum = 0.0;
    for (int64_t r = threadIdx.x; r < rows; r += kTotalThreads) {
        const double l = row_loss[r];
        const double w = weight ? (double)weight[r] : 1.0;
        sum += w == 0.0 ? 0.0 : w * l;
    }
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    sum = s[threadIdx.x];
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (threadIdx.x == 0) *loss = (float)sum;
}

template <int kMode>
so_status run_loss(const LossArgs &a, int32_t dtype, float *loss, cudaStream_t st)
{
    int sms = 0;
    so_status s = device_sms(&sms);
    if (s != SO_OK) return s;
    if (a.rows > 0) {
        const unsigned grid = (unsigned)(a.rows < 4 * sms ? a.rows : 4 * sms);
        if (dtype == SO_DTYPE_BF16) s = launch(loss_two_pass_kernel<bf16_t, kMode>, grid, kRowThreads, 0, st, false, a);
        else if (dtype == SO_DTYPE_FP16) s = launch(loss_two_pass_kernel<f16_t, kMode>, grid, kRowThreads, 0, st, false, a);
        else s = launch(loss_two_pass_kernel<float, kMode>, grid, kRowThreads, 0, st, false, a);
        if (s != SO_OK) return s;
    }
    return launch(loss_total_kernel, 1, kTotalThreads, 0, st, true, a.row_loss, a.weight, a.rows, loss);
}

// What both losses check; fills the shared part of the arguments.
so_status common_args(LossArgs &a, const void *logits, int64_t stride, const float *weight, int64_t rows,
                      int64_t vocab, int32_t dtype, double temperature, double grad_scale, void *grad,
                      int64_t grad_stride, float *row_loss, float *loss, const void *ids, int32_t ids_dtype)
{
    if (!valid_dtype(dtype) || !valid_ids(ids_dtype)) return SO_ERR_INVALID_ARG;
    if (rows < 0 || vocab < 1 || vocab > (int64_t(1) << 30)) return SO_ERR_INVALID_ARG;
    if (!(temperature > 0.0) || !std::isfinite(temperature) || !std::isfinite(grad_scale)) return SO_ERR_INVALID_ARG;
    const float t = (float)temperature, inv = (float)(1.0 / temperature);
    if (!(t > 0.0f) || !std::isfinite(t) || !(inv > 0.0f) || !std::isfinite(inv) || !std::isfinite((float)grad_scale))
        return SO_ERR_INVALID_ARG;
    if (!loss || !aligned(loss, 4) || !aligned(weight, 4)) return SO_ERR_INVALID_ARG;
    const int es = elem_size(dtype);
    if (rows > 0) {
        if (!logits || !aligned(logits, es) || !row_loss || !aligned(row_loss, 4)) return SO_ERR_INVALID_ARG;
        if (!ids || !aligned(ids, ids_dtype == SO_IDS_INT64 ? 8 : 4)) return SO_ERR_INVALID_ARG;
        if (!valid_in_stride(rows, stride, vocab) || !valid_extent(rows, stride)) return SO_ERR_INVALID_ARG;
        if (grad) {
            if (!aligned(grad, es)) return SO_ERR_INVALID_ARG;
            if (!valid_out_stride(rows, grad_stride, vocab) || !valid_extent(rows, grad_stride)) return SO_ERR_INVALID_ARG;
            if (grad == logits && rows > 1 && grad_stride != stride) return SO_ERR_INVALID_ARG;
        }
    }
    a.logits = logits; a.grad = grad; a.weight = weight; a.row_loss = row_loss; a.stride = stride;
    a.grad_stride = grad_stride; a.rows = rows; a.vocab = vocab; a.temperature = t; a.inv_temperature = inv;
    a.log2e_over_t = (float)(1.4426950408889634 / temperature); a.grad_scale = (float)grad_scale;
    a.ids = ids; a.ids_dtype = ids_dtype;
    return SO_OK;
}

}  // namespace

extern "C" {

so_status so_distill_loss(const void *logits, int64_t logits_stride, const void *teacher_ids,
                          int32_t ids_dtype, int64_t ids_stride, const void *teacher_logits,
                          int64_t teacher_stride, int32_t teacher_dtype, int32_t top_k,
                          const float *weight, int64_t rows, int64_t vocab, int32_t dtype,
                          double temperature, double grad_scale, void *grad, int64_t grad_stride,
                          float *row_loss, float *loss, void *stream)
{
    LossArgs a = {};
    const so_status s = common_args(a, logits, logits_stride, weight, rows, vocab, dtype, temperature, grad_scale,
                                    grad, grad_stride, row_loss, loss, teacher_ids, ids_dtype);
    if (s != SO_OK) return s;
    if (!valid_dtype(teacher_dtype) || top_k < 1 || top_k > SO_DISTILL_MAX_TOP_K) return SO_ERR_INVALID_ARG;
    if (rows > 0) {
        if (!teacher_logits || !aligned(teacher_logits, elem_size(teacher_dtype))) return SO_ERR_INVALID_ARG;
        if (!valid_in_stride(rows, ids_stride, top_k) || !valid_in_stride(rows, teacher_stride, top_k)) return SO_ERR_INVALID_ARG;
        if (!valid_extent(rows, ids_stride) || !valid_extent(rows, teacher_stride)) return SO_ERR_INVALID_ARG;
    }
    a.teacher = teacher_logits; a.ids_stride = ids_stride; a.teacher_stride = teacher_stride;
    a.top_k = top_k; a.teacher_dtype = teacher_dtype;
    return run_loss<kDistill>(a, dtype, loss, static_cast<cudaStream_t>(stream));
}

so_status so_policy_loss(const void *logits, int64_t logits_stride, const void *tokens,
                         int32_t ids_dtype, const float *advantage, const float *old_logp,
                         const float *ref_logp, const float *weight, int64_t rows, int64_t vocab,
                         int32_t dtype, double temperature, double clip_low, double clip_high,
                         double kl_coef, double grad_scale, void *grad, int64_t grad_stride,
                         float *logp, float *row_loss, float *loss, void *stream)
{
    LossArgs a = {};
    const so_status s = common_args(a, logits, logits_stride, weight, rows, vocab, dtype, temperature, grad_scale,
                                    grad, grad_stride, row_loss, loss, tokens, ids_dtype);
    if (s != SO_OK) return s;
    if (!(clip_low >= 0.0 && clip_low <= 1.0) || !(clip_high >= 0.0)) return SO_ERR_INVALID_ARG;
    if (!(kl_coef >= 0.0) || !std::isfinite(kl_coef) || (kl_coef != 0.0 && !ref_logp)) return SO_ERR_INVALID_ARG;
    if (!aligned(advantage, 4) || !aligned(old_logp, 4) || !aligned(ref_logp, 4) || !aligned(logp, 4))
        return SO_ERR_INVALID_ARG;
    if (rows > 0 && !advantage) return SO_ERR_INVALID_ARG;
    a.advantage = advantage; a.old_logp = old_logp; a.ref_logp = kl_coef != 0.0 ? ref_logp : nullptr; a.logp = logp;
    a.clip_lo = (float)(1.0 - clip_low); a.clip_hi = (float)(1.0 + clip_high); a.kl_coef = (float)kl_coef;
    return run_loss<kPolicy>(a, dtype, loss, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
