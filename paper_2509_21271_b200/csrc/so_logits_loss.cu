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
        a.s = a.m == -kInf ? a.s : a.s * exp2_fast((a.m - z) * c);
        a.m = z;
    }
    a.s += exp2_fast((z - (a.m == -kInf ? 0.0f : a.m)) * c);
}

__device__ __forceinline__ MaxSum merge(const MaxSum &a, const MaxSum &b, float c)
{
    const float m = fmaxf(a.m, b.m);
    MaxSum r;
    r.m = m;
    r.s = (a.m == m || a.m == -kInf ? a.s : a.s * exp2_fast((a.m - m) * c)) +
          (b.m == m || b.m == -kInf ? b.s : b.s * exp2_fast((b.m - m) * c));
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
__device__ bool load_teacher(const LossArgs &a, int64_t row, int32_t *t_id, float *t_p, float *t_logp, float *t_z)
{
    const int lane = threadIdx.x & 31;
    const T *z = static_cast<const T *>(a.logits) + row * a.stride;
    MaxSum ms{-kInf, 0.0f};
    bool any = false;
    for (int k = lane; k < a.top_k; k += 32) {
        const int64_t id = load_id(a.ids, row * a.ids_stride + k, a.ids_dtype);
        const float x = load_any(a.teacher, row * a.teacher_stride + k, a.teacher_dtype);
        const bool ok = id >= 0 && id < a.vocab && x != -kInf;
        t_id[k] = ok ? (int32_t)id : -1;
        t_logp[k] = x;
        t_z[k] = ok ? to_f32(z[id]) : 0.0f;
        if (ok) {
            any = true;
            if (x > ms.m) {
                ms.s = ms.m == -kInf ? ms.s : ms.s * expf((ms.m - x) * a.inv_temperature);
                ms.m = x;
            }
            ms.s += expf((x - (ms.m == -kInf ? 0.0f : ms.m)) * a.inv_temperature);
        }
    }
    for (int o = 16; o > 0; o >>= 1) {
        MaxSum b;
        b.m = __shfl_xor_sync(0xFFFFFFFFu, ms.m, o);
        b.s = __shfl_xor_sync(0xFFFFFFFFu, ms.s, o);
        const float m = fmaxf(ms.m, b.m);
        const float sa = ms.m == m || ms.m == -kInf ? ms.s : ms.s * expf((ms.m - m) * a.inv_temperature);
        const float sb = b.m == m || b.m == -kInf ? b.s : b.s * expf((b.m - m) * a.inv_temperature);
        ms.m = m;
        ms.s = sa + sb;
    }
    const float inv = 1.0f / ms.s, log_s = logf(ms.s);
    for (int k = lane; k < a.top_k; k += 32) {
        const float d = (t_logp[k] - ms.m) * a.inv_temperature;
        t_p[k] = t_id[k] >= 0 ? expf(d) * inv : 0.0f;
        t_logp[k] = d - log_s;
    }
    any = __any_sync(0xFFFFFFFFu, any);
    __syncwarp();
    return any;
}

// T^2 sum_k p_k (log p_k - log q[id_k]) by one warp, log q a function of the logit.
template <typename LogQ>
__device__ float distill_row_loss(const LossArgs &a, const int32_t *t_id, const float *t_p, const float *t_logp,
                                  const float *t_z, LogQ log_q)
{
    float sum = 0.0f;
    for (int k = threadIdx.x & 31; k < a.top_k; k += 32)
        if (t_id[k] >= 0 && t_p[k] != 0.0f) sum = fmaf(t_p[k], t_logp[k] - log_q(t_z[k]), sum);
    return warp_sum(sum) * a.temperature * a.temperature;
}

// Loss and slope d loss / d logp of a policy row.
__device__ __forceinline__ void policy_row(const LossArgs &a, float logp, float adv, float old_logp, float ref_logp,
                                           float &loss, float &slope)
{
    const float ratio = a.old_logp ? expf(logp - old_logp) : 1.0f;
    const float free_gain = ratio * adv;
    const float held_gain = fminf(fmaxf(ratio, a.clip_lo), a.clip_hi) * adv;
    // written so that a NaN ratio or advantage stays NaN in both
    const bool held = held_gain < free_gain;
    loss = -(held ? held_gain : free_gain);
    slope = held ? 0.0f : -free_gain;
    if (a.ref_logp) {
        const float d = ref_logp - logp;
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
            if (kMode == kDistill) {
                const bool any = load_teacher<T>(a, row, t.id, t.p, t.logp, t.z);
                if (lane == 0) t.live = any;
            } else if (lane == 0) {
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
        MaxSum ms{-kInf, 0.0f};
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
                const float loss = distill_row_loss(a, t.id, t.p, t.logp, t.z, [&](float x) { return (x - ms.m) * a.inv_temperature - log_s; });
                if (lane == 0) a.row_loss[row] = loss;
            }
            coef = a.grad_scale * w * a.temperature;
        } else {
            const float logp = (t.z[0] - ms.m) * a.inv_temperature - log_s;
            float loss, slope;
            policy_row(a, logp, a.advantage[row], a.old_logp ? a.old_logp[row] : 0.0f, a.ref_logp ? a.ref_logp[row] : 0.0f, loss, slope);
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

// ---- a cluster per row, the row held in shared memory ------------------------------
//
// A row of logits is needed twice, for its sum of exponentials and for its gradient.
// A cluster of 1, 2, 4 or 8 blocks holds it in shared memory in between, so that
// memory sees it once: each block takes a share, which comes in chunks through a
// ring of bulk copies.  The chunks of a row stay until their gradient is written;
// the ring is larger than a share, so the next row is on its way meanwhile.
//
//   producer warp   keeps the ring full, row after row
//   target warp     loads the teacher's list (or the token) of the next row, the
//                   student's logits there and the teacher's softmax
//   the others      phase 1: maximum and sum over the chunks as they arrive; the
//                   blocks of the cluster exchange theirs through each other's
//                   shared memory; phase 2: gradient, chunk by chunk, each freed after;
//                   then the row's few targets are written over
//
// The elements before a row's first 16-byte boundary and after its last are loaded by
// single threads.  Rows may start anywhere; a gradient whose rows start at another
// offset from a 16-byte boundary than the logits' is stored element by element.
//
// A wait that runs out of polls makes the loss and the gradient of its row, and of
// those after it, NaN (the optimizer's gradient check then skips the iteration).

constexpr int kPerThread = 2;             // 16-byte vectors of a chunk per thread
constexpr int kMaxSlots = 32;
constexpr int kMaxCluster = 8;

struct RingShape {
    int threads;                          // that compute; the block has two warps more
    int cluster, slots;
    int chunk_bytes;
    size_t smem;
};

struct RowInfo {
    float weight;
    int32_t load, live;                   // read the row at all; its loss and gradient are not zero
};

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t remote_addr(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// Two floats into the shared memory of a block of the cluster, counted by its mbarrier.
__device__ __forceinline__ void remote_store(uint32_t addr, float x, float y, uint32_t bar)
{
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(addr),
                 "f"(x), "f"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Reference of the exponents in units of log2: z c - ref(m) is the exponent of z.  The
// same rounded number is used everywhere, so its rounding cancels.  Beyond kPlain
// the product may overflow and (z - m) c is used instead.
constexpr float kPlain = 1e38f;
__device__ __forceinline__ bool plain(float m) { return fabsf(m) <= kPlain; }

__device__ __forceinline__ float rescale(float from, float to, float c)   // exp2(ref(from) - ref(to))
{
    if (plain(from) && plain(to)) return exp2_fast(__fsub_rn(from * c, to * c));
    return exp2_fast((from - to) * c);
}

__device__ __forceinline__ MaxSum join(const MaxSum &a, const MaxSum &b, float c)
{
    MaxSum r;
    r.m = fmaxf(a.m, b.m);
    r.s = (a.m == r.m || a.m == -kInf ? a.s : a.s * rescale(a.m, r.m, c)) +
          (b.m == r.m || b.m == -kInf ? b.s : b.s * rescale(b.m, r.m, c));
    return r;
}

template <int kLanes>
__device__ __forceinline__ MaxSum join_lanes(MaxSum a, float c)
{
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) {
        MaxSum b;
        b.m = __shfl_xor_sync(0xFFFFFFFFu, a.m, o);
        b.s = __shfl_xor_sync(0xFFFFFFFFu, a.s, o);
        a = join(a, b, c);
    }
    return a;
}

// Largest element of a vector (NaN is passed over: it shows in the sum).
template <typename T> __device__ __forceinline__ float largest(const uint4 &v);
template <> __device__ __forceinline__ float largest<float>(const uint4 &v)
{
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
}
template <> __device__ __forceinline__ float largest<bf16_t>(const uint4 &v)
{
    uint32_t a, b;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
    asm("max.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
    asm("max.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
    return fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u));
}
template <> __device__ __forceinline__ float largest<f16_t>(const uint4 &v)
{
    uint32_t a, b;
    asm("max.f16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
    asm("max.f16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
    asm("max.f16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
    return fmaxf(__half2float(__ushort_as_half((unsigned short)(a & 0xFFFFu))),
                 __half2float(__ushort_as_half((unsigned short)(a >> 16))));
}

// exp((z - m) / T) of a vector
template <int E>
__device__ __forceinline__ Vals<E> exponentials(const Vals<E> &z, float m, float ref, bool is_plain, float c)
{
    const Vals<E> x = is_plain ? fma(z, c, -ref) : (z + -m) * c;
    float f[E];
    x.get(f);
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = exp2_fast(f[e]);
    Vals<E> r;
    r.put(f);
    return r;
}

// Running maximum and sum of a thread.
template <typename T>
struct Running {
    static constexpr int E = Vec<T>::kElems;
    float m, ref;
    bool is_plain;
    Vals<E> s;

    __device__ __forceinline__ Running() : m(-kInf), ref(0.0f), is_plain(false) { s.set(0.0f); }
    __device__ __forceinline__ void raise(float to, float c)
    {
        const float k = m == -kInf ? 1.0f : rescale(m, to, c);   // a sum of nothing (or NaN) stays
        s = s * k;
        m = to;
        is_plain = plain(m);
        ref = m * c;
    }
    __device__ __forceinline__ void add(const uint4 &v, float c)
    {
        // while everything was -inf: (-inf) - 0 = -inf, nothing to add
        s = s + exponentials<E>(widen16<T>(v), m == -kInf ? 0.0f : m, ref, is_plain, c);
    }
};

template <typename T, int kMode, bool kGrad>
__global__ void __launch_bounds__(576, 1) loss_ring_kernel(LossArgs a, RingShape shape)
{
    constexpr int E = Vec<T>::kElems;
    extern __shared__ __align__(128) uint8_t s_ring[];   // [slots][chunk], then the targets of two rows
    __shared__ __align__(8) uint64_t s_full[kMaxSlots], s_empty[kMaxSlots], s_target_full[2], s_target_empty[2], s_exchange[2];
    __shared__ __align__(8) MaxSum s_warp[2][16], s_block[2][kMaxCluster];
    __shared__ RowInfo s_info[2];
    const int warps = shape.threads >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cluster = shape.cluster, slots = shape.slots;
    const uint32_t rank = cluster > 1 ? cluster_rank() : 0u;
    const int64_t first_row = blockIdx.x / cluster, row_step = gridDim.x / cluster;
    const int top_k = kMode == kDistill ? a.top_k : 1;
    // targets of row buffer b: id, probability, its logarithm, logit
    float *s_targets = reinterpret_cast<float *>(s_ring + (size_t)slots * shape.chunk_bytes);
    const auto target_id = [&](int b) { return reinterpret_cast<int32_t *>(s_targets + (size_t)b * 4 * top_k); };
    const auto target_p = [&](int b) { return s_targets + (size_t)b * 4 * top_k + top_k; };
    const auto target_logp = [&](int b) { return s_targets + (size_t)b * 4 * top_k + 2 * top_k; };
    const auto target_z = [&](int b) { return s_targets + (size_t)b * 4 * top_k + 3 * top_k; };

    if (threadIdx.x == 0) {
        for (int i = 0; i < slots; ++i) {
            mbar_init(smem_addr(&s_full[i]), 1);
            mbar_init(smem_addr(&s_empty[i]), warps);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&s_target_full[i]), 1);
            mbar_init(smem_addr(&s_target_empty[i]), warps);
            mbar_init(smem_addr(&s_exchange[i]), 1);
        }
        mbar_init_fence();
    }
    __syncwarp();
    if (cluster > 1) cluster_sync();
    else __syncthreads();
    grid_dependency_release();            // the sum over rows may be set up meanwhile

    // a row's 16-byte part: `head` elements before it, then `count` vectors, of which
    // this block has [from, from + mine)
    struct Part { int head, count, from, mine; };
    const auto part_of = [&](int64_t row) {
        Part p;
        const uintptr_t at = reinterpret_cast<uintptr_t>(static_cast<const T *>(a.logits) + row * a.stride);
        const int64_t head = (int64_t)(((16u - (unsigned)(at & 15u)) & 15u) / sizeof(T));
        p.head = (int)(head < a.vocab ? head : a.vocab);
        p.count = (int)((a.vocab - p.head) / E);
        const int per = (p.count + cluster - 1) / cluster;
        p.from = per * (int)rank < p.count ? per * (int)rank : p.count;
        p.mine = p.count - p.from < per ? p.count - p.from : per;
        return p;
    };
    const auto wanted = [&](int64_t row, float &w) {      // is the row read at all
        w = a.weight ? a.weight[row] : 1.0f;
        if (kMode == kDistill) return w != 0.0f;
        const int64_t token = load_id(a.ids, row, a.ids_dtype);
        return w != 0.0f && token >= 0 && token < a.vocab;
    };
    const int per_chunk = shape.chunk_bytes / 16;
    uint32_t limit = kPolls;

    if (warp == warps) {
        // ---- producer ----
        uint32_t slot = 0, phase = 0, issued = 0;
        float w;
        bool load = first_row < a.rows && wanted(first_row, w);
        for (int64_t row = first_row; row < a.rows; row += row_step) {
            const bool load_next = row + row_step < a.rows && wanted(row + row_step, w);
            if (load) {
                const Part p = part_of(row);
                const T *src = static_cast<const T *>(a.logits) + row * a.stride + p.head + (int64_t)p.from * E;
                for (int v = 0; v < p.mine && limit != 0; v += per_chunk) {
                    if (!mbar_wait(smem_addr(&s_empty[slot]), phase ^ 1, limit)) limit = 0;
                    if (lane == 0 && limit != 0) {
                        const uint32_t bytes = (uint32_t)(p.mine - v < per_chunk ? p.mine - v : per_chunk) * 16;
                        const uint32_t bar = smem_addr(&s_full[slot]);
                        mbar_expect(bar, bytes);
                        bulk_load(smem_addr(s_ring) + slot * shape.chunk_bytes, src + (int64_t)v * E, bytes, bar);
                    }
                    if (limit == 0) break;
                    ++issued;
                    if (++slot == (uint32_t)slots) slot = 0, phase ^= 1;
                }
            }
            load = load_next;
        }
        // whatever was issued lands before the block goes (consumed already, unless a wait ran out)
        for (uint32_t i = issued > (uint32_t)slots ? issued - slots : 0; i < issued; ++i)
            mbar_wait(smem_addr(&s_full[i % slots]), (i / slots) & 1, kPolls);
    } else if (warp == warps + 1) {
        // ---- targets ----
        int buf = 0;
        uint32_t phase = 0;
        float w = 0.0f;
        bool load = first_row < a.rows && wanted(first_row, w);
        for (int64_t row = first_row; row < a.rows; row += row_step) {
            float w_next = 0.0f;
            const bool load_next = row + row_step < a.rows && wanted(row + row_step, w_next);
            if (limit != 0 && !mbar_wait(smem_addr(&s_target_empty[buf]), phase ^ 1, limit)) limit = 0;
            bool live = load;
            if (load && kMode == kDistill) {
                live = load_teacher<T>(a, row, target_id(buf), target_p(buf), target_logp(buf), target_z(buf));
            } else if (load && lane == 0) {
                const int64_t token = load_id(a.ids, row, a.ids_dtype);
                target_id(buf)[0] = (int32_t)token;
                target_p(buf)[0] = 1.0f;
                target_z(buf)[0] = to_f32(static_cast<const T *>(a.logits)[row * a.stride + token]);
            }
            if (lane == 0) s_info[buf] = RowInfo{w, load, live};
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&s_target_full[buf]));
            load = load_next;
            w = w_next;
            if (++buf == 2) buf = 0, phase ^= 1;
        }
    } else {
        // ---- the rest ----
        const float c = a.log2e_over_t;
        uint32_t slot = 0, phase = 0, row_phase = 0, computed = 0;   // rows computed so far: even and odd ones take turns
        int buf = 0;
        for (int64_t row = first_row; row < a.rows; row += row_step) {
            if (limit != 0 && !mbar_wait(smem_addr(&s_target_full[buf]), row_phase, limit)) limit = 0;
            const RowInfo info = s_info[buf];
            const Part p = part_of(row);
            const T *z = static_cast<const T *>(a.logits) + row * a.stride;
            T *g = kGrad ? static_cast<T *>(a.grad) + row * a.grad_stride : nullptr;
            const bool same_offset = kGrad && ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0;
            // the single element of a few threads: the first block's head, the last block's tail
            int64_t edge = -1;
            if (rank == 0 && (int)threadIdx.x < p.head) edge = threadIdx.x;
            const int64_t tail = p.head + (int64_t)p.count * E + ((int)threadIdx.x - 32);
            if (rank == (uint32_t)cluster - 1 && threadIdx.x >= 32 && tail < a.vocab) edge = tail;

            if (!info.live) {
                // nothing to compute: a chunk that is on its way is let go, the gradient is zero
                if (info.load)
                    for (int v = 0; v < p.mine; v += per_chunk) {
                        if (limit != 0 && !mbar_wait(smem_addr(&s_full[slot]), phase, limit)) limit = 0;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_addr(&s_empty[slot]));
                        if (++slot == (uint32_t)slots) slot = 0, phase ^= 1;
                    }
                if (kGrad) {
                    T *out = g + p.head + (int64_t)p.from * E;
                    if (same_offset) {
                        for (int v = threadIdx.x; v < p.mine; v += shape.threads)
                            reinterpret_cast<uint4 *>(out)[v] = make_uint4(0, 0, 0, 0);
                    } else {
                        for (int64_t i = threadIdx.x; i < (int64_t)p.mine * E; i += shape.threads) out[i] = from_f32<T>(0.0f);
                    }
                    if (edge >= 0) g[edge] = from_f32<T>(0.0f);
                }
                if (rank == 0 && threadIdx.x == 0) {
                    a.row_loss[row] = 0.0f;
                    if (kMode == kPolicy && a.logp) a.logp[row] = 0.0f;
                }
            } else {
                float edge_z = 0.0f;
                if (edge >= 0) edge_z = to_f32(z[edge]);
                float adv = 0.0f, old_logp = 0.0f, ref_logp = 0.0f;
                if (kMode == kPolicy) {
                    adv = a.advantage[row];
                    if (a.old_logp) old_logp = a.old_logp[row];
                    if (a.ref_logp) ref_logp = a.ref_logp[row];
                }
                // phase 1
                const uint32_t slot0 = slot;
                Running<T> run;
                for (int v = 0; v < p.mine; v += per_chunk) {
                    if (limit != 0 && !mbar_wait(smem_addr(&s_full[slot]), phase, limit)) limit = 0;
                    const uint32_t at = smem_addr(s_ring) + slot * shape.chunk_bytes + threadIdx.x * 16;
                    const int i0 = v + (int)threadIdx.x, i1 = i0 + shape.threads;
                    if (i1 < p.mine) {
                        const uint4 q0 = lds16(at), q1 = lds16(at + shape.threads * 16);
                        const float top = fmaxf(largest<T>(q0), largest<T>(q1));
                        if (top > run.m) run.raise(top, c);
                        run.add(q0, c);
                        run.add(q1, c);
                    } else if (i0 < p.mine) {
                        const uint4 q0 = lds16(at);
                        const float top = largest<T>(q0);
                        if (top > run.m) run.raise(top, c);
                        run.add(q0, c);
                    }
                    if (!kGrad) {
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_addr(&s_empty[slot]));
                    }
                    if (++slot == (uint32_t)slots) slot = 0, phase ^= 1;
                }
                MaxSum ms{run.m, total(run.s)};
                if (edge >= 0) {
                    // exp2 of its exponent against its own reference: 1 but for the rounding of that
                    const float own = plain(edge_z) ? exp2_fast(fmaf(edge_z, c, -(edge_z * c))) : exp2_fast(edge_z - edge_z);
                    ms = join(ms, MaxSum{edge_z, edge_z == -kInf ? 0.0f : own}, c);
                }
                if (limit == 0) ms.s = kNan;
                ms = join_lanes<32>(ms, c);
                const int turn = computed & 1;
                if (lane == 0) s_warp[turn][warp] = ms;
                asm volatile("bar.sync 1, %0;" ::"r"(shape.threads) : "memory");
                if (cluster == 1 || warp == 0) {
                    // at most 16 warps, the same in both halves of this one
                    ms = (lane & 15) < warps ? s_warp[turn][lane & 15] : MaxSum{-kInf, 0.0f};
                    ms = join_lanes<16>(ms, c);
                }
                if (cluster > 1) {
                    const uint32_t bar = smem_addr(&s_exchange[turn]);
                    if (warp == 0) {
                        if (lane == 0) mbar_expect(bar, (uint32_t)cluster * sizeof(MaxSum));
                        __syncwarp();
                        if (lane < cluster)
                            remote_store(remote_addr(smem_addr(&s_block[turn][rank]), lane), ms.m, ms.s, remote_addr(bar, lane));
                    }
                    if (limit != 0 && !mbar_wait(bar, (computed >> 1) & 1, limit)) limit = 0;
                    ms = (lane & 7) < cluster ? s_block[turn][lane & 7] : MaxSum{-kInf, 0.0f};
                    ms = join_lanes<8>(ms, c);
                    if (limit == 0) ms.s = kNan;
                }
                ++computed;

                // log q = ln 2 (z c - ref) - ln S
                const bool is_plain = plain(ms.m);
                const float ref = ms.m * c, log_s = logf(ms.s), inv_s = 1.0f / ms.s;
                const auto exponent = [&](float x) { return is_plain ? fmaf(x, c, -ref) : (x - ms.m) * c; };
                const auto log_q = [&](float x) { return fmaf(exponent(x), 0.693147180559945f, -log_s); };
                float coef;
                if (kMode == kDistill) {
                    if (rank == 0 && warp == 0) {
                        const float loss = distill_row_loss(a, target_id(buf), target_p(buf), target_logp(buf), target_z(buf), log_q);
                        if (lane == 0) a.row_loss[row] = loss;
                    }
                    coef = a.grad_scale * info.weight * a.temperature;
                } else {
                    const float logp = log_q(target_z(buf)[0]);
                    float loss, slope;
                    policy_row(a, logp, adv, old_logp, ref_logp, loss, slope);
                    if (rank == 0 && threadIdx.x == 0) {
                        a.row_loss[row] = loss;
                        if (a.logp) a.logp[row] = logp;
                    }
                    coef = -a.grad_scale * info.weight * slope * a.inv_temperature;
                }

                if (kGrad) {
                    // phase 2
                    const float scaled = coef * inv_s;
                    uint32_t s2 = slot0;
                    T *out = g + p.head + (int64_t)p.from * E;
                    const auto one = [&](uint32_t at, int i) {
                        const Vals<E> e = exponentials<E>(widen16<T>(lds16(at)), ms.m, ref, is_plain, c) * scaled;
                        if (same_offset) {
                            reinterpret_cast<uint4 *>(out)[i] = narrow16<T>(e);
                        } else {
                            float f[E];
                            e.get(f);
#pragma unroll
                            for (int k = 0; k < E; ++k) out[(int64_t)i * E + k] = from_f32<T>(f[k]);
                        }
                    };
                    for (int v = 0; v < p.mine; v += per_chunk) {
                        const uint32_t at = smem_addr(s_ring) + s2 * shape.chunk_bytes + threadIdx.x * 16;
                        const int i0 = v + (int)threadIdx.x, i1 = i0 + shape.threads;
                        if (i0 < p.mine) one(at, i0);
                        if (i1 < p.mine) one(at + shape.threads * 16, i1);
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_addr(&s_empty[s2]));
                        if (++s2 == (uint32_t)slots) s2 = 0;
                    }
                    if (edge >= 0) g[edge] = from_f32<T>(exp2_fast(exponent(edge_z)) * scaled);
                    asm volatile("bar.sync 1, %0;" ::"r"(shape.threads) : "memory");
                    // the targets, by the block that has their element
                    const int32_t *ids = target_id(buf);
                    const float *probs = target_p(buf), *zs = target_z(buf);
                    for (int k = threadIdx.x; k < top_k; k += shape.threads) {
                        const int32_t id = ids[k];
                        if (id < 0) continue;
                        const int v = (id - p.head) / E;
                        const uint32_t owner_is_me = id < p.head ? rank == 0
                                                     : v >= p.count ? rank == (uint32_t)cluster - 1
                                                                    : v >= p.from && v < p.from + p.mine;
                        if (!owner_is_me) continue;
                        float prob = 0.0f;
                        for (int i = 0; i < top_k; ++i)
                            if (ids[i] == id) prob += probs[i];
                        g[id] = from_f32<T>(coef * fmaf(exp2_fast(exponent(zs[k])), inv_s, -prob));
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&s_target_empty[buf]));
            if (++buf == 2) buf = 0, row_phase ^= 1;
        }
    }
    // no block goes while another may still write into its shared memory
    if (cluster > 1) {
        __syncwarp();
        cluster_sync();
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

// The ring's shape for `vocab` elements of `es` bytes: false if no cluster holds a row.
#ifndef L_T
#define L_T 512
#endif
#ifndef L_FILL
#define L_FILL 70
#endif
bool ring_shape(int64_t rows, int64_t vocab, int es, int top_k, bool grad, int sms, RingShape *out)
{
    const int64_t row_bytes = vocab * es;
    int threads = L_T;
    int64_t share_max = 0;
    RingShape r;
    const size_t targets = (size_t)2 * 16 * top_k;
    const auto fit = [&](int t) {
        r.threads = t;
        r.chunk_bytes = t * 16 * kPerThread;
        const size_t per_block = (size_t)225 * 1024 * t / 512 - 3 * 1024;
        if (per_block < targets + 2 * (size_t)r.chunk_bytes) return false;
        r.slots = (int)((per_block - targets) / r.chunk_bytes);
        if (r.slots > kMaxSlots) r.slots = kMaxSlots;
        r.smem = (size_t)r.slots * r.chunk_bytes + targets;
        share_max = (int64_t)r.slots * r.chunk_bytes;
        return true;
    };
    // short rows: fewer threads each, more blocks per SM
    while (threads > 64 && row_bytes < (int64_t)threads * 16 * kPerThread) threads /= 2;
    while (!fit(threads)) {
        if (threads >= 512) return false;
        threads *= 2;
    }
    r.cluster = 1;
    const auto chunks = [&](int c) { return ((row_bytes / 16 + c - 1) / c * 16 + r.chunk_bytes - 1) / r.chunk_bytes; };
    if (grad)
        while (r.cluster < kMaxCluster && chunks(r.cluster) * 100 > (int64_t)r.slots * L_FILL) r.cluster *= 2;
    if (grad && chunks(r.cluster) > r.slots) return false;
    // few rows: more blocks each, while SMs are idle
    while (r.cluster < kMaxCluster && rows * r.cluster * 2 <= sms && chunks(r.cluster) > 1) r.cluster *= 2;
    *out = r;
    return true;
}

constexpr int kMaxShared = 224 * 1024;

template <typename T, int kMode, bool kGrad>
so_status launch_ring(const LossArgs &a, const RingShape &shape, int sms, cudaStream_t st)
{
    struct Known { std::atomic<uint64_t> key; std::atomic<int> clusters; };
    static Known cache[kMaxDevices];
    const auto kernel = loss_ring_kernel<T, kMode, kGrad>;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return SO_ERR_CUDA;
    if (dev < 0 || dev >= kMaxDevices) return SO_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)shape.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.blockDim = dim3((unsigned)shape.threads + 64);
    cfg.dynamicSmemBytes = shape.smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    // how many clusters of this shape run at a time; one word per device says for which shape
    const uint64_t key = ((uint64_t)shape.smem << 20) | ((uint64_t)shape.threads << 8) | (uint64_t)shape.cluster;
    int clusters = cache[dev].clusters.load(std::memory_order_acquire);
    if (cache[dev].key.load(std::memory_order_acquire) != key || clusters == 0) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxShared) != cudaSuccess)
            return SO_ERR_CUDA;
        cfg.gridDim = dim3((unsigned)shape.cluster);
        if (cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) != cudaSuccess || clusters < 1) return SO_ERR_CUDA;
        cache[dev].key.store(0, std::memory_order_release);
        cache[dev].clusters.store(clusters, std::memory_order_release);
        cache[dev].key.store(key, std::memory_order_release);
    }
    const int64_t n = a.rows < clusters ? a.rows : clusters;
    cfg.gridDim = dim3((unsigned)(n * shape.cluster));
    return cudaLaunchKernelEx(&cfg, kernel, a, shape) == cudaSuccess ? SO_OK : SO_ERR_CUDA;
}

template <typename T, int kMode>
so_status launch_loss(const LossArgs &a, int sms, cudaStream_t st)
{
    RingShape shape;
    if (ring_shape(a.rows, a.vocab, (int)sizeof(T), kMode == kDistill ? a.top_k : 1, a.grad != nullptr, sms, &shape))
        return a.grad ? launch_ring<T, kMode, true>(a, shape, sms, st) : launch_ring<T, kMode, false>(a, shape, sms, st);
    const unsigned grid = (unsigned)(a.rows < 4 * sms ? a.rows : 4 * sms);
    return launch(loss_two_pass_kernel<T, kMode>, grid, kRowThreads, 0, st, false, a);
}

template <int kMode>
so_status run_loss(const LossArgs &a, int32_t dtype, float *loss, cudaStream_t st)
{
    int sms = 0;
    so_status s = device_sms(&sms);
    if (s != SO_OK) return s;
    if (a.rows > 0) {
        if (dtype == SO_DTYPE_BF16) s = launch_loss<bf16_t, kMode>(a, sms, st);
        else if (dtype == SO_DTYPE_FP16) s = launch_loss<f16_t, kMode>(a, sms, st);
        else s = launch_loss<float, kMode>(a, sms, st);
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
