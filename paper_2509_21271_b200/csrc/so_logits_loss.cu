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
    void *grad;                           // nullptr: the loss alone (not in loss_two_pass_kernel)
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
    Patience patience;
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

// One warp fills the targets of a distillation row: ids, the student's logits there, the
// teacher's softmax over the entries that are there and its logarithm.  False if none is.
template <typename T>
__device__ bool load_teacher(const LossArgs &a, int64_t row, int32_t *t_id, float *t_p, float *t_logp, float *t_z)
{
    constexpr int kAtOnce = 4;            // loads in flight per lane; the logits wait for the ids
    const int lane = threadIdx.x & 31;
    const T *z = static_cast<const T *>(a.logits) + row * a.stride;
    float top = -kInf;
    bool any = false;
    for (int k0 = lane; k0 < a.top_k; k0 += 32 * kAtOnce) {
        int32_t id[kAtOnce];
        float x[kAtOnce], zk[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int k = k0 + 32 * u;
            id[u] = -1;
            x[u] = -kInf;
            if (k < a.top_k) {
                const int64_t wide = load_id(a.ids, row * a.ids_stride + k, a.ids_dtype);
                x[u] = load_any(a.teacher, row * a.teacher_stride + k, a.teacher_dtype);
                id[u] = wide >= 0 && wide < a.vocab ? (int32_t)wide : -1;
            }
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (x[u] == -kInf) id[u] = -1;
            zk[u] = id[u] >= 0 ? to_f32(z[id[u]]) : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int k = k0 + 32 * u;
            if (k >= a.top_k) break;
            t_id[k] = id[u];
            t_logp[k] = x[u];
            t_z[k] = zk[u];
            if (id[u] >= 0) {
                any = true;
                top = fmaxf(top, x[u]);
            }
        }
    }
    any = __any_sync(0xFFFFFFFFu, any);
    asm("redux.sync.max.f32 %0, %0, 0xFFFFFFFF;" : "+f"(top));
    float sum = 0.0f;
    for (int k = lane; k < a.top_k; k += 32) {
        const float d = (t_logp[k] - top) * a.inv_temperature;
        const float e = t_id[k] >= 0 ? expf(d) : 0.0f;
        t_logp[k] = d;
        t_p[k] = e;
        sum += e;
    }
    sum = warp_sum(sum);
    const float inv = 1.0f / sum, log_s = logf(sum);
    for (int k = lane; k < a.top_k; k += 32) {
        t_p[k] *= inv;
        t_logp[k] -= log_s;
    }
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
    float ratio = a.old_logp ? expf(logp - old_logp) : 1.0f;
    if (ratio == kInf && adv == 0.0f) ratio = 1.0f;      // beyond fp32, but times 0
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
//
// For rows with a gradient that the shared memory of a cluster does not hold (1.7 MB, 1.3
// with the longest lists), element by element.

constexpr int kRowThreads = 512;

template <typename T, int kMode>
__global__ void __launch_bounds__(kRowThreads) loss_two_pass_kernel(LossArgs a)
{
    __shared__ Targets t;
    __shared__ MaxSum s_ms[kRowThreads / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *z = static_cast<const T *>(a.logits) + row * a.stride;
        T *g = static_cast<T *>(a.grad) + row * a.grad_stride;
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
//   row warp        deals out the cluster's rows
//   producer warp   keeps the ring full, row after row
//   target warps    take the rows in turn, `depth` of them: load the teacher's list (or
//                   the token) of a row to come, the student's logits there and the
//                   teacher's softmax; when the row is done, its loss, and its
//                   gradient at the targets
//   the others      phase 1: maximum and sum over the chunks as they arrive; the
//                   warps of the cluster exchange theirs through each other's
//                   shared memory; phase 2: gradient, chunk by chunk, each freed after
//
// The elements before a row's first 16-byte boundary and after its last are loaded by
// single threads.  Rows may start anywhere; a gradient whose rows start at another
// offset from a 16-byte boundary than the logits' is stored element by element.
//
// Bound: 4-byte logits, memory (8192 x 50304 fp32: 511 us, 6.45 TB/s, 98 % of a copy's
// rate).  2-byte logits, the two exponentials an element (16 a clock and SM: 70 % of
// either phase) and the stores of phase 2 (an SM stores 27 to 30 bytes a clock), one after
// the other: 4096 x 128256 bf16 with 64 teacher logits and a fifth of the rows masked
// 364 to 373 us, 5.1 TB/s, 79 %; the policy loss of 8191 x 128256 with 30 % masked 657 to
// 676 us, 5.4 TB/s, 82 %; the loss alone of 8192 x 128256 464 us (policy) for 321 of bytes.
// The chunks are always there before they are asked for.  Few rows: a chain of waits, each
// polled with sleeps, from the row's number to its targets' softmax: 63 x 50257 fp16 16 us,
// the sum over rows included, for 1.9 of bytes.  Measured and not taken: a quarter of the
// exponentials on the multipliers (391 us), 640 or 768 threads (394, 405), two blocks of 256
// an SM with clusters of four (441), the maximum kept exactly (397).  A row read twice from
// memory took 1771 and 2311 us.
//
// A wait that runs out of polls ends its block's work.  When all blocks of the cluster have
// come to their end they hear of it, and write NaN over all rows of the cluster: their
// losses, log probabilities and whole gradients, those of masked rows too.

constexpr int kBigThreads = 512;          // that compute, in a block that has an SM to itself
constexpr int kPerThread = 2;             // 16-byte vectors of a chunk per thread
constexpr int kMaxSlots = 32;
constexpr int kMaxCluster = 8;
constexpr int kMaxDepth = 4;
constexpr int kQueue = 8;                 // rows dealt out ahead

struct RingShape {
    int threads;                          // that compute; the block has 2 + depth warps more
    int cluster, slots, depth;            // blocks a row, chunks of the ring, rows whose targets are at hand
    int chunk_bytes;
    size_t smem;
};

struct RowInfo {
    int64_t row;                          // -1: no more
    float weight;
    int32_t load, live;                   // read the row at all; its loss and gradient are not zero
    int32_t repeats;                      // some id is in its list more than once
    // its 16-byte part: `head` elements before it, then `count` vectors, of which this
    // block has [from, from + mine)
    int32_t head, count, from, mine;
    float advantage, old_logp, ref_logp;
};

// Places of the table that finds repeated ids: a power of two, at least twice the list; none
// for a list short enough to be compared with itself.
__host__ __device__ inline int table_places(int top_k)
{
    if (top_k <= 128) return 0;
    int n = 256;
    while (n < 2 * top_k) n *= 2;
    return n;
}

// Whether the condition holds for any of the computing threads; a barrier for them.
__device__ __forceinline__ bool any_of(bool condition, int threads)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, %2, p;\n\t"
                 "selp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)condition), "r"(threads) : "memory");
    return r != 0;
}

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
__device__ __forceinline__ void remote_set(uint32_t addr, uint32_t rank)
{
    asm volatile("st.shared::cluster.u32 [%0], 1;" ::"r"(remote_addr(addr, rank)) : "memory");
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

// Reference of the exponents in units of log2: the exponent of z is z c - ref with
// ref = m c rounded.  The same rounded number is used everywhere, so its rounding
// cancels.  Beyond kPlain that rounding is not small any more (and the product may
// overflow), and (z - m) c is used instead.
constexpr float kPlain = 1048576.0f;
__device__ __forceinline__ bool plain(float ref) { return fabsf(ref) <= kPlain; }

// Exponent of z against the reference of m.
__device__ __forceinline__ float exponent_of(float z, float m, float c)
{
    const float ref = m * c;
    return plain(ref) ? fmaf(z, c, -ref) : (z - m) * c;
}

constexpr float kLn2 = 0.693147180559945f;

// log q of a logit: ln 2 (z c - ref) - ln S, or (z - m) / T - ln S where the exponent in units
// of log2 exceeds what fp32 holds (a logit of the type's lowest value).
__device__ __forceinline__ float log_prob(const LossArgs &a, float z, float m, float log_s)
{
    const float x = exponent_of(z, m, a.log2e_over_t);
    return x == -kInf && z != -kInf ? (z - m) * a.inv_temperature - log_s : fmaf(x, kLn2, -log_s);
}

// Factor that takes a sum from one reference to another.
__device__ __forceinline__ float rescale(float from, float to, float c)
{
    const float rf = from * c, rt = to * c;
    if (plain(rf) && plain(rt)) return exp2_fast(rf - rt);
    float d = (from - to) * c;
    if (plain(rf)) d -= fmaf(from, c, -rf);
    if (plain(rt)) d += fmaf(to, c, -rt);
    return exp2_fast(d);
}

__device__ __forceinline__ MaxSum join(const MaxSum &a, const MaxSum &b, float c)
{
    MaxSum r;
    r.m = fmaxf(a.m, b.m);
    r.s = (a.m == r.m || a.m == -kInf ? a.s : a.s * rescale(a.m, r.m, c)) +
          (b.m == r.m || b.m == -kInf ? b.s : b.s * rescale(b.m, r.m, c));
    return r;
}

// The same over the lanes of a warp.
__device__ __forceinline__ MaxSum join_lanes(MaxSum a, float c)
{
    float top;
    asm("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;" : "=f"(top) : "f"(a.m));
    a.s = warp_sum(a.m == top || a.m == -kInf ? a.s : a.s * rescale(a.m, top, c));
    a.m = top;
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

// A vector of -inf.
template <typename T> __device__ __forceinline__ uint4 nothing()
{
    const uint32_t w = sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, bf16_t>::value ? 0xFF80FF80u : 0xFC00FC00u;
    return make_uint4(w, w, w, w);
}

// exp((z - m) / T) of a vector
template <bool kPlainRow, int E>
__device__ __forceinline__ Vals<E> exponentials(const Vals<E> &z, float m, float ref, float c)
{
    Vals<E> x = kPlainRow ? fma(z, c, -ref) : (z + -m) * c;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
        float lo, hi;
        split(x.p[i], lo, hi);
        x.p[i] = pair(exp2_fast(lo), exp2_fast(hi));
    }
    return x;
}

// Running sum of a thread, against a reference that need not be the maximum: it is the
// largest of the first vectors that have a finite element.  Where the row stays at hand, the
// elements after that are added without a look at their size, and a sum that came out above
// kMost is done again with one; otherwise the reference moves when something exceeds it by
// a factor of 2^kSlack.  (Were it the maximum, some lane of a warp would move it with almost
// every vector.)
//
// kMost is far below what fp32 holds, for three reasons.  The sums of a cluster's 4096
// threads are added: 2^72 at most.  A sum is taken to a reference above its own by a factor
// that the exponential unit flushes to 0 below 2^-126: what is lost of a sum of 2^60 is
// below 2^-66 of the total.  And the gradient's factor coef / S has to be a normal number:
// it is, down to |coef| = 2^-54.  Exponents up to 60 round to 2^-19, 1.3e-6 of an exponential.
// Rows that need the second sum take longer: 8192 x 50257 bf16 with an element 50 (72 in
// units of log2) above the others 435 us, without one 331 us.
constexpr float kSlack = 16.0f, kMost = 0x1p60f;

template <typename T>
struct Running {
    static constexpr int E = Vec<T>::kElems;
    float m, ref, bound;                  // reference, the same in units of log2, and where it moves
    bool is_plain;
    Vals<E> s;

    __device__ __forceinline__ Running() : m(-kInf), ref(0.0f), bound(-kInf), is_plain(false) { s.set(0.0f); }

    // Against the reference as it is, if there is one.  The sum may exceed kMost, up to
    // infinity, for the caller to find.
    template <int N>
    __device__ __forceinline__ void add_unchecked(const uint4 (&v)[N], float c, float slack)
    {
        if (is_plain) {
#pragma unroll
            for (int i = 0; i < N; ++i) s = s + exponentials<true>(widen16<T>(v[i]), m, ref, c);
        } else {
            add(v, c, slack);
        }
    }

    template <int N>
    __device__ __forceinline__ void add(const uint4 (&v)[N], float c, float slack)   // slack = kSlack / c
    {
        float top = largest<T>(v[0]);
#pragma unroll
        for (int i = 1; i < N; ++i) top = fmaxf(top, largest<T>(v[i]));
        if (top > bound) {
            if (m != -kInf) s = s * rescale(m, top, c);   // a sum of nothing (or NaN) stays
            m = top;
            ref = m * c;
            bound = m + slack;
            is_plain = plain(ref);
        }
        if (is_plain) {
#pragma unroll
            for (int i = 0; i < N; ++i) s = s + exponentials<true>(widen16<T>(v[i]), m, ref, c);
        } else {
            // while everything was -inf: (-inf) - 0 = -inf, nothing to add
            const float base = m == -kInf ? 0.0f : m;
#pragma unroll
            for (int i = 0; i < N; ++i) s = s + exponentials<false>(widen16<T>(v[i]), base, ref, c);
        }
    }
};

// ---- a block per row, the row held in registers ----------------------------------------
//
// For short rows, where a cluster's set-up would cost more than the row: as many threads
// as hold its vectors, four each, and as many rows at a time as the SMs have room for.
// A thread keeps the exponentials against its own maximum, so each is taken once; the
// gradient is that times one factor per thread.  8191 rows of 4001 bf16 logits, policy
// loss: 38 us against 71 us by clusters, for 20 us of bytes; of 16000, distillation: 189
// against 205 us, for 80 (with 64 teacher logits 202 us, the policy loss 128).  Loads, the
// list by one warp, barriers and stores of a row follow each other, and two blocks an SM
// (60 registers) hide little of that.

constexpr int kShortVectors = 4, kShortThreads = 512;

template <typename T, int kMode, bool kGrad>
__global__ void __launch_bounds__(kShortThreads) loss_short_kernel(LossArgs a)
{
    constexpr int E = Vec<T>::kElems;
    __shared__ MaxSum s_warp[kShortThreads / 32];
    __shared__ float4 s_result;           // reference, logarithm of the sum, its inverse, the gradient's factor
    __shared__ int s_any;
    extern __shared__ __align__(16) float s_lists[];      // ids, probabilities, their logarithms, logits
    const int top_k = kMode == kDistill ? a.top_k : 1, threads = blockDim.x, tid = threadIdx.x;
    const int warp = tid >> 5, lane = tid & 31;
    int32_t *ids = reinterpret_cast<int32_t *>(s_lists);
    float *probs = s_lists + top_k, *logs = probs + top_k, *zs = logs + top_k;
    const float c = a.log2e_over_t;
    grid_dependency_release();            // the sum over rows may be set up meanwhile
    const int64_t row = blockIdx.x;
    const T *z = static_cast<const T *>(a.logits) + row * a.stride;
    T *g = kGrad ? static_cast<T *>(a.grad) + row * a.grad_stride : nullptr;
    const int vocab = (int)a.vocab;
    const int to_boundary = (int)((16u - (unsigned)(reinterpret_cast<uintptr_t>(z) & 15u)) & 15u) / (int)sizeof(T);
    const int head = to_boundary < vocab ? to_boundary : vocab, count = (vocab - head) / E;
    const bool same_offset = kGrad && ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0;
    // single elements: the head by the first threads, the tail by others
    int edge = -1;
    if (tid < head) edge = tid;
    else if (tid >= 8 && tid < 16 && head + count * E + (tid - 8) < vocab) edge = head + count * E + (tid - 8);

    const float w = a.weight ? a.weight[row] : 1.0f;
    int64_t token = -1;
    if (kMode == kPolicy) token = load_id(a.ids, row, a.ids_dtype);
    bool live = w != 0.0f && (kMode == kDistill || (token >= 0 && token < a.vocab));
    uint4 q[kShortVectors];
    float edge_z = -kInf;
    if (live) {
#pragma unroll
        for (int i = 0; i < kShortVectors; ++i)
            q[i] = tid + i * threads < count ? __ldcs(reinterpret_cast<const uint4 *>(z + head) + tid + i * threads) : nothing<T>();
        if (edge >= 0) edge_z = to_f32(z[edge]);
        if (warp == 0) {
            bool any = true;
            if (kMode == kDistill) {
                any = load_teacher<T>(a, row, ids, probs, logs, zs);
            } else if (lane == 0) {
                ids[0] = (int32_t)token;
                probs[0] = 1.0f;
                zs[0] = to_f32(z[token]);
            }
            if (lane == 0) s_any = any;
        }
    }
    const auto put = [&](const Vals<E> &v, int i) {
        T *at = g + head + (int64_t)i * E;
        if (same_offset) {
            *reinterpret_cast<uint4 *>(at) = narrow16<T>(v);
        } else {
            float f[E];
            v.get(f);
#pragma unroll
            for (int k = 0; k < E; ++k) at[k] = from_f32<T>(f[k]);
        }
    };

    Vals<E> e[kShortVectors];
    MaxSum ms{-kInf, 0.0f};
    if (live) {
        float top = edge_z == edge_z ? edge_z : -kInf;
#pragma unroll
        for (int i = 0; i < kShortVectors; ++i) top = fmaxf(top, largest<T>(q[i]));
        const float base = top == -kInf ? 0.0f : top, ref = base * c;
        Vals<E> sum;
        sum.set(0.0f);
#pragma unroll
        for (int i = 0; i < kShortVectors; ++i) {
            e[i] = plain(ref) ? exponentials<true>(widen16<T>(q[i]), base, ref, c) : exponentials<false>(widen16<T>(q[i]), base, ref, c);
            sum = sum + e[i];
        }
        if (edge >= 0) edge_z = exp2_fast(exponent_of(edge_z, base, c));
        ms = MaxSum{top, total(sum) + (edge >= 0 ? edge_z : 0.0f)};
        const MaxSum joined = join_lanes(ms, c);
        if (lane == 0) s_warp[warp] = joined;
    }
    __syncthreads();
    live = live && s_any;
    if (!live) {
        if (kGrad) {
            Vals<E> none;
            none.set(0.0f);
            for (int i = tid; i < count; i += threads) put(none, i);
            if (edge >= 0) g[edge] = from_f32<T>(0.0f);
        }
        if (tid == 0) {
            a.row_loss[row] = 0.0f;
            if (kMode == kPolicy && a.logp) a.logp[row] = 0.0f;
        }
        return;
    }
    if (warp == 0) {
        const MaxSum all = join_lanes(lane < threads / 32 ? s_warp[lane] : MaxSum{-kInf, 0.0f}, c);
        const float log_s = logf(all.s);
        const auto log_q = [&](float x) { return log_prob(a, x, all.m, log_s); };
        float coef, loss, slope;
        if (kMode == kDistill) {
            loss = distill_row_loss(a, ids, probs, logs, zs, log_q);
            coef = a.grad_scale * w * a.temperature;
        } else {
            const float logp = log_q(zs[0]);
            policy_row(a, logp, a.advantage[row], a.old_logp ? a.old_logp[row] : 0.0f, a.ref_logp ? a.ref_logp[row] : 0.0f, loss, slope);
            if (lane == 0 && a.logp) a.logp[row] = logp;
            coef = -a.grad_scale * w * slope * a.inv_temperature;
        }
        if (lane == 0) {
            a.row_loss[row] = loss;
            s_result = make_float4(all.m, log_s, 1.0f / all.s, coef);
        }
    }
    if (!kGrad) return;
    __syncthreads();
    const float4 done = s_result;
    // a thread without a finite element has exponentials of 0, or NaN that stay so
    const float scaled = done.w * done.z * (ms.m == -kInf ? (done.x == -kInf ? kNan : 1.0f) : rescale(ms.m, done.x, c));
#pragma unroll
    for (int i = 0; i < kShortVectors; ++i)
        if (tid + i * threads < count) put(e[i] * scaled, tid + i * threads);
    if (edge >= 0) g[edge] = from_f32<T>(edge_z * scaled);
    __syncthreads();
    for (int k = tid; k < top_k; k += threads) {
        const int32_t id = ids[k];
        if (id < 0) continue;
        float p = 0.0f;
        for (int i = 0; i < top_k; ++i)
            if (ids[i] == id) p += probs[i];
        g[id] = from_f32<T>(done.w * fmaf(exp2_fast(exponent_of(zs[k], done.x, c)), done.z, -p));
    }
}

// The rows of a cluster, in ascending order, by one warp.  Masked rows, which cost less
// than the others, are dealt out separately, both kinds in turn by their own count: the
// warp looks at 32 rows at a time, a few hundred clocks beside rows of 32 KB and more, and
// all clusters come to the same counts.
template <typename Wanted, typename Give>
__device__ void walk_rows(const Wanted &wanted, int64_t rows, int n, int mine, Give give)
{
    const int lane = threadIdx.x & 31;
    if (rows == n) {                      // one row each
        give(mine, wanted(mine));
        return;
    }
    constexpr int kAhead = 4;             // windows whose loads are in flight
    bool next[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) next[i] = 32 * i + lane < rows && wanted(32 * i + lane);
    int live_turn = 0, dead_turn = 0;     // whose turn it is
    for (int64_t base = 0; base < rows; base += 32) {
        const bool here = base + lane < rows, live = next[0];
#pragma unroll
        for (int i = 0; i + 1 < kAhead; ++i) next[i] = next[i + 1];
        const int64_t ahead = base + 32 * kAhead + lane;
        next[kAhead - 1] = ahead < rows && wanted(ahead);
        const uint32_t lives = __ballot_sync(0xFFFFFFFFu, here && live), deads = __ballot_sync(0xFFFFFFFFu, here && !live);
        const uint32_t before = (1u << lane) - 1u;
        const int turn = live ? live_turn + __popc(lives & before) : dead_turn + __popc(deads & before);
        uint32_t todo = __ballot_sync(0xFFFFFFFFu, here && turn % n == mine);
        live_turn = (live_turn + __popc(lives)) % n;
        dead_turn = (dead_turn + __popc(deads)) % n;
        for (; todo; todo &= todo - 1) {
            const int at = __ffs(todo) - 1;
            if (!give(base + at, (lives >> at) & 1u)) return;
        }
    }
}

// kBig: one block an SM of 512 computing threads, else two of 256
template <typename T, int kMode, bool kGrad, bool kBig>
__global__ void __launch_bounds__(kBig ? kBigThreads + 32 * (2 + kMaxDepth) : 384, kBig ? 1 : 2) loss_ring_kernel(LossArgs a, RingShape shape)
{
    constexpr int E = Vec<T>::kElems;
    extern __shared__ __align__(128) uint8_t s_ring[];   // [slots][chunk], then the targets of `depth` rows and a table
    __shared__ __align__(8) uint64_t s_full[kMaxSlots], s_empty[kMaxSlots], s_exchange[2];
    __shared__ __align__(8) uint64_t s_target_full[kMaxDepth], s_target_empty[kMaxDepth];
    __shared__ __align__(8) uint64_t s_queue_full[kQueue], s_queue_empty[kQueue];
    __shared__ int64_t s_queue[kQueue];                  // 2 row + (is it read), -1: no more
    __shared__ uint32_t s_gave_up;                       // some wait of the cluster ran out
    __shared__ __align__(8) MaxSum s_block[2][kMaxCluster * kBigThreads / 32];
    __shared__ RowInfo s_info[kMaxDepth];
    __shared__ float4 s_result[kMaxDepth];               // reference, sum: its logarithm and inverse; the gradient's factor
    const int warps = shape.threads >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cluster = shape.cluster, slots = shape.slots, depth = shape.depth;
    const uint32_t rank = cluster > 1 ? cluster_rank() : 0u;
    const int my_cluster = (int)(blockIdx.x / cluster), clusters = (int)(gridDim.x / cluster);
    // targets of a row buffer: id, probability, its logarithm, logit, each padded to whole vectors
    const int top_k = kMode == kDistill ? a.top_k : 1, pad_k = (top_k + 3) & ~3;   // lists start at 16 bytes
    float *s_targets = reinterpret_cast<float *>(s_ring + (size_t)slots * shape.chunk_bytes);
    const auto target_id = [&](int b) { return reinterpret_cast<int32_t *>(s_targets + (size_t)b * 4 * pad_k); };
    const auto target_p = [&](int b) { return s_targets + (size_t)b * 4 * pad_k + pad_k; };
    const auto target_logp = [&](int b) { return s_targets + (size_t)b * 4 * pad_k + 2 * pad_k; };
    const auto target_z = [&](int b) { return s_targets + (size_t)b * 4 * pad_k + 3 * pad_k; };

    if (threadIdx.x == 0) {
        for (int i = 0; i < slots; ++i) {
            mbar_init(smem_addr(&s_full[i]), 1);
            mbar_init(smem_addr(&s_empty[i]), warps);
        }
        for (int i = 0; i < depth; ++i) {
            mbar_init(smem_addr(&s_target_full[i]), 1);
            mbar_init(smem_addr(&s_target_empty[i]), warps);
        }
        for (int i = 0; i < kQueue; ++i) {
            mbar_init(smem_addr(&s_queue_full[i]), 1);
            mbar_init(smem_addr(&s_queue_empty[i]), 2);
        }
        for (int i = 0; i < 2; ++i) mbar_init(smem_addr(&s_exchange[i]), 1);
        mbar_init_fence();
        s_gave_up = 0;
    }
    __syncwarp();
    if (cluster > 1) cluster_sync();
    else __syncthreads();
    grid_dependency_release();            // the sum over rows may be set up meanwhile

    const auto set_part = [&](RowInfo &p, int64_t row) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(static_cast<const T *>(a.logits) + row * a.stride);
        const int64_t head = (int64_t)(((16u - (unsigned)(at & 15u)) & 15u) / sizeof(T));
        p.head = (int)(head < a.vocab ? head : a.vocab);
        p.count = (int)((a.vocab - p.head) / E);
        const int per = (p.count + cluster - 1) / cluster;
        p.from = per * (int)rank < p.count ? per * (int)rank : p.count;
        p.mine = p.count - p.from < per ? p.count - p.from : per;
    };
    const auto wanted = [&](int64_t row) {                // is the row read at all
        if (a.weight && a.weight[row] == 0.0f) return false;
        if (kMode == kDistill) return true;
        const int64_t token = load_id(a.ids, row, a.ids_dtype);
        return token >= 0 && token < a.vocab;
    };
    const int per_chunk = shape.chunk_bytes / 16;
    uint32_t limit = a.patience.of(my_cluster);
    // the next row of the queue (by the producer and the target warp), -1 at the end
    const auto next_row = [&](uint32_t taken, bool &load) {
        const uint32_t at = taken % kQueue;
        if (limit != 0 && !mbar_wait_idle(smem_addr(&s_queue_full[at]), (taken / kQueue) & 1, limit)) limit = 0;
        limit = __shfl_sync(0xFFFFFFFFu, limit, 0);
        const int64_t v = limit == 0 ? -1 : s_queue[at];
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&s_queue_empty[at]));
        load = v >= 0 && (v & 1) != 0;
        return v >= 0 ? v >> 1 : -1;
    };

    if (warp == warps + 1) {
        // ---- rows ----
        uint32_t given = 0;
        const auto give = [&](int64_t row, uint32_t load) {
            const uint32_t at = given % kQueue;
            if (limit != 0 && !mbar_wait_idle(smem_addr(&s_queue_empty[at]), ((given / kQueue) & 1) ^ 1, limit)) limit = 0;
            limit = __shfl_sync(0xFFFFFFFFu, limit, 0);
            if (limit == 0) return false;
            if (lane == 0) {
                s_queue[at] = row < 0 ? -1 : 2 * row + load;
                mbar_arrive(smem_addr(&s_queue_full[at]));
            }
            ++given;
            return true;
        };
        walk_rows(wanted, a.rows, clusters, my_cluster, give);
        for (int i = 0; i < depth; ++i)       // an end mark for every target warp
            if (!give(-1, 0)) break;
    } else if (warp == warps) {
        // ---- producer ----
        uint32_t slot = 0, phase = 0, issued = 0;
        bool load;
        uint32_t taken = 0;
        for (int64_t row = next_row(taken++, load); row >= 0; row = next_row(taken++, load)) {
            if (!load) continue;
            RowInfo p;
            set_part(p, row);
            const T *src = static_cast<const T *>(a.logits) + row * a.stride + p.head + (int64_t)p.from * E;
            for (int v = 0; v < p.mine && limit != 0; v += per_chunk) {
                if (!mbar_wait_idle(smem_addr(&s_empty[slot]), phase ^ 1, limit)) limit = 0;
                limit = __shfl_sync(0xFFFFFFFFu, limit, 0);
                if (limit == 0) break;
                if (lane == 0) {
                    const uint32_t bytes = (uint32_t)(p.mine - v < per_chunk ? p.mine - v : per_chunk) * 16;
                    const uint32_t bar = smem_addr(&s_full[slot]);
                    mbar_expect(bar, bytes);
                    bulk_load(smem_addr(s_ring) + slot * shape.chunk_bytes, src + (int64_t)v * E, bytes, bar);
                }
                ++issued;
                if (++slot == (uint32_t)slots) slot = 0, phase ^= 1;
            }
        }
        // whatever was issued lands before the block goes (consumed already, unless a wait ran out)
        for (uint32_t i = issued > (uint32_t)slots ? issued - slots : 0; i < issued; ++i)
            mbar_wait(smem_addr(&s_full[i % slots]), (i / slots) & 1, kPolls);
    } else if (warp >= warps + 2) {
        // ---- targets: the lists of rows to come; of the rows that are done, the
        // loss and the gradient at the targets, over what phase 2 wrote there ----
        const auto finish = [&](int buf, uint32_t parity) {
            if (limit != 0 && !mbar_wait_idle(smem_addr(&s_target_empty[buf]), parity, limit)) limit = 0;
            limit = __shfl_sync(0xFFFFFFFFu, limit, 0);
            if (limit == 0) return;
            const RowInfo info = s_info[buf];
            const float4 done = s_result[buf];
            const auto exponent = [&](float z) { return exponent_of(z, done.x, a.log2e_over_t); };
            if (!info.live) {
                if (rank == 0 && lane == 0) {
                    a.row_loss[info.row] = 0.0f;
                    if (kMode == kPolicy && a.logp) a.logp[info.row] = 0.0f;
                }
                return;
            }
            const int32_t *ids = target_id(buf);
            const float *probs = target_p(buf);
            if (kMode == kDistill && rank == 0) {
                const float loss = distill_row_loss(a, ids, probs, target_logp(buf), target_z(buf),
                                                    [&](float z) { return log_prob(a, z, done.x, done.y); });
                if (lane == 0) a.row_loss[info.row] = loss;
            }
            if (kGrad) {
                const RowInfo &p = info;
                T *g = static_cast<T *>(a.grad) + info.row * a.grad_stride;
                for (int k = lane; k < top_k; k += 32) {
                    const int32_t id = ids[k];
                    if (id < 0) continue;
                    // the block that has the element
                    const int v = (id - p.head) / E;
                    const bool my_part = id < p.head ? rank == 0
                                         : v >= p.count ? rank == (uint32_t)cluster - 1
                                                        : v >= p.from && v < p.from + p.mine;
                    if (!my_part) continue;
                    float prob = probs[k];
                    if (info.repeats) {
                        prob = 0.0f;
                        for (int i = 0; i < top_k; ++i)
                            if (ids[i] == id) prob += probs[i];
                    }
                    g[id] = from_f32<T>(done.w * fmaf(exp2_fast(exponent(target_z(buf)[k])), done.z, -prob));
                }
            }
            __syncwarp();
        };
        // Does an id occur twice in a list?  A short list is compared with itself.  The ids of
        // a long one are put into a table of at least twice as many places, each at the
        // first free one from where its hash points.
        const int buf = warp - (warps + 2), places = table_places(top_k);
        int32_t *table = reinterpret_cast<int32_t *>(s_targets + (size_t)depth * 4 * pad_k) + buf * places;
        const auto repeats = [&](const int32_t *ids) {
            bool twice = false;
            if (places == 0) {
                for (int k = lane; k < top_k; k += 32) {
                    int same = 0;
#pragma unroll 4
                    for (int i = 0; i < pad_k; i += 4) {
                        const int4 q = *reinterpret_cast<const int4 *>(ids + i);
                        same += (q.x == ids[k]) + (q.y == ids[k]) + (q.z == ids[k]) + (q.w == ids[k]);
                    }
                    twice |= ids[k] >= 0 && same > 1;
                }
                return __any_sync(0xFFFFFFFFu, twice) != 0;
            }
            for (int i = lane; i < places; i += 32) table[i] = -1;
            __syncwarp();
            for (int k = lane; k < top_k; k += 32) {
                const int32_t id = ids[k];
                uint32_t at = ((uint32_t)id * 2654435761u) >> 16;
                for (int tries = 0; id >= 0 && tries < places; ++tries, ++at) {
                    const int32_t was = atomicCAS(&table[at & (places - 1)], -1, id);
                    twice |= was == id;
                    if (was == -1 || was == id) break;
                }
            }
            return __any_sync(0xFFFFFFFFu, twice) != 0;
        };
        bool load = false;
        for (uint32_t it = buf;; it += depth) {
            const int64_t row = next_row(it, load);
            if (it >= (uint32_t)depth) finish(buf, ((it / depth) & 1) ^ 1);
            if (limit == 0) break;            // the buffer may still be in use: it stays as it is
            bool live = row >= 0 && load, twice = false;
            if (live && kMode == kDistill) {
                live = load_teacher<T>(a, row, target_id(buf), target_p(buf), target_logp(buf), target_z(buf));
                if (lane < pad_k - top_k) target_id(buf)[top_k + lane] = -1;
                __syncwarp();
                twice = kGrad && live && repeats(target_id(buf));
            } else if (live && lane == 0) {
                const int64_t token = load_id(a.ids, row, a.ids_dtype);
                target_id(buf)[0] = (int32_t)token;
                target_p(buf)[0] = 1.0f;
                target_z(buf)[0] = to_f32(static_cast<const T *>(a.logits)[row * a.stride + token]);
            }
            if (lane == 0) {
                RowInfo info = {};
                info.row = row;
                if (row >= 0) {
                    info.weight = a.weight ? a.weight[row] : 1.0f;
                    info.load = load;
                    info.live = live;
                    info.repeats = twice;
                    set_part(info, row);
                    if (kMode == kPolicy && live) {
                        info.advantage = a.advantage[row];
                        info.old_logp = a.old_logp ? a.old_logp[row] : 0.0f;
                        info.ref_logp = a.ref_logp ? a.ref_logp[row] : 0.0f;
                    }
                }
                s_info[buf] = info;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&s_target_full[buf]));
            if (row < 0) break;
        }
    } else {
        // ---- the rest ----
        const float c = a.log2e_over_t, slack = kSlack / c;
        const uint32_t ring = smem_addr(s_ring) + threadIdx.x * 16, vector_step = (uint32_t)shape.threads * 16;
        const uint32_t full_bar = smem_addr(s_full), empty_bar = smem_addr(s_empty), ring_bytes = (uint32_t)slots * shape.chunk_bytes;
        // a chunk of the ring: its bytes, its barriers' offset, and their phase
        struct Place { uint32_t at, bar, phase; };
        const auto advance = [&](Place &p) {
            p.at += shape.chunk_bytes;
            p.bar += 8;
            if (p.at == ring_bytes) p = Place{0, 0, p.phase ^ 1};
        };
        Place place = {0, 0, 0};
        uint32_t row_phase = 0, computed = 0;   // rows computed so far: even and odd ones take turns
        int buf = 0;
        while (true) {
            // one warp waits for the row's targets, the others for that warp; all agree
            // on whether some wait ran out, which ends the block's work
            if (warp == 0 && limit != 0 && !mbar_wait(smem_addr(&s_target_full[buf]), row_phase, limit)) limit = 0;
            if (any_of(limit == 0, shape.threads)) break;
            const RowInfo info = s_info[buf];
            const int64_t row = info.row;
            if (row < 0) break;
            const RowInfo &p = info;
            const T *z = static_cast<const T *>(a.logits) + row * a.stride;
            T *g = kGrad ? static_cast<T *>(a.grad) + row * a.grad_stride : nullptr;
            const bool same_offset = kGrad && ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0;
            // the single element of a few threads: the first block's head, the last block's tail
            int64_t edge = -1;
            if (rank == 0 && (int)threadIdx.x < p.head) edge = threadIdx.x;
            if (rank == (uint32_t)cluster - 1 && warp == 1 && p.head + p.count * E + lane < a.vocab) edge = p.head + p.count * E + lane;

            if (!info.live) {
                // nothing to compute: a chunk that is on its way is let go, the gradient is zero
                if (info.load)
                    for (int left = p.mine; left > 0; left -= per_chunk) {
                        if (limit != 0 && !mbar_wait(full_bar + place.bar, place.phase, limit)) limit = 0;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(empty_bar + place.bar);
                        advance(place);
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
            } else {
                float edge_z = 0.0f;
                if (edge >= 0) edge_z = to_f32(z[edge]);
                // phase 1
                const Place place0 = place;
                Running<T> run;
                for (int left = p.mine; left > 0; left -= per_chunk) {
                    if (!mbar_test(full_bar + place.bar, place.phase) && limit != 0 &&
                        !mbar_wait(full_bar + place.bar, place.phase, limit))
                        limit = 0;
                    const uint32_t at = ring + place.at;
                    if (left >= per_chunk) {
                        uint4 q[kPerThread];
#pragma unroll
                        for (int i = 0; i < kPerThread; ++i) q[i] = lds16(at + i * vector_step);
                        if constexpr (kGrad) run.add_unchecked(q, c, slack);
                        else run.add(q, c, slack);
                    } else {
                        // the last chunk: -inf where there is nothing
                        uint4 q[kPerThread];
#pragma unroll
                        for (int i = 0; i < kPerThread; ++i)
                            q[i] = (int)threadIdx.x + i * shape.threads < left ? lds16(at + i * vector_step) : nothing<T>();
                        if constexpr (kGrad) run.add_unchecked(q, c, slack);
                        else run.add(q, c, slack);
                    }
                    if (!kGrad) {
                        __syncwarp();
                        if (lane == 0) mbar_arrive(empty_bar + place.bar);
                    }
                    advance(place);
                }
                MaxSum ms{run.m, total(run.s)};
                if (kGrad && !(ms.s < kMost)) {
                    // once more, with a look at every vector's largest element
                    run = Running<T>();
                    Place there = place0;
                    for (int left = p.mine; left > 0; left -= per_chunk) {
                        for (int i = threadIdx.x, u = 0; i < left && u < kPerThread; i += shape.threads, ++u) {
                            const uint4 q[1] = {lds16(ring + there.at + u * vector_step)};
                            run.add(q, c, slack);
                        }
                        advance(there);
                    }
                    ms = MaxSum{run.m, total(run.s)};
                }
                if (edge >= 0) {
                    // exp2 of its exponent against its own reference: 1 but for the rounding of that
                    const float own = plain(edge_z * c) ? exp2_fast(fmaf(edge_z, c, -(edge_z * c))) : exp2_fast(edge_z - edge_z);
                    ms = join(ms, MaxSum{edge_z, edge_z == -kInf ? 0.0f : own}, c);
                }
                ms = join_lanes(ms, c);
                if (limit == 0) ms.s = kNan;
                // every warp's part to every block of the cluster, where one warp joins them and
                // works out what the row comes to
                const int turn = computed & 1;
                const uint32_t bar = smem_addr(&s_exchange[turn]);
                if (cluster > 1) {
                    if (threadIdx.x == 0) mbar_expect(bar, (uint32_t)(cluster * warps) * sizeof(MaxSum));
                    if (lane < cluster)
                        remote_store(remote_addr(smem_addr(&s_block[turn][rank * warps + warp]), lane), ms.m, ms.s, remote_addr(bar, lane));
                } else {
                    if (lane == 0) s_block[turn][warp] = ms;
                    asm volatile("bar.sync 1, %0;" ::"r"(shape.threads) : "memory");
                }
                if (warp == 0) {
                    if (cluster > 1 && limit != 0 && !mbar_wait(bar, (computed >> 1) & 1, limit)) limit = 0;
                    ms = lane < cluster * warps ? s_block[turn][lane] : MaxSum{-kInf, 0.0f};
                    for (int i = lane + 32; i < cluster * warps; i += 32) ms = join(ms, s_block[turn][i], c);
                    ms = join_lanes(ms, c);
                    if (limit == 0) ms.s = kNan;
                    const float log_s = logf(ms.s);
                    float coef;
                    if (kMode == kDistill) {
                        coef = a.grad_scale * info.weight * a.temperature;
                    } else {
                        const float logp = log_prob(a, target_z(buf)[0], ms.m, log_s);
                        float loss, slope;
                        policy_row(a, logp, info.advantage, info.old_logp, info.ref_logp, loss, slope);
                        if (rank == 0 && lane == 0) {
                            a.row_loss[row] = loss;
                            if (a.logp) a.logp[row] = logp;
                        }
                        coef = -a.grad_scale * info.weight * slope * a.inv_temperature;
                    }
                    if (lane == 0) s_result[buf] = make_float4(ms.m, log_s, 1.0f / ms.s, coef);
                }
                ++computed;
                asm volatile("bar.sync 1, %0;" ::"r"(shape.threads) : "memory");

                if (kGrad) {
                    // phase 2
                    const float4 done = s_result[buf];
                    const float m = done.x, ref = m * c, scaled = done.w * done.z;
                    const bool is_plain = plain(ref);
                    T *out = g + p.head + (int64_t)p.from * E;
                    const auto write_chunks = [&](auto plain_row, auto vectors) {
                        const auto put = [&](const uint4 &q, T *at) {
                            const Vals<E> e = exponentials<decltype(plain_row)::value>(widen16<T>(q), m, ref, c) * scaled;
                            if constexpr (decltype(vectors)::value) {
                                *reinterpret_cast<uint4 *>(at) = narrow16<T>(e);
                            } else {
                                float f[E];
                                e.get(f);
#pragma unroll
                                for (int k = 0; k < E; ++k) at[k] = from_f32<T>(f[k]);
                            }
                        };
                        Place there = place0;
                        T *to = out + (int64_t)threadIdx.x * E;
                        for (int left = p.mine; left > 0; left -= per_chunk, to += (int64_t)per_chunk * E) {
                            const uint32_t at = ring + there.at;
                            if (left >= per_chunk) {
                                uint4 q[kPerThread];
#pragma unroll
                                for (int i = 0; i < kPerThread; ++i) q[i] = lds16(at + i * vector_step);
#pragma unroll
                                for (int i = 0; i < kPerThread; ++i) put(q[i], to + i * shape.threads * E);
                            } else {
                                uint4 q[kPerThread];
#pragma unroll
                                for (int i = 0; i < kPerThread; ++i)
                                    q[i] = (int)threadIdx.x + i * shape.threads < left ? lds16(at + i * vector_step) : nothing<T>();
#pragma unroll
                                for (int i = 0; i < kPerThread; ++i)
                                    if ((int)threadIdx.x + i * shape.threads < left) put(q[i], to + i * shape.threads * E);
                            }
                            __syncwarp();
                            if (lane == 0) mbar_arrive(empty_bar + there.bar);
                            advance(there);
                        }
                    };
                    if (is_plain && same_offset) write_chunks(std::true_type{}, std::true_type{});
                    else if (same_offset) write_chunks(std::false_type{}, std::true_type{});
                    else if (is_plain) write_chunks(std::true_type{}, std::false_type{});
                    else write_chunks(std::false_type{}, std::false_type{});
                    if (edge >= 0) g[edge] = from_f32<T>(exp2_fast(exponent_of(edge_z, m, c)) * scaled);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&s_target_empty[buf]));
            if (++buf == depth) buf = 0, row_phase ^= 1;
        }
    }
    // No block goes while another may still write into its shared memory, and all hear of a
    // wait that ran out.
    if (__any_sync(0xFFFFFFFFu, limit == 0) && lane < cluster) {
        if (cluster > 1) remote_set(smem_addr(&s_gave_up), lane);
        else s_gave_up = 1;
    }
    __syncwarp();
    if (cluster > 1) cluster_sync();
    else __syncthreads();
    if (s_gave_up == 0) return;
    walk_rows(wanted, a.rows, clusters, my_cluster, [&](int64_t row, uint32_t) {
        if (rank == 0 && threadIdx.x == 0) {
            a.row_loss[row] = kNan;
            if (kMode == kPolicy && a.logp) a.logp[row] = kNan;
        }
        if (kGrad) {
            T *g = static_cast<T *>(a.grad) + row * a.grad_stride;
            for (int64_t j = (int64_t)rank * blockDim.x + threadIdx.x; j < a.vocab; j += (int64_t)cluster * blockDim.x) g[j] = from_f32<T>(kNan);
        }
        return true;
    });
    // An exchange that was not waited for may still be under way to this block (a store takes
    // about a microsecond, and nothing tells of the last one): it stays for a millisecond.
    if (cluster > 1)
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
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

// The ring's shape for rows of more than kShortVectors * kShortThreads vectors: false if no
// cluster holds one for its gradient.
bool ring_shape(int64_t rows, int64_t vocab, int es, int top_k, bool grad, int sms, RingShape *out)
{
    const int64_t row_bytes = vocab * es;
    RingShape r;
    const size_t list = (size_t)16 * ((top_k + 3) & ~3), table = (size_t)4 * table_places(top_k);
    const int lists = top_k <= 256 ? kMaxDepth : 2;
    // the ring takes what the lists leave: 7 chunks at least (1024 entries, 256 threads)
    const auto fit = [&](int t) {
        r.threads = t;
        r.depth = t > 256 ? lists : 2;
        r.chunk_bytes = t * 16 * kPerThread;
        const size_t per_block = (size_t)224 * 1024 / (kBigThreads / t) - 5 * 1024, targets = (list + table) * r.depth;
        r.slots = (int)((per_block - targets) / r.chunk_bytes);
        if (r.slots > kMaxSlots) r.slots = kMaxSlots;
        r.smem = (size_t)r.slots * r.chunk_bytes + targets;
    };
    // two blocks of 256 threads an SM where each holds whole rows: what one waits for, the
    // other hides
    fit(256);
    if (grad ? (row_bytes + r.chunk_bytes - 1) / r.chunk_bytes > r.slots : row_bytes >= 64 * 1024) fit(kBigThreads);
    r.cluster = 1;
    const auto chunks = [&](int c) { return ((row_bytes / 16 + c - 1) / c * 16 + r.chunk_bytes - 1) / r.chunk_bytes; };
    if (grad)
        while (r.cluster < kMaxCluster && chunks(r.cluster) > r.slots) r.cluster *= 2;
    if (grad && chunks(r.cluster) > r.slots) return false;
    // few rows: more blocks each, while SMs are idle
    while (r.cluster < kMaxCluster && rows * r.cluster * 2 <= sms && chunks(r.cluster) > 1) r.cluster *= 2;
    *out = r;
    return true;
}

constexpr int kMaxShared = 220 * 1024;

template <typename T, int kMode, bool kGrad, bool kBig>
so_status launch_ring(const LossArgs &a, const RingShape &shape, int sms, cudaStream_t st)
{
    struct Known { std::atomic<uint64_t> key; std::atomic<int> clusters; };
    static Known cache[kMaxDevices];
    const auto kernel = loss_ring_kernel<T, kMode, kGrad, kBig>;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return SO_ERR_CUDA;
    if (dev < 0 || dev >= kMaxDevices) return SO_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)shape.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.blockDim = dim3((unsigned)(shape.threads + 32 * (2 + shape.depth)));
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
    const int64_t vectors = a.vocab / Vec<T>::kElems;
    if (vectors <= kShortVectors * kShortThreads) {
        const int per_thread = (int)((vectors + kShortVectors - 1) / kShortVectors);
        const unsigned threads = per_thread <= 32 ? 32u : (unsigned)((per_thread + 31) / 32 * 32);
        const size_t lists = (size_t)16 * (kMode == kDistill ? a.top_k : 1);
        return launch(a.grad ? loss_short_kernel<T, kMode, true> : loss_short_kernel<T, kMode, false>, (unsigned)a.rows, threads, lists, st, false, a);
    }
    RingShape shape;
    if (ring_shape(a.rows, a.vocab, (int)sizeof(T), kMode == kDistill ? a.top_k : 1, a.grad != nullptr, sms, &shape))
    {
        if (shape.threads > 256)
            return a.grad ? launch_ring<T, kMode, true, true>(a, shape, sms, st) : launch_ring<T, kMode, false, true>(a, shape, sms, st);
        return a.grad ? launch_ring<T, kMode, true, false>(a, shape, sms, st) : launch_ring<T, kMode, false, false>(a, shape, sms, st);
    }
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
    if (rows < 0 || rows > INT32_MAX || vocab < 1 || vocab > (int64_t(1) << 30)) return SO_ERR_INVALID_ARG;
    if (!(temperature > 0.0) || !std::isfinite(temperature) || !std::isfinite(grad_scale)) return SO_ERR_INVALID_ARG;
    // what the kernels hold of them in fp32: T, 1 / T, and log2(e) / T, the largest of the three
    const float t = (float)temperature, inv = (float)(1.0 / temperature), log2e_over_t = (float)(1.4426950408889634 / temperature);
    if (!(t > 0.0f) || !std::isfinite(t) || !(inv > 0.0f) || !std::isfinite(log2e_over_t) || !std::isfinite((float)grad_scale))
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
    a.log2e_over_t = log2e_over_t; a.grad_scale = (float)grad_scale;
    a.ids = ids; a.ids_dtype = ids_dtype;
    a.patience = patience();
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
    if (!(kl_coef >= 0.0) || !std::isfinite((float)kl_coef) || (kl_coef != 0.0 && !ref_logp)) return SO_ERR_INVALID_ARG;
    if (!aligned(advantage, 4) || !aligned(old_logp, 4) || !aligned(ref_logp, 4) || !aligned(logp, 4))
        return SO_ERR_INVALID_ARG;
    if (rows > 0 && !advantage) return SO_ERR_INVALID_ARG;
    a.advantage = advantage; a.old_logp = old_logp; a.ref_logp = kl_coef != 0.0 ? ref_logp : nullptr; a.logp = logp;
    a.clip_lo = (float)(1.0 - clip_low); a.clip_hi = (float)(1.0 + clip_high); a.kl_coef = (float)kl_coef;
    return run_loss<kPolicy>(a, dtype, loss, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
