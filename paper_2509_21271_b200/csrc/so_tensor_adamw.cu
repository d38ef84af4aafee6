// AdamW over a list of tensors where they lie, with its moments in 32 or in 8 bits.
//
//   g  = grad * (grad_scale * clip),  clip = min(1, max_norm / (norm + 1e-6))
//   m' = beta1 m + (1 - beta1) g,     v' = beta2 v + (1 - beta2) g g
//   p' = p - (lr wd p + lr / (1 - beta1^t) * m' / (sqrt(v') / sqrt(1 - beta2^t) + eps))
//
// in fp32, m and v with every operation rounded by itself (no contraction).  The moments lie in arenas
// of the optimizer, each tensor's from a block of 256 elements on.
//
// An 8-bit moment has 4 bits of fraction and, for m, 3 bits of exponent and a sign, for v,
// 4 bits of exponent.  With f and e those bits it stands for f units where e = 0, for
// (16 + f) 2^(e - 1) otherwise; a unit is 2^(s - 127) with s a byte of the block, chosen so
// that the block's largest value fits.  The largest m is 1984 units, the largest v 507904,
// so that a block spans 2^11 in m and, as v is a square, 2^9.5 in the size of gradients.
// s = 0 marks a block of zeros, s = 255 one that holds a value which is not finite (all of
// it is NaN then).  A v that is not zero is never rounded to zero: a moment without a
// second moment would be divided by eps alone.
//
// That code is the bit pattern of an fp32 number of as many units of 2^-130, cut off above
// its last 19 bits: fp32 has the same step from its subnormal to its normal numbers.  So a
// value is encoded by two multiplications (the second rounds to 2^-19 of a unit), the
// addition of 2^18 (to nearest) or of 16 random bits (stochastically) to the bits below,
// and a shift.
#include "so_ops.cuh"

using namespace so_ops;

namespace {

constexpr int kBlock = SO_TENSOR_BLOCK;   // elements that share a scale, and what a warp takes at a time
constexpr int kLane = kBlock / 32;        // consecutive elements of a lane
constexpr int kThreads = 256, kWarps = kThreads / 32;
// Tensors of a launch: the table is a kernel parameter of 25 KB, or of 2.5 KB where that is enough.
constexpr int kMaxTensors = 640, kFewTensors = 64;
// Blocks a warp takes in a row, at most.  589 M parameters with 8-bit moments, which are then written out in bf16
// (0.6 ms of it): 2.53 ms with runs of 1, 2.80 with 8, 2.70 with 32, 2.32 with 100, 2.34 with 128, 2.73 with one
// run a warp; with 32 bits the same up to 100.
constexpr int kMaxRun8 = 100, kMaxRun32 = 8;
constexpr int kNormBlocks = 1184;         // thread blocks of a norm launch, at most; the same on every device

struct Entry {
    float *param;
    const void *grad;
    void *copy;
    int64_t numel, first;                 // its first block, counted over the list
};

// What the device knows of an optimizer's progress: SO_TENSOR_RECORD_BYTES of the caller's.
struct Record {
    int64_t t;                            // steps taken
    float norm, coef, skipped;            // of the last step: norm of the gradients, clip factor, 1 if it was skipped
    float factor;                         // grad_scale * clip
    float rsqrt_bc2, step_size;           // 1 / sqrt(1 - beta2^t), lr / (1 - beta1^t)
    uint32_t key;                         // of the step's random numbers
    uint32_t done;                        // thread blocks whose sums are in place
};
static_assert(sizeof(Record) <= SO_TENSOR_RECORD_BYTES, "the record fits");

struct Hyper {
    double lr, beta1, beta2, max_norm, grad_scale;
    uint64_t seed;
    int32_t clip;
};

// MurmurHash3's 32-bit finalizer (Appleby; public domain).
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x85EBCA6Bu;
    x ^= x >> 13;
    x *= 0xC2B2AE35u;
    return x ^ (x >> 16);
}

// Closes the gradients' look and opens the step: one thread.
__device__ void begin_step(Record *r, double sumsq, const Hyper &h)
{
    float norm = 0.0f, coef = 1.0f;
    bool skip = false;
    if (h.clip) {
        const double wide = sqrt(sumsq) * fabs(h.grad_scale);
        skip = !(wide <= 1.7976931348623157e308);        // infinite, or NaN
        norm = (float)wide;
        if (h.max_norm > 0.0) coef = (float)fmin(1.0, h.max_norm / (wide + 1e-6));
        if (skip) coef = 0.0f;
    }
    r->norm = norm;
    r->coef = coef;
    r->skipped = skip ? 1.0f : 0.0f;
    r->factor = __fmul_rn((float)h.grad_scale, coef);
    if (skip) return;
    const int64_t t = r->t + 1;
    r->t = t;
    r->rsqrt_bc2 = (float)(1.0 / sqrt(1.0 - pow(h.beta2, (double)t)));
    r->step_size = (float)(h.lr / (1.0 - pow(h.beta1, (double)t)));
    r->key = mix(mix((uint32_t)h.seed) ^ mix((uint32_t)(h.seed >> 32) ^ 0x9E3779B9u) ^ (uint32_t)t);
}

__global__ void begin_kernel(Record *r, const __grid_constant__ Hyper h) { begin_step(r, 0.0, h); }

template <int kMax>
struct TableOf {
    static constexpr int kRoom = kMax;
    int32_t n;
    int64_t blocks;                       // of all its tensors
    int64_t first;                        // of its first tensor
    Entry e[kMax];
};

// Index of the tensor that holds block b (tensors without elements have none).
template <typename Table>
__device__ __forceinline__ int tensor_of(const Table &t, int64_t b)
{
    int lo = 0, hi = t.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.e[mid].first <= b) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// kLane elements of a matrix of any alignment, those from `n` on as zeros.
template <typename T>
__device__ __forceinline__ void load_lane(const T *p, int n, bool vectors, float (&f)[kLane])
{
    if (vectors && n >= kLane) {
        if constexpr (sizeof(T) == 4) {
            uint32_t w[8];
            asm("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
        } else {
            unpack<T>(__ldcs(reinterpret_cast<const uint4 *>(p)), f);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kLane; ++i) f[i] = i < n ? to_f32(p[i]) : 0.0f;
    }
}

// The same of an array that this kernel writes.
__device__ __forceinline__ void load_own(const float *p, int n, bool vectors, float (&f)[kLane])
{
    if (vectors && n >= kLane) {
        asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7]) : "l"(p));
    } else {
#pragma unroll
        for (int i = 0; i < kLane; ++i) f[i] = i < n ? p[i] : 0.0f;
    }
}
__device__ __forceinline__ void store_own(float *p, int n, bool vectors, const float (&f)[kLane])
{
    if (vectors && n >= kLane) {
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]),
                     "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]) : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < kLane; ++i)
            if (i < n) p[i] = f[i];
    }
}
template <typename T>
__device__ __forceinline__ void store_copy(T *p, int n, bool vectors, const float (&f)[kLane])
{
    if (vectors && n >= kLane) {
        __stcs(reinterpret_cast<uint4 *>(p), pack<T>(f));
    } else {
#pragma unroll
        for (int i = 0; i < kLane; ++i)
            if (i < n) p[i] = from_f32<T>(f[i]);
    }
}

// Bound: memory: 76 % of DRAM's peak rate by the counters, 28 % of the issue slots.
//
// Sum of the squares of all gradients: fp32 over 32 bytes of a lane's, fp64 from there on, in a fixed
// order.  The thread block that comes last adds the blocks' sums and opens the step.
template <typename G, typename Table>
__global__ void __launch_bounds__(kThreads) norm_kernel(const __grid_constant__ Table t, const __grid_constant__ Hyper h, Record *record,
                                                        double *sums, uint32_t first_sum, uint32_t all_sums)
{
    __shared__ double s_sum[kWarps];
    __shared__ bool s_last;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double sum = 0.0;
    // consecutive blocks a warp, eight at a time: where they lie in one tensor, 32 bytes a lane and load
    const int64_t warps = (int64_t)gridDim.x * kWarps, me = (int64_t)blockIdx.x * kWarps + warp, each = (t.blocks + warps - 1) / warps;
    int64_t i = me * each, end = i + each;
    if (end > t.blocks) end = t.blocks;
    int k = i < end ? tensor_of(t, t.first + i) : 0;
    constexpr int kAtOnce = 8, kElems = 32 / (int)sizeof(G), kLoads = kAtOnce * kBlock / (32 * kElems);
    while (i < end) {
        const int64_t b = t.first + i;
        while (k + 1 < t.n && t.e[k + 1].first <= b) ++k;
        const Entry &e = t.e[k];
        const int64_t at = (b - e.first) * kBlock;
        const G *grad = static_cast<const G *>(e.grad) + at;
        if (i + kAtOnce <= end && at + kAtOnce * kBlock <= e.numel && (reinterpret_cast<uintptr_t>(grad) & 31) == 0) {
            uint32_t w[kLoads][8];
#pragma unroll
            for (int u = 0; u < kLoads; ++u)
                asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                             : "=r"(w[u][0]), "=r"(w[u][1]), "=r"(w[u][2]), "=r"(w[u][3]), "=r"(w[u][4]), "=r"(w[u][5]), "=r"(w[u][6]), "=r"(w[u][7])
                             : "l"(grad + (u * 32 + lane) * kElems));
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                float q = 0.0f;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float f[Vec<G>::kElems];
                    unpack<G>(make_uint4(w[u][4 * h], w[u][4 * h + 1], w[u][4 * h + 2], w[u][4 * h + 3]), f);
#pragma unroll
                    for (int j = 0; j < Vec<G>::kElems; ++j) q = fmaf(f[j], f[j], q);
                }
                sum += (double)q;
            }
            i += kAtOnce;
        } else {
            float f[kLane];
            const int64_t left = e.numel - at - lane * kLane;
            load_lane(grad + lane * kLane, left > kLane ? kLane : (int)left, (reinterpret_cast<uintptr_t>(grad) & (sizeof(G) * kLane - 1)) == 0, f);
            float q = 0.0f;
#pragma unroll
            for (int j = 0; j < kLane; ++j) q = fmaf(f[j], f[j], q);
            sum += (double)q;
            ++i;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int i = 0; i < kWarps; ++i) s += s_sum[i];
        sums[first_sum + blockIdx.x] = s;
        __threadfence();
        s_last = atomicAdd(&record->done, 1u) == all_sums - 1;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    sum = 0.0;
    for (uint32_t i = threadIdx.x; i < all_sums; i += kThreads) sum += __ldcg(sums + i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int i = 0; i < kWarps; ++i) s += s_sum[i];
        record->done = 0;
        begin_step(record, s, h);
    }
}

struct Step {
    float beta1, omb1, beta2, omb2, eps, decay;
    void *m, *v;
    uint8_t *m_scale, *v_scale;
    const Record *record;
    int32_t run, stochastic, sms;
};

// One step of an element.  m and v operation by operation (packed pairs of operations come out
// fused, although they name their rounding); the square root and the quotient are the hardware's,
// good to 2^-22 together; a second moment below 2^-126 counts as 0 there.
struct Update {
    float factor, beta1, omb1, beta2, omb2, rsqrt_bc2, eps, decay, step;
    __device__ __forceinline__ void operator()(float grad, float &m, float &v, float &p) const
    {
        const float g = __fmul_rn(grad, factor);
        m = __fadd_rn(__fmul_rn(m, beta1), __fmul_rn(g, omb1));
        v = __fadd_rn(__fmul_rn(v, beta2), __fmul_rn(__fmul_rn(g, omb2), g));
        float root, inverse;
        asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(root) : "f"(v));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"(fmaf(root, rsqrt_bc2, eps)));
        p = fmaf(__fmul_rn(m, inverse), -step, fmaf(p, -decay, p));
    }
};

// What 8 codes stand for.  As the top bits of binary16 numbers they are multiples of 2^-18, from
// its subnormal numbers on; so two at a time go through binary16 to fp32.
template <bool kSigned>
__device__ __forceinline__ void decode(uint2 codes, uint32_t scale, float (&f)[kLane])
{
    // 2^(scale - 127 + 18), in two factors where fp32 has none
    const bool large = scale > 236;
    const float wide = scale == 255 ? kNan : __uint_as_float((scale + (large ? 9 : 18)) << 23);
#pragma unroll
    for (int i = 0; i < kLane / 2; ++i) {
        const uint32_t w = __byte_perm(i < 2 ? codes.x : codes.y, 0, i & 1 ? 0x4342 : 0x4140);   // a byte to each half
        const uint32_t bits = kSigned ? ((w << 6) & 0x1FC01FC0u) | ((w << 8) & 0x80008000u) : (w << 6) & 0x3FC03FC0u;
        float lo, hi;
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(bits));
        f[2 * i] = lo;
        f[2 * i + 1] = hi;
    }
    if (large) {
#pragma unroll
        for (int i = 0; i < kLane; ++i) f[i] *= 512.0f;
    }
#pragma unroll
    for (int i = 0; i < kLane; ++i) f[i] *= wide;
}

// The scale of a block from the bit pattern of its largest magnitude: the largest code
// stands for 31/16 2^kTop units.
template <int kTop>
__device__ __forceinline__ uint32_t scale_of(uint32_t most)
{
    const int exponent = (int)(most >> 23);
    if (exponent == 255) return 255;
    if (most == 0) return 0;
    const int s = exponent + ((most & 0x7FFFFFu) > 0x780000u) - kTop;
    return s < 1 ? 1u : (uint32_t)s;
}

// 8 codes.  `noise` is what is added below a code, times 32: the code is then the top byte of
// 32 (bits + noise), whose multiplication drops the sign.
template <bool kSigned>
__device__ __forceinline__ uint2 encode(const float (&f)[kLane], uint32_t scale, const uint32_t (&noise)[kLane])
{
    if (scale == 255) return make_uint2(0, 0);
    const uint32_t s = scale < 1 ? 1u : scale;
    float y[kLane];                       // f 2^(127 - s - 130): in one product where that factor is a normal number
    if (s <= 123) {
        const float factor = __uint_as_float((124u - s) << 23);
#pragma unroll
        for (int i = 0; i < kLane; ++i) y[i] = f[i] * factor;
    } else {
        const float up = __uint_as_float((254u - s) << 23);
#pragma unroll
        for (int i = 0; i < kLane; ++i) y[i] = f[i] * up * 0x1p-130f;
    }
    uint32_t t[kLane];
#pragma unroll
    for (int i = 0; i < kLane; ++i) {
        uint32_t c = __float_as_uint(y[i]) * 32u + noise[i];
        if (kSigned) c = (c & 0x7FFFFFFFu) | (__float_as_uint(f[i]) & 0x80000000u);
        else if (f[i] != 0.0f) c = max(c, 1u << 24);
        t[i] = c;
    }
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = __byte_perm(__byte_perm(t[4 * i], t[4 * i + 1], 0x0073), __byte_perm(t[4 * i + 2], t[4 * i + 3], 0x0073), 0x5410);
    return make_uint2(w[0], w[1]);
}

// Bits of the warp's largest magnitude; those of a NaN are larger than all others'.
__device__ __forceinline__ uint32_t most_of(const float (&f)[kLane])
{
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < kLane; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(most) : "f"(fabsf(f[i])));
    return __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most));
}

// What a lane reads of a block.
template <int kBits, typename G>
struct Block {
    static constexpr int kWords = kLane * (int)sizeof(G) / 4;
    float *param;
    void *copy;
    int n;                                // elements of this lane that there are
    float p[kLane];
    uint32_t g[kWords];
    uint2 mc, vc;
    uint32_t ms, vs;
    // k: the tensor of the block before, brought up to this one's
    template <typename Table>
    __device__ __forceinline__ void load(const Table &t, const Step &s, int &k, int64_t b, int lane)
    {
        while (k + 1 < t.n && t.e[k + 1].first <= b) ++k;
        const Entry &e = t.e[k];
        const int64_t at = (b - e.first) * kBlock + lane * kLane, left = e.numel - at;
        n = left >= kLane ? kLane : left > 0 ? (int)left : 0;
        param = e.param + at;
        copy = static_cast<char *>(e.copy) + at * 2;
        const G *grad = static_cast<const G *>(e.grad) + at;
        load_own(param, n, (reinterpret_cast<uintptr_t>(param) & 31) == 0, p);
        if (n >= kLane && (reinterpret_cast<uintptr_t>(grad) & (sizeof(G) * kLane - 1)) == 0) {
            if constexpr (sizeof(G) == 4) {
                asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                             : "=r"(g[0]), "=r"(g[1]), "=r"(g[2]), "=r"(g[3]), "=r"(g[4]), "=r"(g[5]), "=r"(g[6]), "=r"(g[7]) : "l"(grad));
            } else {
                const uint4 q = __ldcs(reinterpret_cast<const uint4 *>(grad));
                g[0] = q.x, g[1] = q.y, g[2] = q.z, g[3] = q.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                if constexpr (sizeof(G) == 4) g[i] = i < n ? __float_as_uint(grad[i]) : 0u;
                else g[i] = (2 * i < n ? (uint32_t)grad[2 * i].bits : 0u) | (2 * i + 1 < n ? (uint32_t)grad[2 * i + 1].bits << 16 : 0u);
            }
        }
        if constexpr (kBits == 8) {
            const int64_t slot = b * kBlock + lane * kLane;
            mc = *reinterpret_cast<const uint2 *>(static_cast<uint8_t *>(s.m) + slot);
            vc = *reinterpret_cast<const uint2 *>(static_cast<uint8_t *>(s.v) + slot);
            ms = s.m_scale[b];
            vs = s.v_scale[b];
        }
    }
    __device__ __forceinline__ void gradients(float (&f)[kLane]) const
    {
        if constexpr (sizeof(G) == 4) {
#pragma unroll
            for (int i = 0; i < kLane; ++i) f[i] = __uint_as_float(g[i]);
        } else {
            unpack<G>(make_uint4(g[0], g[1], g[2], g[3]), f);
        }
    }
};

// A warp takes `run` blocks in a row, a lane eight consecutive elements of each; the grid goes through
// the list from its begin to its end, and a warp finds its tensors by going on from the last one's.
//
// Bound: memory, with 8-bit moments together with instructions.  589 M parameters, bf16 gradients and
// copies: 32 bits 2.54 ms, 28 bytes a parameter at 6.5 TB/s, a copy's rate; 8 bits 2.29 ms together with writing the
// moments out.  With 8 bits some 580 instructions a warp and block take 70 % of the issue slots, DRAM is at 69 %.
template <int kBits, typename G, typename C, typename Table>
__global__ void __launch_bounds__(kThreads) step_kernel(const __grid_constant__ Table t, const __grid_constant__ Step s)
{
    const int lane = threadIdx.x & 31;
    const int64_t begin = ((int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5)) * s.run, stride = (int64_t)gridDim.x * kWarps * s.run;
    int k = begin < t.blocks ? tensor_of(t, t.first + begin) : 0;
    grid_dependency_wait();
    if (s.record->skipped != 0.0f) return;
    const uint32_t key = s.record->key;
    const Update update = {s.record->factor, s.beta1, s.omb1, s.beta2, s.omb2, s.record->rsqrt_bc2, s.eps, s.decay, s.record->step_size};
    Block<kBits, G> now;
    for (int64_t i = begin, left = s.run; i < t.blocks; --left, left > 0 ? ++i : (i += stride - s.run + 1, left = s.run)) {
        const int64_t b = t.first + i;
        now.load(t, s, k, b, lane);
        const int n = now.n;
        const int64_t slot = b * kBlock + lane * kLane;
        float *param = now.param;
        const bool own = (reinterpret_cast<uintptr_t>(param) & 31) == 0;
        float p[kLane], g[kLane], m[kLane], v[kLane];
#pragma unroll
        for (int i = 0; i < kLane; ++i) p[i] = now.p[i];
        now.gradients(g);
        if constexpr (kBits == 8) {
            decode<true>(now.mc, now.ms, m);
            decode<false>(now.vc, now.vs, v);
        } else {
            load_own(static_cast<float *>(s.m) + slot, kLane, true, m);
            load_own(static_cast<float *>(s.v) + slot, kLane, true, v);
        }
#pragma unroll
        for (int i = 0; i < kLane; ++i) update(g[i], m[i], v[i], p[i]);
        store_own(param, n, own, p);
        if constexpr (!std::is_same<C, void>::value) {
            C *copy = static_cast<C *>(now.copy);
            store_copy<C>(copy, n, (reinterpret_cast<uintptr_t>(copy) & 15) == 0, p);
        }
        // (behind a tensor's end gradients and moments are zeros, and stay so)
        if constexpr (kBits == 8) {
            const uint32_t ms = scale_of<10>(most_of(m)), vs = scale_of<18>(most_of(v));
            uint32_t nm[kLane], nv[kLane];
            if (s.stochastic) {
                const uint32_t lane_key = mix(key + (uint32_t)(slot >> 32)) ^ (uint32_t)slot;
#pragma unroll
                for (int i = 0; i < kLane; ++i) {
                    // 8 r + 4 below the code for 16 random bits r, times 32
                    const uint32_t x = mix(lane_key ^ i);
                    nm[i] = __byte_perm(x, 128u, 0x5104);
                    nv[i] = __byte_perm(x, 128u, 0x5324);
                }
            } else {
#pragma unroll
                for (int i = 0; i < kLane; ++i) nm[i] = nv[i] = 1u << 23;
            }
            *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(s.m) + slot) = encode<true>(m, ms, nm);
            *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(s.v) + slot) = encode<false>(v, vs, nv);
            if (lane == 0) {
                s.m_scale[b] = (uint8_t)ms;
                s.v_scale[b] = (uint8_t)vs;
            }
        } else {
            store_own(static_cast<float *>(s.m) + slot, kLane, true, m);
            store_own(static_cast<float *>(s.v) + slot, kLane, true, v);
        }
    }
}

// 8-bit moments as the values they stand for; bf16 holds each of them.
__global__ void __launch_bounds__(kThreads) moments_kernel(const uint8_t *m, const uint8_t *v, const uint8_t *m_scale,
                                                           const uint8_t *v_scale, bf16_t *m_out, bf16_t *v_out, int64_t blocks)
{
    const int lane = threadIdx.x & 31;
    const int64_t b = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (b >= blocks) return;
    const int64_t slot = b * kBlock + lane * kLane;
    float f[kLane];
    decode<true>(__ldcs(reinterpret_cast<const uint2 *>(m + slot)), m_scale[b], f);
    __stcs(reinterpret_cast<uint4 *>(m_out + slot), pack<bf16_t>(f));
    decode<false>(__ldcs(reinterpret_cast<const uint2 *>(v + slot)), v_scale[b], f);
    __stcs(reinterpret_cast<uint4 *>(v_out + slot), pack<bf16_t>(f));
}

// ---- host ------------------------------------------------------------------------

int64_t blocks_of(int64_t numel) { return numel / kBlock + (numel % kBlock != 0); }

bool finite32(double x) { return std::isfinite(x) && std::isfinite((float)x); }

// Blocks of the whole list, -1 if a size or their sum is not one of a list.
int64_t list_blocks(const so_tensor *t, int32_t n)
{
    int64_t sum = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (t[i].numel < 0 || t[i].numel > int64_t(1) << 40) return -1;
        sum += blocks_of(t[i].numel);
        if (sum > SO_TENSOR_MAX_BLOCKS) return -1;
    }
    return sum;
}

unsigned norm_grid(int64_t blocks)
{
    // a warp takes several blocks at a time
    const int64_t want = (blocks + 4 * kWarps - 1) / (4 * kWarps);
    return want < 1 ? 1u : want > kNormBlocks ? (unsigned)kNormBlocks : (unsigned)want;
}

// Calls `fn(table)` for every kMaxTensors of the list.
template <typename Table, typename F>
so_status for_tables_of(const so_tensor *t, int32_t n, F fn)
{
    Table table;
    int64_t block = 0;
    int32_t i = 0;
    while (i < n) {
        table.n = 0;
        table.first = block;
        for (; i < n && table.n < Table::kRoom; ++i) {
            if (t[i].numel == 0) continue;
            Entry &e = table.e[table.n++];
            e.param = static_cast<float *>(t[i].param);
            e.grad = t[i].grad;
            e.copy = t[i].copy;
            e.numel = t[i].numel;
            e.first = block;
            block += blocks_of(t[i].numel);
        }
        table.blocks = block - table.first;
        if (table.n == 0) continue;
        const so_status st = fn(table);
        if (st != SO_OK) return st;
    }
    return SO_OK;
}

template <typename F>
so_status for_tables(const so_tensor *t, int32_t n, F fn)
{
    if (n <= kFewTensors) return for_tables_of<TableOf<kFewTensors>>(t, n, fn);
    return for_tables_of<TableOf<kMaxTensors>>(t, n, fn);
}

template <int kBits, typename G, typename C, typename Table>
so_status launch_step(const Table &t, const Step &s, cudaStream_t stream)
{
    const int64_t runs = (t.blocks + s.run - 1) / s.run;
    const int64_t grid = (runs + kWarps - 1) / kWarps, most = (int64_t)s.sms * 4;   // four blocks an SM
    return launch(step_kernel<kBits, G, C, Table>, (unsigned)(kBits == 32 || grid < most ? grid : most), kThreads, 0, stream, true, t, s);
}
template <int kBits, typename G, typename Table>
so_status launch_step(int32_t copy_dtype, const Table &t, const Step &s, cudaStream_t stream)
{
    if (copy_dtype == SO_DTYPE_BF16) return launch_step<kBits, G, bf16_t>(t, s, stream);
    if (copy_dtype == SO_DTYPE_FP16) return launch_step<kBits, G, f16_t>(t, s, stream);
    return launch_step<kBits, G, void>(t, s, stream);
}
template <int kBits, typename Table>
so_status launch_step(int32_t grad_dtype, int32_t copy_dtype, const Table &t, const Step &s, cudaStream_t stream)
{
    if (grad_dtype == SO_DTYPE_BF16) return launch_step<kBits, bf16_t>(copy_dtype, t, s, stream);
    if (grad_dtype == SO_DTYPE_FP16) return launch_step<kBits, f16_t>(copy_dtype, t, s, stream);
    return launch_step<kBits, float>(copy_dtype, t, s, stream);
}

}  // namespace

extern "C" {

so_status so_tensor_adamw_layout(const so_tensor *tensors, int32_t n_tensors, int32_t state_bits, so_tensor_adamw_info *info)
{
    if (!info || n_tensors < 0 || (n_tensors > 0 && !tensors) || (state_bits != 8 && state_bits != 32)) return SO_ERR_INVALID_ARG;
    const int64_t blocks = list_blocks(tensors, n_tensors);
    if (blocks < 0) return SO_ERR_INVALID_ARG;
    info->blocks = blocks;
    info->bytes_moment = (uint64_t)blocks * kBlock * (state_bits / 8);
    info->bytes_scale = state_bits == 8 ? (uint64_t)blocks : 0;
    info->bytes_record = SO_TENSOR_RECORD_BYTES;
    // one sum per thread block of the norm's launches
    info->bytes_scratch = ((uint64_t)n_tensors / kMaxTensors + 1) * kNormBlocks * sizeof(double);
    return SO_OK;
}

so_status so_tensor_adamw_step(const so_tensor *tensors, int32_t n_tensors, int32_t grad_dtype, int32_t copy_dtype,
                               int32_t state_bits, void *m, void *v, uint8_t *m_scale, uint8_t *v_scale,
                               const so_hparams *hp, double grad_scale, int32_t clip, int32_t stochastic,
                               uint64_t seed, void *record, void *scratch, uint64_t scratch_bytes, void *stream)
{
    so_tensor_adamw_info info;
    const so_status st = so_tensor_adamw_layout(tensors, n_tensors, state_bits, &info);
    if (st != SO_OK) return st;
    if (!valid_dtype(grad_dtype) || (copy_dtype != SO_TENSOR_NO_COPY && copy_dtype != SO_DTYPE_BF16 && copy_dtype != SO_DTYPE_FP16))
        return SO_ERR_INVALID_ARG;
    if ((clip != 0 && clip != 1) || (stochastic != 0 && stochastic != 1) || (stochastic && state_bits != 8)) return SO_ERR_INVALID_ARG;
    if (!hp || !record || !aligned(record, 16) || !finite32(grad_scale)) return SO_ERR_INVALID_ARG;
    if (!(hp->lr >= 0.0) || !finite32(hp->lr) || !(hp->beta1 >= 0.0 && hp->beta1 < 1.0) || !(hp->beta2 >= 0.0 && hp->beta2 < 1.0) ||
        !((float)hp->eps >= 0x1p-126f) || !finite32(hp->eps) || !(hp->weight_decay >= 0.0) || !finite32(hp->lr * hp->weight_decay) ||
        !finite32(hp->lr / (1.0 - hp->beta1)) || std::isnan(hp->max_grad_norm))
        return SO_ERR_INVALID_ARG;
    if (clip && (!scratch || !aligned(scratch, 16) || scratch_bytes < info.bytes_scratch)) return SO_ERR_INVALID_ARG;
    if (info.blocks > 0) {
        if (!m || !v || !aligned(m, 32) || !aligned(v, 32)) return SO_ERR_INVALID_ARG;
        if (state_bits == 8 && (!m_scale || !v_scale)) return SO_ERR_INVALID_ARG;
    }
    for (int32_t i = 0; i < n_tensors; ++i) {
        const so_tensor &t = tensors[i];
        if (t.numel == 0) continue;
        if (!t.param || !aligned(t.param, 4) || !t.grad || !aligned(t.grad, elem_size(grad_dtype))) return SO_ERR_INVALID_ARG;
        if (copy_dtype != SO_TENSOR_NO_COPY && (!t.copy || !aligned(t.copy, 2))) return SO_ERR_INVALID_ARG;
    }
    int sms;
    const so_status dev = device_sms(&sms);
    if (dev != SO_OK) return dev;
    const cudaStream_t cs = static_cast<cudaStream_t>(stream);
    Record *r = static_cast<Record *>(record);
    const Hyper h = {hp->lr, hp->beta1, hp->beta2, hp->max_grad_norm, grad_scale, seed, clip};
    so_status done;
    if (clip && info.blocks > 0) {
        uint32_t sums = 0, at = 0;
        for_tables(tensors, n_tensors, [&](const auto &t) { sums += norm_grid(t.blocks); return SO_OK; });
        done = for_tables(tensors, n_tensors, [&](const auto &t) {
            using Table = std::decay_t<decltype(t)>;
            const unsigned grid = norm_grid(t.blocks);
            const auto kernel = grad_dtype == SO_DTYPE_BF16 ? norm_kernel<bf16_t, Table> : grad_dtype == SO_DTYPE_FP16 ? norm_kernel<f16_t, Table> : norm_kernel<float, Table>;
            const so_status one = launch(kernel, grid, kThreads, 0, cs, false, t, h, r, static_cast<double *>(scratch), at, sums);
            at += grid;
            return one;
        });
    } else {
        done = launch(begin_kernel, 1, 1, 0, cs, false, r, h);
    }
    if (done != SO_OK) return done;
    Step s = {(float)hp->beta1, (float)(1.0 - hp->beta1), (float)hp->beta2, (float)(1.0 - hp->beta2), (float)hp->eps,
              (float)(hp->lr * hp->weight_decay), m, v, m_scale, v_scale, r, 1, stochastic, sms};
    return for_tables(tensors, n_tensors, [&](const auto &t) {
        // as many turns for every warp of the grid as keep runs below the limit
        const int64_t warps = (int64_t)sms * 4 * kWarps, mine = (t.blocks + warps - 1) / warps, limit = state_bits == 8 ? kMaxRun8 : kMaxRun32;
        const int64_t turns = mine < 2 * kMaxRun32 ? mine : (mine + limit - 1) / limit;   // short lists: a block a turn
        s.run = (int32_t)((mine + turns - 1) / (turns < 1 ? 1 : turns));
        return state_bits == 8 ? launch_step<8>(grad_dtype, copy_dtype, t, s, cs) : launch_step<32>(grad_dtype, copy_dtype, t, s, cs);
    });
}

so_status so_tensor_adamw_moments(const void *m, const void *v, const uint8_t *m_scale, const uint8_t *v_scale, int64_t blocks,
                                  void *m_out, void *v_out, void *stream)
{
    if (blocks < 0 || blocks > SO_TENSOR_MAX_BLOCKS) return SO_ERR_INVALID_ARG;
    if (blocks == 0) return SO_OK;
    if (!m || !v || !m_scale || !v_scale || !m_out || !v_out || !aligned(m, 8) || !aligned(v, 8) || !aligned(m_out, 16) || !aligned(v_out, 16))
        return SO_ERR_INVALID_ARG;
    return launch(moments_kernel, (unsigned)((blocks + kWarps - 1) / kWarps), kThreads, 0, static_cast<cudaStream_t>(stream), false,
                  static_cast<const uint8_t *>(m), static_cast<const uint8_t *>(v), m_scale, v_scale, static_cast<bf16_t *>(m_out),
                  static_cast<bf16_t *>(v_out), blocks);
}

}  // extern "C"
