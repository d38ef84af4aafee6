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
    Patience patience;
};

// ---- rows through shared memory ----------------------------------------------------
//
// A group of threads takes a row: a warp, or as many as its elements ask for, several
// groups to a block if they are small.  A thread holds its columns' weight and bias in
// registers for all its rows: kNV vectors of 16 bytes, or, where the rows do not all
// start at a 16-byte boundary (E = 1), kNV single elements.

template <typename T, int E>
__device__ __forceinline__ void store_vec(T *p, const Vals<E> &f)
{
    if constexpr (E == 1) *p = from_f32<T>(f.v);
    else *reinterpret_cast<uint4 *>(p) = narrow16<T>(f);
}

// E parameters from element c, as fp32 (`fill` where the array is absent)
template <int E>
__device__ __forceinline__ Vals<E> load_params(const void *p, int c, int32_t dtype, float fill)
{
    Vals<E> f;
    if (!p) {
        f.set(fill);
    } else if constexpr (E == 1) {
        f.v = load_any(p, c, dtype);
    } else if (dtype == SO_DTYPE_FP32) {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            const float4 q = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + c + e);
            f.p[e / 2] = pair(q.x, q.y);
            f.p[e / 2 + 1] = pair(q.z, q.w);
        }
    } else if constexpr (E == 8) {
        const uint4 q = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + c);
        f = dtype == SO_DTYPE_BF16 ? widen16<bf16_t>(q) : widen16<f16_t>(q);
    }
    return f;
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

constexpr int kRingBars = 64;             // groups x stages of a block, at most
constexpr size_t kRingBytes = 50 * 1024;  // shared memory a ring aims for
constexpr int kLongThreads = 512;         // threads of a long row, at most
constexpr int kRowThreads = 256;
constexpr int kGroupThreads = 128;        // a block has several groups up to this many threads

// Where R rows of a matrix lie in a stage of the ring, and their copies.  Rows of
// vectors are copied as they are.  Otherwise the 16-byte granules that a row touches
// are copied whole, so that it starts as far from a boundary as in memory; the granule
// in front of the first row and that behind the last one may reach out of the matrix,
// and their elements are loaded one by one.
template <typename T, int E>
struct RowCopies {
    const char *base;
    int64_t step;                         // bytes between rows
    uintptr_t end;                        // of the matrix
    uint32_t bytes, pitch;                // of a row, in memory and in the ring

    __device__ RowCopies(const void *p, int64_t stride, int64_t rows, int64_t cols)
        : base(static_cast<const char *>(p)), step(stride * (int64_t)sizeof(T)),
          end(reinterpret_cast<uintptr_t>(p) + (uintptr_t)((rows - 1) * stride * (int64_t)sizeof(T)) + (uintptr_t)cols * sizeof(T)),
          bytes((uint32_t)cols * sizeof(T)), pitch(E == 1 ? (bytes + 30 + 15) / 16 * 16 : bytes)
    {
    }
    // bytes from the row's place in the ring to its first element
    __device__ __forceinline__ uint32_t shift(int64_t row) const
    {
        return E == 1 ? ((uint32_t)reinterpret_cast<uintptr_t>(base) + (uint32_t)row * (uint32_t)step) & 15u : 0u;
    }
    __device__ __forceinline__ void load(int64_t row, uint32_t dst, uint32_t bar) const
    {
        const char *src = base + row * step;
        if constexpr (E > 1) {
            bulk_load(dst, src, bytes, bar);
        } else {
            const uint32_t before = shift(row), whole = (before + bytes + 15) / 16 * 16;
            uint32_t from = 0, to = whole;
            if (src - before < base) {
                from = 16;
                for (uint32_t i = before; i < 16 && i < before + bytes; i += sizeof(T)) put(dst + i, src + (i - before));
            }
            if (reinterpret_cast<uintptr_t>(src) - before + whole > end && whole > from) {
                to = whole - 16;
                for (uint32_t i = to < before ? before : to; i < before + bytes; i += sizeof(T)) put(dst + i, src + (i - before));
            }
            // ordinary stores into a place that a later bulk copy will overwrite: ordered between
            // the two kinds of access here, by the thread that issues that copy (two rows have any)
            if (from != 0 || to != whole) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            if (to > from) {
                asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(to - from) : "memory");
                bulk_load(dst + from, src - before + from, to - from, bar);
            }
        }
    }
    static __device__ __forceinline__ void put(uint32_t dst, const char *src)
    {
        if constexpr (sizeof(T) == 4)
            asm volatile("st.shared.u32 [%0], %1;" ::"r"(dst), "r"(*reinterpret_cast<const uint32_t *>(src)) : "memory");
        else
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(dst), "h"(*reinterpret_cast<const uint16_t *>(src)) : "memory");
    }
};

// E elements from shared memory
template <typename T, int E>
__device__ __forceinline__ Vals<E> from_shared(uint32_t at)
{
    if constexpr (E > 1) {
        return widen16<T>(lds16(at));
    } else if constexpr (sizeof(T) == 4) {
        float f;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f) : "r"(at));
        return Vals<1>{f};
    } else {
        uint16_t h;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(at));
        return Vals<1>{to_f32(T{h})};
    }
}

// Sum over the warp of each of the N values (a power of two), all of them at
// once: every exchange halves the values a lane still carries, so it takes N - 1 +
// 5 - log2 N exchanges instead of 5 N.  Lane l ends with the sum of value
// l >> (5 - log2 N).
template <int N>
__device__ __forceinline__ float warp_sum_many(float (&v)[N])
{
    const int lane = threadIdx.x & 31;
    int mask = 16;
#pragma unroll
    for (int n = N / 2; n > 0; n >>= 1, mask >>= 1) {
        const bool high = (lane & mask) != 0;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float give = high ? v[i] : v[i + n], keep = high ? v[i + n] : v[i];
            v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, mask);
        }
    }
    float r = v[0];
    for (; mask > 0; mask >>= 1) r += __shfl_xor_sync(0xFFFFFFFFu, r, mask);
    return r;
}

// The wait for a stage, once a look has not found it there.  What a group's threads know
// of a wait that ran out is in shared memory: a register for it would be one too many.
__device__ __forceinline__ bool has_given_up(uint32_t flag)
{
    uint32_t v;
    asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(v) : "r"(flag));
    return v != 0;
}
__device__ __forceinline__ void wait_or_give_up(uint32_t bar, uint32_t parity, uint32_t polls, uint32_t flag)
{
    if (!has_given_up(flag) && !mbar_wait(bar, parity, polls))
        asm volatile("st.volatile.shared.u32 [%0], 1;" ::"r"(flag) : "memory");
}

// Waits, with the full limit, for the last fills of a ring: fill k went into stage
// k % stages, and one is issued only when the one before it in its stage has been seen.
__device__ __forceinline__ void land(uint32_t bars, int issued, int stages)
{
    for (int k = issued > stages ? issued - stages : 0; k < issued; ++k)
        mbar_wait(bars + (k % stages) * 8, (uint32_t)(k / stages) & 1u, kPolls);
}

// Forward: rows come through a ring of bulk copies in shared memory, so that no register waits for memory and the loads of several
// groups of rows are always on their way.  A group takes R rows at a time, whose
// sums share one exchange and one barrier; that barrier also tells the group's
// first thread that everyone is done with the rows before, whose place in the ring
// it refills.
//
// Statistics in one exchange: a thread has the mean m_t of its n_t elements and
// their squares around it, Q_t.  With c the first lane's mean, a warp sums
//   D = sum n_t (m_t - c),  Q = sum (Q_t + n_t (m_t - c)^2)
// so its mean is c + D / n and its squares around that Q - D^2 / n; c is within
// sqrt(32) standard deviations of the mean, so the difference loses 5 bits at most,
// however large the mean.  Warps are joined by M2 = sum M2_w + sum n_w (mean_w - mean)^2.
//
// Bound: memory (one read, one write of the matrix).  32768 x 4096 bf16: 95 to 99 us, 5.4 to
// 5.7 TB/s, 83 to 86 % of a copy's rate; what is left is the exchange of each row's sums.
// Registers that prefetch the next row instead of the ring: 125 us; a warp per row with 16
// vectors a lane (244 registers, 8 warps an SM): 185 us.  Widths that leave lanes idle with
// four vectors a thread spill: 16384 x 8184 bf16 166 us for 82 of bytes.  Elements one by one
// (E = 1), each a shared-memory access and a store: 65536 x 1001 bf16 140 us for 40 of bytes.
//
// A copy that does not arrive in time turns the rows that the group has not written into
// NaN, statistics and gradients of the weights included (the optimizer's gradient check
// then skips the iteration).
template <typename T, int E, int kNV, int R, bool kFull, int kMaxThreads>
__global__ void __launch_bounds__(kMaxThreads, kMaxThreads <= kRowThreads ? 2 : 1) norm_forward_ring_kernel(NormArgs a, int per_row, int stages)
{
    extern __shared__ __align__(128) uint8_t s_ring[];   // [groups][stages][R][cols]
    constexpr int kSums = 2 * R;
    __shared__ __align__(16) float s_part[2][32][kSums], s_centre[2][32][R];
    __shared__ float s_count[32];
    __shared__ __align__(8) uint64_t s_full[kRingBars];
    __shared__ int s_issued[kGroupThreads / 32];         // fills of a group's stages so far
    __shared__ int s_gave_up[kGroupThreads / 32];        // a wait of the group ran out
    const Group g(per_row);
    const int cols = (int)a.cols, lane = threadIdx.x & 31;
    const RowCopies<T, E> xs(a.x, a.x_stride, a.rows, a.cols);
    const uint32_t stage_bytes = xs.pitch * R;
    const uint32_t ring = smem_addr(s_ring) + (uint32_t)(g.index * stages) * stage_bytes;
    const uint32_t bars = smem_addr(s_full) + (uint32_t)(g.index * stages) * 8;
    const int64_t step = (int64_t)gridDim.x * g.per_block * R;
    const int64_t row = ((int64_t)blockIdx.x * g.per_block + g.index) * R;
    const auto has = [&](int i) { return kFull || (g.thread + i * g.threads) * E < cols; };
    float mine_n = 0.0f;                  // elements of this thread
#pragma unroll
    for (int i = 0; i < kNV; ++i)
        if (has(i)) mine_n += E;
    const float inv_n = mine_n > 0.0f ? 1.0f / mine_n : 0.0f, warp_n = warp_sum(mine_n);
    if (lane == 0) s_count[threadIdx.x >> 5] = warp_n;
    if (threadIdx.x < (unsigned)(g.per_block * stages)) {
        mbar_init(smem_addr(s_full + threadIdx.x), 1);
        mbar_init_fence();                // before any group's first thread issues a copy
    }
    if (g.thread == 0) s_gave_up[g.index] = a.patience.of((int)blockIdx.x) == 0;
    __syncthreads();
    const float first_inv = 1.0f / s_count[g.index * g.warps];

    const auto load_rows = [&](int64_t from, int s) {
        const int n = a.rows - from < R ? (int)(a.rows - from) : R;
        const uint32_t bar = bars + s * 8, dst = ring + s * stage_bytes;
        if (E > 1) mbar_expect(bar, xs.bytes * n);
        for (int r = 0; r < n; ++r) xs.load(from + r, dst + r * xs.pitch, bar);
        if (E == 1) mbar_arrive(bar);
    };
    if (g.thread == 0) {
        int n = 0;
        for (; n < stages && row + n * step < a.rows; ++n) load_rows(row + n * step, n);
        s_issued[g.index] = n;
    }

    Vals<E> w[kNV], b[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i)
        if (has(i)) {
            w[i] = load_params<E>(a.weight, (g.thread + i * g.threads) * E, a.param_dtype, 1.0f);
            b[i] = load_params<E>(a.bias, (g.thread + i * g.threads) * E, a.param_dtype, 0.0f);
        }
    T *y = static_cast<T *>(a.y) + row * a.y_stride + g.thread * E;
    const int64_t y_step = (step - R) * a.y_stride;
    constexpr uint32_t kBytes = E * sizeof(T);
    const uint32_t mine = ring + (uint32_t)g.thread * kBytes, vector_step = (uint32_t)g.threads * kBytes;
    uint32_t phase = 0;
    int stage = 0, turn = 0;
    bool first = true;

    for (int64_t left = a.rows - row; left > 0; left -= step) {
        if (!mbar_test(bars + stage * 8, phase)) wait_or_give_up(bars + stage * 8, phase, a.patience.of((int)blockIdx.x), smem_addr(s_gave_up + g.index));
        const uint32_t at = mine + stage * stage_bytes;
        const int n = left < R ? (int)left : R;
        const auto row_at = [&](int r) { return at + r * xs.pitch + xs.shift(a.rows - left + r); };
        float sums[kSums], centre[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float m = 0.0f, q = 0.0f;
            if (r < n) {
                Vals<E> f[kNV], acc;
                acc.set(0.0f);
#pragma unroll
                for (int i = 0; i < kNV; ++i)
                    if (has(i)) {
                        f[i] = from_shared<T, E>(row_at(r) + i * vector_step);
                        acc = acc + f[i];
                    }
                m = total(acc) * inv_n;
                acc.set(0.0f);
#pragma unroll
                for (int i = 0; i < kNV; ++i)
                    if (has(i)) {
                        const Vals<E> d = f[i] + -m;
                        acc = fma(d, d, acc);
                    }
                q = total(acc);
            }
            centre[r] = __shfl_sync(0xFFFFFFFFu, m, 0);
            const float d = mine_n > 0.0f ? m - centre[r] : 0.0f;
            sums[2 * r] = d * mine_n;
            sums[2 * r + 1] = fmaf(d * mine_n, d, q);
        }
        const float one = warp_sum_many<kSums>(sums);
        float (*part)[kSums] = s_part[turn] + g.index * g.warps;
        float (*cent)[R] = s_centre[turn] + g.index * g.warps;
        const float *count = s_count + g.index * g.warps;
        turn ^= 1;
        if (lane % (32 / kSums) == 0) part[g.warp][lane / (32 / kSums)] = one;
        if (lane == 0) {
#pragma unroll
            for (int r = 0; r < R; ++r) cent[g.warp][r] = centre[r];
        }
        if (g.warps > 1) g.sync();
        else __syncwarp();
        const bool gave_up = has_given_up(smem_addr(s_gave_up + g.index));
        if (g.thread == 0 && !first && !gave_up) {      // the stage before this one is free
            const int before = stage == 0 ? stages - 1 : stage - 1;
            const int64_t ahead = (int64_t)(stages - 1) * step;
            if (left > ahead) {
                load_rows(a.rows - left + ahead, before);
                ++s_issued[g.index];
            }
        }
        first = false;
        // the warps' sums, moved to a common centre (the first warp's mean), one warp a lane
        float mean[R], m2[R], rstd[R];
        if (g.warps > 1) {
            float base[R], both[kSums];
#pragma unroll
            for (int r = 0; r < R; ++r) base[r] = fmaf(part[0][2 * r], first_inv, cent[0][r]);
            const bool in = lane < g.warps;
            const float n_w = in ? count[lane] : 0.0f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float k = in ? cent[lane][r] - base[r] : 0.0f, d = in ? part[lane][2 * r] : 0.0f;
                both[2 * r] = fmaf(n_w, k, d);
                both[2 * r + 1] = in ? fmaf(k, fmaf(n_w, k, 2.0f * d), part[lane][2 * r + 1]) : 0.0f;
            }
            const float joined = warp_sum_many<kSums>(both);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float d = __shfl_sync(0xFFFFFFFFu, joined, 2 * r * (32 / kSums));
                const float q = __shfl_sync(0xFFFFFFFFu, joined, (2 * r + 1) * (32 / kSums));
                const float shift = d * a.inv_cols;
                mean[r] = base[r] + shift;
                m2[r] = fmaf(-d, shift, q);
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float d = part[0][2 * r], shift = d * a.inv_cols;
                mean[r] = cent[0][r] + shift;
                m2[r] = fmaf(-d, shift, part[0][2 * r + 1]);
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            rstd[r] = 1.0f / sqrtf(fmaf(fmaxf(m2[r], 0.0f), a.inv_cols, a.eps));
            if (m2[r] != m2[r]) rstd[r] = kNan;
            if (gave_up) mean[r] = rstd[r] = kNan;
            if (a.mean && g.thread == r && r < n) {
                a.mean[a.rows - left + r] = mean[r];
                a.rstd[a.rows - left + r] = rstd[r];
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r < n) {
#pragma unroll
                for (int i = 0; i < kNV; ++i)
                    if (has(i)) {
                        const Vals<E> x = from_shared<T, E>(row_at(r) + i * vector_step);
                        store_vec<T, E>(y + i * g.threads * E, fma((x + -mean[r]) * rstd[r], w[i], b[i]));
                    }
                y += a.y_stride;
            }
        y += y_step;
        if (++stage == stages) {
            stage = 0;
            phase ^= 1;
        }
    }
    // the copies that were issued land before the block goes (all have, unless the wait ran out)
    if (s_gave_up[g.index] && g.thread == 0) land(bars, s_issued[g.index], stages);
    __syncthreads();
}

// Backward: the rows of x and dy come through a ring of bulk copies.  A group takes R rows at a time: their two sums each share one exchange
// and one barrier.  That barrier also tells the group's first thread that
// everyone is done with the rows before, whose place in the ring it refills.
// A thread keeps its columns' part of dweight and dbias for all its rows.
//
// Bound: memory (two reads, one write).  32768 x 2048 bf16: 78 to 80 us with the sum over
// blocks, 5.1 TB/s, 78 % of a copy's rate (this kernel alone 73 us); 32768 x 4096 bf16 190 us
// for 123 of bytes, 65536 x 1001 bf16 element by element 153 us for 60; 2047 x 768 fp16 14 us
// on the device, for the 512 partial rows of blocks with one turn each.  The work per
// row and thread that does not depend on the elements is what costs: 8 elements a
// thread 86 us, 16 elements 81 us; one row at a time 102 us, two 88 us, four 81 us.
//
// A copy that does not arrive in time turns the rows that the group has not written into
// NaN, statistics and gradients of the weights included (the optimizer's gradient check
// then skips the iteration).
template <typename T, int E, int kNV, int R, bool kFull, int kMaxThreads>
__global__ void __launch_bounds__(kMaxThreads, kMaxThreads <= kRowThreads ? 2 : 1) norm_backward_ring_kernel(NormArgs a, int per_row, int stages)
{
    extern __shared__ __align__(128) uint8_t s_ring[];   // [groups][stages][R][x, dy][cols]
    constexpr int kSums = 2 * R;          // of each row: sum(g), sum(g xhat)
    // x - mean first, or xhat = x rstd + (-mean rstd), an operation less in either pass, whose
    // constant rounds to 2^-24 of |mean| / std?  At 10^4 deviations that is 6e-4 of an fp32
    // result, and less than x itself was rounded to in 2 bytes.  32768 x 4096 fp32 278 us
    // against 255 (2048 and fewer columns the same), 32768 x 2048 bf16 82 against 80; a choice
    // by each row's mean 273 and, at 65536 x 1001 bf16, 177 against 153.
    constexpr bool kCentred = sizeof(T) == 4;
    __shared__ __align__(16) float s_part[2][32][kSums];
    __shared__ __align__(8) uint64_t s_full[kRingBars];
    __shared__ int s_issued[kGroupThreads / 32];         // fills of a group's stages so far
    __shared__ int s_gave_up[kGroupThreads / 32];        // a wait of the group ran out
    const Group g(per_row);
    const int cols = (int)a.cols;
    const RowCopies<T, E> xs(a.x, a.x_stride, a.rows, a.cols), ys(a.dy, a.dy_stride, a.rows, a.cols);
    const uint32_t stage_bytes = xs.pitch * 2 * R;
    const uint32_t ring = smem_addr(s_ring) + (uint32_t)(g.index * stages) * stage_bytes;
    const uint32_t bars = smem_addr(s_full) + (uint32_t)(g.index * stages) * 8;
    const int64_t step = (int64_t)gridDim.x * g.per_block * R;
    const int64_t row = ((int64_t)blockIdx.x * g.per_block + g.index) * R;
    const auto has = [&](int i) { return kFull || (g.thread + i * g.threads) * E < cols; };
    if (threadIdx.x < (unsigned)(g.per_block * stages)) {
        mbar_init(smem_addr(s_full + threadIdx.x), 1);
        mbar_init_fence();                // before any group's first thread issues a copy
    }
    if (g.thread == 0) s_gave_up[g.index] = a.patience.of((int)blockIdx.x) == 0;
    __syncthreads();
    grid_dependency_release();            // the sum over blocks may be set up meanwhile

    // the group's first thread: the copies of the R rows from `from`, into stage s
    const auto load_rows = [&](int64_t from, int s) {
        const int n = a.rows - from < R ? (int)(a.rows - from) : R;
        const uint32_t bar = bars + s * 8, dst = ring + s * stage_bytes;
        if (E > 1) mbar_expect(bar, xs.bytes * 2 * n);
        for (int r = 0; r < n; ++r) {
            xs.load(from + r, dst + r * 2 * xs.pitch, bar);
            ys.load(from + r, dst + (r * 2 + 1) * xs.pitch, bar);
        }
        if (E == 1) mbar_arrive(bar);
    };
    if (g.thread == 0) {
        int n = 0;
        for (; n < stages && row + n * step < a.rows; ++n) load_rows(row + n * step, n);
        s_issued[g.index] = n;
    }

    Vals<E> w[kNV], dw[kNV], db[kNV];
    float mean[R], rstd[R];
    const float *mean_at = a.mean + row, *rstd_at = a.rstd + row;
    const auto load_stats = [&](int n) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r < n) {
                mean[r] = mean_at[r];
                rstd[r] = rstd_at[r];
            }
    };
    int64_t left = a.rows - row;          // rows from here on
    if (left > 0) load_stats(left < R ? (int)left : R);
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
        if (has(i)) w[i] = load_params<E>(a.weight, (g.thread + i * g.threads) * E, a.param_dtype, 1.0f);
        dw[i].set(0.0f);
        db[i].set(0.0f);
    }
    T *dx = static_cast<T *>(a.y) + row * a.y_stride + g.thread * E;
    const int64_t dx_step = (step - R) * a.y_stride;
    constexpr uint32_t kBytes = E * sizeof(T);
    const uint32_t mine = ring + (uint32_t)g.thread * kBytes, vector_step = (uint32_t)g.threads * kBytes;
    uint32_t phase = 0;
    int stage = 0, turn = 0;
    bool first = true;

    for (; left > 0; left -= step) {
        if (!mbar_test(bars + stage * 8, phase)) wait_or_give_up(bars + stage * 8, phase, a.patience.of((int)blockIdx.x), smem_addr(s_gave_up + g.index));
        const uint32_t at = mine + stage * stage_bytes;
        const int n = left < R ? (int)left : R;
        const auto x_at = [&](int r) { return at + r * 2 * xs.pitch + xs.shift(a.rows - left + r); };
        const auto dy_at = [&](int r) { return at + (r * 2 + 1) * xs.pitch + ys.shift(a.rows - left + r); };
        float sums[kSums];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            Vals<E> ag, agx;
            ag.set(0.0f);
            agx.set(0.0f);
            if (r < n) {
                const float off = -mean[r] * rstd[r];
#pragma unroll
                for (int i = 0; i < kNV; ++i) {
                    if (!has(i)) break;
                    const Vals<E> x = from_shared<T, E>(x_at(r) + i * vector_step);
                    const Vals<E> d = from_shared<T, E>(dy_at(r) + i * vector_step);
                    const Vals<E> t = d * (kCentred ? (x + -mean[r]) * rstd[r] : fma(x, rstd[r], off));
                    ag = fma(d, w[i], ag);
                    agx = fma(t, w[i], agx);
                    dw[i] = dw[i] + t;
                    db[i] = db[i] + d;
                }
            }
            sums[2 * r] = total(ag);
            sums[2 * r + 1] = total(agx);
        }
        const int lane = threadIdx.x & 31;
        const float one = warp_sum_many<kSums>(sums);
        float (*part)[kSums] = s_part[turn] + g.index * g.warps;
        turn ^= 1;
        if (lane % (32 / kSums) == 0) part[g.warp][lane / (32 / kSums)] = one;
        if (g.warps > 1) g.sync();
        else __syncwarp();
        const bool gave_up = has_given_up(smem_addr(s_gave_up + g.index));
        if (g.thread == 0 && !first && !gave_up) {      // the stage before this one is free
            const int before = stage == 0 ? stages - 1 : stage - 1;
            const int64_t ahead = (int64_t)(stages - 1) * step;
            if (left > ahead) {
                load_rows(a.rows - left + ahead, before);
                ++s_issued[g.index];
            }
        }
        first = false;
        Vals<kSums> all;
        all.set(0.0f);
        for (int j = 0; j < g.warps; ++j) {
            Vals<kSums> p;
#pragma unroll
            for (int i = 0; i < R; ++i) p.p[i] = *reinterpret_cast<const f32x2 *>(&part[j][2 * i]);
            all = all + p;
        }
        float row_sum[kSums];
        all.get(row_sum);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r < n) {
                // dx = rstd (dy w - m_g - xhat m_gx), gathered by factors of dy w and of x - mean
                const float rs = gave_up ? kNan : rstd[r];
                const float by_x = -rs * rs * (row_sum[2 * r + 1] * a.inv_cols);
                const float rest = fmaf(kCentred ? 0.0f : -mean[r], by_x, -rs * (row_sum[2 * r] * a.inv_cols));
#pragma unroll
                for (int i = 0; i < kNV; ++i) {
                    if (!has(i)) break;
                    const Vals<E> x = from_shared<T, E>(x_at(r) + i * vector_step);
                    const Vals<E> d = from_shared<T, E>(dy_at(r) + i * vector_step);
                    store_vec<T, E>(dx + i * g.threads * E, fma(d * w[i], rs, fma(kCentred ? x + -mean[r] : x, by_x, rest)));
                }
                dx += a.y_stride;
            }
        }
        dx += dx_step;
        mean_at += step;
        rstd_at += step;
        if (left > step) load_stats(left - step < R ? (int)(left - step) : R);
        if (++stage == stages) {
            stage = 0;
            phase ^= 1;
        }
    }
    if (s_gave_up[g.index]) {
        // the copies that were issued land before the block goes and the ring is used again
        if (g.thread == 0) land(bars, s_issued[g.index], stages);
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            dw[i].set(kNan);
            db[i].set(kNan);
        }
    }
    __syncthreads();

    if (!a.partials) return;
    float *out = a.partials + (int64_t)blockIdx.x * 2 * a.cols;
    float *sums = g.per_block > 1 ? reinterpret_cast<float *>(s_ring) : out;   // the ring is done with
    for (int turn = 0; turn < g.per_block; ++turn) {
        if (turn > 0) __syncthreads();
        if (g.index != turn) continue;
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
            const int c = (g.thread + i * g.threads) * E;
            if (c >= cols) break;
            float fw[E], fb[E];
            dw[i].get(fw);
            db[i].get(fb);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float pw = turn > 0 ? sums[c + e] + fw[e] : fw[e];
                const float pb = turn > 0 ? sums[a.cols + c + e] + fb[e] : fb[e];
                float *to = turn == g.per_block - 1 ? out : sums;
                to[c + e] = pw;
                to[a.cols + c + e] = pb;
            }
        }
    }
}

// ---- rows too long for that ------------------------------------------------------
//
// Forward beyond 32 KB a row of vectors, backward beyond 16 KB (512 threads of four and two
// vectors), and rows of more than 8192 elements that are not aligned.  The rows come from L2
// again, and the backward pass updates its partial row in memory: 8192 x 5120 fp32 backward
// 273 us for 77 of bytes, 16384 x 16384 bf16 1957 us for 246.

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

constexpr int kMaxPartials = 1024;        // blocks that may leave a partial row

// ---- which kernel ----------------------------------------------------------------

// How a row is dealt out: `per_row` threads with `nv` vectors of E elements each,
// blocks of `block` threads; per_row = 0: the row does not fit, use the loop.
struct Plan { int per_row, nv, block; };

inline Plan make_plan(int64_t vectors, int nv)
{
    Plan p;
    p.per_row = (int)(((vectors + nv - 1) / nv + 31) / 32 * 32);
    p.nv = nv;
    p.block = p.per_row >= kGroupThreads ? p.per_row : kGroupThreads / p.per_row * p.per_row;
    return p;
}

constexpr int kMaxShared = 220 * 1024;    // dynamic shared memory of a block, at most

// Resident blocks per SM of a kernel, asked for again only when its block or its shared
// memory changes.  The grid follows from the answer, and with it the order in which the
// backward pass sums dweight and dbias: the key is exact, so that a width's sums do not
// depend on the widths called before it.
template <typename K>
so_status resident(K kernel, int block, size_t smem, std::atomic<uint64_t> (&cache)[kMaxDevices], int *out)
{
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return SO_ERR_CUDA;
    if (dev < 0 || dev >= kMaxDevices) return SO_ERR_UNSUPPORTED;
    // one word: the block size and shared memory it was asked for, and the answer
    const uint64_t tag = (uint64_t)smem << 24 | (uint64_t)block << 8;
    uint64_t v = cache[dev].load(std::memory_order_relaxed);
    if ((v & ~uint64_t(255)) != tag) {
        int n = 0;
        if (smem > 40 * 1024 &&
            cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxShared) != cudaSuccess)
            return SO_ERR_CUDA;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, block, smem) != cudaSuccess || n < 1)
            return SO_ERR_CUDA;
        v = tag | (uint64_t)(n < 255 ? n : 255);
        cache[dev].store(v, std::memory_order_relaxed);
    }
    *out = (int)(v & 255);
    return SO_OK;
}

// Stages of a ring: up to four, in the shared memory that four blocks share an SM with
// (two blocks' if only two stages of long rows fit there).
inline int ring_stages(size_t stage_bytes, int groups)
{
    int stages = (int)(kRingBytes / stage_bytes);
    if (stages > 4) stages = 4;
    if (stages < 2) stages = 2;
    return stages < kRingBars / groups ? stages : kRingBars / groups;
}

// Bytes of a row in the ring.
template <typename T, int E>
size_t ring_pitch(int64_t cols)
{
    const size_t bytes = (size_t)cols * sizeof(T);
    return E == 1 ? (bytes + 30 + 15) / 16 * 16 : bytes;
}

template <typename T, int E, int kNV, int R, bool kFull, int kMaxThreads>
so_status launch_forward_ring(const NormArgs &a, const Plan &p, int sms, cudaStream_t st)
{
    const int groups = p.block / p.per_row;
    const size_t stage = ring_pitch<T, E>(a.cols) * R * groups;
    const int stages = ring_stages(stage, groups);
    static std::atomic<uint64_t> cache[kMaxDevices];
    int per_sm = 0;
    const auto kernel = norm_forward_ring_kernel<T, E, kNV, R, kFull, kMaxThreads>;
    const so_status s = resident(kernel, p.block, stage * stages, cache, &per_sm);
    if (s != SO_OK) return s;
    const int64_t want = (a.rows + groups * R - 1) / (groups * R), most = (int64_t)per_sm * sms;
    return launch(kernel, (unsigned)(want < most ? want : most), p.block, stage * stages, st, false, a, p.per_row, stages);
}

template <typename T, int E, int kNV, int R, bool kFull, int kMaxThreads>
so_status launch_backward_ring(const NormArgs &a, const Plan &p, int sms, cudaStream_t st, int *blocks)
{
    const int groups = p.block / p.per_row;
    const size_t stage = ring_pitch<T, E>(a.cols) * 2 * R * groups;
    const int stages = ring_stages(stage, groups);
    static std::atomic<uint64_t> cache[kMaxDevices];
    int per_sm = 0;
    const auto kernel = norm_backward_ring_kernel<T, E, kNV, R, kFull, kMaxThreads>;
    const so_status s = resident(kernel, p.block, stage * stages, cache, &per_sm);
    if (s != SO_OK) return s;
    const int64_t want = (a.rows + groups * R - 1) / (groups * R);
    int64_t most = (int64_t)per_sm * sms;
    if (most > kMaxPartials) most = kMaxPartials;
    *blocks = (int)(want < most ? want : most);
    return launch(kernel, (unsigned)*blocks, p.block, stage * stages, st, false, a, p.per_row, stages);
}

// Vectors per thread for the ring kernels: the choice that leaves the fewest lanes
// idle, and the largest of equals (fewer warps share a row, less goes into the
// exchange).
inline Plan plan_ring(int64_t vectors, int most_nv)
{
    Plan best = {0, 0, 0};
    int64_t waste = INT64_MAX;
    for (int nv = most_nv; nv > 0; --nv) {
        const Plan p = make_plan(vectors, nv);
        const int64_t idle = (int64_t)p.per_row * nv - vectors;
        if (p.per_row <= kLongThreads && idle < waste) best = p, waste = idle;
    }
    return best;
}

template <typename T, int E, int kNV, int R>
so_status forward_ring(const NormArgs &a, const Plan &p, int sms, cudaStream_t st)
{
    const bool full = E > 1 && (int64_t)p.per_row * kNV * E == a.cols;
    if (p.block <= kRowThreads)
        return full ? launch_forward_ring<T, E, kNV, R, E != 1, kRowThreads>(a, p, sms, st)
                    : launch_forward_ring<T, E, kNV, R, false, kRowThreads>(a, p, sms, st);
    return launch_forward_ring<T, E, kNV, R, false, kLongThreads>(a, p, sms, st);
}

template <typename T>
so_status forward(const NormArgs &a, bool vec, int sms, cudaStream_t st)
{
    constexpr int E = Vec<T>::kElems;
    const bool fits = a.cols * (int64_t)sizeof(T) * 2 + 128 <= kMaxShared;   // two stages of one row
    if (vec && fits) {
        const Plan p = plan_ring(a.cols / E, 4);
        if (p.nv == 4) return forward_ring<T, E, 4, 1>(a, p, sms, st);
        if (p.nv == 3) return forward_ring<T, E, 3, 1>(a, p, sms, st);
        if (p.nv == 2) return forward_ring<T, E, 2, 2>(a, p, sms, st);
        if (p.nv == 1) return forward_ring<T, E, 1, 4>(a, p, sms, st);
    } else if (fits) {
        const Plan p = make_plan(a.cols, a.cols <= 8 * kLongThreads ? 8 : 16);
        if (p.nv == 8) return forward_ring<T, 1, 8, 2>(a, p, sms, st);
        if (p.per_row <= kLongThreads) return forward_ring<T, 1, 16, 1>(a, p, sms, st);
    }
    const unsigned grid = (unsigned)(a.rows < 4 * sms ? a.rows : 4 * sms);
    return launch(norm_forward_loop_kernel<T>, grid, kLoopThreads, 0, st, false, a);
}

template <typename T, int E, int kNV, int R>
so_status backward_ring(const NormArgs &a, const Plan &p, int sms, cudaStream_t st, int *blocks)
{
    const bool full = E > 1 && (int64_t)p.per_row * kNV * E == a.cols;
    if (p.block <= kRowThreads)
        return full ? launch_backward_ring<T, E, kNV, R, E != 1, kRowThreads>(a, p, sms, st, blocks)
                    : launch_backward_ring<T, E, kNV, R, false, kRowThreads>(a, p, sms, st, blocks);
    return launch_backward_ring<T, E, kNV, R, false, kLongThreads>(a, p, sms, st, blocks);
}

template <typename T>
so_status backward(const NormArgs &a, bool vec, int sms, cudaStream_t st, int *blocks)
{
    constexpr int E = Vec<T>::kElems;
    const int64_t row = a.cols * (int64_t)sizeof(T) + (vec ? 0 : 48);
    // rows at a time: four, or two where that leaves less than three stages in shared memory
    // (more than 9 KB a row; the plans below hold at most 16 KB, or take one row themselves)
    const int r = row * 24 <= kMaxShared ? 4 : 2;
    if (vec && row * 4 <= kMaxShared) {
        const Plan p = plan_ring(a.cols / E, 2);
        if (p.nv == 2) {
            if (r == 4) return backward_ring<T, E, 2, 4>(a, p, sms, st, blocks);
            return backward_ring<T, E, 2, 2>(a, p, sms, st, blocks);
        }
        if (p.nv == 1) return backward_ring<T, E, 1, 4>(a, p, sms, st, blocks);   // 8 KB a row at most
    } else if (row * 4 <= kMaxShared) {
        const Plan p = make_plan(a.cols, a.cols <= 8 * kLongThreads ? 8 : 16);
        if (p.nv == 8) {
            if (r == 4) return backward_ring<T, 1, 8, 4>(a, p, sms, st, blocks);
            return backward_ring<T, 1, 8, 2>(a, p, sms, st, blocks);
        }
        if (p.per_row <= kLongThreads) return backward_ring<T, 1, 16, 1>(a, p, sms, st, blocks);
    }
    const int64_t most = 2 * sms < kMaxPartials ? 2 * sms : kMaxPartials;
    *blocks = (int)(a.rows < most ? a.rows : most);
    return launch(norm_backward_loop_kernel<T>, (unsigned)*blocks, kLoopThreads, 0, st, false, a);
}

}  // namespace

extern "C" {

so_status so_debug_set_operator_polls(int64_t polls, int32_t unit)
{
    if (polls < 0 || polls > (int64_t)kPolls || unit < -1) return SO_ERR_INVALID_ARG;
    g_patience.store((uint64_t)polls << 32 | (uint32_t)unit, std::memory_order_relaxed);
    return SO_OK;
}

so_status so_layer_norm_forward(const void *x, int64_t x_stride, const void *weight,
                                const void *bias, void *y, int64_t y_stride, float *mean,
                                float *rstd, int64_t rows, int64_t cols, int32_t dtype,
                                int32_t param_dtype, double eps, void *stream)
{
    if (!valid_dtype(dtype) || (param_dtype != dtype && param_dtype != SO_DTYPE_FP32)) return SO_ERR_INVALID_ARG;
    if (rows < 0 || cols < 1 || cols > INT32_MAX || !(eps >= 0.0) || !std::isfinite((float)eps)) return SO_ERR_INVALID_ARG;
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
    a.patience = patience();
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
    a.patience = patience();
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
