// Shared by the norms: rows of a matrix that groups of threads hold in registers, and the
// ring of bulk copies that they come through.
#pragma once

#include "so_ops.cuh"

namespace so_ops {

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

}  // namespace so_ops
