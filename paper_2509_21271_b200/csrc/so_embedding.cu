// Token embedding: lookup with scaling, and the table's gradient by sorted
// tokens.
//
//   forward   out[t] = scale * table[ids[t]]
//   backward  dtable[v] = scale * sum of dout[t] over t with ids[t] = v
//
// The backward pass first puts the tokens in the order of their ids (stably, so
// each row's sum runs over ascending t), then sums runs of equal ids.
#include "so_ops.cuh"

using namespace so_ops;

namespace {

constexpr int64_t kMaxTokens = int64_t(1) << 30;   // tokens, and table rows, in one call

struct LookupArgs {
    const void *ids, *table;
    void *out;
    int32_t *bad_id;
    int64_t n, vocab, cols, table_stride, out_stride;
    int32_t ids_dtype;
    float scale;
};

constexpr int kLookupThreads = 256;

template <typename T, bool kVec>
__global__ void __launch_bounds__(kLookupThreads) embedding_forward_kernel(LookupArgs a)
{
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * (kLookupThreads / 32);
    for (int64_t t = (int64_t)blockIdx.x * (kLookupThreads / 32) + (threadIdx.x >> 5); t < a.n; t += warps) {
        const int64_t id = load_id(a.ids, t, a.ids_dtype);
        T *out = static_cast<T *>(a.out) + t * a.out_stride;
        const bool ok = id >= 0 && id < a.vocab;
        if (!ok && a.bad_id && lane == 0) *a.bad_id = 1;
        const T *row = static_cast<const T *>(a.table) + (ok ? id : 0) * a.table_stride;
        if constexpr (kVec) {
            constexpr int E = Vec<T>::kElems;
            for (int64_t v = lane; v < a.cols / E; v += 32) {
                float f[E];
                uint4 raw = make_uint4(0, 0, 0, 0);
                if (ok) raw = reinterpret_cast<const uint4 *>(row)[v];
                unpack<T>(raw, f);
#pragma unroll
                for (int i = 0; i < E; ++i) f[i] *= a.scale;
                reinterpret_cast<uint4 *>(out)[v] = ok ? pack<T>(f) : raw;
            }
        } else {
            for (int64_t c = lane; c < a.cols; c += 32)
                out[c] = ok ? from_f32<T>(to_f32(row[c]) * a.scale) : from_f32<T>(0.0f);
        }
    }
}

// ---- tokens in the order of their ids ------------------------------------------
//
// A stable counting sort in one launch with no exchange between blocks.  Block b
// owns the ids [b kRange, (b + 1) kRange) and reads every token: it counts the
// tokens of its ids, and those of smaller ids, which gives the place where its
// part of the sorted order begins.  Each warp takes a contiguous run of
// tokens and keeps counters of its own, so that ranks follow from prefix sums
// and do not depend on the order of the (integer, shared-memory) additions.

constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kRange = 1024;              // ids a block owns, at most one per thread

struct SortArgs {
    const void *ids;
    int32_t *order;                       // [n] token positions by (id, position)
    int32_t *start;                       // [vocab + 1] where each id's tokens begin
    int32_t n, vocab, range;
    int64_t padding_id;
    int32_t ids_dtype;
};

__device__ __forceinline__ int32_t usable_id(const SortArgs &a, int32_t t)
{
    const int64_t id = load_id(a.ids, t, a.ids_dtype);
    return (id >= 0 && id < a.vocab && id != a.padding_id) ? (int32_t)id : -1;
}

__global__ void __launch_bounds__(kSortThreads) embedding_sort_kernel(SortArgs a)
{
    extern __shared__ int32_t s_hist[];   // [kSortWarps][range]
    __shared__ int32_t s_below[kSortWarps], s_scan[kSortWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int32_t lo = (int32_t)blockIdx.x * a.range;
    const int32_t hi = a.vocab - lo < a.range ? a.vocab : lo + a.range;
    for (int i = threadIdx.x; i < kSortWarps * a.range; i += kSortThreads) s_hist[i] = 0;
    __syncthreads();

    const int32_t per_warp = (int32_t)(((int64_t)a.n + kSortThreads - 1) / kSortThreads) * 32;
    const int64_t first = (int64_t)warp * per_warp;
    const int32_t t0 = first < a.n ? (int32_t)first : a.n;
    const int32_t t1 = a.n - t0 < per_warp ? a.n : t0 + per_warp;
    int32_t *hist = s_hist + warp * a.range;
    int32_t below = 0;
    for (int32_t t = t0 + lane; t < t1; t += 32) {
        const int32_t id = usable_id(a, t);
        if (id >= 0 && id < lo) ++below;
        else if (id >= lo && id < hi) atomicAdd(&hist[id - lo], 1);
    }
    for (int o = 16; o > 0; o >>= 1) below += __shfl_xor_sync(0xFFFFFFFFu, below, o);
    if (lane == 0) s_below[warp] = below;
    __syncthreads();

    // thread i: the tokens of id lo + i, exclusive prefix over the block's ids
    const bool mine = (int32_t)threadIdx.x < hi - lo;
    int32_t count = 0;
    if (mine)
        for (int w = 0; w < kSortWarps; ++w) count += s_hist[w * a.range + threadIdx.x];
    int32_t incl = count;
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += up;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    int32_t base = 0;
    for (int w = 0; w < kSortWarps; ++w) base += s_below[w] + (w < warp ? s_scan[w] : 0);
    int32_t at = base + incl - count;
    if (mine) {
        a.start[lo + threadIdx.x] = at;
        if (lo + (int32_t)threadIdx.x == a.vocab - 1) a.start[a.vocab] = at + count;
        for (int w = 0; w < kSortWarps; ++w) {
            const int32_t c = s_hist[w * a.range + threadIdx.x];
            s_hist[w * a.range + threadIdx.x] = at;
            at += c;
        }
    }
    __syncthreads();

    for (int32_t t = t0; t < t1; t += 32) {
        const int32_t id = t + lane < t1 ? usable_id(a, t + lane) : -1;
        const bool in = id >= lo && id < hi;
        const unsigned active = __ballot_sync(0xFFFFFFFFu, in);
        if (in) {
            const unsigned same = __match_any_sync(active, id);
            const int rank = __popc(same & ((1u << lane) - 1u));
            const int32_t pos = hist[id - lo];
            __syncwarp(active);
            if (rank == 0) hist[id - lo] = pos + __popc(same);
            a.order[pos + rank] = t + lane;
        }
        __syncwarp();
    }
}

struct SumArgs {
    const void *dout;
    const int32_t *order, *start;
    void *dtable;
    int64_t vocab, cols, dout_stride, dtable_stride;
    int32_t grad_dtype, accumulate;
    float scale;
};

// One warp per table row.
template <typename T>
__global__ void __launch_bounds__(kLookupThreads) embedding_sum_kernel(SumArgs a)
{
    grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * (kLookupThreads / 32);
    for (int64_t v = (int64_t)blockIdx.x * (kLookupThreads / 32) + (threadIdx.x >> 5); v < a.vocab; v += warps) {
        const int32_t s0 = a.start[v], s1 = a.start[v + 1];
        if (s0 == s1 && a.accumulate) continue;
        for (int64_t c = lane; c < a.cols; c += 32) {
            float sum = 0.0f;
            for (int32_t i = s0; i < s1; ++i)
                sum += to_f32(static_cast<const T *>(a.dout)[(int64_t)a.order[i] * a.dout_stride + c]);
            sum *= a.scale;
            const int64_t at = v * a.dtable_stride + c;
            if (a.accumulate) sum += load_any(a.dtable, at, a.grad_dtype);
            store_any(a.dtable, at, a.grad_dtype, sum);
        }
    }
}

// scratch: order [n], then start [vocab + 1], each rounded up to 16 bytes
uint64_t round16(uint64_t b) { return (b + 15) & ~uint64_t(15); }

so_status sort_tokens(const SortArgs &a, cudaStream_t st)
{
    static std::atomic<bool> ready[kMaxDevices];
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return SO_ERR_CUDA;
    if (dev < 0 || dev >= kMaxDevices) return SO_ERR_UNSUPPORTED;
    if (!ready[dev].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(embedding_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 kSortWarps * kRange * (int)sizeof(int32_t)) != cudaSuccess)
            return SO_ERR_CUDA;
        ready[dev].store(true, std::memory_order_release);
    }
    const unsigned grid = (unsigned)((a.vocab + a.range - 1) / a.range);
    return launch(embedding_sort_kernel, grid, kSortThreads, (size_t)kSortWarps * a.range * sizeof(int32_t), st, false, a);
}

}  // namespace

extern "C" {

so_status so_embedding_forward(const void *ids, int32_t ids_dtype, int64_t n, const void *table,
                               int64_t table_stride, int64_t vocab, int64_t cols, int32_t dtype,
                               double scale, void *out, int64_t out_stride, int32_t *bad_id,
                               void *stream)
{
    if (!valid_ids(ids_dtype) || !valid_dtype(dtype) || !std::isfinite(scale)) return SO_ERR_INVALID_ARG;
    if (n < 0 || n > kMaxTokens || vocab < 1 || vocab > kMaxTokens || cols < 1 || cols > INT32_MAX)
        return SO_ERR_INVALID_ARG;
    const int es = elem_size(dtype);
    if (!aligned(bad_id, 4)) return SO_ERR_INVALID_ARG;
    if (n == 0) return SO_OK;
    if (!ids || !table || !out) return SO_ERR_INVALID_ARG;
    if (!aligned(ids, ids_dtype == SO_IDS_INT64 ? 8 : 4) || !aligned(table, es) || !aligned(out, es))
        return SO_ERR_INVALID_ARG;
    if (!valid_in_stride(vocab, table_stride, cols) || !valid_out_stride(n, out_stride, cols)) return SO_ERR_INVALID_ARG;
    if (!valid_extent(vocab, table_stride) || !valid_extent(n, out_stride)) return SO_ERR_INVALID_ARG;

    LookupArgs a = {};
    a.ids = ids; a.table = table; a.out = out; a.bad_id = bad_id; a.n = n; a.vocab = vocab; a.cols = cols;
    a.table_stride = table_stride; a.out_stride = out_stride; a.ids_dtype = ids_dtype; a.scale = (float)scale;
    int sms = 0;
    const so_status s = device_sms(&sms);
    if (s != SO_OK) return s;
    const int64_t want = (n + kLookupThreads / 32 - 1) / (kLookupThreads / 32);
    const unsigned grid = (unsigned)(want < 8 * sms ? want : 8 * sms);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool vec = aligned(table, 16) && aligned(out, 16) && (table_stride * es) % 16 == 0 &&
                     (out_stride * es) % 16 == 0 && (cols * es) % 16 == 0;
    if (dtype == SO_DTYPE_BF16)
        return launch(vec ? embedding_forward_kernel<bf16_t, true> : embedding_forward_kernel<bf16_t, false>, grid,
                      kLookupThreads, 0, st, false, a);
    if (dtype == SO_DTYPE_FP16)
        return launch(vec ? embedding_forward_kernel<f16_t, true> : embedding_forward_kernel<f16_t, false>, grid,
                      kLookupThreads, 0, st, false, a);
    return launch(vec ? embedding_forward_kernel<float, true> : embedding_forward_kernel<float, false>, grid,
                  kLookupThreads, 0, st, false, a);
}

so_status so_embedding_backward_scratch(int64_t n, int64_t vocab, int64_t cols, uint64_t *bytes)
{
    if (!bytes || n < 0 || n > kMaxTokens || vocab < 1 || vocab > kMaxTokens || cols < 1 || cols > INT32_MAX)
        return SO_ERR_INVALID_ARG;
    *bytes = round16((uint64_t)n * 4) + round16(((uint64_t)vocab + 1) * 4);
    return SO_OK;
}

so_status so_embedding_backward(const void *ids, int32_t ids_dtype, int64_t n, const void *dout,
                                int64_t dout_stride, int64_t vocab, int64_t cols, int32_t dtype,
                                double scale, int64_t padding_id, void *dtable,
                                int64_t dtable_stride, int32_t grad_dtype, int32_t accumulate,
                                void *scratch, uint64_t scratch_bytes, void *stream)
{
    uint64_t need = 0;
    if (!valid_ids(ids_dtype) || !valid_dtype(dtype) || !valid_dtype(grad_dtype) || !std::isfinite(scale) ||
        (accumulate != 0 && accumulate != 1))
        return SO_ERR_INVALID_ARG;
    if (so_embedding_backward_scratch(n, vocab, cols, &need) != SO_OK) return SO_ERR_INVALID_ARG;
    const int es = elem_size(dtype), gs = elem_size(grad_dtype);
    if (!dtable || !aligned(dtable, gs) || !valid_out_stride(vocab, dtable_stride, cols) || !valid_extent(vocab, dtable_stride))
        return SO_ERR_INVALID_ARG;
    if (!scratch || !aligned(scratch, 16) || scratch_bytes < need) return SO_ERR_INVALID_ARG;
    if (n > 0) {
        if (!ids || !dout || !aligned(ids, ids_dtype == SO_IDS_INT64 ? 8 : 4) || !aligned(dout, es))
            return SO_ERR_INVALID_ARG;
        if (!valid_in_stride(n, dout_stride, cols) || !valid_extent(n, dout_stride)) return SO_ERR_INVALID_ARG;
    }
    if (n == 0 && accumulate) return SO_OK;

    int sms = 0;
    so_status s = device_sms(&sms);
    if (s != SO_OK) return s;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    SortArgs k = {};
    k.ids = ids; k.order = static_cast<int32_t *>(scratch);
    k.start = reinterpret_cast<int32_t *>(static_cast<char *>(scratch) + round16((uint64_t)n * 4));
    k.n = (int32_t)n; k.vocab = (int32_t)vocab; k.padding_id = padding_id; k.ids_dtype = ids_dtype;
    k.range = (int32_t)((vocab + sms - 1) / sms);
    if (k.range > kRange) k.range = kRange;
    s = sort_tokens(k, st);
    if (s != SO_OK) return s;

    SumArgs a = {};
    a.dout = dout; a.order = k.order; a.start = k.start; a.dtable = dtable; a.vocab = vocab; a.cols = cols;
    a.dout_stride = dout_stride; a.dtable_stride = dtable_stride; a.grad_dtype = grad_dtype;
    a.accumulate = accumulate; a.scale = (float)scale;
    const int64_t want = (vocab + kLookupThreads / 32 - 1) / (kLookupThreads / 32);
    const unsigned grid = (unsigned)(want < 8 * sms ? want : 8 * sms);
    if (dtype == SO_DTYPE_BF16) return launch(embedding_sum_kernel<bf16_t>, grid, kLookupThreads, 0, st, true, a);
    if (dtype == SO_DTYPE_FP16) return launch(embedding_sum_kernel<f16_t>, grid, kLookupThreads, 0, st, true, a);
    return launch(embedding_sum_kernel<float>, grid, kLookupThreads, 0, st, true, a);
}

}  // extern "C"
