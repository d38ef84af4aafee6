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

constexpr int kLookupThreads = 256, kLookupBatch = 8;

// A warp per token.  Bound: memory (the rows written, and each distinct row read once:
// L2 keeps the rows of frequent tokens, but for an eighth that is read again).  32767 x 4096
// fp16 from 128256 rows: 68 us, of which the bytes take 56 us at a copy's rate; one load in
// flight per lane: 79 us.  Rows that are not aligned, element by element: 32768 x 1001 bf16
// 39 us for 17 of bytes.
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
        // loads of a batch before its stores: several are in flight
        if constexpr (kVec) {
            constexpr int E = Vec<T>::kElems;
            const int vectors = (int)(a.cols / E);
            for (int v0 = lane; v0 < vectors; v0 += 32 * kLookupBatch) {
                uint4 raw[kLookupBatch];
#pragma unroll
                for (int u = 0; u < kLookupBatch; ++u) {
                    raw[u] = make_uint4(0, 0, 0, 0);
                    if (ok && v0 + 32 * u < vectors) raw[u] = __ldg(reinterpret_cast<const uint4 *>(row) + v0 + 32 * u);
                }
#pragma unroll
                for (int u = 0; u < kLookupBatch; ++u)
                    if (v0 + 32 * u < vectors) {
                        // streamed out: the table's rows keep their place in L2
                        __stcs(reinterpret_cast<uint4 *>(out) + v0 + 32 * u,
                               ok && a.scale != 1.0f ? narrow16<T>(widen16<T>(raw[u]) * a.scale) : raw[u]);
                    }
            }
        } else {
            const uint32_t cols = (uint32_t)a.cols;   // up to 2^31 - 1: the last step passes 2^31
            for (uint32_t c0 = lane; c0 < cols; c0 += 32 * kLookupBatch) {
                T raw[kLookupBatch];
#pragma unroll
                for (int u = 0; u < kLookupBatch; ++u)
                    raw[u] = ok && c0 + 32 * u < cols ? row[c0 + 32 * u] : from_f32<T>(0.0f);
#pragma unroll
                for (int u = 0; u < kLookupBatch; ++u)
                    if (c0 + 32 * u < cols) out[c0 + 32 * u] = from_f32<T>(to_f32(raw[u]) * (ok ? a.scale : 1.0f));
            }
        }
    }
}

// ---- tokens in the order of their ids ------------------------------------------
//
// A stable counting sort in one launch with no exchange between blocks.  Block b
// owns the ids [b range, (b + 1) range) and reads every token: it counts the
// tokens of its ids, and those of smaller ids, which gives the place where its
// part of the sorted order begins.  Each warp takes a contiguous run of
// tokens and keeps counters of its own, so that ranks follow from prefix sums
// and do not depend on the order of the (integer, shared-memory) additions.
//
// A token goes out with all that the sum needs to know of its run, so that a block of
// the sum has one load to wait for before it reads rows.  Which ids occur at all goes
// out as bits: the rows of the others are zeroed by further blocks of the sum's launch.

// Bound: the instructions of looking at every token in every block: 8 us for 8192 tokens,
// 17 us for 32768, 26 us for 65536 (ids of 64 bits).  Reading the tokens a second time
// for the placing, instead of keeping the block's own: 24 us for 32768.

constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kRange = 1024;              // ids a block owns, at most one per thread
constexpr int kUnroll = 4;                // token loads in flight per lane
constexpr int kKeep = 256;                // tokens of its ids that a warp keeps from the count for the placing

// Runs of equal ids are summed by whoever owns the stretch of `chunk` sorted positions
// (16, 32 or 64) in which they begin; a run longer than two stretches is cut at the
// boundaries of the stretches instead, and the pieces are joined.
constexpr int kMinChunk = 16, kMaxChunk = 64;

// A token in sorted order: its position, its id, and where the tokens of that id are.
struct __align__(16) Sorted { int32_t token, id, start, count; };

struct SortArgs {
    const void *ids;
    Sorted *sorted;                       // [n] by (id, position)
    int32_t *total;                       // tokens that take part
    uint32_t *present;                    // bit per id: it has tokens
    uint32_t *arrived;                    // [n / (2 chunk) + 1][tiles] pieces of a long run summed so far
    int64_t padding_id;
    int32_t n, vocab, range, tiles, chunk, ids_dtype;
};

__device__ __forceinline__ int32_t usable_id(const SortArgs &a, int32_t t)
{
    const int64_t id = load_id(a.ids, t, a.ids_dtype);
    return (id >= 0 && id < a.vocab && id != a.padding_id) ? (int32_t)id : -1;
}

__global__ void __launch_bounds__(kSortThreads) embedding_sort_kernel(SortArgs a)
{
    extern __shared__ int32_t s_hist[];   // [kSortWarps][range], then [kSortWarps][kKeep] kept tokens, and ids
    __shared__ int32_t s_below[kSortWarps], s_scan[kSortWarps], s_first[kRange], s_count[kRange];
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
    int32_t *kept_token = s_hist + kSortWarps * a.range + warp * kKeep, *kept_id = kept_token + kSortWarps * kKeep;
    const uint32_t lower_lanes = (1u << lane) - 1u, width = (uint32_t)(hi - lo);
    int32_t below = 0, kept = 0;
    for (int32_t t = t0; t < t1; t += 32 * kUnroll) {
        int32_t id[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) id[u] = t + 32 * u + lane < t1 ? usable_id(a, t + 32 * u + lane) : -1;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            below += (uint32_t)id[u] < (uint32_t)lo;
            const bool in = (uint32_t)(id[u] - lo) < width && id[u] >= 0;
            const uint32_t found = __ballot_sync(0xFFFFFFFFu, in);
            if (found == 0) continue;
            const int at = kept + __popc(found & lower_lanes);
            if (in) {
                atomicAdd(&hist[id[u] - lo], 1);
                if (at < kKeep) {
                    kept_token[at] = t + 32 * u + lane;
                    kept_id[at] = id[u];
                }
            }
            kept += __popc(found);
        }
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
    // ranges are multiples of 32: a warp's ids are one word of the bits
    const uint32_t bits = __ballot_sync(0xFFFFFFFFu, mine && count > 0);
    if (lane == 0 && lo + warp * 32 < hi) a.present[(lo >> 5) + warp] = bits;
    __syncthreads();
    int32_t base = 0;
    for (int w = 0; w < kSortWarps; ++w) base += s_below[w] + (w < warp ? s_scan[w] : 0);
    int32_t at = base + incl - count;
    if (mine) {
        s_first[threadIdx.x] = at;
        s_count[threadIdx.x] = count;
        if (lo + (int32_t)threadIdx.x == a.vocab - 1) *a.total = at + count;
        if (count > 2 * a.chunk)          // two long runs never begin in the same 2 chunk positions
            for (int i = 0; i < a.tiles; ++i) a.arrived[(int64_t)(at / (2 * a.chunk)) * a.tiles + i] = 0;
        for (int w = 0; w < kSortWarps; ++w) {
            const int32_t c = s_hist[w * a.range + threadIdx.x];
            s_hist[w * a.range + threadIdx.x] = at;
            at += c;
        }
    }
    __syncthreads();

    // 32 tokens in order: those of one id follow each other
    const auto place = [&](int32_t token, int32_t id, bool in) {
        const unsigned active = __ballot_sync(0xFFFFFFFFu, in);
        if (in) {
            const unsigned same = __match_any_sync(active, id);
            const int rank = __popc(same & lower_lanes);
            const int32_t pos = hist[id - lo];
            __syncwarp(active);
            if (rank == 0) hist[id - lo] = pos + __popc(same);
            a.sorted[pos + rank] = Sorted{token, id, s_first[id - lo], s_count[id - lo]};
        }
        __syncwarp();
    };
    if (kept <= kKeep) {
        for (int32_t i = 0; i < kept; i += 32) {
            const bool in = i + lane < kept;
            place(in ? kept_token[i + lane] : 0, in ? kept_id[i + lane] : lo, in);
        }
        return;
    }
    for (int32_t t = t0; t < t1; t += 32 * kUnroll) {
        int32_t id[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) id[u] = t + 32 * u + lane < t1 ? usable_id(a, t + 32 * u + lane) : -1;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) place(t + 32 * u + lane, id[u], id[u] >= lo && id[u] < hi);
    }
}

// ---- sums over runs of equal ids ------------------------------------------------
//
// A block takes one stretch of sorted positions and one tile of columns
// (one vector per thread).  It sums the runs that begin in the stretch, in order,
// kBatch rows in flight; of a long run it sums the piece inside the stretch into
// fp32 scratch, and the last block to finish a piece of that run adds the
// pieces in their order (which block that is does not show in the result).

// Bound: memory where the table or the batch is large.  With the sort, 32768 x 2048 bf16
// into 128256 fp32 rows: 203 us for 181 us of bytes at a copy's rate; 8192 x 768 into
// 50257 bf16 rows: 25 us for 14 us of bytes (the sort is 8 us of it); unaligned rows, four
// columns a thread: 32768 x 1001 into 50257 bf16 rows 106 us for 25 of bytes.  A warp per
// table row, runs summed one after the other: 17.0 ms and 1.74 ms (the most frequent
// token has 6 % of them); zero rows written by the sort's blocks: 232 and 35 us.

constexpr int kSumThreads = 256, kBatch = 8;
constexpr int kStrided = 4;               // columns of a thread where rows are not aligned
constexpr int kZeroRows = 64;             // ids that a block of the zeroing looks at

struct SumArgs {
    const void *dout;
    const Sorted *sorted;
    const int32_t *total;
    const uint32_t *present;
    uint32_t *arrived;
    float *pieces;                        // [chunks][2][cols]: of a run that began before, of one that begins here
    void *dtable;
    int64_t vocab, cols, dout_stride, dtable_stride;
    int32_t tiles, sum_blocks, chunk, grad_dtype, accumulate;
    bool wide;                            // 16-byte stores fit the rows
    float scale;
};

// The rows of ids [64 block, ...) that have no token become zero, a warp at a time.
__device__ __forceinline__ void zero_rows(const SumArgs &a, int64_t block)
{
    const int lane = threadIdx.x & 31, size = a.grad_dtype == SO_DTYPE_FP32 ? 4 : 2;
    const int64_t row_bytes = a.cols * size;
    for (int i = threadIdx.x >> 5; i < kZeroRows; i += blockDim.x >> 5) {
        const int64_t v = block * kZeroRows + i;
        if (v >= a.vocab) return;
        if ((a.present[v >> 5] >> (v & 31)) & 1u) continue;
        char *row = static_cast<char *>(a.dtable) + v * a.dtable_stride * size;
        if (a.wide) {
            for (int64_t j = lane; j < row_bytes / 16; j += 32) __stcs(reinterpret_cast<uint4 *>(row) + j, make_uint4(0, 0, 0, 0));
        } else if (size == 4) {
            for (int64_t j = lane; j < a.cols; j += 32) reinterpret_cast<uint32_t *>(row)[j] = 0;
        } else {
            for (int64_t j = lane; j < a.cols; j += 32) reinterpret_cast<uint16_t *>(row)[j] = 0;
        }
    }
}

// A thread's E columns: a vector of them, or (kVec false) one in every blockDim.x, for rows
// that are not aligned.
template <int E, bool kVec>
struct Columns {
    int64_t first;
    int32_t step, count;                  // between them, and how many there are
    __device__ Columns(int tile, int64_t cols)
    {
        first = (int64_t)tile * blockDim.x * E + (int64_t)threadIdx.x * (kVec ? E : 1);
        step = kVec ? 1 : (int)blockDim.x;
        const int64_t left = cols - first;
        count = left <= 0 ? 0 : kVec ? E : (int)((left + step - 1) / step < E ? (left + step - 1) / step : E);
    }
};

template <int E, bool kVec>
__device__ __forceinline__ void write_row(const SumArgs &a, int64_t id, const Columns<E, kVec> &c, const float (&sum)[E])
{
    const int64_t at = id * a.dtable_stride + c.first;
    float f[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        f[i] = sum[i] * a.scale;
        if (a.accumulate && i < c.count) f[i] += load_any(a.dtable, at + i * c.step, a.grad_dtype);
    }
    if constexpr (!kVec) {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i < c.count) store_any(a.dtable, at + i * c.step, a.grad_dtype, f[i]);
    } else if (a.grad_dtype == SO_DTYPE_FP32) {
        float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(a.dtable) + at);
#pragma unroll
        for (int i = 0; i < E / 4; ++i) p[i] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
    } else {
        uint2 *p = reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.dtable) + at);
        const bool bf = a.grad_dtype == SO_DTYPE_BF16;
#pragma unroll
        for (int i = 0; i < E / 4; ++i)
            p[i] = bf ? make_uint2(pack2_bf16(f[4 * i], f[4 * i + 1]), pack2_bf16(f[4 * i + 2], f[4 * i + 3]))
                      : make_uint2(pack2_f16(f[4 * i], f[4 * i + 1]), pack2_f16(f[4 * i + 2], f[4 * i + 3]));
    }
}

template <int E, bool kVec>
__device__ __forceinline__ void store_piece(float *piece, const Columns<E, kVec> &c, const float (&sum)[E])
{
    if constexpr (kVec) {
#pragma unroll
        for (int e = 0; e < E; e += 4)
            *reinterpret_cast<float4 *>(piece + c.first + e) = make_float4(sum[e], sum[e + 1], sum[e + 2], sum[e + 3]);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < c.count) piece[c.first + e * c.step] = sum[e];
    }
}

template <int E, bool kVec>
__device__ __forceinline__ void load_piece(const float *piece, const Columns<E, kVec> &c, float (&f)[E])
{
    if constexpr (kVec) {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            const float4 q = __ldcg(reinterpret_cast<const float4 *>(piece + c.first + e));
            f[e] = q.x; f[e + 1] = q.y; f[e + 2] = q.z; f[e + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = e < c.count ? __ldcg(piece + c.first + e * c.step) : 0.0f;
    }
}

template <typename T, int E, bool kVec>
__global__ void __launch_bounds__(kSumThreads) embedding_sum_kernel(SumArgs a)
{
    __shared__ int32_t s_order[3 * kMaxChunk], s_key[3 * kMaxChunk + 1];
    __shared__ uint32_t s_last;
    grid_dependency_wait();
    if ((int32_t)blockIdx.x >= a.sum_blocks) {
        zero_rows(a, (int64_t)blockIdx.x - a.sum_blocks);
        return;
    }
    const int32_t chunk = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles;
    const int32_t total = *a.total, p0 = chunk * a.chunk;
    const int32_t p1 = total - p0 < a.chunk ? total : p0 + a.chunk;
    // looked at before they are known to be there: the array has room for whole chunks
    const Sorted first = a.sorted[p0], last = a.sorted[p1 > p0 ? p1 - 1 : p0];
    if (p0 >= total) return;
    const int32_t first_id = first.id, last_id = last.id;
    const int32_t first_start = first.start, first_end = first.start + first.count;
    const int32_t last_start = last.start, last_end = last.start + last.count;
    const bool first_long = first.count > 2 * a.chunk, last_long = last.count > 2 * a.chunk;
    // a short run that began before belongs to another block; one that begins here is finished here
    const int32_t begin = first_start < p0 && !first_long ? first_end : p0;
    const int32_t end = last_long ? p1 : last_end;
    if (begin >= p1) return;
    for (int32_t i = threadIdx.x; i < end - begin; i += blockDim.x) {
        const Sorted q = a.sorted[begin + i];
        s_order[i] = q.token;
        s_key[i] = q.id;
    }
    if (threadIdx.x == 0) s_key[end - begin] = -1;
    __syncthreads();

    const Columns<E, kVec> c(tile, a.cols);
    const T *dout = static_cast<const T *>(a.dout) + (c.count ? c.first : 0);
    float *head = a.pieces + (int64_t)chunk * 2 * a.cols, *tail = head + a.cols;
    const int32_t count = end - begin;
    float sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = 0.0f;
    if (c.count) {
        for (int32_t i = 0; i < count; i += kBatch) {
            uint4 raw[kVec ? kBatch : 1];
            T one[kVec ? 1 : kBatch][kVec ? 1 : E];
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
                if (i + u < count) {
                    const T *src = dout + (int64_t)s_order[i + u] * a.dout_stride;
                    if constexpr (kVec) {
                        raw[u] = __ldcs(reinterpret_cast<const uint4 *>(src));
                    } else {
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            if (e < c.count) one[u][e] = src[e * c.step];
                    }
                }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                if (i + u >= count) break;
                float f[E];
                if constexpr (kVec) {
                    unpack<T>(raw[u], f);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) f[e] = e < c.count ? to_f32(one[u][e]) : 0.0f;
                }
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] += f[e];
                const int32_t id = s_key[i + u];
                if (s_key[i + u + 1] == id) continue;
                const bool from_before = first_long && id == first_id && first_start < p0;
                if (from_before || (last_long && id == last_id)) store_piece(from_before ? head : tail, c, sum);
                else write_row(a, id, c, sum);
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] = 0.0f;
            }
        }
    }

    // at most two long runs have a piece here: one from before, one that goes on
    for (int which = 0; which < 2; ++which) {
        if (which == 0 ? !(first_long && first_start < p0) : !(last_long && last_start >= p0)) continue;
        const int32_t id = which == 0 ? first_id : last_id;
        const int32_t s0 = which == 0 ? first_start : last_start, s1 = which == 0 ? first_end : last_end;
        const int32_t c0 = s0 / a.chunk, c1 = (s1 - 1) / a.chunk;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) s_last = atomicAdd(&a.arrived[(int64_t)(s0 / (2 * a.chunk)) * a.tiles + tile], 1u);
        __syncthreads();
        if (s_last != (uint32_t)(c1 - c0)) continue;
        __threadfence();
        if (!c.count) continue;
        // the tail of the first stretch, then the heads of the others
        const float *piece = a.pieces + ((int64_t)c0 * 2 + 1) * a.cols;
        load_piece(piece, c, sum);
        piece += a.cols;
        for (int32_t k = c0 + 1; k <= c1; k += kBatch) {
            float f[kBatch][E];
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
                if (k + u <= c1) load_piece(piece + (int64_t)(k + u - c0 - 1) * 2 * a.cols, c, f[u]);
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
                if (k + u <= c1)
#pragma unroll
                    for (int e = 0; e < E; ++e) sum[e] += f[u][e];
        }
        write_row(a, id, c, sum);
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = 0.0f;
    }
}

// Scratch: sorted [n], total, present [vocab / 32], arrived, pieces, at their sizes for the
// shortest stretches, each rounded up to 16 bytes.  A tile is at least 32 columns.
uint64_t round16(uint64_t b) { return (b + 15) & ~uint64_t(15); }

struct Scratch {
    uint64_t sorted, total, present, arrived, pieces, bytes;
    Scratch(int64_t n, int64_t vocab, int64_t cols)
    {
        const uint64_t tiles = ((uint64_t)cols + 31) / 32, chunks = ((uint64_t)n + kMinChunk - 1) / kMinChunk;
        sorted = 0;
        total = sorted + ((uint64_t)n + kMaxChunk) * sizeof(Sorted);
        present = total + 16;
        arrived = present + round16(((uint64_t)vocab + 31) / 32 * 4);
        pieces = arrived + round16(((uint64_t)n / (2 * kMinChunk) + 1) * tiles * 4);
        bytes = pieces + round16(chunks * 2 * (uint64_t)cols * 4);
    }
};

so_status sort_tokens(const SortArgs &a, cudaStream_t st)
{
    static std::atomic<bool> ready[kMaxDevices];
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return SO_ERR_CUDA;
    if (dev < 0 || dev >= kMaxDevices) return SO_ERR_UNSUPPORTED;
    if (!ready[dev].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(embedding_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 kSortWarps * (kRange + 2 * kKeep) * (int)sizeof(int32_t)) != cudaSuccess)
            return SO_ERR_CUDA;
        ready[dev].store(true, std::memory_order_release);
    }
    const unsigned grid = (unsigned)((a.vocab + a.range - 1) / a.range);
    return launch(embedding_sort_kernel, grid, kSortThreads, (size_t)kSortWarps * (a.range + 2 * kKeep) * sizeof(int32_t), st, false, a);
}

template <typename T>
so_status sum_runs(const SumArgs &a, bool vec, unsigned grid, unsigned threads, cudaStream_t st)
{
    return vec ? launch(embedding_sum_kernel<T, Vec<T>::kElems, true>, grid, threads, 0, st, true, a)
               : launch(embedding_sum_kernel<T, kStrided, false>, grid, threads, 0, st, true, a);
}

}  // namespace

extern "C" {

so_status so_embedding_forward(const void *ids, int32_t ids_dtype, int64_t n, const void *table,
                               int64_t table_stride, int64_t vocab, int64_t cols, int32_t dtype,
                               double scale, void *out, int64_t out_stride, int32_t *bad_id,
                               void *stream)
{
    if (!valid_ids(ids_dtype) || !valid_dtype(dtype) || !std::isfinite((float)scale)) return SO_ERR_INVALID_ARG;
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
    *bytes = Scratch(n, vocab, cols).bytes;
    return SO_OK;
}

so_status so_embedding_backward(const void *ids, int32_t ids_dtype, int64_t n, const void *dout,
                                int64_t dout_stride, int64_t vocab, int64_t cols, int32_t dtype,
                                double scale, int64_t padding_id, void *dtable,
                                int64_t dtable_stride, int32_t grad_dtype, int32_t accumulate,
                                void *scratch, uint64_t scratch_bytes, void *stream)
{
    uint64_t need = 0;
    if (!valid_ids(ids_dtype) || !valid_dtype(dtype) || !valid_dtype(grad_dtype) || !std::isfinite((float)scale) ||
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
    // a vector of dout per thread, if whole rows of both sides allow it
    const bool vec = aligned(dout, 16) && (dout_stride * es) % 16 == 0 && (cols * es) % 16 == 0 && aligned(dtable, 16) &&
                     (dtable_stride * gs) % 16 == 0 && (cols * gs) % 16 == 0;
    const int64_t lanes = vec ? cols * es / 16 : (cols + kStrided - 1) / kStrided;
    const unsigned threads = lanes < kSumThreads ? (unsigned)((lanes + 31) / 32 * 32) : kSumThreads;
    const int64_t tiles = (lanes + threads - 1) / threads;
    // short stretches spread few tokens over the SMs, long ones spend less on finding out
    // what to do: the longest with eight blocks an SM
    int chunk = kMinChunk;
    while (chunk < kMaxChunk && n / (2 * chunk) * tiles >= (int64_t)8 * sms) chunk *= 2;
    const int64_t chunks = (n + chunk - 1) / chunk;
    const int64_t zero_blocks = accumulate ? 0 : (vocab + kZeroRows - 1) / kZeroRows;
    if (chunks * tiles + zero_blocks > INT32_MAX) return SO_ERR_TOO_LARGE;
    char *ws = static_cast<char *>(scratch);
    const Scratch at(n, vocab, cols);

    SortArgs k = {};
    k.ids = ids; k.sorted = reinterpret_cast<Sorted *>(ws + at.sorted); k.total = reinterpret_cast<int32_t *>(ws + at.total);
    k.present = reinterpret_cast<uint32_t *>(ws + at.present); k.arrived = reinterpret_cast<uint32_t *>(ws + at.arrived);
    k.padding_id = padding_id; k.n = (int32_t)n; k.vocab = (int32_t)vocab; k.tiles = (int32_t)tiles; k.chunk = chunk;
    k.ids_dtype = ids_dtype;
    k.range = (int32_t)((vocab + sms - 1) / sms + 31) / 32 * 32;
    if (k.range > kRange) k.range = kRange;
    s = sort_tokens(k, st);
    if (s != SO_OK) return s;

    SumArgs a = {};
    a.dout = dout; a.sorted = k.sorted; a.total = k.total; a.present = k.present; a.arrived = k.arrived;
    a.pieces = reinterpret_cast<float *>(ws + at.pieces); a.dtable = dtable; a.vocab = vocab; a.cols = cols;
    a.dout_stride = dout_stride; a.dtable_stride = dtable_stride; a.tiles = (int32_t)tiles; a.chunk = chunk;
    a.sum_blocks = (int32_t)(chunks * tiles); a.grad_dtype = grad_dtype; a.accumulate = accumulate; a.scale = (float)scale;
    a.wide = aligned(dtable, 16) && (dtable_stride * gs) % 16 == 0 && (cols * gs) % 16 == 0;
    const unsigned grid = (unsigned)(chunks * tiles + zero_blocks);
    if (dtype == SO_DTYPE_BF16) return sum_runs<bf16_t>(a, vec, grid, threads, st);
    if (dtype == SO_DTYPE_FP16) return sum_runs<f16_t>(a, vec, grid, threads, st);
    return sum_runs<float>(a, vec, grid, threads, st);
}

}  // extern "C"
