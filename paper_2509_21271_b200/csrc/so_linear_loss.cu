// Cross entropy of labels from the hidden states and the table of the head, with both
// gradients, in pieces of the vocabulary: the logits of a large batch are never all there.
//
//   z = H W^T,  row_loss = log sum_j exp z_j - z_label,  loss = sum w row_loss
//   P = w (softmax(z) - [label]),  dH = s P W,  dW = s P^T H
//
// Rows of weight 0 or without a label in the vocabulary are left out from the start: the
// others are gathered into a matrix of their own, which also gives every row an aligned
// start and whole tiles.  Then
//   statistics     a pass over all logits, tile by tile: each row's maximum and sum
//   for each piece the piece's logits once more (a small batch has kept them), as P in 16 bits;
//                  dH += P W; dW = P^T H
// are all one kernel, a persistent matrix product on the tensor cores (tcgen05: operands
// through TMA into swizzled shared memory, two accumulators of 256 columns in tensor
// memory, so that one is read while the next is computed) with four ways to end a tile.
//
// With top = max z and others = sum of exp(z_j - top) but for the label's,
//   q_j = exp(z_j - top) / total,  total = others + exp(z_label - top),  q_label - 1 = -others / total,
// and the loss is log(1 + others / exp(z_label - top)): where a label has nearly all the probability,
// both are as good relative to 1 - q as other rows' are to 1.  (One number for log sum exp z would do
// for q, but its rounding, 1e-6 for logits near 20, is all of q - 1 there.)
//
// P is w (q - [label]) as a multiple of the largest |w| (for fp16 of 2^-15 of it: its normal
// numbers then reach down to 2^-29 of a row's largest).  A mean's weights are all the same: as
// multiples of a power of two, P at the labels would be rounded the same way in every row, which made
// dW of 255 rows 0.4 % too long; so it is close to -1.  Its
// rounding to 16 bits is one rounding of every term of sums that are themselves
// rounded to 16 bits; where dW is fp32, it sums P in parts of 16 bits that together hold 24
// bits (bf16, three parts) or 22 (fp16, two).
#include <cuda.h>

#include "so_ops.cuh"

using namespace so_ops;

namespace {

constexpr int kTileN = 256;               // columns of a tile
constexpr int kTileK = 64;                // of a step: 128 bytes, the width of the swizzle
constexpr int kRowsOfCta = 128;           // rows of a tile that a block holds
constexpr int kEnders = 8;                // warps that end tiles: two for each 32 rows, with half of the columns each
constexpr int kThreads = 64 + 32 * kEnders;   // and a warp that copies, one that multiplies
constexpr int kEndCols = kTileN / 2;
constexpr uint32_t kBox = 32 * 128;       // what such a warp copies out at a time: 32 rows of 128 bytes
constexpr int kRowPad = 256;              // rows are padded to whole tiles of a pair of blocks
constexpr float kLog2e = 1.44269504088896340736f;

// What a launch computes, and a tile of one: the tiles of both gradients are in one launch, as they
// need the same P and fill each other's last wave.
enum Mode { kStats, kProb, kHidden, kTable, kGradients };

// What the device finds out about a call, in scratch.
struct Control {
    int32_t live;                         // rows that take part
    float unit;                           // P is held as a multiple of this
    uint32_t ticket;                      // blocks of the statistics' join that are done
    int32_t gave_up;                      // a wait ran out: every result becomes NaN
};

// ---- tensor memory, matrix instructions, tensor copies -----------------------------

__device__ __forceinline__ uint32_t cta_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address of this block's `addr` in the block of rank `rank`
__device__ __forceinline__ uint32_t of_rank(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
template <int kCtas>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    if constexpr (kCtas == 2)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// The same from a matrix seen as groups of 64 columns: 64 rows of two groups.
template <int kCtas>
__device__ __forceinline__ void tma_load_groups(uint32_t dst, const CUtensorMap *map, int y, int group, uint32_t bar)
{
    if constexpr (kCtas == 2)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(0), "r"(y), "r"(group), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(0), "r"(y), "r"(group), "r"(bar) : "memory");
}
// A box in shared memory to its place in a matrix, or added to what is there (fp32); what lies
// outside of the matrix is left out.  By the same thread of a warp each time.
__device__ __forceinline__ void tma_store(const CUtensorMap *map, int x, int y, uint32_t src, bool add)
{
    if (add)
        asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];"
                     ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void tma_stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void tma_stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

template <int kCtas>
__device__ __forceinline__ void tmem_alloc(uint32_t dst, uint32_t cols)
{
    if constexpr (kCtas == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <int kCtas>
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t cols)
{
    if constexpr (kCtas == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(cols) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(cols) : "memory");
}
template <int kCtas>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    if constexpr (kCtas == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// The barrier (of both blocks of a pair) is arrived at once the instructions so far are done.
template <int kCtas>
__device__ __forceinline__ void commit(uint32_t bar)
{
    if constexpr (kCtas == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of the warp's 32 lanes of tensor memory
__device__ __forceinline__ void tmem_load(uint32_t at, float (&f)[32])
{
    uint32_t r[32];
    __syncwarp();                         // all lanes, whatever they did with the columns before
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
                   "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
                   "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(r[i]);
}

// Descriptors.  An operand whose K elements are contiguous lies in rows of 128 bytes (64 of
// them), groups of eight rows 1024 bytes apart.  One whose M (or N) elements are contiguous
// lies in rows of 128 bytes for each k: groups of eight k 1024 bytes apart, groups of 64 of its
// M (or N) elements kMajorStep bytes apart.  Either is swizzled over 128 bytes.
constexpr uint32_t kMajorStep = kTileK * 128;
constexpr uint64_t kDescBase = (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
__device__ __forceinline__ uint64_t descriptor(uint32_t addr, bool k_contiguous)
{
    return kDescBase | (uint64_t)((k_contiguous ? 16 : kMajorStep) >> 4) << 16 | (uint64_t)((addr & 0x3FFFF) >> 4);
}
// bytes from one instruction's operand (16 elements of K) to the next one's
template <bool kContiguous> constexpr uint32_t kStepBytes = kContiguous ? 32 : 16 * 128;

// fp32 accumulators; A and B bf16 or fp16; contiguous in K (0) or in M, N (1)
template <typename T>
__host__ __device__ constexpr uint32_t instruction(int m, int n, bool a_k, bool b_k)
{
    const uint32_t type = std::is_same<T, bf16_t>::value ? 1 : 0;
    return 1u << 4 | type << 7 | type << 10 | (a_k ? 0u : 1u) << 15 | (b_k ? 0u : 1u) << 16 | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}

// ---- the product ----------------------------------------------------------------------

struct Product {
    Control *control;
    int64_t width;                        // vocabulary of this launch
    int64_t first;                        // its first entry
    int64_t table_row;                    // row of the (perhaps packed) table where that is
    int64_t vocab, cols;
    int32_t rows_pad;
    int32_t splits;                       // kHidden: parts that the vocabulary is summed in
    int32_t planes;                       // kProb, kTable: parts of P
    int32_t table_groups;                 // kHidden: the table's map is of groups of 64 columns
    int32_t begin;                        // kHidden: the sums begin here rather than going on
    const int32_t *label;                 // [rows_pad], of the gathered rows
    float *label_logit;                   // [rows_pad]
    const float4 *terms;                  // [rows_pad]: largest logit, log2 of the sum relative to it, w over the unit, q - 1 of the label
    float *residual;                      // [rows_pad]: what P at the label lost when it was rounded
    float2 *stats;                        // [half tiles of the vocabulary][rows_pad]: maximum, sum without the label's
    float *kept;                          // kStats: [rows_pad][prob_stride], where all logits are kept
    void *prob;                           // [planes][rows_pad][prob_stride]
    int64_t prob_stride;
    float *part;                          // [splits][rows_pad][part_stride]
    int64_t part_stride;
    int32_t want_hidden;
    void *table_grad;
    int64_t grad_stride;
    int32_t grad_dtype, accumulate, grad_boxes;
    float grad_scale;
    Patience patience;
};

// Which tile, and which steps of K.
struct Item {
    int kind, m, n, split, steps, k0;     // k0: first step
};

// The tiles of one kind.
template <int kCtas>
struct Tiles {
    int m, n, k_steps, splits;
    int64_t items;
    __device__ Tiles(const Product &p, int kind, int live)
    {
        constexpr int kTileM = kRowsOfCta * kCtas;
        const int row_tiles = (live + kTileM - 1) / kTileM, col_tiles = (int)((p.cols + kTileN - 1) / kTileN);
        splits = 1;
        if (kind == kStats || kind == kProb) {
            m = row_tiles;
            n = (int)((p.width + kTileN - 1) / kTileN);
            k_steps = (int)((p.cols + kTileK - 1) / kTileK);
        } else if (kind == kHidden) {
            m = row_tiles;
            n = col_tiles;
            k_steps = (int)((p.width + kTileK - 1) / kTileK);
            splits = p.splits;
        } else {
            m = live ? (int)((p.width + kTileM - 1) / kTileM) : 0;
            n = col_tiles;
            k_steps = (live + kTileK - 1) / kTileK;
        }
        items = (int64_t)m * n * splits;
    }
    __device__ __forceinline__ Item item(const Product &p, int kind, int64_t i) const
    {
        Item r;
        r.kind = kind;
        r.split = 0;
        r.k0 = 0;
        r.steps = k_steps;
        if (kind == kStats || kind == kProb) {
            // the rows' tiles one after the other: a tile of the table is read once, the hidden states stay in L2
            r.n = (int)(i / m);
            r.m = (int)(i - (int64_t)r.n * m);
        } else {
            const int64_t q = i / n;
            r.n = (int)(i - q * n);
            r.m = (int)(q % m);
            r.split = (int)(q / m);
        }
        if (kind == kHidden) {
            r.k0 = (int)((int64_t)k_steps * r.split / splits);
            r.steps = (int)((int64_t)k_steps * (r.split + 1) / splits) - r.k0;
        } else if (kind == kTable) {
            r.steps = k_steps * p.planes;
        }
        return r;
    }
};

template <int kMode, int kCtas>
struct Work {
    static constexpr int kFirst = kMode == kGradients ? (int)kHidden : kMode;
    Tiles<kCtas> first, second;           // second: kGradients' of the table, behind the longer ones of dH
    int64_t items;
    __device__ Work(const Product &p, int live) : first(p, kFirst, live), second(p, kTable, live)
    {
        if (kMode == kGradients && !p.want_hidden) first.items = 0;
        items = first.items + (kMode == kGradients && p.table_grad ? second.items : 0);
    }
    __device__ __forceinline__ Item item(const Product &p, int64_t i) const
    {
        if (kMode != kGradients || i < first.items) return first.item(p, kFirst, i);
        return second.item(p, kTable, i - first.items);
    }
    __device__ __forceinline__ int k_steps(const Item &it) const { return kMode == kGradients && it.kind == kTable ? second.k_steps : first.k_steps; }
};

template <int kCtas>
struct Shape {
    static constexpr uint32_t kA = kRowsOfCta * 128, kB = kTileN / kCtas * 128, kStage = kA + kB;
    static constexpr int kStages = kCtas == 2 ? 6 : 4;       // 192 KB
    static constexpr size_t kBytes = (size_t)kStage * kStages + kEnders * kBox + 1024;
};

struct Shared {
    uint64_t full[8], empty[8], done[2], free[2], last;
    uint32_t tmem;
    int issued[2];                        // stages that this block has filled; of the second block of a pair
    volatile uint32_t gave_up;
};

// Waits, after a wait that ran out, for the copies that are still on their way into the first block's
// stages, and the second's, which are counted by the first's barriers too.  Where one of them had
// gone on further than the other, the barrier is given what the other left out.
template <int kCtas>
__device__ __noinline__ void land_stages(Shared &s)
{
    using S = Shape<kCtas>;
    const int mine = s.issued[0], other = kCtas == 2 ? s.issued[1] : mine, most = mine > other ? mine : other;
    for (int k = most > S::kStages ? most - S::kStages : 0; k < most; ++k) {
        const uint32_t bar = smem_addr(s.full + k % S::kStages);
        if (k >= mine) mbar_expect(bar, S::kStage);
        else if (k >= other) asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(S::kStage) : "memory");
        mbar_wait(bar, (uint32_t)(k / S::kStages) & 1u, kPolls);
    }
}

// A wait that ends when the barrier's phase does, when it runs out, or when another of the block
// has run out; false unless the first.
__device__ __noinline__ bool await_long(uint32_t bar, uint32_t parity, uint32_t polls, Shared &s, Control *c)
{
    if (s.gave_up) return false;
    for (uint32_t left = polls; left > 0;) {
        const uint32_t now = left < 1024 ? left : 1024;
        if (mbar_wait(bar, parity, now)) return true;
        if (s.gave_up) return false;
        left -= now;
    }
    s.gave_up = 1;
    atomicExch(&c->gave_up, 1);
    return false;
}
// All lanes of a warp, which go on together.
__device__ __forceinline__ bool await(uint32_t bar, uint32_t parity, uint32_t polls, Shared &s, Control *c)
{
    bool ok = mbar_test(bar, parity);
    if (!__all_sync(0xFFFFFFFFu, ok)) ok = await_long(bar, parity, polls, s, c);
    return __all_sync(0xFFFFFFFFu, ok);
}

// One lane of a converged warp, the same one each time.
__device__ __forceinline__ bool elected()
{
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}

// 32 bytes
__device__ __forceinline__ void load32(const void *p, uint32_t (&w)[8])
{
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p) : "memory");
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    if constexpr (std::is_same<T, bf16_t>::value) return pack2_bf16(lo, hi);
    else return pack2_f16(lo, hi);
}
template <typename T> __device__ __forceinline__ void unpack2(uint32_t w, float &lo, float &hi)
{
    lo = to_f32(T{(uint16_t)(w & 0xFFFFu)});
    hi = to_f32(T{(uint16_t)(w >> 16)});
}

// 128 bytes of each lane's row, swizzled, through shared memory to rows y.. and columns x.. of a
// matrix.  Stores of a lane's own 32 bytes into 32 rows take a cycle or two for every row: 1 x 128256 x
// 4096 bf16 as a whole 654 us with them, 580 us this way.
__device__ __forceinline__ void copy_out(const CUtensorMap *map, uint32_t box, int x, int y, const uint32_t (&w)[32], bool add)
{
    const int lane = threadIdx.x & 31;
    if (lane == 0) tma_stores_read();     // the box is free again
    __syncwarp();
#pragma unroll
    for (int u = 0; u < 8; ++u)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(box + lane * 128 + ((u ^ (lane & 7)) << 4)), "r"(w[4 * u]), "r"(w[4 * u + 1]),
                     "r"(w[4 * u + 2]), "r"(w[4 * u + 3]) : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) tma_store(map, x, y, box, add);
}

// Half a tile, n-th of the columns.  A row's maximum and sum over it, its label's logit if that is
// here (which the sum leaves out), and the logits themselves where they are kept.
__device__ __forceinline__ void end_stats(const Product &p, const CUtensorMap *map, uint32_t box, uint32_t tmem, int64_t row, int live, int n)
{
    const int64_t n0 = p.first + (int64_t)n * kEndCols;
    const int cols = p.vocab - n0 < kEndCols ? (int)(p.vocab - n0) : kEndCols;
    if (cols <= 0) return;                // the second half of a last tile
    const bool in = row < live;
    const int64_t label = in ? (int64_t)p.label[row] - n0 : -1;
    float top = -kInf;
    for (int c = 0; c < cols; c += 32) {
        float f[32];
        tmem_load(tmem + c, f);
        if (c + 32 <= cols) {
#pragma unroll
            for (int i = 0; i < 32; ++i) top = fmaxf(top, f[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (c + i < cols) top = fmaxf(top, f[i]);
        }
        if (__any_sync(0xFFFFFFFFu, label >= c && label < c + 32)) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (label == c + i) p.label_logit[row] = f[i];
        }
    }
    const float ref = top == -kInf ? 0.0f : top;            // a tile of nothing else adds nothing
    float sum0 = 0.0f, sum1 = 0.0f;
    for (int c = 0; c < cols; c += 32) {
        float f[32];
        tmem_load(tmem + c, f);
        if (p.kept && row - (int64_t)(threadIdx.x & 31) < live) {
            uint32_t w[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(f[i]);
            copy_out(map, box, (int)n0 + c, (int)row - (int)(threadIdx.x & 31), w, false);
        }
        if (__any_sync(0xFFFFFFFFu, label >= c && label < c + 32)) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (label == c + i) f[i] = -kInf;
        }
        // (the difference first: large logits keep their digits)
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            sum0 += c + i < cols ? exp2_fast((f[i] - ref) * kLog2e) : 0.0f;
            sum1 += c + i + 1 < cols ? exp2_fast((f[i + 1] - ref) * kLog2e) : 0.0f;
        }
    }
    if (in) p.stats[(n0 / kEndCols) * p.rows_pad + row] = make_float2(top, sum0 + sum1);
}

// P of the tile, in `planes` parts of 16 bits; zero in rows and columns that are not there.
template <typename T>
__device__ __forceinline__ void end_prob(const Product &p, const CUtensorMap *map, uint32_t box, uint32_t tmem, int64_t row, int live, int n)
{
    const int64_t n0 = p.first + (int64_t)n * kEndCols;
    const int cols = p.vocab - n0 < kEndCols ? (int)(p.vocab - n0) : kEndCols;
    const bool in = row < live;
    const int64_t label = in ? (int64_t)p.label[row] - n0 : -1;
    const float4 t = in ? p.terms[row] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const int y = (int)row - (int)(threadIdx.x & 31);
    for (int c = 0; c < kEndCols; c += 64) {
        float f[2][32];
        uint32_t w[32];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            tmem_load(tmem + c + 32 * h, f[h]);
            const int c0 = c + 32 * h;
            const bool here = __any_sync(0xFFFFFFFFu, label >= c0 && label < c0 + 32);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                float q = exp2_fast(fmaf(f[h][i] - t.x, kLog2e, -t.y));
                if (here && label == c0 + i) q = t.w;
                f[h][i] = in && c0 + i < cols ? q * t.z : 0.0f;
                if (here && label == c0 + i) p.residual[row] = f[h][i] - to_f32(from_f32<T>(f[h][i]));
            }
        }
        for (int plane = 0;; ++plane) {
#pragma unroll
            for (int i = 0; i < 32; ++i) w[i] = pack2<T>(f[i / 16][2 * (i % 16)], f[i / 16][2 * (i % 16) + 1]);
            copy_out(map, box, n * kEndCols + c, plane * p.rows_pad + y, w, false);
            if (plane + 1 == p.planes) break;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                float lo, hi;
                unpack2<T>(w[i], lo, hi);
                f[i / 16][2 * (i % 16)] -= lo;
                f[i / 16][2 * (i % 16) + 1] -= hi;
            }
        }
    }
}

// The tile added to (or begun as) a part of dH, fp32; `nothing`: a short piece had no columns for it.
// One tile of a launch adds to an element, so that the order of the sums is that of the launches.
__device__ __forceinline__ void end_hidden(const Product &p, const CUtensorMap *map, uint32_t box, uint32_t tmem, int64_t row, int n, int split, bool nothing)
{
    if (nothing && !p.begin) return;
    const int y = split * p.rows_pad + (int)row - (int)(threadIdx.x & 31);
    for (int c = 0; c < kEndCols; c += 32) {
        float f[32];
        uint32_t w[32];
        tmem_load(tmem + c, f);
#pragma unroll
        for (int i = 0; i < 32; ++i) w[i] = nothing ? 0u : __float_as_uint(f[i]);
        copy_out(map, box, n * kEndCols + c, y, w, !p.begin);
    }
}

// The tile as rows of dW, in the gradient's type.
__device__ __forceinline__ void end_table(const Product &p, const CUtensorMap *map, uint32_t box, uint32_t tmem, int64_t row, int n, float scale)
{
    const int c0 = n * kEndCols, y = (int)(p.first + row) - (int)(threadIdx.x & 31);
    if (p.grad_dtype == SO_DTYPE_FP32) {
        for (int c = 0; c < kEndCols && c0 + c < p.cols; c += 32) {
            float f[32];
            uint32_t w[32];
            tmem_load(tmem + c, f);
#pragma unroll
            for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(f[i] * scale);
            copy_out(map, box, c0 + c, y, w, p.accumulate != 0);
        }
        return;
    }
    const bool bf = p.grad_dtype == SO_DTYPE_BF16;
    for (int c = 0; c < kEndCols && c0 + c < p.cols; c += 64) {
        uint32_t w[32];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float f[32];
            tmem_load(tmem + c + 32 * h, f);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float lo = f[2 * i] * scale, hi = f[2 * i + 1] * scale;
                w[16 * h + i] = bf ? pack2_bf16(lo, hi) : pack2_f16(lo, hi);
            }
        }
        copy_out(map, box, c0 + c, y, w, false);
    }
}

// The same where 16-bit numbers are added to what is there, or where rows do not start at 16-byte
// boundaries: through shared memory too, then a row at a time, a column a lane.  Both gradients of 300
// x 128256 x 77 bf16 take 90 us this way; with a lane to its own row's columns they took 142 us.
__device__ __forceinline__ void end_table_by_rows(const Product &p, uint32_t box, uint32_t tmem, int64_t row, int n, float scale)
{
    const int lane = threadIdx.x & 31;
    const int64_t c0 = (int64_t)n * kEndCols, first = row - lane;
    const int64_t left = p.width - first < p.vocab - p.first - first ? p.width - first : p.vocab - p.first - first;
    const int rows = left < 32 ? (int)left : 32;
    if (lane == 0) tma_stores_read();     // the box may still be on its way out with a tile of dH
    __syncwarp();
    for (int c = 0; c < kEndCols && c0 + c < p.cols; c += 32) {
        float f[32];
        tmem_load(tmem + c, f);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(box + lane * 128 + ((u ^ (lane & 7)) << 4)), "f"(f[4 * u] * scale),
                         "f"(f[4 * u + 1] * scale), "f"(f[4 * u + 2] * scale), "f"(f[4 * u + 3] * scale) : "memory");
        __syncwarp();
        if (c0 + c + lane < p.cols) {
            int64_t at = (p.first + first) * p.grad_stride + c0 + c + lane;
#pragma unroll 4
            for (int r = 0; r < rows; ++r, at += p.grad_stride) {
                float x;
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(box + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4));
                if (p.accumulate) x += load_any(p.table_grad, at, p.grad_dtype);
                store_any(p.table_grad, at, p.grad_dtype, x);
            }
        }
        __syncwarp();
    }
}

// A block, or a pair of blocks that share an instruction's tile of 256 x 256 (tiles of 128 x 256 where
// there are at most 128 rows), takes every units-th tile.  Its warps: one copies 64 columns (K) of A and
// B a stage, one issues the instructions, eight end the tile before while the next is computed.
//
// Bound: the tensor cores and the power limit.  8192 x 128256 x 4096 bf16 with 5734 rows that take part
// does 2.4e13 operations in 17.0 (a short run) to 18.9 ms, 1.28 to 1.42 PFLOP/s; a library's product sustains
// 1.41.  The statistics alone of 4095 x 128256 x 2048: 1.29 to 1.56 ms, 1.38 to 1.66 PFLOP/s (a library's burst: 1.68).
// On the way: one lane alone in the loops of the first two warps 22.1 ms, six or seven stages the same
// within 0.1 %, P in pieces of 128 MB instead of 256 MB 5 % more, both gradients in two launches 2 % more.
// Small batches are bound by the chain of six launches and the table's reading: 63 x 50257 x 768 85 to 93
// us for 24 us of bytes.  The sums of a logit's 16-column products are rounded to fp32 one after the
// other, d / 16 of them: losses come out good to 4e-7 (d = 512) to 1.6e-6 (d = 4096).
//
// a, b, out: of kStats and kProb, and of the tiles of dH; a2, b2, out2: of those of dW.
struct Maps {
    CUtensorMap a, b, out, a2, b2, out2;
};

template <typename T, int kMode, int kCtas>
__global__ void __launch_bounds__(kThreads, 1) product_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Product p)
{
    using S = Shape<kCtas>;
    constexpr bool kBK = kMode != kGradients;                // B contiguous in K: W by its columns, else W and H by their rows
    extern __shared__ uint8_t s_raw[];
    __shared__ __align__(8) Shared s;
    const uint32_t tiles = (smem_addr(s_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = kCtas == 2 ? cta_rank() : 0;
    const int unit = (int)(blockIdx.x / kCtas), units = (int)(gridDim.x / kCtas);
    const uint32_t polls = p.patience.of(unit);
    const uint32_t full = smem_addr(s.full), empty = smem_addr(s.empty), done = smem_addr(s.done), free = smem_addr(s.free);

    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(done + 8 * i, 1);
            mbar_init(free + 8 * i, kEnders * kCtas);
        }
        mbar_init(smem_addr(&s.last), 1);
        mbar_init_fence();
        s.gave_up = polls == 0;
    }
    if (warp == 1) tmem_alloc<kCtas>(smem_addr(&s.tmem), 512);
    fence_before();
    __syncthreads();
    if (kCtas == 2) cluster_sync();
    fence_after();
    const uint32_t tmem = s.tmem;
    grid_dependency_wait();
    grid_dependency_release();            // the next launch waits for this one's end before it reads anything
    if (polls == 0 && threadIdx.x == 0) atomicExch(&p.control->gave_up, 1);
    const int live = p.control->live;
    const Work<kMode, kCtas> work(p, live);

    // The warps that copy and multiply go through their loops with all lanes, so that addresses and
    // descriptors stay in uniform registers, and one lane issues: with one lane alone in the loop a
    // step took 800 clocks, of which the tensor cores need 512.
    if (warp == 0) {
        // copies: this block's rows of A and its share of B
        int stage = 0, issued = 0;
        uint32_t phase = 1;
        bool ok = true;
        for (int64_t i = unit; ok && i < work.items; i += units) {
            const Item it = work.item(p, i);
            const int m0 = (it.m * kCtas + (int)rank) * kRowsOfCta, n0 = it.n * kTileN + (int)rank * (kTileN / kCtas);
            const int k_steps = work.k_steps(it);
            int step = it.k0, row0 = 0;                      // row0: of the part of P
            for (int k = 0; k < it.steps; ++k) {
                if (!(ok = await(empty + 8 * stage, phase, polls, s, p.control))) break;
                const uint32_t bar = kCtas == 2 ? of_rank(full + 8 * stage, 0) : full + 8 * stage;
                const uint32_t a = tiles + stage * S::kStage, b = a + S::kA;
                const int k0 = step * kTileK;
                if (elected()) {
                    if (rank == 0) mbar_expect(full + 8 * stage, S::kStage * kCtas);
                    if (kBK) {
                        tma_load<kCtas>(a, &maps.a, k0, m0, bar);
#pragma unroll
                        for (int g = 0; g < 2 / kCtas; ++g) tma_load<kCtas>(b + g * 128 * 128, &maps.b, k0, (int)p.table_row + n0 + 128 * g, bar);
                    } else if (it.kind == kTable) {
                        tma_load_groups<kCtas>(a, &maps.a2, row0 + k0, m0 / 64, bar);
#pragma unroll
                        for (int g = 0; g < 2 / kCtas; ++g) tma_load_groups<kCtas>(b + 2 * g * kMajorStep, &maps.b2, k0, n0 / 64 + 2 * g, bar);
                    } else {
                        tma_load<kCtas>(a, &maps.a, k0, m0, bar);
                        if (p.table_groups) {
#pragma unroll
                            for (int g = 0; g < 2 / kCtas; ++g) tma_load_groups<kCtas>(b + 2 * g * kMajorStep, &maps.b, (int)p.table_row + k0, n0 / 64 + 2 * g, bar);
                        } else {
#pragma unroll
                            for (int g = 0; g < kTileN / kCtas / 64; ++g) tma_load<kCtas>(b + g * kMajorStep, &maps.b, n0 + 64 * g, (int)p.table_row + k0, bar);
                        }
                    }
                }
                __syncwarp();
                ++issued;
                if (++stage == S::kStages) stage = 0, phase ^= 1;
                if (++step == k_steps && it.kind == kTable) step = 0, row0 += p.rows_pad;
            }
        }
        if (lane == 0) {
            if (rank == 0) s.issued[0] = issued;
            else asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(of_rank(smem_addr(s.issued + 1), 0)), "r"(issued) : "memory");
        }
    } else if (warp == 1 && rank == 0) {
        int stage = 0, buffer = 0;
        uint32_t phase = 0, free_phase = 1;
        bool ok = true, ready = false;                       // ready: the stage is known to be filled
        for (int64_t i = unit; ok && i < work.items; i += units) {
            const Item it = work.item(p, i);
            if (!(ok = await(free + 8 * buffer, free_phase, polls, s, p.control))) break;
            const uint32_t d = tmem + buffer * kTileN;
            // A: H, H, P contiguous in K; P transposed is not
            const bool a_k = kMode != kGradients || it.kind != kTable;
            const uint32_t what = a_k ? instruction<T>(kRowsOfCta * kCtas, kTileN, true, kBK) : instruction<T>(kRowsOfCta * kCtas, kTileN, false, kBK);
            const uint32_t a_step = (a_k ? kStepBytes<true> : kStepBytes<false>) >> 4;
            for (int k = 0; k < it.steps; ++k) {
                if (!ready && !(ok = await(full + 8 * stage, phase, polls, s, p.control))) break;
                fence_after();
                const uint32_t a = tiles + stage * S::kStage, b = a + S::kA, used = empty + 8 * stage;
                if (++stage == S::kStages) stage = 0, phase ^= 1;
                // a look at the next stage while this one's instructions are still to come
                ready = k + 1 < it.steps && __all_sync(0xFFFFFFFFu, mbar_test(full + 8 * stage, phase));
                const uint64_t da = descriptor(a, a_k), db = descriptor(b, kBK);
                if (elected()) {
#pragma unroll
                    for (int j = 0; j < kTileK / 16; ++j)
                        mma<kCtas>(d, da + j * a_step, db + (j * kStepBytes<kBK> >> 4), what, (k | j) != 0);
                    commit<kCtas>(used);
                }
                __syncwarp();
            }
            if (!ok) break;
            if (elected()) commit<kCtas>(done + 8 * buffer);
            __syncwarp();
            buffer ^= 1;
            if (buffer == 0) free_phase ^= 1;
        }
        if (!ok) {
            if (elected()) commit<kCtas>(smem_addr(&s.last));
            __syncwarp();
            mbar_wait(smem_addr(&s.last), 0, kPolls);
        }
    } else if (warp >= 2) {
        const uint32_t lanes = (uint32_t)(warp & 3) * 32;    // of tensor memory that this warp reaches
        const int half = (warp - 2) / (kEnders / 2);
        const uint32_t box = tiles + S::kStage * S::kStages + (warp - 2) * kBox;
        const float scale = p.grad_scale * p.control->unit;
        int buffer = 0;
        uint32_t phase = 0;
        for (int64_t i = unit; i < work.items; i += units) {
            const Item it = work.item(p, i);
            if (!await(done + 8 * buffer, phase, polls, s, p.control)) break;
            fence_after();
            const uint32_t at = tmem + buffer * kTileN + half * kEndCols + (lanes << 16);
            const int64_t row = ((int64_t)it.m * kCtas + rank) * kRowsOfCta + lanes + lane;
            if (kMode == kStats) end_stats(p, &maps.out, box, at, row, live, 2 * it.n + half);
            else if (kMode == kProb) end_prob<T>(p, &maps.out, box, at, row, live, 2 * it.n + half);
            else if (it.kind == kHidden) end_hidden(p, &maps.out, box, at, row, 2 * it.n + half, it.split, it.steps == 0);
            else if (p.grad_boxes) end_table(p, &maps.out2, box, at, row, 2 * it.n + half, scale);
            else end_table_by_rows(p, box, at, row, 2 * it.n + half, scale);
            fence_before();
            __syncwarp();
            if (lane == 0) {
                if (kCtas == 2) arrive_at(of_rank(free + 8 * buffer, 0));
                else mbar_arrive(free + 8 * buffer);
            }
            buffer ^= 1;
            if (buffer == 0) phase ^= 1;
        }
        if (lane == 0) tma_stores_done();
    }
    __syncthreads();
    if (kCtas == 2) cluster_sync();
    if (rank == 0 && threadIdx.x == 0 && s.gave_up) land_stages<kCtas>(s);
    __syncwarp();
    if (kCtas == 2) cluster_sync();       // the second block stays as long as its copies do
    if (warp == 1) tmem_free<kCtas>(tmem, 512);
}

// ---- around the products ----------------------------------------------------------------

struct Rows {
    Control *control;
    const void *hidden;
    int64_t hidden_stride;
    const void *labels;
    int32_t ids_dtype;
    const float *weight;
    int64_t rows, vocab, cols;
    int32_t rows_pad;
    void *gathered;                       // [rows_pad][gathered_stride]
    int64_t gathered_stride;
    int32_t *index, *label;               // [rows_pad]: where a gathered row is from
    float *w;                             // [rows_pad]
    float *row_loss;
    void *dhidden;
    int64_t dhidden_stride;
    float2 *counts;                       // [chunks]: rows that take part (as bits), largest weight; NULL: one chunk
    int32_t fp16, vectors, dhidden_vectors;
};

__device__ __forceinline__ bool is_live(const Rows &r, int64_t i)
{
    if (r.weight && r.weight[i] == 0.0f) return false;
    const int64_t label = load_id(r.labels, i, r.ids_dtype);
    return label >= 0 && label < r.vocab;
}

constexpr int kGatherThreads = 256, kGatherRows = kGatherThreads / 32;
constexpr int kChunk = 4096;              // rows that one block counts; batches beyond it are counted by chunks first

// 16-bit elements [0, n) of a row of `n_pad` (a multiple of 8), zeros behind; `src` NULL: zeros.
__device__ __forceinline__ void copy_row(uint16_t *dst, const uint16_t *src, int64_t n, int64_t n_pad, bool vectors, int lane)
{
#pragma unroll 4
    for (int64_t c = lane * 8; c < n_pad; c += 256) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (src && vectors && c + 8 <= n) {
            v = *reinterpret_cast<const uint4 *>(src + c);
        } else if (src) {
            uint16_t e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = c + i < n ? src[c + i] : (uint16_t)0;
            v = make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16);
        }
        *reinterpret_cast<uint4 *>(dst + c) = v;
    }
}

// Rows that take part among [from, to), and the largest weight there; known to every thread.
__device__ __forceinline__ int count_rows(const Rows &r, int64_t from, int64_t to, float *top)
{
    __shared__ int s_count[kGatherThreads / 32];
    __shared__ float s_top[kGatherThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int count = 0;
    float most = 0.0f;
#pragma unroll 4
    for (int64_t i = from + threadIdx.x; i < to; i += kGatherThreads) {
        const float w = r.weight ? r.weight[i] : 1.0f;
        const int64_t label = load_id(r.labels, i, r.ids_dtype);
        if (w != 0.0f && label >= 0 && label < r.vocab) {
            ++count;
            most = fmaxf(most, fabsf(w));
        }
    }
    count = __reduce_add_sync(0xFFFFFFFFu, count);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
    if (lane == 0) s_count[warp] = count, s_top[warp] = most;
    __syncthreads();
    count = 0;
#pragma unroll
    for (int i = 0; i < kGatherThreads / 32; ++i) count += s_count[i], most = fmaxf(most, s_top[i]);
    *top = most;
    return count;
}

// Counts of chunks of rows, for batches of many.
__global__ void __launch_bounds__(kGatherThreads) count_kernel(const __grid_constant__ Rows r)
{
    grid_dependency_wait();
    const int64_t from = (int64_t)blockIdx.x * kChunk, to = from + kChunk;
    float top;
    const int count = count_rows(r, from, to < r.rows ? to : r.rows, &top);
    if (threadIdx.x == 0) r.counts[blockIdx.x] = make_float2(__int_as_float(count), top);
}

// Gathers the rows that take part, a row a warp; a block counts the rows before its own for
// itself (those of its chunk, behind what earlier chunks have).  Eight more blocks know them all.
__global__ void __launch_bounds__(kGatherThreads) gather_kernel(const __grid_constant__ Rows r)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t row0 = (int64_t)blockIdx.x * kGatherRows;
    const bool behind = row0 >= r.rows;   // one of the blocks behind the last row: they know all rows
    if (behind) row0 = r.rows;
    const int64_t chunk = r.counts ? row0 / kChunk : 0;
    grid_dependency_wait();
    grid_dependency_release();
    float top;
    int base = count_rows(r, chunk * kChunk, row0, &top);
    for (int64_t i = 0; i < chunk; ++i) {
        const float2 c = r.counts[i];
        base += __float_as_int(c.x);
        top = fmaxf(top, c.y);
    }
    // lane k of every warp looks at the block's k-th row
    const bool in = lane < kGatherRows && row0 + lane < r.rows && is_live(r, row0 + lane);
    const uint32_t mask = __ballot_sync(0xFFFFFFFFu, in);
    const int64_t i = row0 + warp;
    if (i < r.rows) {
        if (mask >> warp & 1u) {
            const int at = base + __popc(mask & ((1u << warp) - 1u));
            copy_row(static_cast<uint16_t *>(r.gathered) + at * r.gathered_stride, static_cast<const uint16_t *>(r.hidden) + i * r.hidden_stride,
                     r.cols, r.gathered_stride, r.vectors, lane);
            if (lane == 0) {
                r.index[at] = (int32_t)i;
                r.label[at] = (int32_t)load_id(r.labels, i, r.ids_dtype);
                r.w[at] = r.weight ? r.weight[i] : 1.0f;
            }
        } else {
            if (lane == 0) r.row_loss[i] = 0.0f;
            if (r.dhidden) {
                uint16_t *out = static_cast<uint16_t *>(r.dhidden) + i * r.dhidden_stride;
                if (r.dhidden_vectors) copy_row(out, nullptr, r.cols, r.cols, true, lane);
                else
                    for (int64_t c = lane; c < r.cols; c += 32) out[c] = 0;
            }
        }
    }
    if (!behind) return;
    // rows up to the end of a step of the sums over rows count there, with factors of zero
    const int first = (int)(((r.rows + kGatherRows - 1) / kGatherRows)), at = base + ((int)blockIdx.x - first) * kGatherRows + warp;
    if (at < (base + kTileK - 1) / kTileK * kTileK)
        copy_row(static_cast<uint16_t *>(r.gathered) + at * r.gathered_stride, nullptr, r.cols, r.gathered_stride, true, lane);
    if (blockIdx.x != gridDim.x - 1) return;
    const int live = base;
    if (threadIdx.x == 0) {
        const float unit = (top > 0.0f && top < kInf ? top : 1.0f) * (r.fp16 ? 0x1p-15f : 1.0f);
        r.control->live = live;
        r.control->unit = fminf(fmaxf(unit, 0x1p-126f), 0x1p126f);
        r.control->ticket = 0;
        r.control->gave_up = 0;
    }
}

// P from logits that were kept: 8 columns of a row a thread, rows up to whole steps of the sums over them.
template <typename T>
__global__ void __launch_bounds__(256) prob_kernel(const __grid_constant__ Product p)
{
    grid_dependency_wait();
    grid_dependency_release();
    const int live = p.control->live;
    const int64_t groups = p.prob_stride / 8, all = (int64_t)((live + kTileK - 1) / kTileK * kTileK) * groups;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / groups, c = (i - row * groups) * 8;
        float f[8] = {};
        if (row < live) {
            const int64_t label = p.label[row] - c;
            const float4 t = p.terms[row];
            uint32_t w[8];
            load32(p.kept + row * p.prob_stride + c, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float q = exp2_fast(fmaf(__uint_as_float(w[j]) - t.x, kLog2e, -t.y));
                if (label == j) q = t.w;
                f[j] = c + j < p.vocab ? q * t.z : 0.0f;
                if (label == j) p.residual[row] = f[j] - to_f32(from_f32<T>(f[j]));
            }
        }
        T *to = static_cast<T *>(p.prob) + row * p.prob_stride + c;
        for (int plane = 0;; ++plane) {
            const uint4 w = pack<T>(f);
            *reinterpret_cast<uint4 *>(to) = w;
            if (plane + 1 == p.planes) break;
            to += (int64_t)p.rows_pad * p.prob_stride;
            float held[8];
            unpack<T>(w, held);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] -= held[j];
        }
    }
}

struct Join {
    Control *control;
    const float2 *stats;
    const float *label_logit, *w;
    const int32_t *index;
    float4 *terms;
    float *row_loss, *loss;
    double *sums;                         // [blocks]
    int32_t rows_pad, halves;
    int64_t rows;
};

constexpr int kJoinWarps = 32;

// Joins the tiles' statistics, 32 rows a block (a lane each, the tiles dealt out to warps); the
// block that comes last adds up the loss.  After a wait that ran out both are NaN, masked rows too.
__global__ void __launch_bounds__(32 * kJoinWarps) join_kernel(const __grid_constant__ Join j)
{
    __shared__ float2 s_part[kJoinWarps][32];
    __shared__ double s_sum[kJoinWarps];
    __shared__ bool s_last;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_dependency_wait();
    grid_dependency_release();
    const int live = j.control->live;
    const int row = blockIdx.x * 32 + lane;
    if (j.control->gave_up) {
        if (warp == 0 && row < j.rows) j.row_loss[row] = kNan;
        if (blockIdx.x == 0 && threadIdx.x == 0) *j.loss = kNan;
        return;
    }
    float top = -kInf, sum = 0.0f;
    if (blockIdx.x * 32 < live) {
        // rows behind the last one are read as they lie in scratch, and dropped
        const float2 *at = j.stats + row;
        for (int t0 = warp; t0 < j.halves; t0 += 8 * kJoinWarps) {
            float2 v[8];
            float most = top;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int t = t0 + u * kJoinWarps;
                v[u] = t < j.halves && row < live ? at[(int64_t)t * j.rows_pad] : make_float2(-kInf, 0.0f);
                most = fmaxf(most, v[u].x);
            }
            const float ref = most == -kInf ? 0.0f : most;
            sum *= exp2_fast((top - ref) * kLog2e);
#pragma unroll
            for (int u = 0; u < 8; ++u) sum += v[u].y == 0.0f ? 0.0f : v[u].y * exp2_fast((v[u].x - ref) * kLog2e);
            top = most;
        }
    }
    s_part[warp][lane] = make_float2(top, sum);
    __syncthreads();
    if (warp == 0) {
        double mine = 0.0;
        if (row < live) {
            float most = -kInf;
            for (int i = 0; i < kJoinWarps; ++i) most = fmaxf(most, s_part[i][lane].x);
            float others = 0.0f;
            for (int i = 0; i < kJoinWarps; ++i)
                others += s_part[i][lane].y == 0.0f ? 0.0f : s_part[i][lane].y * exp2_fast((s_part[i][lane].x - most) * kLog2e);
            const float w = j.w[row], below = most - j.label_logit[row], own = exp2_fast(-below * kLog2e), total = others + own;
            const float loss = own > 0.5f ? log1pf(others / own) : below + logf(total);
            j.row_loss[j.index[row]] = loss;
            j.terms[row] = make_float4(most, log2f(total), w / j.control->unit, -(others / total));
            mine = (double)w * (double)loss;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xFFFFFFFFu, mine, o);
        if (lane == 0) {
            j.sums[blockIdx.x] = mine;
            __threadfence();
            s_last = atomicAdd(&j.control->ticket, 1u) == gridDim.x - 1;
        }
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    double all = 0.0;
    for (unsigned i = threadIdx.x; i < gridDim.x; i += 32 * kJoinWarps) all += __ldcg(j.sums + i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, o);
    if (lane == 0) s_sum[warp] = all;
    __syncthreads();
    if (threadIdx.x == 0) {
        all = 0.0;
        for (int i = 0; i < kJoinWarps; ++i) all += s_sum[i];
        *j.loss = (float)all;
    }
}

struct Finish {
    Control *control;
    const float *part, *residual;
    const int32_t *index, *label;
    const void *table;
    int64_t table_stride;
    void *dhidden, *table_grad;
    float *row_loss, *loss;
    int64_t rows, vocab, cols, dhidden_stride, grad_stride, part_stride;
    int32_t rows_pad, splits, grad_dtype, vectors, table_vectors, accumulate;
    float grad_scale;
};

constexpr int kFinishThreads = 128;

// dH from its parts, and what the label's P lost in its rounding times the label's row: where one row
// of the table outweighs the others, that rounding would be all of dH's.  dW where no row took part: zeros, unless it
// is added to.  NaN everywhere after a wait that ran out.
template <typename T>
__global__ void __launch_bounds__(kFinishThreads) finish_kernel(const __grid_constant__ Finish f)
{
    grid_dependency_wait();
    const int live = f.control->live;
    const bool gave_up = f.control->gave_up != 0;
    const int64_t me = (int64_t)blockIdx.x * kFinishThreads + threadIdx.x, all = (int64_t)gridDim.x * kFinishThreads;
    if (f.table_grad && (gave_up || (live == 0 && !f.accumulate)))
        for (int64_t i = me; i < f.vocab * f.cols; i += all)
            store_any(f.table_grad, i / f.cols * f.grad_stride + i % f.cols, f.grad_dtype, gave_up ? kNan : 0.0f);
    if (gave_up) {
        for (int64_t i = me; i < f.rows; i += all) f.row_loss[i] = kNan;
        if (me == 0) *f.loss = kNan;
        if (f.dhidden)
            for (int64_t i = me; i < f.rows * f.cols; i += all) static_cast<T *>(f.dhidden)[i / f.cols * f.dhidden_stride + i % f.cols] = from_f32<T>(kNan);
        return;
    }
    if (!f.dhidden) return;
    const float scale = f.grad_scale * f.control->unit;
    // a warp has 256 columns; where there are many parts, the block's four share them
    __shared__ float s_sum[3][32][9];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool share = f.splits >= 8;
    const int64_t per_row = (f.cols + 255) / 256, step = (int64_t)f.rows_pad * f.part_stride, items = live * per_row;
    for (int64_t first = share ? blockIdx.x : (int64_t)blockIdx.x * 4; first < items; first += share ? gridDim.x : (int64_t)gridDim.x * 4) {
        const int64_t item = share ? first : first + warp, row = item / per_row, c = (item - row * per_row) * 256 + lane * 8;
        const bool in = item < items && c < f.cols;
        float sum[8] = {};
        if (in) {
            const float *at = f.part + row * f.part_stride + c;
#pragma unroll 8
            for (int k = share ? warp : 0; k < f.splits; k += share ? 4 : 1) {
                uint32_t w[8];
                load32(at + k * step, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] += __uint_as_float(w[i]);
            }
        }
        if (share) {
            if (warp > 0)
#pragma unroll
                for (int i = 0; i < 8; ++i) s_sum[warp - 1][lane][i] = sum[i];
            __syncthreads();
            if (warp == 0)
#pragma unroll
                for (int w = 0; w < 3; ++w)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[i] += s_sum[w][lane][i];
            __syncthreads();
        }
        if (!in || (share && warp > 0)) continue;
        T *out = static_cast<T *>(f.dhidden) + (int64_t)f.index[row] * f.dhidden_stride + c;
        const T *at = static_cast<const T *>(f.table) + (int64_t)f.label[row] * f.table_stride + c;
        const float residual = f.residual[row];
        float w[8] = {};
        if (f.table_vectors && c + 8 <= f.cols) {
            unpack<T>(*reinterpret_cast<const uint4 *>(at), w);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < f.cols) w[i] = to_f32(at[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = fmaf(residual, w[i], sum[i]) * scale;
        if (f.vectors && c + 8 <= f.cols) {
            *reinterpret_cast<uint4 *>(out) = pack<T>(sum);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < f.cols) out[i] = from_f32<T>(sum[i]);
        }
    }
}

// A piece of a table whose rows cannot be copied as they are, rows padded to whole steps.
__global__ void __launch_bounds__(256) pack_kernel(const uint16_t *table, int64_t stride, int64_t rows, int64_t cols, uint16_t *out, int64_t out_stride)
{
    grid_dependency_wait();
    grid_dependency_release();
    for (int64_t v = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); v < rows; v += (int64_t)gridDim.x * 8)
        copy_row(out + v * out_stride, table + v * stride, cols, out_stride, false, threadIdx.x & 31);
}

// ---- host ---------------------------------------------------------------------------------

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Where everything lies in scratch.
struct Layout {
    int64_t rows_pad, ld, pieces, piece, splits, planes, part_stride, halves;
    bool packed, keep;
    uint64_t control, counts, index, label, w, label_logit, terms, residual, sums, stats, gathered, kept, prob, part, table, bytes;
};

constexpr int64_t kPieceBytes = int64_t(256) << 20;   // of P, unless rows are so many that pieces would get short
constexpr int64_t kShortPiece = 4096;
// Logits are kept from the statistics to P where multiplying again would cost more than writing and
// reading them, 8 bytes each, which goes by the row's length; the bytes are a limit of what scratch
// should take, all logits of 1025 x 50257 with some left.  Kept / again 596 / 655 us for 1025 x 50257 x 1600 (fp16,
// fp32 gradient), 281 / 343 us for 300 x 50257 x 2048, 88 / 101 us for 63 x 50257 x 768, but
// 146 / 137 us for 500 x 50257 x 512 and 198 / 171 us for 1000 x 50257 x 256.
constexpr int64_t kKeptBytes = int64_t(256) << 20;
constexpr int64_t kKeptCols = 768;        // with shorter rows only a quarter of that, which L2 may hold, is worth it

constexpr int kSms = 148;                 // of a B200: sums are split alike on every device

Layout layout(int64_t rows, int64_t vocab, int64_t cols, int32_t dtype, int32_t grad_dtype, bool gradients, bool packed)
{
    const int units = rows > kRowsOfCta ? kSms / 2 : kSms;   // blocks, or pairs of them, that work at a time
    Layout l = {};
    l.packed = packed;
    l.rows_pad = up(rows > 0 ? rows : 1, kRowPad);
    l.ld = up(cols, kTileK);
    l.halves = (vocab + kEndCols - 1) / kEndCols;
    l.planes = grad_dtype != SO_DTYPE_FP32 ? 1 : dtype == SO_DTYPE_BF16 ? 3 : 2;
    l.piece = up(vocab, kTileN);
    if (gradients || packed) {
        int64_t c = kPieceBytes / (2 * l.planes * l.rows_pad) / kTileN * kTileN;
        if (c < kShortPiece) c = kShortPiece;
        if (c < l.piece) l.piece = c;
    }
    l.pieces = (vocab + l.piece - 1) / l.piece;
    l.part_stride = up(cols, kTileN);
    // parts of the sums over the vocabulary: as many as fill the units best, each split costing
    // its write and reading
    const int64_t tile_m = rows > kRowsOfCta ? 2 * kRowsOfCta : kRowsOfCta;
    const int64_t tiles = up(rows > 0 ? rows : 1, tile_m) / tile_m * (l.part_stride / kTileN);
    l.splits = 1;
    double best = 1e30;
    for (int64_t s = 1; s <= 64 && s * 4 <= l.piece / kTileK; ++s) {
        const double cost = (double)((tiles * s + units - 1) / units) / (double)s * (1.0 + 0.01 * (double)(s - 1));
        if (cost < best * 0.999) best = cost, l.splits = s;
    }
    uint64_t at = 0;
    const auto take = [&](uint64_t bytes) {
        const uint64_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    const uint64_t rp = (uint64_t)l.rows_pad;
    l.control = take(sizeof(Control));
    l.counts = take((rp / kChunk + 1) * sizeof(float2));
    l.index = take(rp * 4);
    l.label = take(rp * 4);
    l.w = take(rp * 4);
    l.label_logit = take(rp * 4);
    l.terms = take(rp * sizeof(float4));
    l.residual = take(rp * 4);
    l.sums = take(rp / 32 * 8);
    l.stats = take(rp * (uint64_t)l.halves * 8);
    l.gathered = take(rp * (uint64_t)l.ld * 2);
    l.keep = gradients && l.pieces == 1 && l.rows_pad * l.piece * 4 <= (cols >= kKeptCols ? kKeptBytes : kKeptBytes / 4);
    if (l.keep) l.kept = take(rp * (uint64_t)l.piece * 4);
    if (gradients) {
        l.prob = take(rp * (uint64_t)(l.planes * l.piece) * 2);
        l.part = take(rp * (uint64_t)(l.splits * l.part_stride) * 4);
    }
    if (packed) l.table = take((uint64_t)(l.piece * l.ld) * 2);
    l.bytes = at;
    return l;
}

using EncodeFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                              const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

CUtensorMapDataType type_of(int32_t dtype)
{
    return dtype == SO_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : dtype == SO_DTYPE_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
}

EncodeFn encoder()
{
    static std::atomic<void *> found{nullptr};
    void *fn = found.load(std::memory_order_acquire);
    if (!fn) {
        cudaDriverEntryPointQueryResult how;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &how) != cudaSuccess || how != cudaDriverEntryPointSuccess) return nullptr;
        found.store(fn, std::memory_order_release);
    }
    return reinterpret_cast<EncodeFn>(fn);
}

// A matrix, copied 128 bytes of `box_rows` rows at a time.
bool make_map(CUtensorMap *m, const void *base, int32_t dtype, int64_t rows, int64_t cols, int64_t stride, int box_rows)
{
    const EncodeFn fn = encoder();
    if (!fn) return false;
    const int size = elem_size(dtype);
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)(stride * size)};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / size), (cuuint32_t)box_rows}, step[2] = {1, 1};
    return fn(m, type_of(dtype), 2, const_cast<void *>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// One of 16-bit elements as groups of 64 columns (the stride is a multiple of 64), 64 rows of two groups at a time.
bool make_group_map(CUtensorMap *m, const void *base, int32_t dtype, int64_t rows, int64_t cols, int64_t stride)
{
    const EncodeFn fn = encoder();
    if (!fn) return false;
    const cuuint64_t dims[3] = {64, (cuuint64_t)rows, (cuuint64_t)(cols + 63) / 64}, strides[2] = {(cuuint64_t)stride * 2, 128};
    const cuuint32_t box[3] = {64, kTileK, 2}, step[3] = {1, 1, 1};
    return fn(m, type_of(dtype), 3, const_cast<void *>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int kMode, int kCtas>
so_status launch_product(const Maps &maps, const Product &p, int units, cudaStream_t st)
{
    static std::atomic<bool> ready[kMaxDevices];
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return SO_ERR_CUDA;
    const auto kernel = product_kernel<T, kMode, kCtas>;
    if (!ready[dev].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<kCtas>::kBytes) != cudaSuccess) return SO_ERR_CUDA;
        ready[dev].store(true, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * kCtas));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Shape<kCtas>::kBytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kCtas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, maps, p) == cudaSuccess ? SO_OK : SO_ERR_CUDA;
}

struct Call {
    const void *hidden, *table, *labels;
    const float *weight;
    int64_t hidden_stride, table_stride, rows, vocab, cols, dhidden_stride, dtable_stride;
    int32_t ids_dtype, dtype, grad_dtype, accumulate;
    float grad_scale;
    void *dhidden, *dtable;
    float *row_loss, *loss;
};

#define SO_TRY(x) do { const so_status so_try_ = (x); if (so_try_ != SO_OK) return so_try_; } while (0)

template <typename T, int kCtas>
so_status run(const Call &c, const Layout &l, char *scratch, int sms, cudaStream_t st)
{
    const bool gradients = c.dhidden || c.dtable;
    const int units = sms / kCtas;
    Control *control = reinterpret_cast<Control *>(scratch + l.control);
    int32_t *index = reinterpret_cast<int32_t *>(scratch + l.index), *label = reinterpret_cast<int32_t *>(scratch + l.label);
    float *w = reinterpret_cast<float *>(scratch + l.w);
    Rows r = {};
    r.control = control, r.hidden = c.hidden, r.hidden_stride = c.hidden_stride, r.labels = c.labels, r.ids_dtype = c.ids_dtype, r.weight = c.weight;
    r.rows = c.rows, r.vocab = c.vocab, r.cols = c.cols, r.rows_pad = (int32_t)l.rows_pad;
    r.gathered = scratch + l.gathered, r.gathered_stride = l.ld, r.index = index, r.label = label, r.w = w, r.row_loss = c.row_loss;
    r.dhidden = c.dhidden, r.dhidden_stride = c.dhidden_stride, r.fp16 = c.dtype == SO_DTYPE_FP16;
    r.vectors = aligned(c.hidden, 16) && (c.rows <= 1 || c.hidden_stride % 8 == 0);
    r.dhidden_vectors = aligned(c.dhidden, 16) && c.cols % 8 == 0 && (c.rows <= 1 || c.dhidden_stride % 8 == 0);
    r.counts = c.rows > kChunk ? reinterpret_cast<float2 *>(scratch + l.counts) : nullptr;
    if (r.counts) SO_TRY(launch(count_kernel, (unsigned)((c.rows + kChunk - 1) / kChunk), kGatherThreads, 0, st, false, r));
    SO_TRY(launch(gather_kernel, (unsigned)((c.rows + kGatherRows - 1) / kGatherRows + kTileK / kGatherRows), kGatherThreads, 0, st, r.counts != nullptr, r));

    Product p = {};
    p.control = control, p.vocab = c.vocab, p.cols = c.cols, p.rows_pad = (int32_t)l.rows_pad, p.splits = (int32_t)l.splits, p.planes = (int32_t)l.planes;
    p.label = label;
    p.label_logit = reinterpret_cast<float *>(scratch + l.label_logit);
    float4 *terms = reinterpret_cast<float4 *>(scratch + l.terms);
    p.terms = terms;
    p.residual = reinterpret_cast<float *>(scratch + l.residual);
    p.stats = reinterpret_cast<float2 *>(scratch + l.stats);
    p.prob = scratch + l.prob, p.prob_stride = l.piece;
    p.kept = l.keep ? reinterpret_cast<float *>(scratch + l.kept) : nullptr;
    p.part = reinterpret_cast<float *>(scratch + l.part), p.part_stride = l.part_stride;
    p.table_grad = c.dtable, p.grad_stride = c.dtable_stride, p.grad_dtype = c.grad_dtype, p.accumulate = c.accumulate, p.grad_scale = c.grad_scale;
    p.table_groups = l.packed || c.cols % 64 == 0;           // a row's last group ends with it
    p.patience = patience();

    // the table as it is, or a packed piece of it
    const uint16_t *table = static_cast<const uint16_t *>(c.table);
    uint16_t *packed = reinterpret_cast<uint16_t *>(scratch + l.table);
    Maps logits, gradient;                // of the products for z, and of those with P
    CUtensorMap table_m;
    p.want_hidden = c.dhidden != nullptr;
    if (!make_map(&logits.a, r.gathered, c.dtype, l.rows_pad, c.cols, l.ld, kRowsOfCta) || !make_group_map(&gradient.b2, r.gathered, c.dtype, l.rows_pad, c.cols, l.ld))
        return SO_ERR_CUDA;
    logits.out = logits.a2 = logits.b2 = logits.out2 = logits.a;
    if (l.keep && !make_map(&logits.out, p.kept, SO_DTYPE_FP32, l.rows_pad, l.piece, l.piece, 32)) return SO_ERR_CUDA;
    const auto table_maps = [&](int64_t rows) {
        const void *at = l.packed ? static_cast<const void *>(packed) : c.table;
        const int64_t stride = l.packed ? l.ld : c.vocab == 1 ? l.ld : c.table_stride;
        return make_map(&logits.b, at, c.dtype, rows, c.cols, stride, 128) &&
               (p.table_groups ? make_group_map(&table_m, at, c.dtype, rows, c.cols, stride) : make_map(&table_m, at, c.dtype, rows, c.cols, stride, kTileK));
    };
    const auto pack_piece = [&](int64_t first, int64_t width) {
        return launch(pack_kernel, (unsigned)(4 * sms), 256, 0, st, true, table + first * c.table_stride, c.table_stride, width, c.cols, packed, l.ld);
    };

    if (l.packed) {
        for (int64_t first = 0; first < c.vocab; first += l.piece) {
            const int64_t width = c.vocab - first < l.piece ? c.vocab - first : l.piece;
            SO_TRY(pack_piece(first, width));
            if (!table_maps(width)) return SO_ERR_CUDA;
            Product q = p;
            q.first = first, q.width = width, q.table_row = 0;
            SO_TRY((launch_product<T, kStats, kCtas>(logits, q, units, st)));
        }
    } else {
        if (!table_maps(c.vocab)) return SO_ERR_CUDA;
        p.width = c.vocab;
        SO_TRY((launch_product<T, kStats, kCtas>(logits, p, units, st)));
    }
    Join j = {control, p.stats, p.label_logit, w, index, terms, c.row_loss, c.loss, reinterpret_cast<double *>(scratch + l.sums), (int32_t)l.rows_pad, (int32_t)l.halves, c.rows};
    SO_TRY(launch(join_kernel, (unsigned)(l.rows_pad / 32), 32 * kJoinWarps, 0, st, true, j));
    if (gradients) {
        // (what a warp copies out is 32 rows)
        if (!make_map(&gradient.a, p.prob, c.dtype, l.rows_pad * l.planes, l.piece, l.piece, kRowsOfCta) ||
            !make_group_map(&gradient.a2, p.prob, c.dtype, l.rows_pad * l.planes, l.piece, l.piece) ||
            (!l.keep && !make_map(&logits.out, p.prob, c.dtype, l.rows_pad * l.planes, l.piece, l.piece, 32)) ||
            !make_map(&gradient.out, p.part, SO_DTYPE_FP32, l.rows_pad * l.splits, l.part_stride, l.part_stride, 32))
            return SO_ERR_CUDA;
        gradient.out2 = gradient.out;
        const int grad_size = elem_size(c.grad_dtype);
        const int64_t grad_stride = c.vocab == 1 ? l.ld : c.dtable_stride;   // (of one row: any)
        p.grad_boxes = c.dtable && (!c.accumulate || c.grad_dtype == SO_DTYPE_FP32) && aligned(c.dtable, 16) && grad_stride * grad_size % 16 == 0;
        if (p.grad_boxes && !make_map(&gradient.out2, c.dtable, c.grad_dtype, c.vocab, c.cols, grad_stride, 32)) return SO_ERR_CUDA;
        for (int64_t first = 0; first < c.vocab; first += l.piece) {
            Product q = p;
            q.first = q.table_row = first;
            q.width = c.vocab - first < l.piece ? c.vocab - first : l.piece;
            q.begin = first == 0;
            if (l.packed) {
                if (l.pieces > 1) SO_TRY(pack_piece(first, q.width));   // (one piece is still there)
                if (!table_maps(q.width)) return SO_ERR_CUDA;
                q.table_row = 0;
            }
            if (l.keep) SO_TRY(launch(prob_kernel<T>, (unsigned)(8 * sms), 256, 0, st, true, q));
            else SO_TRY((launch_product<T, kProb, kCtas>(logits, q, units, st)));
            gradient.b = table_m;
            SO_TRY((launch_product<T, kGradients, kCtas>(gradient, q, units, st)));
        }
    }
    if (!gradients) return SO_OK;
    Finish f = {control, p.part, p.residual, index, label, c.table, c.table_stride, c.dhidden, c.dtable, c.row_loss, c.loss, c.rows, c.vocab, c.cols, c.dhidden_stride, c.dtable_stride, l.part_stride,
                (int32_t)l.rows_pad, (int32_t)l.splits, c.grad_dtype, r.dhidden_vectors, !l.packed, c.accumulate, c.grad_scale};
    return launch(finish_kernel<T>, (unsigned)(16 * sms), kFinishThreads, 0, st, true, f);
}

so_status check_sizes(int64_t rows, int64_t vocab, int64_t cols, int32_t dtype, int32_t grad_dtype)
{
    if ((dtype != SO_DTYPE_BF16 && dtype != SO_DTYPE_FP16) || !valid_dtype(grad_dtype)) return SO_ERR_INVALID_ARG;
    if (rows < 0 || rows > SO_LINEAR_MAX_ROWS || vocab < 1 || vocab > SO_LINEAR_MAX_VOCAB || cols < 1 || cols > SO_LINEAR_MAX_COLS) return SO_ERR_INVALID_ARG;
    return SO_OK;
}

bool needs_packing(const void *table, int64_t stride, int64_t vocab) { return !aligned(table, 16) || (vocab > 1 && stride % 8 != 0); }

}  // namespace

extern "C" {

so_status so_linear_cross_entropy_scratch(int64_t rows, int64_t vocab, int64_t cols, int32_t dtype, int32_t grad_dtype, int32_t gradients,
                                          int32_t packed, uint64_t *bytes)
{
    if (!bytes || (gradients != 0 && gradients != 1) || (packed != 0 && packed != 1)) return SO_ERR_INVALID_ARG;
    SO_TRY(check_sizes(rows, vocab, cols, dtype, grad_dtype));
    *bytes = layout(rows, vocab, cols, dtype, grad_dtype, gradients != 0, packed != 0).bytes;
    return SO_OK;
}

so_status so_linear_cross_entropy(const void *hidden, int64_t hidden_stride, const void *table, int64_t table_stride, const void *labels,
                                  int32_t ids_dtype, const float *weight, int64_t rows, int64_t vocab, int64_t cols, int32_t dtype,
                                  double grad_scale, void *dhidden, int64_t dhidden_stride, void *dtable, int64_t dtable_stride,
                                  int32_t grad_dtype, int32_t accumulate, float *row_loss, float *loss, void *scratch,
                                  uint64_t scratch_bytes, void *stream)
{
    SO_TRY(check_sizes(rows, vocab, cols, dtype, grad_dtype));
    if (!valid_ids(ids_dtype) || (accumulate != 0 && accumulate != 1) || !std::isfinite(grad_scale) || !std::isfinite((float)grad_scale)) return SO_ERR_INVALID_ARG;
    if (!loss || !aligned(loss, 4) || (rows > 0 && !row_loss) || !aligned(row_loss, 4) || !aligned(weight, 4)) return SO_ERR_INVALID_ARG;
    if (!table || !aligned(table, 2) || !valid_extent(vocab, table_stride) || !valid_out_stride(vocab, table_stride, cols)) return SO_ERR_INVALID_ARG;
    if (dtable && (!aligned(dtable, elem_size(grad_dtype)) || !valid_extent(vocab, dtable_stride) || !valid_out_stride(vocab, dtable_stride, cols))) return SO_ERR_INVALID_ARG;
    if (rows > 0) {
        if (!hidden || !aligned(hidden, 2) || !valid_extent(rows, hidden_stride) || !valid_in_stride(rows, hidden_stride, cols)) return SO_ERR_INVALID_ARG;
        if (!labels || !aligned(labels, ids_dtype == SO_IDS_INT64 ? 8 : 4)) return SO_ERR_INVALID_ARG;
        if (dhidden && (!aligned(dhidden, 2) || !valid_extent(rows, dhidden_stride) || !valid_out_stride(rows, dhidden_stride, cols))) return SO_ERR_INVALID_ARG;
    }
    // dhidden may take hidden's place, row for row; otherwise the gradients are apart
    const int size = elem_size(dtype);
    const Span at_hidden(hidden, rows, hidden_stride, cols, size), at_table(table, vocab, table_stride, cols, size),
        at_dhidden(dhidden, dhidden ? rows : 0, dhidden_stride, cols, size), at_dtable(dtable, dtable ? vocab : 0, dtable_stride, cols, elem_size(grad_dtype));
    if ((!at_dhidden.same(at_hidden) && overlap(at_dhidden, at_hidden)) || overlap(at_dhidden, at_table) || overlap(at_dtable, at_hidden) ||
        overlap(at_dtable, at_table) || overlap(at_dtable, at_dhidden))
        return SO_ERR_INVALID_ARG;
    if (!scratch || !aligned(scratch, 256)) return SO_ERR_INVALID_ARG;
    const Layout l = layout(rows, vocab, cols, dtype, grad_dtype, dhidden || dtable, needs_packing(table, table_stride, vocab));
    if (scratch_bytes < l.bytes) return SO_ERR_INVALID_ARG;
    int sms;
    SO_TRY(device_sms(&sms));
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const Call c = {hidden, table, labels, weight, hidden_stride, table_stride, rows, vocab, cols, dhidden_stride, dtable_stride, ids_dtype, dtype, grad_dtype,
                    accumulate, (float)grad_scale, rows > 0 ? dhidden : nullptr, dtable, row_loss, loss};
    if (dtype == SO_DTYPE_BF16) return rows > kRowsOfCta ? run<bf16_t, 2>(c, l, static_cast<char *>(scratch), sms, st) : run<bf16_t, 1>(c, l, static_cast<char *>(scratch), sms, st);
    return rows > kRowsOfCta ? run<f16_t, 2>(c, l, static_cast<char *>(scratch), sms, st) : run<f16_t, 1>(c, l, static_cast<char *>(scratch), sms, st);
}

}  // extern "C"
