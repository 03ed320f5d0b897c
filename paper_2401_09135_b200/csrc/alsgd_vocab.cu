// Losses over a vocabulary whose logits are never kept: the cross entropy with a label per row, and the distillation from a
// teacher's highest logits, which is the same loss with a few weighted labels per row.
//
//     z[i][j] = scale x_i . w_j,   lse_i = log sum_j exp z[i][j],   loss_i = sum_k t_ik (log t_ik - z[i][index_ik] + lse_i)
//     dz[i][j] = dloss_i scale (exp(z[i][j] - lse_i) - sum_k t_ik [index_ik = j]),   dx = dz w,   dw = dz^T x
//
// Forward: tiles of 256 rows x 256 words; a tile's maxima, sums of exponentials and the labels' logits leave the chip, the
// logits do not.  Backward, a piece of the vocabulary at a time: the logits again, dz of the piece in bf16, then dx += dz w and
// dw = dz^T x in one launch.
//
// The rows that take part are gathered first (a padded batch pays for its tokens, not for its padding; what the other rows
// hold reaches nothing) and everything behind works on their number, which only the device knows.  Few rows and short passes stay
// where they are: there is little to save, and the two launches in front would cost more than the rest
// (77 rows x 32000 words x 384: forward 18.4 -> 15.4 us, backward 43.9 -> 35.3 us when this was measured).
//
// dz becomes an operand of the tensor cores and is rounded to bf16 for it.  The roundings of a sum's terms are independent of one
// another, as the terms are, so that a sum is off by about the same share as each of them, and that is about what rounding the
// result costs once more: together 0.0018 to 0.0023 of it, against 0.0017 (the squares add up).  Up to 64 rows the tiles have room for
// dz in two parts, the rounded value and what rounding left, as so many more rows, and only the result's rounding stays.  More rows
// are off as above and would take longer for it: from 65 to 128 a step more of every product (28.5 -> 33.0 us at 77 rows), many
// rows twice the products with dz, two thirds more in all.
//
// Times in this file are those of calls captured in a loop over one set of inputs: what fits the L2 is found there.
//
// The matrix products bound it.  Two blocks of a cluster form one 256 x 256 tile: each holds 128 of its rows and copies half
// of either operand, so that a tile needs half of the shared memory traffic of two single ones.  (Up to 128 rows there is no
// second half of the rows: every block then forms logits by itself, 128 x 256.)  One warp copies, one
// issues products, sixteen take the finished tile out of tensor memory while the next one is formed in its other half.
#include "../../include/alsgd.h"
#include "alsgd_ops.cuh"
#include "alsgd_pair.cuh"

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>

namespace {

using namespace alsgd_ops;
using namespace alsgd_tc;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kTile = 256;             // rows and columns of a pair's tile
constexpr int kStep = 64;              // of the products' inner axis: one 128-byte row of bf16
constexpr int kPairs = kSMs / 2;
constexpr int kMaxTop = 128;
constexpr uint64_t kPieceBytes = 256ull << 20;
constexpr int kLeastPiece = 16;        // tiles of a piece: below that, adding dx up would cost more than the memory is worth
constexpr int kMaxSplits = 64;
constexpr uint64_t kPlainProducts = 9000000000;                // 13 us of them
constexpr int kMostRest = 64;          // rows up to which dz is kept to two bf16 parts

// ---------------------------------------------------------------------------------------------- rows that take part

struct Labels {
    const void* index;                 // [rows] or [rows][top]
    const void* teacher;               // [rows][top]; null: a label per row
    int wide, bf16;                    // 64-bit indices; teacher's type
    int rows, top, vocab;
};

__device__ __forceinline__ int label_at(const Labels& l, size_t i) {
    const int64_t v = l.wide ? static_cast<const int64_t*>(l.index)[i] : static_cast<const int32_t*>(l.index)[i];
    return v >= 0 && v < l.vocab ? (int)v : -1;
}
__device__ __forceinline__ float teacher_at(const Labels& l, size_t i) {
    return l.bf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(l.teacher)[i] << 16) : static_cast<const float*>(l.teacher)[i];
}

constexpr int kCountRows = 64;         // rows of a counting block

// Which rows take part: their number in each block of rows, and each row's place among its block's (-1 - place among those
// that do not).  A teacher's entries are read in a row by as many threads as a block may have.
__global__ void __launch_bounds__(1024) count_kernel(Labels l, int* block_count, int* place) {
    __shared__ int warp_count[kCountRows / 32];
    __shared__ uint8_t any[kCountRows];
    grid_dependency_sync();
    const int r0 = blockIdx.x * kCountRows, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    bool mine = false;
    if (l.teacher) {
        if (threadIdx.x < kCountRows) any[threadIdx.x] = 0;
        __syncthreads();
        const int n = max(0, min(kCountRows, l.rows - r0)) * l.top;
        const size_t from = (size_t)r0 * l.top;
#pragma unroll 8
        for (int i = threadIdx.x; i < n; i += 1024)
            if ((label_at(l, from + i) >= 0) & (teacher_at(l, from + i) != -INFINITY)) any[i / l.top] = 1;
        __syncthreads();
        if (threadIdx.x >= kCountRows) return;
        mine = any[threadIdx.x];
    } else {
        const int r = r0 + threadIdx.x;
        mine = r < l.rows && label_at(l, r) >= 0;
    }
    const uint32_t votes = __ballot_sync(~0u, mine);
    if (lane == 0) warp_count[warp] = __popc(votes);
    asm volatile("bar.sync 1, %0;" ::"n"(kCountRows) : "memory");
    int before = __popc(votes & ((1u << lane) - 1)), total = 0;
    for (int w = 0; w < kCountRows / 32; ++w) {
        if (w < warp) before += warp_count[w];
        total += warp_count[w];
    }
    place[r0 + threadIdx.x] = mine ? before : -1 - ((int)threadIdx.x - before);
    if (threadIdx.x == 0) block_count[blockIdx.x] = total;
}

constexpr int kPrefixThreads = 1024;
// Counting blocks up to which every block of the gathering kernel adds up all counts for itself: that saves a launch, and grows with
// the square of the rows.  Forward of one word x 8, labels and two entries a row, each block by itself and with prefixes: 16384 rows
// 16.6 and 17.6, 21.7 and 21.5 us; 32768 25.4 and 26.8, 35.1 and 32.7; 65536 38.8 and 39.6, 56.9 and 50.6; 131072 71 and 67,
// 107 and 89; 2^22 14400 and 2010, 15500 and 2850.
constexpr int kFewBlocks = 512;

// Rows that take part before each counting block's, in place of their number in it, and all of them: by one block, a run of counts
// a thread.
__global__ void __launch_bounds__(kPrefixThreads) prefix_kernel(int* block_count, int blocks, int* count) {
    __shared__ int warp_sum[kPrefixThreads / 32];
    grid_dependency_sync();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, run = (blocks + kPrefixThreads - 1) / kPrefixThreads;
    const int from = min(blocks, (int)threadIdx.x * run), to = min(blocks, from + run);
    int sum = 0;
#pragma unroll 8
    for (int i = from; i < to; ++i) sum += block_count[i];
    int before = sum;                                              // with the thread's own, at first
    for (int d = 1; d < 32; d *= 2) {
        const int other = __shfl_up_sync(~0u, before, d);
        if (lane >= d) before += other;
    }
    if (lane == 31) warp_sum[warp] = before;
    before -= sum;
    __syncthreads();
    int total = 0;
    for (int w = 0; w < kPrefixThreads / 32; ++w) {
        if (w < warp) before += warp_sum[w];
        total += warp_sum[w];
    }
    for (int i = from; i < to; ++i) {
        const int n = block_count[i];
        block_count[i] = before;
        before += n;
    }
    if (threadIdx.x == 0) *count = total;
}

struct GatherArgs {
    Labels l;
    const uint16_t* x;
    int64_t x_step;
    const float *lse, *dloss;          // backward only
    int64_t dloss_step;
    float scale;
    int padded, blocks, dim, tiles;    // rows in whole tiles; counting blocks; tiles of the vocabulary
    int direct;                        // where all rows take part, the products read x itself
    int plain;                         // rows stay in their places; only the teacher's lists are made
    uint16_t* dx;                      // backward only: zeros for the rows that take no part
    int64_t dx_step;
    const int *block_count, *place;
    int summed;                        // block_count: rows that take part before the block's; count is there
    int* count;                        // one: rows that take part
    int* slot;                         // [rows]: place among them, or -1
    int* row;                          // [padded]: the row at a place
    uint16_t* xc;                      // [padded][dim]
    int* target;                       // [padded]: a label, or -1.  With a teacher and plain rows: 0, or -1
    int* index;                        // [padded][top] ascending, then places that take no part; teacher only
    float* weight;                     // [padded][top]
    float* entropy;                    // [padded]: sum t log t
    uint32_t* first;                   // [padded][tiles + 1]: four bytes, the entries below the first word of each quarter of a tile
    float *lse2, *coef;                // [padded]; backward only
};

constexpr int kGatherWarps = 4;

// One row's list by one warp: the teacher's softmax over the entries that take part, then the entries in ascending order of
// their words.  E: entries of a lane.
template <int E>
__device__ __forceinline__ void teacher_list(const GatherArgs& a, int r, int slot, bool used, int* keys, uint32_t* counts, int lane) {
    uint32_t* first = a.first + (size_t)slot * (a.tiles + 1);
    if (!used) {
        for (int t = lane; t <= a.tiles; t += 32) first[t] = 0;
        if (a.plain && lane == 0) a.target[slot] = -1;
        return;
    }
    constexpr int kNone = 1 << 30;                                 // behind every word's key
    const float c = a.scale * kLog2e;
    int key[E];                                                    // word, then the entry's number: all different
    float v[E], top = -INFINITY, sum = 0.0f;
    bool nan = false, any = false;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int k = lane + 32 * e;
        key[e] = kNone | k;
        v[e] = -INFINITY;
        if (k < a.l.top) {
            const size_t i = (size_t)r * a.l.top + k;
            const int word = label_at(a.l, i);
            const float t = teacher_at(a.l, i);
            if (word >= 0 && t != -INFINITY) {
                key[e] = word * kMaxTop + k;
                v[e] = t;
                any = true;
            }
        }
        keys[k] = key[e];                                          // those behind the list are behind every entry
        nan |= v[e] != v[e];
        top = fmaxf(top, v[e]);
    }
    any = __any_sync(~0u, any);
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
    if (__any_sync(~0u, nan)) top = NAN;
    if (!any) top = 0.0f;                                          // plain rows: the list is empty; so is everything below
    if (a.plain && lane == 0) a.target[slot] = any ? 0 : -1;
#pragma unroll
    for (int e = 0; e < E; ++e) sum += key[e] >= kNone ? 0.0f : exp2f((v[e] - top) * c);
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
    const float inv = 1.0f / sum, log_sum = logf(sum);
    int rank[E] = {};
    __syncwarp();
    for (int j = 0; j < a.l.top; j += 4) {
        const int4 q = *reinterpret_cast<const int4*>(keys + j);
#pragma unroll
        for (int e = 0; e < E; ++e) rank[e] += (q.x < key[e]) + (q.y < key[e]) + (q.z < key[e]) + (q.w < key[e]);
    }
    float entropy = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const bool is = key[e] < kNone;
        const float t = is ? exp2f((v[e] - top) * c) * inv : 0.0f;
        if (t != 0.0f) entropy += t * ((v[e] - top) * a.scale - log_sum);       // 0 log 0 = 0, also where the logarithm is -inf
        if (lane + 32 * e >= a.l.top) continue;
        const int word = is ? key[e] / kMaxTop : INT_MAX;
        a.index[(size_t)slot * a.l.top + rank[e]] = word;
        a.weight[(size_t)slot * a.l.top + rank[e]] = t;
    }
    for (int d = 16; d; d >>= 1) entropy += __shfl_xor_sync(~0u, entropy, d);
    if (lane == 0) a.entropy[slot] = entropy;
    // entries below each quarter of a tile: counted by quarters, 32 tiles at a time, then summed up: four quarters are the bytes
    // of a word (there are at most 128 entries), and so many ones side by side multiply it into its own running sums.  (A binary
    // search for every quarter took half of this kernel's instructions.)
    int below = 0;
    for (int t0 = 0; t0 <= a.tiles; t0 += 32) {
        counts[lane] = 0;
        __syncwarp();
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int at = key[e] / kMaxTop / (kTile / 4) + 1 - 4 * t0;        // counts for the quarters behind its own
            if (key[e] < kNone && at >= 0 && at < 128) atomicAdd(&counts[at / 4], 1u << (8 * (at & 3)));
        }
        __syncwarp();
        const uint32_t sums = counts[lane] * 0x01010101u;
        int before = sums >> 24;
        for (int d = 1; d < 32; d *= 2) {
            const int other = __shfl_up_sync(~0u, before, d);
            if (lane >= d) before += other;
        }
        const uint32_t off = below + before - (sums >> 24);
        if (t0 + lane <= a.tiles) first[t0 + lane] = sums + off * 0x01010101u;
        below += __shfl_sync(~0u, before, 31);
        __syncwarp();
    }
}

__device__ __forceinline__ void teacher_lists(const GatherArgs& a, int r, int slot, bool used, int* keys, uint32_t* counts, int lane) {
    static_assert(kMaxTop == 128, "one more case");
    if (a.l.top <= 32) teacher_list<1>(a, r, slot, used, keys, counts, lane);
    else if (a.l.top <= 64) teacher_list<2>(a, r, slot, used, keys, counts, lane);
    else teacher_list<4>(a, r, slot, used, keys, counts, lane);
}

// One warp per row: its place, its copy of x, its labels, what the gradient scales by.
__global__ void __launch_bounds__(32 * kGatherWarps) gather_kernel(const __grid_constant__ GatherArgs a) {
    __shared__ __align__(16) int s_index[kGatherWarps][kMaxTop];
    __shared__ uint32_t s_counts[kGatherWarps][32];
    __shared__ int s_sum[2];
    grid_dependency_sync();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int r0 = blockIdx.x * kGatherWarps, r = r0 + warp, block = r0 / kCountRows;     // a block's rows share a counting block
    if (a.plain) {
        teacher_lists(a, r, r, r < a.l.rows, s_index[warp], s_counts[warp], lane);
        return;
    }
    int before, count;
    if (a.summed) {
        before = a.block_count[block];
        count = *a.count;
    } else {
        int total = before = 0;
        for (int i = threadIdx.x; i < a.blocks; i += 32 * kGatherWarps) {
            const int n = a.block_count[i];
            total += n;
            if (i < block) before += n;
        }
        if (threadIdx.x < 2) s_sum[threadIdx.x] = 0;
        __syncthreads();
        before = __reduce_add_sync(~0u, before);
        total = __reduce_add_sync(~0u, total);
        if (lane == 0) {
            atomicAdd(&s_sum[0], before);          // whole numbers: any order
            atomicAdd(&s_sum[1], total);
        }
        __syncthreads();
        before = s_sum[0];
        count = s_sum[1];
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.count = count;
    }
    if (r >= a.padded) return;
    const int place = a.place[r];
    const bool used = place >= 0;
    // rows that do not take part fill the places behind; of those only the last tile's are looked at
    const int slot = used ? before + place : count + (block * kCountRows - before) + (-1 - place);
    if (r < a.l.rows) {
        if (lane == 0) a.slot[r] = used ? slot : -1;
        if (!used && a.dx)
            for (int c = 8 * lane; c < a.dim; c += 256) *reinterpret_cast<uint4*>(a.dx + r * a.dx_step + c) = make_uint4(0, 0, 0, 0);
    }
    if (slot >= (count + kTile - 1) / kTile * kTile) return;

    if (!(a.direct && count == a.l.rows)) {
        uint16_t* to = a.xc + (size_t)slot * a.dim;
        const uint16_t* from = a.x + r * a.x_step;
        for (int c = 8 * lane; c < a.dim; c += 256)
            *reinterpret_cast<uint4*>(to + c) = used ? *reinterpret_cast<const uint4*>(from + c) : make_uint4(0, 0, 0, 0);
    }
    if (lane == 0) {
        a.row[slot] = r;
        if (a.lse) {
            a.lse2[slot] = used ? a.lse[r] * kLog2e : 0.0f;
            a.coef[slot] = used ? a.dloss[r * a.dloss_step] * a.scale : 0.0f;
        }
        if (a.target) a.target[slot] = used ? label_at(a.l, r) : -1;
    }
    if (a.l.teacher) teacher_lists(a, r, slot, used, s_index[warp], s_counts[warp], lane);
}

// ---------------------------------------------------------------------------------------------- the pair's machinery

constexpr int kOutWarps = 16;          // that take tiles out, four for each quarter of the columns (or eight for every other tile)
constexpr int kThreads = 64 + 32 * kOutWarps;                 // and one that copies, one that issues products
constexpr int kOperandBytes = 16384;   // 128 x 64 values of an operand
constexpr int kAccColumns = 256;

template <int STAGES>
struct Bars {
    uint64_t full[STAGES], empty[STAGES], acc_full[2], acc_empty[2];
    uint32_t tmem, dead;
};

// What every warp of a block knows about the shared memory that it works on with the other block of its pair, or alone (TWO
// false): stages of SUBS operands A and one B, half of which the other block of a pair holds.
template <int STAGES, int SUBS, bool TWO>
struct Pair {
    static constexpr int kStageBytes = (SUBS + (TWO ? 1 : 2)) * kOperandBytes;
    uint32_t stage0, full, empty, acc_full, acc_empty, rank, tmem;
    volatile uint32_t* dead;

    __device__ __forceinline__ uint32_t a(int s) const { return stage0 + s * kStageBytes; }
    __device__ __forceinline__ uint32_t b(int s) const { return stage0 + s * kStageBytes + SUBS * kOperandBytes; }
    __device__ __forceinline__ void wait(uint32_t bar, uint32_t parity, uint32_t code) const {
        if (TWO) wait_pair(bar, parity, dead, code);
        else alsgd_tc::wait(bar, parity, dead, code);
    }
    __device__ __forceinline__ void wait_warp(uint32_t bar, uint32_t parity, uint32_t code) const {
        wait(bar, parity, code);
        __syncwarp();
    }
};

// Barriers and tensor memory of both blocks.  Full: one arrival (the first block's copying thread, for the bytes of
// both).  Empty, finished tile: one arrival, by the tensor core, on either block's.  Tile taken out: every warp of both blocks.
template <int STAGES, int SUBS, bool TWO>
__device__ __forceinline__ Pair<STAGES, SUBS, TWO> pair_begin(uint8_t* stages, Bars<STAGES>* bars) {
    Pair<STAGES, SUBS, TWO> p;
    p.stage0 = smem_u32(stages);
    p.full = smem_u32(bars->full);
    p.empty = smem_u32(bars->empty);
    p.acc_full = smem_u32(bars->acc_full);
    p.acc_empty = smem_u32(bars->acc_empty);
    p.rank = TWO ? cluster_rank() : 0;
    p.dead = &bars->dead;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            bar_init(p.full + 8 * s, 1);
            bar_init(p.empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            bar_init(p.acc_full + 8 * b, 1);
            bar_init(p.acc_empty + 8 * b, (TWO ? 2 : 1) * kOutWarps);
        }
        bars->dead = 0;
        bar_init_fence();
    }
    if (threadIdx.x / 32 == 1) {
        if (TWO) tmem_alloc_pair(smem_u32(&bars->tmem), 2 * kAccColumns);
        else tmem_alloc(smem_u32(&bars->tmem), 2 * kAccColumns);
    }
    tc_fence_before();
    __syncthreads();
    if (TWO) cluster_sync();
    tc_fence_after();
    p.tmem = bars->tmem;
    return p;
}

// The blocks leave together: neither's shared memory goes while the other's copies or products may touch it.
template <int STAGES, int SUBS, bool TWO>
__device__ __forceinline__ void pair_end(const Pair<STAGES, SUBS, TWO>& p) {
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (TWO) cluster_sync();
    if (threadIdx.x / 32 == 1) {
        tc_fence_after();
        if (TWO) tmem_free_pair(p.tmem, 2 * kAccColumns);
        else tmem_free(p.tmem, 2 * kAccColumns);
    }
}

// The copying thread's and the product thread's place in the ring of stages.
struct Ring {
    int stage = 0;
    uint32_t phase = 0;
    template <int STAGES>
    __device__ __forceinline__ void next() {
        if (++stage == STAGES) {
            stage = 0;
            phase ^= 1;
        }
    }
};

// Wait codes, one bit each.
enum : uint32_t { kWaitEmpty = 1, kWaitFull = 2, kWaitAccEmpty = 4, kWaitAccFull = 8 };

// Before the copying thread leaves, everything that it started has landed and been consumed (at once, unless it gave up).
template <int STAGES, int SUBS, bool TWO>
__device__ __forceinline__ void ring_drain(const Pair<STAGES, SUBS, TWO>& p, Ring ring) {
    for (int s = 0; s < STAGES; ++s) {
        drain(p.empty + 8 * ring.stage, ring.phase ^ 1);
        ring.next<STAGES>();
    }
}

// The products of `subs` tiles that share B: `steps` stages, each four products of 16 along the inner axis for either tile.
// a, b: descriptors of the i-th.  acc: tiles before these; tensor memory holds two, in turn.
template <int STAGES, int SUBS, bool TWO, typename DESC_A, typename DESC_B>
__device__ __forceinline__ void tile_products(const Pair<STAGES, SUBS, TWO>& p, Ring& ring, uint32_t acc, int subs, int steps, uint32_t desc, DESC_A a, DESC_B b) {
    for (int k = 0; k < steps; ++k) {
        p.wait(p.full + 8 * ring.stage, ring.phase, kWaitFull);
        tc_fence_after();
        const uint32_t sa = p.a(ring.stage), sb = p.b(ring.stage);
#pragma unroll
        for (int s = 0; s < SUBS; ++s) {
            if (s >= subs) break;
            const uint32_t buf = (acc + s) & 1;
            if (k == 0) {
                p.wait(p.acc_empty + 8 * buf, (((acc + s) >> 1) & 1) ^ 1, kWaitAccEmpty);
                tc_fence_after();
            }
#pragma unroll
            for (int i = 0; i < kStep / 16; ++i) {
                if (TWO) mma_ss_pair(p.tmem + buf * kAccColumns, a(sa + s * kOperandBytes, i), b(sb, i), desc, k || i);
                else mma_ss(p.tmem + buf * kAccColumns, a(sa + s * kOperandBytes, i), b(sb, i), desc, k || i);
            }
        }
        if (TWO) mma_commit_pair(p.empty + 8 * ring.stage);
        else mma_commit(p.empty + 8 * ring.stage);
        ring.next<STAGES>();
    }
    for (int s = 0; s < subs; ++s) {
        if (TWO) mma_commit_pair(p.acc_full + 8 * ((acc + s) & 1));
        else mma_commit(p.acc_full + 8 * ((acc + s) & 1));
    }
}

// The warp has taken its part of the tile out of tensor memory: of its columns a quarter, or a half, which counts twice.
template <int STAGES, int SUBS, bool TWO>
__device__ __forceinline__ void tile_taken(const Pair<STAGES, SUBS, TWO>& p, uint32_t acc, int lane, uint32_t quarters = 1) {
    tc_fence_before();
    __syncwarp();
    if (lane == 0) {
        if (TWO) bar_arrive_cluster(at_rank(p.acc_empty + 8 * (acc & 1), 0), quarters);
        else bar_arrive(p.acc_empty + 8 * (acc & 1), quarters);
    }
}

// ---------------------------------------------------------------------------------------------- logits

struct LogitArgs {
    CUtensorMap x, x_all, w;           // gathered rows, the rows as they are, words: boxes of 64 x 128
    const int* count;
    int all_rows;                      // with as many rows that take part, x_all is read; -1: never
    int plain, rows;                   // rows stay in their places
    int rest;                          // backward: where what rounding left of dz begins; 0: it is dropped
    Labels l;
    const float *lse, *dloss;          // backward, plain
    int64_t dloss_step;
    float scale;
    const uint16_t* x_rows;
    int64_t x_step;
    uint16_t* xc;
    int* row;
    int dim, vocab, top;
    int tile0, tiles, all_tiles;       // of the vocabulary: this launch's, all of them
    Divide by_group;                   // tiles of a group of row tiles
    float scale2;                      // scale * log2 e
    const int* target;
    const int* index;
    const float* weight;
    const uint8_t* first;
    int padded;
    float2* stats;                     // forward: [all_tiles][padded]: maximum of z / scale, sum of exponentials
    float* label_z;                    // forward: [padded][max(1, top)]: z / scale at the labels
    const float *lse2, *coef;          // backward
    uint8_t* dz;                       // backward: blocks of 128 rows x 64 words, [row block][word block][8 words][row]: a warp's
                                       // stores, the copies and the products of either direction all see 16-byte pieces in a row
};

constexpr int kGroup = 8;              // row tiles whose x stays in the L2 while the words go by

// Tiles in an order that lets the blocks at work share operands: the words' tiles in turn for a group of row tiles.
__device__ __forceinline__ void tile_at(const LogitArgs& a, int i, int row_tiles, int& rt, int& ct) {
    const int group = a.by_group(i), g0 = group * kGroup, n = min(kGroup, row_tiles - g0), rest = i - g0 * a.tiles;
    ct = n == kGroup ? rest / kGroup : n == 1 ? rest : rest / n;
    rt = g0 + rest - ct * n;
}

constexpr int kTurnTiles = 2;          // tiles of a pair from which on warps take turns

template <bool BACKWARD, bool TWO>
struct LogitSmem {
    static constexpr int kStages = !TWO ? 4 : BACKWARD ? 7 : 6;
    uint8_t stages[kStages * (TWO ? 2 : 3) * kOperandBytes];
    float2 stats[BACKWARD ? 1 : 2 * 4 * 128];                      // forward, of two tiles: by part of the columns, by row
    Bars<kStages> bars;
};

// One of 32 registers, chosen at run time.
__device__ __forceinline__ float pick(const uint32_t (&z)[32], int at) {
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) v = i == at ? __uint_as_float(z[i]) : v;
    return v;
}

// The arithmetic on a thread's 32 logits, two at a time where there is an instruction for it.
__device__ __forceinline__ float largest(const uint32_t (&z)[32], float m) {
    float part[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        part[g] = max3(__uint_as_float(z[8 * g]), __uint_as_float(z[8 * g + 1]), __uint_as_float(z[8 * g + 2]));
        part[g] = max3(part[g], __uint_as_float(z[8 * g + 3]), __uint_as_float(z[8 * g + 4]));
        part[g] = max3(part[g], __uint_as_float(z[8 * g + 5]), __uint_as_float(z[8 * g + 6]));
    }
    return max3(max3(part[0], part[1], part[2]), max3(part[3], __uint_as_float(z[7]), __uint_as_float(z[15])),
                max3(__uint_as_float(z[23]), __uint_as_float(z[31]), m));
}
// z <- 2^(z scale + shift)
__device__ __forceinline__ void exponentials(uint32_t (&z)[32], float scale, float shift) {
    const uint64_t scale_2 = pack2(scale, scale), shift_2 = pack2(shift, shift);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        float lo, hi;
        unpack2(fma2(pack2(__uint_as_float(z[2 * j]), __uint_as_float(z[2 * j + 1])), scale_2, shift_2), lo, hi);
        z[2 * j] = __float_as_uint(exp2_fast(lo));
        z[2 * j + 1] = __float_as_uint(exp2_fast(hi));
    }
}
__device__ __forceinline__ float total(const uint32_t (&z)[32]) {
    uint64_t part[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        part[g] = pack2(__uint_as_float(z[2 * g]), __uint_as_float(z[2 * g + 1]));
#pragma unroll
        for (int j = 1; j < 4; ++j) part[g] = add2(part[g], pack2(__uint_as_float(z[8 * j + 2 * g]), __uint_as_float(z[8 * j + 2 * g + 1])));
    }
    float lo, hi;
    unpack2(add2(add2(part[0], part[1]), add2(part[2], part[3])), lo, hi);
    return lo + hi;
}
__device__ __forceinline__ void times(uint32_t (&z)[32], float c) {
    const uint64_t c_2 = pack2(c, c);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        float lo, hi;
        unpack2(mul2(pack2(__uint_as_float(z[2 * j]), __uint_as_float(z[2 * j + 1])), c_2), lo, hi);
        z[2 * j] = __float_as_uint(lo);
        z[2 * j + 1] = __float_as_uint(hi);
    }
}

// Takes `t` off one of them.
__device__ __forceinline__ void take_off(uint32_t (&z)[32], int at, float t) {
#pragma unroll
    for (int i = 0; i < 32; ++i) z[i] = __float_as_uint(__uint_as_float(z[i]) - (i == at ? t : 0.0f));
}

// What a row's exponentials and labels are multiplied by.  lost: a wait has run out, and dz shows it in every word, since dw of a
// word is made of its own entries only.
__device__ __forceinline__ float factor_of(float coef, bool lost) { return lost ? NAN : coef; }
// dz in rows that take no part (or fill the last tile) and behind the last word: zeros, whatever the operands hold.
__device__ __forceinline__ void settle(uint32_t (&z)[32], bool used, bool all_used, int words) {
    if (words >= 32 && all_used) return;
#pragma unroll
    for (int j = 0; j < 32; ++j) z[j] = used && j < words ? z[j] : 0;
}

// A row's labels within some words, in ascending order, four of them on the way: a list read one by one costs its warp the
// memory's latency at every label (a piece of 5461 rows x 16384 words x 768 backward, 64 labels a row: 169 to 222 us, so 95 to 110).
struct LabelQueue {
    static constexpr int kAhead = 4;
    const int* indices;
    const float* weights;
    int at, end;
    int index[kAhead];                 // INT_MAX behind the last
    float weight[kAhead];
    __device__ __forceinline__ void load(int i) {
        const bool is = at + i < end;
        index[i] = is ? indices[at + i] : INT_MAX;
        if (weights) weight[i] = is ? weights[at + i] : 0.0f;
    }
    __device__ __forceinline__ void start(const int* all_indices, const float* all_weights, int first, int last) {
        indices = all_indices;
        weights = all_weights;
        at = first;
        end = last;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) load(i);
    }
    __device__ __forceinline__ void next() {
        ++at;
#pragma unroll
        for (int i = 0; i + 1 < kAhead; ++i) {
            index[i] = index[i + 1];
            weight[i] = weight[i + 1];
        }
        load(kAhead - 1);
    }
};

template <bool BACKWARD, bool TOP, bool TWO>
__global__ void __launch_bounds__(kThreads, 1) __cluster_dims__(TWO ? 2 : 1, 1, 1) logit_kernel(const __grid_constant__ LogitArgs a) {
    extern __shared__ uint8_t raw[];
    using Smem = LogitSmem<BACKWARD, TWO>;
    constexpr int STAGES = Smem::kStages, ROWS = TWO ? kTile : kTile / 2, BLOCKS = TWO ? 2 : 1;      // rows of a tile; blocks that form it
    Smem& sm = *reinterpret_cast<Smem*>(raw + ((1024 - (smem_u32(raw) & 1023)) & 1023));
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (threadIdx.x == 0) {
        tma_prefetch(&a.x);
        tma_prefetch(&a.w);
    }
    const Pair<STAGES, 1, TWO> p = pair_begin<STAGES, 1, TWO>(sm.stages, &sm.bars);
    grid_dependency_sync();
    const int count = a.plain ? a.rows : *a.count, row_tiles = (count + ROWS - 1) / ROWS, tiles = row_tiles * a.tiles;
    const int steps = (a.dim + kStep - 1) / kStep, first = blockIdx.x / BLOCKS, pairs = gridDim.x / BLOCKS;

    if (warp == 0) {
        if (elect_one()) {
            const CUtensorMap* x = count == a.all_rows ? &a.x_all : &a.x;
            Ring ring;
            for (int i = first; i < tiles; i += pairs) {
                int rt, ct;
                tile_at(a, i, row_tiles, rt, ct);
                const int row = rt * ROWS + p.rank * 128, word = (a.tile0 + ct) * kTile + p.rank * 128;
                for (int k = 0; k < steps; ++k) {
                    p.wait(p.empty + 8 * ring.stage, ring.phase ^ 1, kWaitEmpty);
                    if (p.rank == 0) bar_expect(p.full + 8 * ring.stage, BLOCKS * p.kStageBytes);
                    if (TWO) {
                        const uint32_t full = at_rank(p.full + 8 * ring.stage, 0);
                        tma_load2_pair(p.a(ring.stage), x, full, k * kStep, row);
                        tma_load2_pair(p.b(ring.stage), &a.w, full, k * kStep, word);
                    } else {
                        const uint32_t full = p.full + 8 * ring.stage;
                        tma_load2(p.a(ring.stage), x, full, k * kStep, row);
                        tma_load2(p.b(ring.stage), &a.w, full, k * kStep, word);
                        tma_load2(p.b(ring.stage) + kOperandBytes, &a.w, full, k * kStep, word + 128);
                    }
                    ring.next<STAGES>();
                }
            }
            ring_drain(p, ring);
        }
    } else if (warp == 1) {
        if (p.rank == 0 && elect_one()) {
            Ring ring;
            uint32_t acc = 0;
            for (int i = first; i < tiles; i += pairs, ++acc)
                tile_products(p, ring, acc, 1, steps, TWO ? mma_desc_pair(kTile, false, false) : mma_desc(kTile, false), [](uint32_t s, int i) { return desc_k_major(s + 32 * i); },
                              [](uint32_t s, int i) { return desc_k_major(s + 32 * i); });
        }
    } else {
        // Tensor memory's lanes that the warp may read; its columns.  Either all sixteen warps share every tile, a quarter each,
        // or, where many tiles follow one another, eight take every other one, a half each: one half's latencies then lie under the
        // other's exponentials (forward of 3420 rows x 74768 words x 72: 118 -> 99 us; of 333 rows x 32000 x 384, 3.4 tiles a pair:
        // 23.6 -> 22.6).
        const int quad = warp & 3, part = (warp - 2) / 4;
        const bool turns = tiles >= kTurnTiles * pairs;
        const int chunks = turns ? 4 : 2, column0 = turns ? 128 * (part & 1) : 64 * part, every = turns ? 2 : 1;
        const uint32_t lanes = p.tmem + ((uint32_t)(32 * quad) << 16) + column0;
        uint32_t acc = turns ? part >> 1 : 0;
        if (BACKWARD && a.plain) {
            // for the products behind: zeros in the rows that take no part
#pragma unroll 4
            for (int place = (warp - 2) * gridDim.x + blockIdx.x; place < a.padded; place += kOutWarps * gridDim.x) {
                const int r = a.rest && place >= a.rest ? place - a.rest : place;      // the rows twice, for either part of dz
                const bool used = r < a.rows && (TOP ? a.target[r] : label_at(a.l, r)) >= 0;
                for (int c = 8 * lane; c < a.dim; c += 256)
                    *reinterpret_cast<uint4*>(a.xc + (size_t)place * a.dim + c) = used ? *reinterpret_cast<const uint4*>(a.x_rows + r * a.x_step + c) : make_uint4(0, 0, 0, 0);
                if (lane == 0 && place == r) a.row[r] = used ? r : ~r;
            }
        }
        for (int i = first + acc * pairs; i < tiles; i += every * pairs, acc += every) {
            int rt, ct;
            tile_at(a, i, row_tiles, rt, ct);
            const int block_row = 32 * quad + lane, row = rt * ROWS + p.rank * 128 + block_row;
            const int c0 = (a.tile0 + ct) * kTile + column0;       // first word
            int label = -1;
            LabelQueue queue;
            const size_t list = (size_t)row * a.top;
            if (TOP) {
                const uint8_t* f = a.first + 4 * ((size_t)row * (a.all_tiles + 1) + a.tile0 + ct) + column0 / 64;
                const bool listed = row < count;                   // what fills the tile up has no list
                queue.start(a.index + list, BACKWARD ? a.weight + list : nullptr, listed ? f[0] : 0, listed ? f[chunks / 2] : 0);
            }
            float lse2 = 0.0f, coef = 0.0f;
            bool used = row < count;
            if (a.plain) {
                if (used) label = TOP ? a.target[row] : label_at(a.l, row);
                used = label >= 0;
                if (BACKWARD && used) {
                    lse2 = a.lse[row] * kLog2e;
                    coef = a.dloss[row * a.dloss_step] * a.scale;
                }
            } else {
                if (!TOP) label = a.target[row];
                if (BACKWARD) {
                    lse2 = a.lse2[row];
                    coef = a.coef[row];
                }
            }
            const bool all_used = __all_sync(~0u, used);
            const bool is_rest = a.rest && row >= a.rest && row < a.rest + count;      // written with the row it is left of
            float top = -INFINITY, sum = 0.0f;
            p.wait_warp(p.acc_full + 8 * (acc & 1), (acc >> 1) & 1, kWaitAccFull);
            tc_fence_after();
            const bool dead = *p.dead != 0;                        // a wait has run out: the results show it
            if (BACKWARD) coef = factor_of(coef, dead);
#pragma unroll 1
            for (int c = 0; c < chunks; ++c) {
                uint32_t z[32];
                tmem_ld32(z, lanes + (acc & 1) * kAccColumns + 32 * c);
                tmem_wait_ld();
                tmem_use(z);
                if (c + 1 == chunks) tile_taken(p, acc, lane, every);
                const int w0 = c0 + 32 * c;
                if (!BACKWARD) {
                    if (w0 + 32 > a.vocab) {                       // words behind the last have no logits
#pragma unroll
                        for (int j = 0; j < 32; ++j) z[j] = w0 + j < a.vocab ? z[j] : 0xFF800000u;
                    }
                    if (TOP) {
                        while (queue.index[0] < w0 + 32) {
                            a.label_z[list + queue.at] = pick(z, queue.index[0] - w0);
                            queue.next();
                        }
                    } else if ((uint32_t)(label - w0) < 32u) {
                        a.label_z[row] = pick(z, label - w0);
                    }
                    __syncwarp();
                    const float m = largest(z, top), ref = m == -INFINITY ? 0.0f : m * a.scale2;
                    sum *= exp2_fast(fmaf(top, a.scale2, -ref));
                    top = m;
                    exponentials(z, a.scale2, -ref);
                    sum += total(z);
                } else {
                    exponentials(z, a.scale2, -lse2);
                    times(z, coef);
                    if (TOP) {
                        while (queue.index[0] < w0 + 32) {
                            take_off(z, queue.index[0] - w0, coef * queue.weight[0]);
                            queue.next();
                        }
                    } else if ((uint32_t)(label - w0) < 32u) {
                        take_off(z, label - w0, coef);
                    }
                    __syncwarp();
                    settle(z, used, all_used, a.vocab - w0);
                    uint8_t* const to = a.dz + ((size_t)(rt * BLOCKS + p.rank) * (a.tiles * 4) + ct * 4) * 16384 + (column0 / 8 + 4 * c) * 2048 + block_row * 16;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t v[4];
#pragma unroll
                        for (int h = 0; h < 4; ++h) v[h] = pack_bf16(__uint_as_float(z[8 * j + 2 * h]), __uint_as_float(z[8 * j + 2 * h + 1]));
                        if (TWO || !is_rest) *reinterpret_cast<uint4*>(to + j * 2048) = make_uint4(v[0], v[1], v[2], v[3]);
                        if (!TWO && a.rest && row < count) {       // what rounding left
#pragma unroll
                            for (int h = 0; h < 4; ++h)
                                v[h] = pack_bf16(__uint_as_float(z[8 * j + 2 * h]) - bf16_lo(v[h]), __uint_as_float(z[8 * j + 2 * h + 1]) - bf16_hi(v[h]));
                            *reinterpret_cast<uint4*>(to + a.rest * 16 + j * 2048) = make_uint4(v[0], v[1], v[2], v[3]);
                        }
                    }
                }
            }
            if (!BACKWARD) {
                // the parts' sums of a row become one; a part's place is free again two tiles (of these warps) later
                float2* const stats = sm.stats + (turns ? (part >> 1) * 512 + ((acc >> 1) & 1) * 256 : (acc & 1) * 512) + block_row;
                stats[column0 / (turns ? 128 : 64) * 128] = make_float2(top, dead ? NAN : sum);
                asm volatile("bar.sync %0, %1;" ::"r"(1 + quad + (turns ? 4 * (part >> 1) : 0)), "r"(turns ? 64 : 128) : "memory");
                if (column0 == 0) {
                    const float2 none = make_float2(-INFINITY, 0.0f);
                    const float2 o[3] = {stats[128], turns ? none : stats[256], turns ? none : stats[384]};
                    const float m = max3(top, o[0].x, fmaxf(o[1].x, o[2].x)), ref = m == -INFINITY ? 0.0f : m * a.scale2;
                    sum *= exp2_fast(fmaf(top, a.scale2, -ref));
#pragma unroll
                    for (int q = 0; q < 3; ++q) sum += o[q].y * exp2_fast(fmaf(o[q].x, a.scale2, -ref));
                    a.stats[(size_t)(a.tile0 + ct) * a.padded + row] = make_float2(m, dead ? NAN : sum);
                }
            }
        }
    }
    pair_end(p);
}

// ---------------------------------------------------------------------------------------------- the loss from the tiles' sums

struct LossArgs {
    const float2* stats;
    const float* label_z;
    const float *weight, *entropy;     // teacher only
    const int *index;
    const int *slot, *count;
    int plain;                         // rows stay in their places
    Labels l;
    const int* target;
    int rows, padded, parts, top;      // parts: tiles of the vocabulary
    float scale, scale2;
    float *loss, *lse;
};

constexpr int kLossRows = 32, kLossParts = 16;

// 32 rows in gathered order, sixteen threads for each.  The rows that take no part get zeros.
__global__ void __launch_bounds__(kLossRows * kLossParts) loss_kernel(LossArgs a, const int* row_of) {
    __shared__ float s_top[kLossParts][kLossRows], s_sum[kLossParts][kLossRows], s_z[kLossRows], s_weight[kLossRows];
    grid_dependency_sync();
    const int count = a.plain ? a.rows : *a.count, i = threadIdx.x % kLossRows, part = threadIdx.x / kLossRows, row = blockIdx.x * kLossRows + i;
    if (!a.plain && threadIdx.x < kLossRows && row < a.rows && a.slot[row] < 0) a.loss[row] = a.lse[row] = 0.0f;
    if (blockIdx.x * kLossRows >= count) return;
    float top = -INFINITY, sum = 0.0f;
    constexpr int N = 8;                                       // loads on the way
    for (int t = part; t < a.parts; t += N * kLossParts) {
        float2 s[N];
#pragma unroll
        for (int i = 0; i < N; ++i)
            s[i] = t + i * kLossParts < a.parts ? a.stats[(size_t)(t + i * kLossParts) * a.padded + row] : make_float2(-INFINITY, 0.0f);
        float m = top;
#pragma unroll
        for (int i = 0; i < N; ++i) m = fmaxf(m, s[i].x);
        const float ref = m == -INFINITY ? 0.0f : m * a.scale2;
        sum *= exp2f(fmaf(top, a.scale2, -ref));
#pragma unroll
        for (int i = 0; i < N; ++i) sum += s[i].y * exp2f(fmaf(s[i].x, a.scale2, -ref));
        top = m;
    }
    // a row's labels by sixteen threads next to one another
    const int list_i = threadIdx.x / kLossParts, list_row = blockIdx.x * kLossRows + list_i;
    float z = 0.0f, weight = 0.0f;                             // sum t z, sum t
    if (list_row < count && !(a.plain && a.top && a.target[list_row] < 0))
#pragma unroll 4
        for (int k = threadIdx.x % kLossParts; k < a.top; k += kLossParts) {
            const size_t at = (size_t)list_row * a.top + k;
            const float t = a.index[at] == INT_MAX ? 0.0f : a.weight[at], label = a.label_z[at];
            z += t == 0.0f ? 0.0f : t * label;                 // nothing was written for the entries that take no part
            weight += t;
        }
    for (int d = kLossParts / 2; d; d >>= 1) {
        z += __shfl_xor_sync(~0u, z, d);
        weight += __shfl_xor_sync(~0u, weight, d);
    }
    if (threadIdx.x % kLossParts == 0) {
        s_z[list_i] = z;
        s_weight[list_i] = weight;
    }
    s_top[part][i] = top;
    s_sum[part][i] = sum;
    __syncthreads();
    if (part || row >= count) return;
    for (int q = 1; q < kLossParts; ++q) {
        const float m = fmaxf(top, s_top[q][i]), ref = m == -INFINITY ? 0.0f : m * a.scale2;
        sum = sum * exp2f(fmaf(top, a.scale2, -ref)) + s_sum[q][i] * exp2f(fmaf(s_top[q][i], a.scale2, -ref));
        top = m;
    }
    const float lse = fmaf(top, a.scale, logf(sum));
    if (a.plain && (a.top ? a.target[row] : label_at(a.l, row)) < 0) {
        a.loss[row] = a.lse[row] = 0.0f;
        return;
    }
    const int r = a.plain ? row : row_of[row];
    a.loss[r] = a.top ? a.entropy[row] - a.scale * s_z[i] + lse * s_weight[i] : lse - a.scale * a.label_z[row];
    a.lse[r] = lse;
}

// ---------------------------------------------------------------------------------------------- dx += dz w, dw = dz^T x

struct ProductArgs {
    CUtensorMap dz_block, dz_half;     // dz's blocks: all of one, or half of its rows
    CUtensorMap x, x_all, w;           // boxes of 64 x 64; x as for the logits
    CUtensorMap dw_map;                // boxes of 32 x 32
    const int* count;
    int all_rows;
    int plain, rows;                   // rows stay in their places
    int rest;                          // as for the logits
    int dim, vocab;
    int tile0, tiles;                  // of the vocabulary: the piece
    int wants_dx, wants_dw;            // one of them at least
    int dx_subs, splits, split_steps;  // dx: tiles of an item (where there are as many), parts of the inner axis
    int dw_subs, dw_splits, dw_split_steps, dw_groups;             // dw: the same; items of one part and column
    int n, dim_tiles;                  // columns of a tile, tiles of dim
    Divide by_pairs, by_dim_tiles, by_splits, by_dw_groups;
    int padded, add, last;             // add: dx's sums so far are read; last: dx is written in place of its sums
    float4* sums;                      // [splits][padded / 128][dim / 4][128]: dx so far, four columns of a row in one place
    float4* dw_sums;                   // [dw_splits][2 * tiles][dim / 4][128], where dw has several parts
    const int* row;                    // of a place; ~row: its dx is zero
    uint16_t* dx;
    int64_t dx_step;
    uint16_t* dw;
    int64_t dw_step;
};

// Two tiles, one above the other, share every copy of B where the inner axis is long: a step's copies are then 96 KB for
// two tiles instead of 128, and what a pair can draw from the L2 (about 100 bytes a cycle) is what bounds the steps.  Both
// halves of tensor memory belong to one item then, which its way out is not hidden behind: not worth it for short inner axes.
// Backward passes with two tiles from 8, 16, 32 steps on, and never: 13622 rows x 10070 x 184 244, 244, 276, 250 us; 1686 x 3622 x 816
// 55, 46, 49, 49; 1188 x 53029 x 888 304, 304, 329, 321; 10598 x 10748 x 360 256, 256, 257, 297.
constexpr int kProductStages = 4;
constexpr int kLongSteps = 16;          // fewer: one tile
constexpr int kOutSteps = 4;            // what a tile's way out costs, in steps

struct ProductSmem {
    uint8_t stages[kProductStages * 3 * kOperandBytes];
    uint8_t staging[kOutWarps * 2048];
    Bars<kProductStages> bars;
};

struct Item {
    bool is_dw;
    int rt, subs, dt, split, k0, steps;        // first tile (of rows or of words), tiles
};

// A pair's items: the longer kind first, dealt in turn; then the shorter kind, at first to the pairs that got one less of the
// longer, until they are even; what is left over goes out as single tiles where there are pairs for all of them.
struct Deal {
    bool dw_long;
    int dx_subs, dw_steps, row_tiles, pair, pairs;
    int longs;                                 // of the longer kind, this pair's
    int short_n, extra, late, extra_from;      // extra for each of the `late` pairs from extra_from on
    int from, rounds, over;                    // then these rounds for all pairs, and some left over
    bool halves;                               // which go out as single tiles
};

__device__ __forceinline__ Deal deal_of(const ProductArgs& a, int count, int pair) {
    Deal d;
    d.pair = pair;
    d.pairs = gridDim.x / 2;
    d.row_tiles = (count + kTile - 1) / kTile;
    d.dw_steps = (a.rest + count + kStep - 1) / kStep;
    d.dx_subs = d.row_tiles > 1 ? a.dx_subs : 1;
    // parts of dw that have steps
    const int dw_parts = a.dw_splits == 1 ? 1 : (d.dw_steps + a.dw_split_steps - 1) / a.dw_split_steps;
    const int dx_n = a.wants_dx ? (d.row_tiles + d.dx_subs - 1) / d.dx_subs * a.dim_tiles * a.splits : 0;
    const int dw_n = a.wants_dw ? dw_parts * a.dw_groups * a.dim_tiles : 0;
    const int dx_cost = (a.split_steps + kOutSteps) * d.dx_subs, dw_cost = (min(d.dw_steps, a.dw_split_steps) + kOutSteps) * a.dw_subs;
    d.dw_long = a.wants_dw && (dw_cost >= dx_cost || !a.wants_dx);
    const int long_n = d.dw_long ? dw_n : dx_n, more = d.dw_long ? dw_cost : dx_cost, less = d.dw_long ? dx_cost : dw_cost;
    d.short_n = d.dw_long ? dx_n : dw_n;
    d.longs = a.by_pairs(long_n);
    const int rest = long_n - d.longs * d.pairs;
    d.longs += pair < rest;
    d.extra = rest ? (more + less / 2) / less : 0;
    d.extra_from = rest;
    d.late = d.pairs - rest;
    d.from = d.extra * d.late;
    const int left = max(0, d.short_n - d.from);
    d.rounds = a.by_pairs(left);
    d.over = left - d.rounds * d.pairs;
    d.halves = (d.dw_long ? d.dx_subs : a.dw_subs) == 2 && 2 * d.over <= d.pairs;
    return d;
}

// The pair's i-th item; false behind its last.
__device__ __forceinline__ bool item_at(const ProductArgs& a, const Deal& d, int i, Item& t) {
    int n, only = -1;                                              // only: one tile of the item
    t.is_dw = d.dw_long;
    if (i < d.longs) {
        n = d.pair + i * d.pairs;
    } else {
        t.is_dw = !d.dw_long;
        i -= d.longs;
        const bool late = d.pair >= d.extra_from;
        if (late && i < d.extra) {
            n = d.pair - d.extra_from + i * d.late;
            if (n >= d.short_n) return false;
        } else {
            if (late) i -= d.extra;
            n = d.from + d.pair + i * d.pairs;
            if (i > d.rounds) return false;
            if (i == d.rounds) {
                if (d.halves) {
                    if (d.pair >= 2 * d.over) return false;
                    n = d.from + d.rounds * d.pairs + d.pair / 2;
                    only = d.pair & 1;
                } else if (d.pair >= d.over) {
                    return false;
                }
            }
        }
    }
    const int m = a.by_dim_tiles(n);
    t.dt = n - m * a.dim_tiles;
    if (t.is_dw) {
        t.split = a.by_dw_groups(m);
        n = m - t.split * a.dw_groups;
        t.k0 = t.split * a.dw_split_steps;
        t.steps = min(a.dw_split_steps, d.dw_steps - t.k0);
        t.subs = a.dw_subs;
    } else {
        n = a.by_splits(m);
        t.split = m - n * a.splits;
        t.k0 = t.split * a.split_steps;
        t.steps = min(a.split_steps, a.tiles * 4 - t.k0);
        t.subs = d.dx_subs;
    }
    t.rt = n * t.subs;
    const int end = t.is_dw ? a.tiles : d.row_tiles;
    if (only >= 0) {
        t.rt += only;
        t.subs = 1;
        return t.rt < end;                                         // a pair's last item
    }
    t.subs = min(t.subs, end - t.rt);
    return true;
}

__device__ __forceinline__ void add_to(uint32_t (&v)[32], const float4 (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        v[4 * j] = __float_as_uint(__uint_as_float(v[4 * j]) + x[j].x);
        v[4 * j + 1] = __float_as_uint(__uint_as_float(v[4 * j + 1]) + x[j].y);
        v[4 * j + 2] = __float_as_uint(__uint_as_float(v[4 * j + 2]) + x[j].z);
        v[4 * j + 3] = __float_as_uint(__uint_as_float(v[4 * j + 3]) + x[j].w);
    }
}

__global__ void __launch_bounds__(kThreads, 1) __cluster_dims__(2, 1, 1) product_kernel(const __grid_constant__ ProductArgs a) {
    extern __shared__ uint8_t raw[];
    ProductSmem& sm = *reinterpret_cast<ProductSmem*>(raw + ((1024 - (smem_u32(raw) & 1023)) & 1023));
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (threadIdx.x == 0) {
        tma_prefetch(&a.dz_block);
        tma_prefetch(&a.dz_half);
        tma_prefetch(&a.x);
        tma_prefetch(&a.w);
    }
    const Pair<kProductStages, 2, true> p = pair_begin<kProductStages, 2, true>(sm.stages, &sm.bars);
    // dealt before the kernel in front has ended, as if every row took part, and once more if not
    Deal deal = deal_of(a, a.rows, blockIdx.x / 2);
    asm volatile("" ::"r"(deal.longs), "r"(deal.over), "r"(deal.from));
    grid_dependency_sync();
    const int count = a.plain ? a.rows : *a.count;
    if (count != a.rows) deal = deal_of(a, count, blockIdx.x / 2);
    const int boxes = (a.n / 2 + 63) / 64;                         // of B in either block

    if (count == 0) {
        // nobody takes part: dw of the piece is zero, and nothing reads dx
        const int per_row = a.dim / 8, words = a.wants_dw ? min(a.vocab - a.tile0 * kTile, a.tiles * kTile) : 0;
        for (int64_t i = blockIdx.x * kThreads + threadIdx.x; i < (int64_t)words * per_row; i += (int64_t)gridDim.x * kThreads) {
            const int64_t v = i / per_row;
            *reinterpret_cast<uint4*>(a.dw + (a.tile0 * (int64_t)kTile + v) * a.dw_step + 8 * (i - v * per_row)) = make_uint4(0, 0, 0, 0);
        }
    } else if (warp == 0) {
        if (elect_one()) {
            const CUtensorMap* x = count == a.all_rows ? &a.x_all : &a.x;
            Ring ring;
            Item t;
            for (int i = 0; item_at(a, deal, i, t); ++i) {
                const int d0 = t.dt * a.n + p.rank * (a.n / 2), row_blocks = a.tiles * 4;      // of one block's rows
                for (int k = t.k0; k < t.k0 + t.steps; ++k) {
                    p.wait(p.empty + 8 * ring.stage, ring.phase ^ 1, kWaitEmpty);
                    if (p.rank == 0) bar_expect(p.full + 8 * ring.stage, 2 * (t.subs * kOperandBytes + boxes * 8192));
                    const uint32_t full = at_rank(p.full + 8 * ring.stage, 0);
                    for (int s = 0; s < t.subs; ++s) {
                        const uint32_t to = p.a(ring.stage) + s * kOperandBytes;
                        // dw: 64 rows x 128 words, half of each of two blocks; dx: 128 rows x 64 words, a whole block
                        if (t.is_dw) {
                            const int block = (k / 2) * row_blocks + (t.rt + s) * 4 + p.rank * 2;
                            tma_load3_pair(to, &a.dz_half, full, 0, (k & 1) * 8, block * 8);
                            tma_load3_pair(to + 8192, &a.dz_half, full, 0, (k & 1) * 8, block * 8 + 8);
                        } else {
                            const int block = ((t.rt + s) * 2 + p.rank) * row_blocks + k;
                            tma_load3_pair(to, &a.dz_block, full, 0, 0, block * 8);
                        }
                    }
                    for (int b = 0; b < boxes; ++b)
                        tma_load2_pair(p.b(ring.stage) + b * 8192, t.is_dw ? x : &a.w, full, d0 + 64 * b, t.is_dw ? k * kStep : a.tile0 * kTile + k * kStep);
                    ring.next<kProductStages>();
                }
            }
            ring_drain(p, ring);
        }
    } else if (warp == 1) {
        if (p.rank == 0 && elect_one()) {
            Ring ring;
            Item t;
            uint32_t acc = 0;
            for (int i = 0; item_at(a, deal, i, t); ++i) {
                if (t.is_dw)
                    tile_products(p, ring, acc, t.subs, t.steps, mma_desc_pair(a.n, true, true),
                                  [](uint32_t s, int i) { return desc_plain(s + 256 * i, 128, 1024); },
                                  [](uint32_t s, int i) { return desc_n_major(s + 2048 * i, 8192); });
                else
                    tile_products(p, ring, acc, t.subs, t.steps, mma_desc_pair(a.n, false, true),
                                  [](uint32_t s, int i) { return desc_plain(s + 4096 * i, 2048, 128); },
                                  [](uint32_t s, int i) { return desc_n_major(s + 2048 * i, 8192); });
                acc += t.subs;
            }
        }
    } else {
        const int quad = warp & 3, part = (warp - 2) / 4;
        uint8_t* const box = sm.staging + (warp - 2) * 2048;
        const uint32_t lanes = p.tmem + ((uint32_t)(32 * quad) << 16);
        Item t;
        uint32_t acc = 0;
        for (int i = 0, sub = 0; item_at(a, deal, i, t); ++acc, sub = sub + 1 < t.subs ? sub + 1 : (++i, 0)) {
            const int row = (t.rt + sub) * kTile + p.rank * 128 + 32 * quad + lane;
            p.wait_warp(p.acc_full + 8 * (acc & 1), (acc >> 1) & 1, kWaitAccFull);
            tc_fence_after();
            const bool dead = *p.dead != 0;
            const int block = (t.rt + sub) * 2 + p.rank, word = (a.tile0 + t.rt + sub) * kTile + p.rank * 128 + 32 * quad;
            float4* const sums = (t.is_dw ? a.dw_sums + ((size_t)t.split * (2 * a.tiles) + block) * (a.dim / 4) * 128
                                          : a.sums + ((size_t)t.split * (a.padded / 128) + block) * (a.dim / 4) * 128) + 32 * quad + lane;
            const bool writes = t.is_dw ? word + lane < a.vocab : row < a.rest + count;
            const bool out = t.is_dw ? a.dw_splits == 1 : a.last, adds = !t.is_dw && a.add && writes;
            // the rows that the lane writes in turn: 8 at a time, four lanes for 64 bytes of each
            int64_t to[4];
            bool zero[4] = {};
            if (out && !t.is_dw)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int place = row - lane + 8 * r + lane / 4, at = place < count ? a.row[place] : 0;
                    zero[r] = at < 0;
                    to[r] = place < count ? (at < 0 ? ~at : at) * a.dx_step : -1;
                }
            for (int c = part; c < a.n / 32; c += 4) {
                const int d0 = t.dt * a.n + 32 * c;
                if (d0 >= a.dim) break;
                float4 before[8];
                if (adds)
#pragma unroll
                    for (int j = 0; j < 8; ++j) before[j] = d0 + 4 * j < a.dim ? sums[(size_t)(d0 / 4 + j) * 128] : make_float4(0, 0, 0, 0);
                uint32_t v[32];
                tmem_ld32(v, lanes + (acc & 1) * kAccColumns + 32 * c);
                tmem_wait_ld();
                tmem_use(v);
                if (c + 4 >= a.n / 32 || d0 + 128 >= a.dim) tile_taken(p, acc, lane);
                if (dead) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = 0x7FC00000u;
                }
                if (adds) add_to(v, before);
                const bool joins = !t.is_dw && a.rest && out;      // what rounding left meets its row, by way of its place in the sums
                if (joins ? row >= a.rest && writes : !out && writes)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (d0 + 4 * j < a.dim)
                            sums[(size_t)(d0 / 4 + j) * 128] = make_float4(__uint_as_float(v[4 * j]), __uint_as_float(v[4 * j + 1]),
                                                                           __uint_as_float(v[4 * j + 2]), __uint_as_float(v[4 * j + 3]));
                __syncwarp();
                if (!out) continue;
                if (joins) {
                    asm volatile("bar.sync %0, 128;" ::"r"(1 + part) : "memory");      // the four warps with these columns
                    if (row < count) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) before[j] = d0 + 4 * j < a.dim ? sums[(size_t)(d0 / 4 + j) * 128 + a.rest] : make_float4(0, 0, 0, 0);
                        add_to(v, before);
                    }
                    __syncwarp();
                }
                // 32 rows of 64 bytes, in the 64-byte swizzle that the tensor map reads, when those before have left
                if (lane == 0) tma_store_wait_read();
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t w[4];
#pragma unroll
                    for (int h = 0; h < 4; ++h) w[h] = pack_bf16(__uint_as_float(v[8 * j + 2 * h]), __uint_as_float(v[8 * j + 2 * h + 1]));
                    *reinterpret_cast<uint4*>(box + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                }
                if (t.is_dw) {
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0 && word < a.vocab) {
                        tma_store2(&a.dw_map, smem_u32(box), d0, word);
                        tma_store_commit();
                    }
                } else {
                    __syncwarp();
                    const int at = 8 * (lane & 3);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int line = 8 * r + lane / 4;
                        const uint4 w = *reinterpret_cast<const uint4*>(box + line * 64 + (((lane & 3) ^ ((line >> 1) & 3)) << 4));
                        if (to[r] >= 0 && d0 + at < a.dim) *reinterpret_cast<uint4*>(a.dx + to[r] + d0 + at) = zero[r] ? make_uint4(0, 0, 0, 0) : w;
                    }
                }
            }
            if (part >= a.n / 32 || t.dt * a.n + 32 * part >= a.dim) tile_taken(p, acc, lane);     // nothing was this warp's
        }
        if (lane == 0) tma_store_wait();
    }
    pair_end(p);
}

// dx and dw from several parts: their sums, rounded.
struct Parts {
    const float4* sums;
    int parts, part_steps;             // dw: parts that begin behind the rows' last step hold nothing
    int blocks;                        // of this launch: 32 rows each
    int rows, padded;
    const int* row;                    // of a place; null: the place itself
    uint16_t* out;
    int64_t step;
    int ways;                          // warps that share the parts: 1, 2, 4, 8 or 16
    int rest;                          // so many places further on is what rounding left; 0: nowhere
};

// A block takes 32 rows x 128 / ways columns; the warps that share a column's parts add their sums in order.  Many warps and little
// code: a kernel this short waits for its instructions about as long as for its data (eight warps with loops unrolled eight
// times: 9 us for 2 x 64 parts of 5 rows x 200, 6 us so).
constexpr int kPartWarps = 16;
__global__ void __launch_bounds__(32 * kPartWarps) parts_kernel(const __grid_constant__ Parts dx, const __grid_constant__ Parts dw, const int* count, int rows, int dim) {
    __shared__ float s[kPartWarps][8][32];
    grid_dependency_sync();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, n = count ? *count : rows;
    const bool is_dw = (int)blockIdx.x >= dx.blocks;
    const Parts& p = is_dw ? dw : dx;
    const int row0 = (blockIdx.x - (is_dw ? dx.blocks : 0)) * 32, row = row0 + lane, end = is_dw ? p.rows : n;
    const int parts = is_dw ? min(p.parts, ((n + kStep - 1) / kStep + p.part_steps - 1) / p.part_steps) : p.parts;
    const int all = p.rest ? 2 * parts : parts;                // what rounding left counts as parts of its own
    const int columns = kPartWarps / p.ways, way = warp % p.ways, groups = dim / 8, group0 = blockIdx.y * columns;
    if (row0 >= end || group0 >= groups) return;
    const int group = group0 + warp / p.ways;
    const int64_t part = (int64_t)(p.padded / 128) * (dim / 4) * 128;
    const float4* from = p.sums + ((int64_t)(row / 128) * (dim / 4) + 2 * group) * 128 + row % 128;
    const int to = row < end && p.row && way == 0 ? p.row[row] : row;
    const bool mine = row < end && group < groups;
    float v[8] = {};
    if (mine)
#pragma unroll 1
        for (int k = way; k < all; k += p.ways) {
            const float4* const at = from + (k < parts ? k * part : (k - parts) * part + p.rest);
            const float4 lo = at[0], hi = at[128];
            const float add[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += add[j];
        }
    if (p.ways > 1) {
#pragma unroll
        for (int j = 0; j < 8; ++j) s[warp][j][lane] = v[j];
        __syncthreads();
#pragma unroll 1
        for (int w = 1; way == 0 && w < p.ways; ++w)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += s[warp + w][j][lane];
    }
    if (!mine || way) return;
    const uint4 out = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    *reinterpret_cast<uint4*>(p.out + (to < 0 ? ~to : to) * p.step + 8 * group) = to < 0 ? make_uint4(0, 0, 0, 0) : out;
}

// ---------------------------------------------------------------------------------------------- host

// Parts of an inner axis, so that an item of one tile, or of two that share an operand where the parts stay long, takes no longer
// than `share` steps.
struct Axis {
    int subs, splits, split_steps;
};
Axis split_axis(int64_t steps, int64_t share, bool pairs, int most) {
    Axis a;
    for (a.subs = pairs ? 2 : 1;; a.subs = 1) {
        const int64_t n = std::max<int64_t>(1, std::min<int64_t>(most, (steps * a.subs + share - 1) / share));
        a.split_steps = (int)std::max<int64_t>(1, (steps + n - 1) / n);
        a.splits = (int)std::max<int64_t>(1, (steps + a.split_steps - 1) / a.split_steps);
        if (a.subs == 1 || a.split_steps >= kLongSteps) return a;
    }
}

// Steps until the last pair is done, as deal_of deals the items.
int64_t steps_until_done(int64_t dx_n, const Axis& dx, int64_t dw_n, const Axis& dw) {
    const int64_t dx_cost = (int64_t)(dx.split_steps + kOutSteps) * dx.subs, dw_cost = (int64_t)(dw.split_steps + kOutSteps) * dw.subs;
    const bool dw_long = dw_cost >= dx_cost;
    const int64_t long_n = dw_long ? dw_n : dx_n, short_n = dw_long ? dx_n : dw_n, more = dw_long ? dw_cost : dx_cost, less = dw_long ? dx_cost : dw_cost;
    const int64_t rest = long_n % kPairs, late = kPairs - rest, extra = rest ? (more + less / 2) / less : 0;
    const int64_t left = std::max<int64_t>(0, short_n - extra * late), rounds = left / kPairs, over = left % kPairs;
    const int64_t early_end = (long_n / kPairs + (rest > 0)) * more, late_end = long_n / kPairs * more + std::min(extra, (short_n + late - 1) / late) * less;
    const bool halves = (dw_long ? dx.subs : dw.subs) == 2 && 2 * over <= kPairs;
    return std::max(early_end, late_end) + rounds * less + (over == 0 ? 0 : halves ? less * 5 / 8 : less);
}

// Sizes and places in the workspace.
struct Plan {
    int padded, count_blocks, tiles, labels;
    int piece, pieces, n, dim_tiles;
    Axis dx, dw;                       // how the products' inner axes are split
    uint64_t block_count, place, count, slot, row, xc, target, index, weight, entropy, first, stats, label_z, lse2, coef, dz, sums, dw_sums, bytes;
};

Plan make_plan(const alsgd_vocab_desc& d, bool backward) {
    Plan p;
    std::memset(&p, 0, sizeof p);
    p.padded = (int)((d.rows + kTile - 1) / kTile * kTile);
    p.count_blocks = p.padded / kCountRows;
    p.tiles = (int)((d.vocab + kTile - 1) / kTile);
    p.labels = d.top ? (int)d.top : 1;
    p.dim_tiles = (int)((d.dim + 255) / 256);
    p.n = (int)((d.dim + p.dim_tiles * 32 - 1) / (p.dim_tiles * 32) * 32);
    // pieces of the vocabulary: dz of one in kPieceBytes, or in kLeastPiece tiles' worth where the rows are many; all alike
    const uint64_t tile_bytes = (uint64_t)p.padded * kTile * 2;
    uint64_t piece = tile_bytes ? kPieceBytes / tile_bytes : p.tiles;
    if (piece < kLeastPiece) piece = kLeastPiece;
    piece -= piece % 2;                                            // two tiles share an operand: rounded up, a piece stays within this
    if (piece > (uint64_t)p.tiles) piece = p.tiles;
    p.pieces = (int)((p.tiles + piece - 1) / piece);
    p.piece = (p.tiles + p.pieces - 1) / p.pieces;
    if (p.pieces > 1) p.piece += p.piece % 2;
    p.pieces = (p.tiles + p.piece - 1) / p.piece;
    // an inner axis is split while an item would take longer than a pair's share of the launch, or a half, a third, a quarter of
    // it, whichever leaves the pairs done first.  (One part where two were better: 10598 rows x 10748 words x 360 are 84 equal items for
    // 74 pairs.)
    const int64_t row_tiles = p.padded / kTile, dx_steps = 4ll * p.piece, dw_steps = p.padded / kStep;
    const int64_t all = p.dim_tiles * (row_tiles * dx_steps + p.piece * dw_steps), share = std::max<int64_t>(8, all / kPairs);
    const uint64_t dx_bytes = 4ull * p.padded * d.dim, dw_bytes = 4ull * p.piece * kTile * d.dim;      // of a part's sums
    auto most = [](uint64_t bytes) { return (int)std::min<uint64_t>(kMaxSplits, std::max<uint64_t>(1, kPieceBytes / (bytes + 1))); };
    int64_t best = INT64_MAX;
    Axis dx[4], dw[4];
    for (int i = 0; i < 4 && backward; ++i) {
        dx[i] = split_axis(dx_steps, std::max<int64_t>(8, share / (1 + i)), row_tiles > 1, most(dx_bytes));
        dw[i] = split_axis(dw_steps, std::max<int64_t>(8, share / (1 + i)), p.piece > 1, most(dw_bytes));
    }
    for (int i = 0; i < 16 && backward; ++i) {
        const Axis &x = dx[i % 4], &w = dw[i / 4];
        const int64_t dx_n = (row_tiles + x.subs - 1) / x.subs * p.dim_tiles * x.splits, dw_n = (p.piece + w.subs - 1) / w.subs * p.dim_tiles * w.splits;
        // parts are written and read again (a step's time moves about 1 MB) by one more launch (about 12 steps)
        const int64_t sums = ((x.splits > 1 ? x.splits * dx_bytes : 0) + (w.splits > 1 ? w.splits * dw_bytes : 0)) >> 19;
        const int64_t t = steps_until_done(dx_n, x, dw_n, w) + sums + (x.splits > 1 || w.splits > 1 ? 12 : 0);
        if (t >= best) continue;
        best = t;
        p.dx = x;
        p.dw = w;
    }

    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        const uint64_t start = at;
        at += (bytes + 255) / 256 * 256;
        return start;
    };
    const uint64_t padded = (uint64_t)p.padded;
    p.block_count = take(4ull * p.count_blocks);
    p.place = take(4 * padded);
    p.count = take(4);
    p.slot = take(4ull * d.rows);
    p.row = take(4 * padded);
    p.xc = take(2 * padded * d.dim);
    if (d.top) {
        p.index = take(4 * padded * d.top);
        p.weight = take(4 * padded * d.top);
        p.entropy = take(4 * padded);
        p.first = take(4 * padded * (p.tiles + 1));
    }
    p.target = take(4 * padded);
    if (backward) {
        p.lse2 = take(4 * padded);
        p.coef = take(4 * padded);
        p.dz = take(tile_bytes * p.piece);
        if (p.pieces > 1 || p.dx.splits > 1 || d.rows <= kMostRest) p.sums = take(p.dx.splits * dx_bytes);
        if (p.dw.splits > 1) p.dw_sums = take(p.dw.splits * dw_bytes);
    } else {
        p.stats = take(8 * padded * p.tiles);
        p.label_z = take(4 * padded * p.labels);
    }
    p.bytes = at;
    return p;
}

int check_desc(const alsgd_vocab_desc* d) {
    if (!d) return ALSGD_E_ARG;
    if (d->vocab == 0 || d->dim == 0 || d->dim % 8) return ALSGD_E_ARG;
    if (d->index_dtype != ALSGD_I32 && d->index_dtype != ALSGD_I64) return ALSGD_E_ARG;
    if (d->top && d->teacher_dtype != ALSGD_F32 && d->teacher_dtype != ALSGD_BF16) return ALSGD_E_ARG;
    if (!(d->scale > 0.0f) || !std::isfinite(d->scale) || !std::isfinite(d->scale * kLog2e)) return ALSGD_E_ARG;
    if (d->top > (uint32_t)kMaxTop || d->dim > 1u << 14) return ALSGD_E_UNSUPPORTED;
    if (d->rows > 1u << 22 || d->vocab > 1u << 22) return ALSGD_E_RANGE;
    if (d->device < 0 || d->device >= kMaxDevices) return ALSGD_E_RANGE;
    return ALSGD_OK;
}

int check_matrix(const alsgd_matrix* m, uint32_t rows, uint32_t dim, bool output) {
    if (!m) return ALSGD_E_ARG;
    if (rows == 0) return ALSGD_OK;
    if (!m->data || reinterpret_cast<uintptr_t>(m->data) % 16) return ALSGD_E_ARG;
    if (rows == 1) return ALSGD_OK;
    if (m->stride_row < 0 || m->stride_row % 8 || m->stride_row >= (1ll << 39)) return ALSGD_E_ARG;
    if (output && m->stride_row < (int64_t)dim) return ALSGD_E_ARG;
    return ALSGD_OK;
}

int encode_map(uint32_t rank, const void* data, const cuuint64_t* size, const cuuint64_t* step_bytes, const cuuint32_t* box, CUtensorMapSwizzle swizzle, CUtensorMap* out) {
    EncodeTiled encode = encode_tiled();
    if (!encode) return ALSGD_E_CUDA;
    const cuuint32_t unit[3] = {1, 1, 1};
    const CUresult r = encode(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(data), size, step_bytes, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? ALSGD_OK : ALSGD_E_ARG;
}

// Boxes of 64 columns x box_rows rows of a bf16 matrix, swizzled over their 128-byte rows; zeros outside.
int make_map(const void* data, uint64_t rows, uint64_t cols, uint64_t step_bytes, uint32_t box_rows, CUtensorMap* out) {
    const cuuint64_t size[2] = {cols, rows};
    const cuuint32_t box[2] = {64, box_rows};
    return encode_map(2, data, size, &step_bytes, box, CU_TENSOR_MAP_SWIZZLE_128B, out);
}

// dz's blocks as [block * 8 words][8 rows][64 values]: `groups` of the 16 groups of rows of a block.
int make_dz_map(const void* data, uint64_t blocks, uint32_t groups, CUtensorMap* out) {
    const cuuint64_t size[3] = {64, 16, 8 * blocks}, step_bytes[2] = {128, 2048};
    const cuuint32_t box[3] = {64, groups, 8};
    return encode_map(3, data, size, step_bytes, box, CU_TENSOR_MAP_SWIZZLE_NONE, out);
}

struct Call {
    const alsgd_vocab_desc* d;
    const alsgd_matrix *x, *w;
    const void *index, *teacher;
    void* work;
    uint64_t work_bytes;
    cudaStream_t stream;
};

// x as it is can be an operand of the products, unless its rows overlap.
bool direct_x(const Call& c) { return c.d->rows == 1 || c.x->stride_row >= (int64_t)c.d->dim; }

// Rows that fit two tiles stay in their places, and those of passes so short that a third of their products, which is what padding
// often is, takes no longer than the two launches in front would (about 4.5 us: 1464 rows x 4486 x 128 forward 16.2 -> 13.0 us,
// 1856 x 5124 x 272 forward 20.4 -> 17.4, 10604 x 1240 x 104 backward 40.2 -> 35.8).
bool plain_rows(const Call& c, bool backward) {
    return direct_x(c) && (c.d->rows <= 2 * kTile || (uint64_t)c.d->rows * c.d->vocab * c.d->dim * (backward ? 3 : 1) <= kPlainProducts);
}

uint64_t step_of(const alsgd_matrix& m, uint32_t rows, uint32_t dim) {
    return rows == 1 || m.stride_row == 0 ? (uint64_t)dim : (uint64_t)m.stride_row;
}

int check_call(const Call& c, bool teacher) {
    const int rc = check_desc(c.d);
    if (rc != ALSGD_OK) return rc;
    const alsgd_vocab_desc& d = *c.d;
    if ((d.top != 0) != teacher) return ALSGD_E_ARG;
    int e;
    if ((e = check_matrix(c.x, d.rows, d.dim, false)) != ALSGD_OK) return e;
    if ((e = check_matrix(c.w, d.vocab, d.dim, false)) != ALSGD_OK) return e;
    if (d.vocab > 1 && c.w->stride_row < (int64_t)d.dim) return ALSGD_E_ARG;
    if (d.rows) {
        if (!c.index || reinterpret_cast<uintptr_t>(c.index) % (d.index_dtype == ALSGD_I64 ? 8 : 4)) return ALSGD_E_ARG;
        if (teacher && (!c.teacher || reinterpret_cast<uintptr_t>(c.teacher) % (d.teacher_dtype == ALSGD_BF16 ? 2 : 4))) return ALSGD_E_ARG;
        if (!c.work || reinterpret_cast<uintptr_t>(c.work) % 256) return ALSGD_E_ARG;
    }
    return ALSGD_OK;
}

template <typename T>
T* at(const Call& c, uint64_t offset) {
    return reinterpret_cast<T*>(static_cast<uint8_t*>(c.work) + offset);
}

Labels labels_of(const Call& c) {
    const alsgd_vocab_desc& d = *c.d;
    return {c.index, c.teacher, d.index_dtype == ALSGD_I64, d.teacher_dtype == ALSGD_BF16, (int)d.rows, (int)d.top, (int)d.vocab};
}

// Rows that take part, their copies and labels.
int gather_rows(const Call& c, const Plan& p, const float* lse, const float* dloss, int64_t dloss_step, const alsgd_matrix* dx) {
    const alsgd_vocab_desc& d = *c.d;
    GatherArgs g;
    std::memset(&g, 0, sizeof g);
    g.l = labels_of(c);
    g.plain = plain_rows(c, lse != nullptr);
    if (g.plain && !d.top) return ALSGD_OK;                        // nothing to do
    g.x = static_cast<const uint16_t*>(c.x->data);
    g.x_step = d.rows == 1 ? 0 : c.x->stride_row;
    g.lse = lse;
    g.dloss = dloss;
    g.dloss_step = dloss_step;
    g.scale = d.scale;
    g.direct = direct_x(c);
    if (dx) {
        g.dx = static_cast<uint16_t*>(dx->data);
        g.dx_step = (int64_t)step_of(*dx, d.rows, d.dim);
    }
    g.padded = p.padded;
    g.blocks = p.count_blocks;
    g.dim = (int)d.dim;
    g.tiles = p.tiles;
    g.block_count = at<int>(c, p.block_count);
    g.place = at<int>(c, p.place);
    g.count = at<int>(c, p.count);
    g.slot = at<int>(c, p.slot);
    g.row = at<int>(c, p.row);
    g.xc = at<uint16_t>(c, p.xc);
    if (d.top) {
        g.index = at<int>(c, p.index);
        g.weight = at<float>(c, p.weight);
        g.entropy = at<float>(c, p.entropy);
        g.first = at<uint32_t>(c, p.first);
    }
    if (!d.top || g.plain) g.target = at<int>(c, p.target);
    if (lse) {
        g.lse2 = at<float>(c, p.lse2);
        g.coef = at<float>(c, p.coef);
    }
    g.summed = p.count_blocks > kFewBlocks;
    if (!g.plain && launch_dependent(count_kernel, dim3(p.count_blocks), dim3(d.top ? 1024 : kCountRows), 0, c.stream, g.l, at<int>(c, p.block_count),
                                     at<int>(c, p.place)) != cudaSuccess)
        return ALSGD_E_CUDA;
    if (!g.plain && g.summed && launch_dependent(prefix_kernel, dim3(1), dim3(kPrefixThreads), 0, c.stream, at<int>(c, p.block_count), p.count_blocks,
                                                 at<int>(c, p.count)) != cudaSuccess)
        return ALSGD_E_CUDA;
    const int rows = g.plain ? ((int)d.rows + kGatherWarps - 1) / kGatherWarps * kGatherWarps : p.padded;
    return launch_dependent(gather_kernel, dim3(rows / kGatherWarps), dim3(32 * kGatherWarps), 0, c.stream, g) == cudaSuccess ? ALSGD_OK : ALSGD_E_CUDA;
}

int make_logits(const Call& c, const Plan& p, bool backward, LogitArgs* a) {
    const alsgd_vocab_desc& d = *c.d;
    std::memset(a, 0, sizeof *a);
    int rc;
    if ((rc = make_map(at<void>(c, p.xc), p.padded, d.dim, 2ull * d.dim, 128, &a->x)) != ALSGD_OK) return rc;
    if ((rc = make_map(c.w->data, d.vocab, d.dim, 2 * step_of(*c.w, d.vocab, d.dim), 128, &a->w)) != ALSGD_OK) return rc;
    a->all_rows = direct_x(c) ? (int)d.rows : -1;
    if (direct_x(c) && (rc = make_map(c.x->data, d.rows, d.dim, 2 * step_of(*c.x, d.rows, d.dim), 128, &a->x_all)) != ALSGD_OK) return rc;
    a->plain = plain_rows(c, backward);
    a->rows = (int)d.rows;
    a->l = labels_of(c);
    a->scale = d.scale;
    a->x_rows = static_cast<const uint16_t*>(c.x->data);
    a->x_step = d.rows == 1 ? 0 : c.x->stride_row;
    a->xc = at<uint16_t>(c, p.xc);
    a->row = at<int>(c, p.row);
    a->count = at<int>(c, p.count);
    a->dim = (int)d.dim;
    a->vocab = (int)d.vocab;
    a->top = (int)d.top;
    a->all_tiles = p.tiles;
    a->scale2 = d.scale * kLog2e;
    a->padded = p.padded;
    if (d.top) {
        a->index = at<int>(c, p.index);
        a->weight = at<float>(c, p.weight);
        a->first = at<uint8_t>(c, p.first);
    }
    a->target = at<int>(c, p.target);
    return ALSGD_OK;
}

int grid_of(int64_t tiles) { return 2 * (int)(tiles < kPairs ? tiles : kPairs); }

template <bool BACKWARD, bool TOP, bool TWO>
int launch_logits(const LogitArgs& a, int device, cudaStream_t s) {
    static SmemLimit limit;
    constexpr size_t smem = sizeof(LogitSmem<BACKWARD, TWO>) + 1024;
    if (!limit.raise(logit_kernel<BACKWARD, TOP, TWO>, device, smem)) return ALSGD_E_CUDA;
    const int64_t tiles = (int64_t)(a.padded / kTile) * a.tiles;
    const int grid = TWO ? grid_of(tiles) : std::min(a.tiles, kSMs);
    return launch_dependent(logit_kernel<BACKWARD, TOP, TWO>, dim3(grid), dim3(kThreads), smem, s, a) == cudaSuccess ? ALSGD_OK : ALSGD_E_CUDA;
}

// Up to 128 rows that stay in their places.
bool alone(const LogitArgs& a) { return a.plain && a.rows <= kTile / 2; }

// There every block forms logits by itself: 77 rows x 32000 words x 384 forward 12.3 -> 9.7 us, backward 31.0 -> 28.9 us.
template <bool BACKWARD>
int launch_logits(const LogitArgs& a, int device, cudaStream_t s) {
    if (alone(a))
        return a.top ? launch_logits<BACKWARD, true, false>(a, device, s) : launch_logits<BACKWARD, false, false>(a, device, s);
    return a.top ? launch_logits<BACKWARD, true, true>(a, device, s) : launch_logits<BACKWARD, false, true>(a, device, s);
}

int forward(const Call& c, bool teacher, float* loss, float* lse) {
    int rc = check_call(c, teacher);
    if (rc != ALSGD_OK) return rc;
    const alsgd_vocab_desc& d = *c.d;
    if (d.rows == 0) return ALSGD_OK;
    if (!loss || !lse || reinterpret_cast<uintptr_t>(loss) % 4 || reinterpret_cast<uintptr_t>(lse) % 4) return ALSGD_E_ARG;
    const Plan p = make_plan(d, false);
    if (c.work_bytes < p.bytes) return ALSGD_E_NOMEM;
    UseDevice use(d.device);
    if (!use.ok) return ALSGD_E_CUDA;
    LogitArgs a;
    if ((rc = make_logits(c, p, false, &a)) != ALSGD_OK) return rc;
    if ((rc = gather_rows(c, p, nullptr, nullptr, 0, nullptr)) != ALSGD_OK) return rc;
    a.tiles = p.tiles;
    a.by_group = divide_by(kGroup * a.tiles);
    a.stats = at<float2>(c, p.stats);
    a.label_z = at<float>(c, p.label_z);
    if ((rc = launch_logits<false>(a, d.device, c.stream)) != ALSGD_OK) return rc;
    LossArgs l;
    std::memset(&l, 0, sizeof l);
    l.stats = a.stats;
    l.label_z = a.label_z;
    if (d.top) {
        l.weight = a.weight;
        l.entropy = at<float>(c, p.entropy);
        l.index = a.index;
    }
    l.plain = a.plain;
    l.l = a.l;
    l.target = a.target;
    l.slot = at<int>(c, p.slot);
    l.count = a.count;
    l.rows = (int)d.rows;
    l.padded = p.padded;
    l.parts = p.tiles;
    l.top = (int)d.top;
    l.scale = d.scale;
    l.scale2 = a.scale2;
    l.loss = loss;
    l.lse = lse;
    const int* row_of = at<int>(c, p.row);
    return launch_dependent(loss_kernel, dim3(p.padded / kLossRows), dim3(kLossRows * kLossParts), 0, c.stream, l, row_of) == cudaSuccess ? ALSGD_OK : ALSGD_E_CUDA;
}

// What a piece leaves in parts: dw of its words, with the last piece dx.
int add_parts(const Plan& p, const ProductArgs& m, cudaStream_t stream) {
    const bool dx = m.wants_dx && p.dx.splits > 1 && m.tile0 + m.tiles == p.tiles, dw = m.wants_dw && p.dw.splits > 1;
    if (!dx && !dw) return ALSGD_OK;
    Parts of_dx, of_dw;
    std::memset(&of_dx, 0, sizeof of_dx);
    std::memset(&of_dw, 0, sizeof of_dw);
    auto ways = [](int parts) {
        int n = 1;
        while (2 * n <= parts && n < kPartWarps) n *= 2;
        return n;
    };
    const int words = std::min(m.vocab - m.tile0 * kTile, m.tiles * kTile);
    if (dx) of_dx = {m.sums, p.dx.splits, p.dx.split_steps, (m.rows + 31) / 32, m.rows, p.padded, m.row, m.dx, m.dx_step, ways(m.rest ? 2 * p.dx.splits : p.dx.splits), m.rest};
    if (dw)
        of_dw = {m.dw_sums, p.dw.splits, p.dw.split_steps, (words + 31) / 32, words, m.tiles * kTile, nullptr, m.dw + (int64_t)m.tile0 * kTile * m.dw_step, m.dw_step,
                 ways(p.dw.splits), 0};
    const int columns = kPartWarps / std::max(of_dx.ways, of_dw.ways), groups = m.dim / 8;
    return launch_dependent(parts_kernel, dim3(of_dx.blocks + of_dw.blocks, (groups + columns - 1) / columns), dim3(32 * kPartWarps), 0, stream, of_dx, of_dw,
                            m.plain ? (const int*)nullptr : m.count, m.rows, m.dim) == cudaSuccess
               ? ALSGD_OK
               : ALSGD_E_CUDA;
}

int backward(const Call& c, bool teacher, const float* lse, const float* dloss, int64_t dloss_step, const alsgd_matrix* dx, const alsgd_matrix* dw) {
    int rc = check_call(c, teacher);
    if (rc != ALSGD_OK) return rc;
    const alsgd_vocab_desc& d = *c.d;
    if (!dx && !dw) return ALSGD_E_ARG;
    if (dx && (rc = check_matrix(dx, d.rows, d.dim, true)) != ALSGD_OK) return rc;
    if (dw && (rc = check_matrix(dw, d.vocab, d.dim, true)) != ALSGD_OK) return rc;
    if ((dx && d.rows && dx->data == c.x->data) || (dw && dw->data == c.w->data)) return ALSGD_E_ARG;      // the operands are read until the end
    if (d.rows && (!lse || !dloss || reinterpret_cast<uintptr_t>(lse) % 4 || reinterpret_cast<uintptr_t>(dloss) % 4 || dloss_step < 0)) return ALSGD_E_ARG;
    const Plan p = make_plan(d, true);
    if (d.rows && c.work_bytes < p.bytes) return ALSGD_E_NOMEM;
    UseDevice use(d.device);
    if (!use.ok) return ALSGD_E_CUDA;
    const uint64_t dw_step = dw ? step_of(*dw, d.vocab, d.dim) : 0;
    if (d.rows == 0)
        return !dw || cudaMemset2DAsync(dw->data, 2 * dw_step, 0, 2ull * d.dim, d.vocab, c.stream) == cudaSuccess ? ALSGD_OK : ALSGD_E_CUDA;
    LogitArgs a;
    ProductArgs m;
    std::memset(&m, 0, sizeof m);
    if ((rc = make_logits(c, p, true, &a)) != ALSGD_OK) return rc;
    a.lse2 = at<float>(c, p.lse2);
    a.coef = at<float>(c, p.coef);
    a.dz = at<uint8_t>(c, p.dz);
    a.lse = lse;
    a.dloss = dloss;
    a.dloss_step = dloss_step;
    if ((rc = make_map(at<void>(c, p.xc), p.padded, d.dim, 2ull * d.dim, 64, &m.x)) != ALSGD_OK) return rc;
    if ((rc = make_map(c.w->data, d.vocab, d.dim, 2 * step_of(*c.w, d.vocab, d.dim), 64, &m.w)) != ALSGD_OK) return rc;
    const uint64_t blocks = (uint64_t)(p.padded / 128) * p.piece * 4;
    if ((rc = make_dz_map(a.dz, blocks, 16, &m.dz_block)) != ALSGD_OK || (rc = make_dz_map(a.dz, blocks, 8, &m.dz_half)) != ALSGD_OK) return rc;
    if (dw) {
        const cuuint64_t size[2] = {d.dim, d.vocab}, step_bytes = 2 * dw_step;
        const cuuint32_t box[2] = {32, 32};
        if ((rc = encode_map(2, dw->data, size, &step_bytes, box, CU_TENSOR_MAP_SWIZZLE_64B, &m.dw_map)) != ALSGD_OK) return rc;
    }
    if (direct_x(c) && (rc = make_map(c.x->data, d.rows, d.dim, 2 * step_of(*c.x, d.rows, d.dim), 64, &m.x_all)) != ALSGD_OK) return rc;
    m.plain = a.plain;
    m.rows = a.rows;
    a.rest = m.rest = !alone(a) || a.rows > kMostRest ? 0 : a.rows > kMostRest / 2 ? kMostRest : kMostRest / 2;
    m.all_rows = a.plain ? -1 : a.all_rows;
    m.count = a.count;
    m.dim = (int)d.dim;
    m.vocab = (int)d.vocab;
    m.n = p.n;
    m.dim_tiles = p.dim_tiles;
    m.by_dim_tiles = divide_by(p.dim_tiles);
    m.padded = p.padded;
    m.dx_subs = p.dx.subs;
    m.dw_subs = p.dw.subs;
    m.dw_splits = p.dw.splits;
    m.dw_split_steps = p.dw.split_steps;
    m.sums = at<float4>(c, p.sums);
    m.dw_sums = at<float4>(c, p.dw_sums);
    m.row = at<int>(c, p.row);
    m.wants_dx = dx != nullptr;
    m.wants_dw = dw != nullptr;
    if (dx) {
        m.dx = static_cast<uint16_t*>(dx->data);
        m.dx_step = (int64_t)step_of(*dx, d.rows, d.dim);
    }
    if (dw) {
        m.dw = static_cast<uint16_t*>(dw->data);
        m.dw_step = (int64_t)dw_step;
    }
    if ((rc = gather_rows(c, p, lse, dloss, dloss_step, dx)) != ALSGD_OK) return rc;
    static SmemLimit limit;
    constexpr size_t smem = sizeof(ProductSmem) + 1024;
    if (!limit.raise(product_kernel, d.device, smem)) return ALSGD_E_CUDA;
    for (int i = 0; i < p.pieces; ++i) {
        a.tile0 = m.tile0 = i * p.piece;
        a.tiles = m.tiles = p.tiles - a.tile0 < p.piece ? p.tiles - a.tile0 : p.piece;
        a.by_group = divide_by(kGroup * a.tiles);
        // the first piece writes all of dx's sums; a shorter last one adds to as many as it has steps for
        m.split_steps = p.dx.split_steps;
        m.splits = (4 * m.tiles + p.dx.split_steps - 1) / p.dx.split_steps;
        m.add = i > 0;
        m.last = i + 1 == p.pieces && p.dx.splits == 1;
        if ((rc = launch_logits<true>(a, d.device, c.stream)) != ALSGD_OK) return rc;
        m.dw_groups = (m.tiles + p.dw.subs - 1) / p.dw.subs;
        m.by_dw_groups = divide_by(m.dw_groups);
        const int grid = grid_of(p.dim_tiles * ((dx ? (int64_t)(p.padded / kTile) * p.dx.splits : 0) + (dw ? (int64_t)m.tiles * p.dw.splits : 0)));
        m.by_pairs = divide_by(grid / 2);
        m.by_splits = divide_by(m.splits);
        if (launch_dependent(product_kernel, dim3(grid), dim3(kThreads), smem, c.stream, m) != cudaSuccess) return ALSGD_E_CUDA;
        if ((rc = add_parts(p, m, c.stream)) != ALSGD_OK) return rc;
    }
    return ALSGD_OK;
}

}  // namespace

extern "C" int alsgd_vocab_bytes(const alsgd_vocab_desc* desc, int backward_pass, uint64_t* bytes_out) {
    if (!bytes_out) return ALSGD_E_ARG;
    const int rc = check_desc(desc);
    if (rc != ALSGD_OK) return rc;
    *bytes_out = desc->rows ? make_plan(*desc, backward_pass != 0).bytes : 0;
    return ALSGD_OK;
}

extern "C" int alsgd_xent_fwd(const alsgd_vocab_desc* desc, const alsgd_matrix* x, const alsgd_matrix* w, const void* target, float* loss, float* lse,
                              void* work, uint64_t work_bytes, void* stream) {
    return forward({desc, x, w, target, nullptr, work, work_bytes, static_cast<cudaStream_t>(stream)}, false, loss, lse);
}

extern "C" int alsgd_xent_bwd(const alsgd_vocab_desc* desc, const alsgd_matrix* x, const alsgd_matrix* w, const void* target, const float* lse,
                              const float* dloss, int64_t dloss_step, const alsgd_matrix* dx, const alsgd_matrix* dw, void* work, uint64_t work_bytes,
                              void* stream) {
    return backward({desc, x, w, target, nullptr, work, work_bytes, static_cast<cudaStream_t>(stream)}, false, lse, dloss, dloss_step, dx, dw);
}

extern "C" int alsgd_distill_fwd(const alsgd_vocab_desc* desc, const alsgd_matrix* x, const alsgd_matrix* w, const void* index, const void* teacher,
                                 float* loss, float* lse, void* work, uint64_t work_bytes, void* stream) {
    return forward({desc, x, w, index, teacher, work, work_bytes, static_cast<cudaStream_t>(stream)}, true, loss, lse);
}

extern "C" int alsgd_distill_bwd(const alsgd_vocab_desc* desc, const alsgd_matrix* x, const alsgd_matrix* w, const void* index, const void* teacher,
                                 const float* lse, const float* dloss, int64_t dloss_step, const alsgd_matrix* dx, const alsgd_matrix* dw, void* work,
                                 uint64_t work_bytes, void* stream) {
    return backward({desc, x, w, index, teacher, work, work_bytes, static_cast<cudaStream_t>(stream)}, true, lse, dloss, dloss_step, dx, dw);
}

extern "C" int alsgd_vocab_status(int32_t device, uint32_t* waits_out) {
    if (!waits_out) return ALSGD_E_ARG;
    if (device < 0 || device >= kMaxDevices) return ALSGD_E_RANGE;
    UseDevice use(device);
    if (!use.ok) return ALSGD_E_CUDA;
    unsigned word = 0;
    // the copy alone would wait for the default stream, but not for streams that are independent of it
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&word, g_wait_error, sizeof word) != cudaSuccess) return ALSGD_E_CUDA;
    *waits_out = word;
    return ALSGD_OK;
}
