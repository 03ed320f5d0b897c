// Shared by attention's forward and backward pass: the shape as the kernels see it, the relative position bias, the
// checks of a call's arguments and the tensor maps.
#pragma once
#include "../../include/alsgd.h"
#include "alsgd_ops.cuh"
#include "alsgd_tc.cuh"

#include <algorithm>
#include <cmath>
#include <cstring>

namespace alsgd_attn {

constexpr int kMaxDistance = 2048;     // the bias table by distance has to fit beside the tiles in shared memory
constexpr int kMaxBuckets = 256;
constexpr int kMaxLength = 1 << 22;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kMaskedOut = -1e30f;   // a table entry at or below this takes its bucket out

using alsgd_ops::Divide;
using alsgd_ops::divide_by;

struct Shape {
    int batch, heads_q, heads_kv, group, len_q, len_kv, dim;
    int causal, q_pos, device;
    float scale, scale_log2;
    const int* kv_len;                 // may be null
    int keys_end;                      // keys from here on are no sequence's: len_kv, or the last query's end under a causal mask
    Divide by_heads_q, by_heads_kv, by_all_q, by_all_kv, by_group;     // heads, batch * heads, query heads per key head
    Divide by_rows_q;                  // row blocks of a sequence's queries * heads
};

// Buckets of a distance: below `near` one each, then up to limits[0], limits[1], ..., the last open.
struct Bias {
    const void* table;                 // null: no bias
    int bf16, buckets;
    int per_side, near, two_sided;
    int far;                           // distances from here on share the last bucket of their side
    int far_bucket[2];                 // those, of keys behind (kSpanFarLeft) and ahead of the query
    int n_limits;
    int limits[kMaxBuckets / 2];
};

__device__ __forceinline__ int bucket_of(const Bias& s, int r) {
    const int a = s.two_sided ? abs(r) : max(-r, 0);
    int at = a;
    if (a >= s.near) {
        at = s.near;
        for (int i = 0; i < s.n_limits; ++i) at += a >= s.limits[i];
    }
    return at + (s.two_sided && r > 0 ? s.per_side : 0);
}

// First and last distance r of a bucket (far beyond any tile where it is open; first > last where it is empty).
__device__ __forceinline__ void bucket_span(const Bias& s, int bucket, int& first, int& last) {
    const bool ahead = s.two_sided && bucket >= s.per_side;
    const int n = ahead ? bucket - s.per_side : bucket;
    auto edge = [&](int n) { return n <= s.near ? n : s.limits[n - s.near - 1]; };
    const int low = edge(n), high = n + 1 == s.per_side ? 1 << 14 : edge(n + 1) - 1;     // of |r|
    if (ahead) {
        first = max(low, 1);
        last = high;
    } else {
        first = -high;
        last = n == 0 && !s.two_sided ? 1 << 14 : -low;
    }
}

__device__ __forceinline__ float table_entry(const Bias& s, int head, int bucket) {
    const size_t i = (size_t)head * s.buckets + bucket;
    return s.bf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(s.table)[i] << 16) : static_cast<const float*>(s.table)[i];
}

// Bucket of every distance r = at - pad, once per block.
__device__ __forceinline__ void fill_buckets(const Bias& s, uint8_t* bucket, int pad, int thread, int threads) {
    for (int i = thread; i <= 2 * pad; i += threads) bucket[i] = (uint8_t)bucket_of(s, i - pad);
}

// One head's bias by distance in the exponent's base 2, as the tiles that lie within reach of the buckets' edges read it: a
// thread wants consecutive distances from its own start on, its neighbour the same ones moved by one.  Two copies, the
// second moved by one element, give every thread aligned pairs whatever its start.  They lie 72 bytes (modulo 128) apart:
// the 16 threads of a half-warp then use 32 banks, when the first thread's start is even as `pad` is.
struct LutShape {
    int pad;                           // distances start at -pad
    int copy;                          // floats from one copy to the next
    int floats;                        // of one table: two copies, the values of the two far ends, a word (lut_outs)
};

__host__ __device__ inline LutShape lut_shape(int far, int tile_a, int tile_b, bool causal) {
    LutShape s;
    s.pad = (far + tile_a + tile_b + 1) / 2 * 2;
    const int reach = causal ? tile_a + tile_b : s.pad;        // no allowed key lies ahead; masked ones are read, whatever is there
    s.copy = (s.pad + reach + 2 + 31) / 32 * 32 + 18;
    s.floats = 2 * s.copy + 4;
    return s;
}

// Where a thread reads the bias of distances r, r + 1, ... as pairs.
__device__ __forceinline__ const float* lut_at(const float* lut, const LutShape& s, int r) {
    const int x = r + s.pad;
    return lut + (x & 1 ? s.copy + x - 1 : x);
}
__device__ __forceinline__ float lut_far(const float* lut, const LutShape& s, bool right) { return lut[2 * s.copy + right]; }

// Whether a bucket of the table's head is taken out.  A mask is a bias of -inf, and a score of +inf (finite operands whose
// product overflows) under it is NaN; so is p (dp - delta) of a masked pair whose dp is infinite.  The backward kernels look
// for a NaN in mixed tiles that may hold masked pairs, and take those out by the table.  Together with far_out: 173 -> 183 us at
// 64 x 256 tokens, 355 -> 371 us at 2 x 4096 (the same look at tiles with one bias, in place of far_out: 380 to 390 us).
__device__ __forceinline__ void lut_set_outs(float* lut, const LutShape& s, bool outs) { lut[2 * s.copy + 2] = outs ? 1.0f : 0.0f; }
__device__ __forceinline__ bool lut_outs(const float* lut, const LutShape& s) { return lut[2 * s.copy + 2] != 0.0f; }

__device__ __forceinline__ float lut_value(const Bias& s, int head, int bucket) {
    if (!s.table) return 0.0f;
    const float v = table_entry(s, head, bucket);
    return v <= kMaskedOut ? -INFINITY : v * kLog2e;
}

// Fills one table for distances low .. high; `sign` -1 turns the axis round (distance r is kept at -r).  With a causal mask
// the distances ahead are -inf, which masks: mask_ahead writes them, once, and a head's fill ends at 0.  Returns whether the
// thread met a bucket that is taken out.
__device__ __forceinline__ bool fill_lut(const Bias& s, int head, const uint8_t* bucket, float* lut, const LutShape& l, int low, int high, int sign,
                                         int thread, int threads) {
    low = max(low, -l.pad);
    high = min(high, l.pad);                                   // the bucket list's end; mixed tiles reach no further
    bool out = false;
#pragma unroll 4
    for (int r = low + thread; r <= high; r += threads) {
        const float x = lut_value(s, head, bucket[sign * r + l.pad]);
        out |= x == -INFINITY;
        lut[r + l.pad] = x;
        if (r + l.pad > 0) lut[l.copy + r + l.pad - 1] = x;
    }
    if (thread < 2) lut[2 * l.copy + thread] = lut_value(s, head, bucket[thread ? 2 * l.pad : 0]);
    return out;
}
__device__ __forceinline__ void mask_ahead(float* lut, const LutShape& l, int thread, int threads) {
    for (int x = l.pad + 1 + thread; x < l.copy; x += threads) {
        lut[x] = -INFINITY;
        lut[l.copy + x - 1] = -INFINITY;
    }
}

// The same on the turned axis.
__device__ __forceinline__ void mask_behind(float* lut, const LutShape& l, int thread, int threads) {
    for (int x = thread; x < l.pad; x += threads) {
        lut[x] = -INFINITY;
        if (x > 0) lut[l.copy + x - 1] = -INFINITY;
    }
}

// What every row of a tile has in common: a bias, or (mixed) the table by distance, which also holds a causal mask.
// Rows and columns are positions; r = column - row.
enum Span { kSpanFarLeft, kSpanFarRight, kSpanMixed };
__device__ __forceinline__ Span span_of(const Bias& s, int r_min, int r_max) {
    return r_max <= -s.far ? kSpanFarLeft : r_min >= s.far ? kSpanFarRight : kSpanMixed;
}

bool bwd_wait_word(unsigned* out);     // alsgd_attn_bwd.cu

// Whether a tile of distances r_min .. r_max lies in a far bucket that is taken out for this head: nothing of it is allowed.  The
// backward kernels copy zeros instead of such a tile (coordinates behind the end), so that its scores are finite.  The entry
// is read again for every far tile: kept for a head, with the tiles where it applies, it cost 3 us more of 371.
__device__ __forceinline__ bool far_out(const Bias& s, int head, int r_min, int r_max) {
    const Span span = span_of(s, r_min, r_max);
    return s.table && span != kSpanMixed && table_entry(s, head, s.far_bucket[span]) <= kMaskedOut;
}

// An operand as the copy engine reads it.  A dimension with step 0 (an operand broadcast over the batch or the heads)
// has extent 1 there and its coordinate is multiplied away.
struct Operand {
    CUtensorMap map;
    int head_mul, batch_mul;
    uint16_t* data;
    int64_t step_pos, step_head, step_batch;   // in elements; 0 where the extent is 1
};

// Zeros in a row of an operand: an item without tiles has nothing to compute.
__device__ __forceinline__ void zero_row(const Operand& t, int dim, int batch, int head, int pos) {
    uint16_t* p = t.data + (int64_t)batch * t.step_batch + (int64_t)head * t.step_head + (int64_t)pos * t.step_pos;
    for (int x = 0; x < dim; x += 8) *reinterpret_cast<uint4*>(p + x) = make_uint4(0, 0, 0, 0);
}

// A block's item in each round: forwards through the blocks, then backwards, so that with items sorted by their work the
// blocks' shares come out nearly even.
__device__ __forceinline__ int walk(int round) {
    return round * (int)gridDim.x + (round & 1 ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x);
}

// The sequences of a ragged batch, the longest first, as every block finds them for itself: their lengths are on the device,
// and a walk over items sorted by their work needs them.  Measured against the order in which they come: 4 sequences of 1531 to
// 511 keys, 1000 queries, 16 heads of 128 that share 4: forward 79 -> 61 us, backward 293 -> 200 us (the four blocks of keys
// too many for one per SM were empty ones).  At 128 short sequences both are alike (32 and 34 us forward, 132 and 127 us
// backward): the items are many, and more sequences are taken as they come.  Compiled apart: its arithmetic in a walk that
// does not need it cost 1 to 7 %.
constexpr int kMaxRanked = 128;
struct Ranks {
    static constexpr bool on = true;
    int len[kMaxRanked];               // keys of the sequence with this rank
    uint8_t seq[kMaxRanked];
};
struct KeyRanks : Ranks {              // for items that are blocks of keys
    int before[kMaxRanked];            // (block, sequence) pairs with keys, ahead of the blocks that only ranks up to this one fill
};

struct NoRanks {                       // without lengths, or with more sequences: as they come
    static constexpr bool on = false;
};

inline bool by_rank(const Shape& sh) { return sh.kv_len && sh.batch <= kMaxRanked; }
// A sequence's keys end where its length does or where no query sees further: what lies behind is never used, whatever it holds.
__device__ __forceinline__ int clamped_len(const Shape& sh, int b) { return sh.kv_len ? min(max(sh.kv_len[b], 0), sh.keys_end) : sh.keys_end; }

__device__ __forceinline__ int blocks_of(int len, int rows) { return (len + rows - 1) / rows; }

// All of the block's threads, at least kMaxRanked.
__device__ __forceinline__ void rank_sequences(const Shape& sh, Ranks& ranks) {
    const int b = threadIdx.x;
    int len = 0, rank = 0;
    if (b < sh.batch) ranks.len[b] = len = clamped_len(sh, b);
    __syncthreads();
    if (b < sh.batch)
        for (int s = 0; s < sh.batch; ++s) rank += ranks.len[s] > len || (ranks.len[s] == len && s < b);
    __syncthreads();
    if (b < sh.batch) {
        ranks.len[rank] = len;
        ranks.seq[rank] = (uint8_t)b;
    }
    __syncthreads();
}
__device__ __forceinline__ void rank_sequences(const Shape& sh, int rows, KeyRanks& ranks) {
    rank_sequences(sh, ranks);
    const int r = threadIdx.x;
    if (r < sh.batch) {
        const int blocks = r + 1 < sh.batch ? blocks_of(ranks.len[r + 1], rows) : 0;
        int pairs = 0;
        for (int s = 0; s < sh.batch; ++s) pairs += min(blocks_of(ranks.len[s], rows), blocks);
        ranks.before[r] = pairs;
    }
    __syncthreads();
}

// The i-th (key block, sequence) pair: those with keys, block by block and rank by rank, then those without.  The blocks from
// edge(r) to edge(r - 1) have keys in the sequences up to rank r and in no other.
__device__ __forceinline__ void ranked_pair(const Shape& sh, const KeyRanks& ranks, int rows, int i, int& block, int& rank) {
    auto edge = [&](int r) { return r + 1 < sh.batch ? blocks_of(ranks.len[r + 1], rows) : 0; };
    const int filled = ranks.before[0] + edge(-1) - edge(0);           // pairs with keys: above edge(0) the longest sequence's alone
    const bool keys = i < filled;
    if (!keys) i -= filled;
    auto ahead = [&](int r) {                                          // pairs of the wanted kind ahead of edge(r)
        const int with = r < 0 ? filled : ranks.before[r];
        return keys ? with : edge(r) * sh.batch - with;
    };
    int low = keys ? 0 : -1, high = sh.batch - 1;                      // the smallest r with ahead(r) <= i
    while (low < high) {
        const int mid = (low + high) >> 1;                             // rounds down for -1 too
        if (ahead(mid) <= i) high = mid; else low = mid + 1;
    }
    const int count = keys ? low + 1 : sh.batch - 1 - low, at = i - ahead(low);
    block = edge(low) + at / count;
    rank = at % count + (keys ? 0 : low + 1);
}

// Row block, sequence, head and valid keys of the i-th item of a kernel whose items are query rows, the most keys first: with
// a causal mask the last rows, else the longest sequences.
template <typename RANKS>
__device__ __forceinline__ void query_item(const Shape& sh, const RANKS& ranks, int row_blocks, int i, int& block, int& b, int& h, int& len) {
    if constexpr (RANKS::on) {
        if (!sh.causal) {
            const int rank = sh.by_rows_q(i), rest = i - rank * row_blocks * sh.heads_q;
            block = sh.by_heads_q(rest);
            h = rest - block * sh.heads_q;
            b = ranks.seq[rank];
            len = ranks.len[rank];
            return;
        }
    }
    const int from_end = sh.by_all_q(i), bh = i - from_end * sh.batch * sh.heads_q;
    block = row_blocks - 1 - from_end;
    b = sh.by_heads_q(bh);
    h = bh - b * sh.heads_q;
    if constexpr (RANKS::on) {
        len = ranks.len[b];
        b = ranks.seq[b];
    } else {
        len = clamped_len(sh, b);
    }
}

// The block's next item from `round` on, if there is one; `round` moves behind it.
template <typename ARGS, typename RANKS, typename ITEM>
__device__ __forceinline__ bool next_item(const ARGS& a, const RANKS& ranks, int& round, ITEM& item) {
    for (; round * (int)gridDim.x < a.items; ++round) {
        const int i = walk(round);
        if (i >= a.items) continue;
        item = item_at(a, ranks, i);
        ++round;
        return true;
    }
    return false;
}

// The tiles of a block's items, one after the other.  item_at(ARGS, ranks, i) finds an item, whose `n` is the number of tiles; items
// without any are passed over, by every warp alike: a barrier's phases must not run past one that waits on it.
template <typename ARGS, typename ITEM>
struct Cursor {
    ITEM item;
    int round, ordinal, j, tile;       // the next round, how many of the block's items with tiles came before it, tile within it, tiles before this one
    bool more;
    template <typename RANKS>
    __device__ __forceinline__ void settle(const ARGS& a, const RANKS& ranks) {
        do more = next_item(a, ranks, round, item);
        while (more && item.n == 0);
        j = 0;
    }
    template <typename RANKS>
    __device__ __forceinline__ void start(const ARGS& a, const RANKS& ranks) {
        round = ordinal = tile = 0;
        settle(a, ranks);
    }
    template <typename RANKS>
    __device__ __forceinline__ void next(const ARGS& a, const RANKS& ranks) {
        ++tile;
        if (++j < item.n) return;
        ++ordinal;
        settle(a, ranks);
    }
};

// 32 columns x 32 rows of results (fp32 in registers, one row per lane), scaled and rounded, into 2 KB of the warp's own;
// after a fence the leader stores the box.
__device__ __forceinline__ void stage_box(const uint32_t (&x)[32], float scale, uint8_t* staging, int lane) {
    uint8_t* line = staging + lane * 64;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = alsgd_ops::pack_bf16(__uint_as_float(x[8 * i + 2 * e]) * scale, __uint_as_float(x[8 * i + 2 * e + 1]) * scale);
        *reinterpret_cast<uint4*>(line + ((i ^ ((lane >> 1) & 3)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}


// ---- host ---------------------------------------------------------------------------------------------------

// Edges of the logarithmic buckets: the smallest whole distances a with log(a/near)/log(max/near) * width >= i.
inline void bucket_limits(int per_side, int near, int max_distance, Bias* out) {
    const int width = per_side - near;
    out->n_limits = 0;
    for (int i = 1; i < width; ++i) {
        const long double t = near * powl((long double)max_distance / near, (long double)i / width);
        const long double whole = roundl(t);
        out->limits[out->n_limits++] = (int)(fabsl(t - whole) < 1e-10L * t ? whole : ceill(t));
    }
    out->far = out->n_limits ? out->limits[out->n_limits - 1] : near;
}

// Blocks of a persistent kernel that are resident together: `per_sm` of them, as far as shared memory allows.
inline int blocks_at_once(size_t smem, int per_sm) {
    const size_t room = 228 * 1024, fit = room / (smem + 1024);        // an SM's; each block takes 1 KB for itself
    return alsgd_ops::kSMs * (fit < (size_t)per_sm ? (int)fit : per_sm);
}

inline int make_bias(const alsgd_attn_desc& d, const void* table, Bias* out) {
    std::memset(out, 0, sizeof *out);
    out->far = 1;
    if (d.buckets == 0) return ALSGD_OK;
    const bool two = d.flags & ALSGD_ATTN_BIAS_TWO_SIDED;
    if (d.table_dtype != ALSGD_F32 && d.table_dtype != ALSGD_BF16) return ALSGD_E_ARG;
    if (d.buckets > kMaxBuckets || d.max_distance > kMaxDistance) return ALSGD_E_UNSUPPORTED;
    if (two && d.buckets % 2) return ALSGD_E_ARG;
    const int per_side = (int)d.buckets / (two ? 2 : 1), near = per_side / 2;
    if (near < 1 || (int)d.max_distance <= near) return ALSGD_E_ARG;
    out->table = table;
    out->bf16 = d.table_dtype == ALSGD_BF16;
    out->buckets = (int)d.buckets;
    out->per_side = per_side;
    out->near = near;
    out->two_sided = two;
    bucket_limits(per_side, near, (int)d.max_distance, out);
    out->far_bucket[0] = per_side - 1;
    out->far_bucket[1] = two ? 2 * per_side - 1 : 0;
    return ALSGD_OK;
}

inline int check_desc(const alsgd_attn_desc* d) {
    if (!d) return ALSGD_E_ARG;
    if (d->batch == 0 || d->heads_q == 0 || d->heads_kv == 0 || d->heads_q % d->heads_kv) return ALSGD_E_ARG;
    if (d->dim == 0 || d->dim % 8 || (d->flags & ~(ALSGD_ATTN_CAUSAL | ALSGD_ATTN_BIAS_TWO_SIDED))) return ALSGD_E_ARG;
    if (!(d->scale > 0.0f) || !std::isfinite(d->scale)) return ALSGD_E_ARG;
    if (d->dim > 128) return ALSGD_E_UNSUPPORTED;
    if (d->len_q > kMaxLength || d->len_kv > kMaxLength || d->q_pos > kMaxLength || d->q_pos < -kMaxLength) return ALSGD_E_RANGE;
    if ((uint64_t)d->batch * d->heads_q > 0x7FFFFFFFull) return ALSGD_E_RANGE;
    if (d->device < 0 || d->device >= alsgd_ops::kMaxDevices) return ALSGD_E_RANGE;
    Bias unused;
    return make_bias(*d, nullptr, &unused);
}

// A bias table or its gradient lies where its values may lie: it can be a vector of a flat layout.
inline bool table_aligned(const alsgd_attn_desc& d, const void* table) {
    return reinterpret_cast<uintptr_t>(table) % (d.table_dtype == ALSGD_BF16 ? 2 : 4) == 0;
}

// A [batch, position, head, dim] operand: 16-byte steps, no step of zero between elements that differ in an output.
inline int check_tensor(const alsgd_attn_tensor* t, uint32_t batch, uint32_t len, uint32_t heads, bool output) {
    if (!t) return ALSGD_E_ARG;
    if (len == 0) return ALSGD_OK;
    if (!t->data || reinterpret_cast<uintptr_t>(t->data) % 16) return ALSGD_E_ARG;
    const int64_t step[3] = {t->stride_pos, t->stride_head, t->stride_batch};
    const uint64_t extent[3] = {len, heads, batch};
    for (int i = 0; i < 3; ++i) {
        if (extent[i] == 1) continue;
        if (step[i] < 0 || step[i] % 8 || step[i] >= (1ll << 39)) return ALSGD_E_ARG;
        if (step[i] == 0 && (output || i == 0)) return ALSGD_E_ARG;
    }
    return ALSGD_OK;
}

// `rows`: query rows of a work item
inline Shape make_shape(const alsgd_attn_desc& d, const int32_t* kv_len, int rows) {
    Shape s;
    s.batch = (int)d.batch;
    s.heads_q = (int)d.heads_q;
    s.heads_kv = (int)d.heads_kv;
    s.group = (int)(d.heads_q / d.heads_kv);
    s.len_q = (int)d.len_q;
    s.len_kv = (int)d.len_kv;
    s.dim = (int)d.dim;
    s.causal = (d.flags & ALSGD_ATTN_CAUSAL) != 0;
    s.q_pos = d.q_pos;
    s.device = d.device;
    s.scale = d.scale;
    s.scale_log2 = d.scale * kLog2e;
    s.kv_len = kv_len;
    s.keys_end = s.causal ? std::min(s.len_kv, std::max(0, s.len_q + s.q_pos)) : s.len_kv;
    s.by_heads_q = divide_by(s.heads_q);
    s.by_heads_kv = divide_by(s.heads_kv);
    s.by_all_q = divide_by(s.batch * s.heads_q);
    s.by_all_kv = divide_by(s.batch * s.heads_kv);
    s.by_group = divide_by(s.group);
    s.by_rows_q = divide_by(std::max(1, (s.len_q + rows - 1) / rows) * s.heads_q);
    return s;
}

// Boxes of `cols` elements (64, or 32 for results) x `rows` positions of one head of one sequence, swizzled over their
// 128- or 64-byte rows, zeros outside.
inline int make_operand(const alsgd_attn_tensor& t, uint32_t batch, uint32_t len, uint32_t heads, uint32_t dim, uint32_t rows, uint32_t cols, Operand* out) {
    alsgd_tc::EncodeTiled encode = alsgd_tc::encode_tiled();
    if (!encode) return ALSGD_E_CUDA;
    const uint64_t extent[3] = {len, heads, batch};
    const int64_t step[3] = {t.stride_pos, t.stride_head, t.stride_batch};
    cuuint64_t size[4] = {dim, 0, 0, 0}, bytes[3];
    int mul[3];
    for (int i = 0; i < 3; ++i) {
        const bool one = extent[i] == 1 || step[i] == 0;
        mul[i] = !one;
        size[i + 1] = one ? 1 : extent[i];
        bytes[i] = one ? 16 * ((dim * 2 + 15) / 16) : (uint64_t)step[i] * 2;
    }
    out->head_mul = mul[1];
    out->batch_mul = mul[2];
    out->data = static_cast<uint16_t*>(t.data);
    out->step_pos = mul[0] ? step[0] : 0;
    out->step_head = mul[1] ? step[1] : 0;
    out->step_batch = mul[2] ? step[2] : 0;
    const cuuint32_t box[4] = {cols, rows, 1, 1}, unit[4] = {1, 1, 1, 1};
    const CUresult r = encode(&out->map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, t.data, size, bytes, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? ALSGD_OK : ALSGD_E_ARG;
}

}  // namespace alsgd_attn
