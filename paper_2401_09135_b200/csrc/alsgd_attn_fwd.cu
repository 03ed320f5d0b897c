// alsgd_attn_fwd: attention with a learned relative position bias.
//
//   x_ij = scale q_i.k_j + T[bucket(j - i)]  over the allowed j,   lse_i = log sum_j e^x_ij,   o_i = sum_j e^(x_ij - lse_i) v_j
//
// A work item is 128 query rows of one head; two blocks per SM walk the items, those with the most keys first.  Keys come
// in tiles of 128; a row's running maximum and sum are kept by one thread (the row's lane of tensor memory), so a tile is
// read once and nothing of size len_q x len_kv exists.
//   warps 0-3  softmax: scores from tensor memory, maximum, e^x, sum; probabilities (bf16) back to tensor memory
//   warp 4     copies q, then k and v tiles, through tensor maps, up to two tiles and one item ahead
//   warp 5     issues the products  S = q k^T  (operands in shared memory)
//   warp 6     issues the products  O += P v  (P in tensor memory); a warp of its own, so that neither waits in the other's queue
//   warp 7     lays out the next item's bias by distance, which is also its causal mask
// Warps 4-7 give their registers to the softmax warps, whose 128 scores a thread leave no others room (with 168 registers a
// thread a few spilled words in the tile loop cost a quarter of the time).
// Two blocks share an SM (256 tensor memory columns and about 100 KB each): one's products and waits run under the other's
// exponentials.
//
// Exponents are taken in base 2 relative to a reference that follows the running maximum only when that has grown by
// more than 8: the sums then hold values up to 2^8, which binary32 and bf16 hold as well as values up to 1, and O in
// tensor memory is rescaled a few times per row instead of once per tile.  Scores, maximum, sum and O are binary32;
// the probabilities are rounded to bf16 for the second product (the operand type of v), the sum uses them unrounded.
//
// Bound: the softmax warps.  A score costs one exponential (16 per clock and SM) and about five more instructions (product
// and bias, maximum, sum, rounding, loads and stores of tensor memory); the products of one tile run under another's.
// Measured (B200), causal with 32 buckets: 2 x 4096 tokens, 16 heads of 64: 114 us, 0.60 PFLOP/s (110 us without a bias), where
// the exponentials alone are 61 us and the tensor cores are busy for 27 %.  64 x 256 tokens: 42 us, 3.2 TB/s: items of one or
// two tiles, whose beginning and end (q and table in, O out) do not hide behind each other.  77 tokens, 6 heads: 10 us in the
// kernel, the latency of one item.  Heads of 128 in groups of 4, 1000 queries, 511 to 1531 keys: 59 us, 0.64 PFLOP/s.
// Also built and measured: 64-key tiles with four blocks per SM (189 us at 2 x 4096), eight softmax warps that share a row
// (140 us), the exponential as a polynomial on the multiply-add units for part of the scores (slower at every share).
#include "alsgd_attn.cuh"

using namespace alsgd_attn;
using namespace alsgd_ops;
using namespace alsgd_tc;

namespace {

constexpr int kRows = 128;              // query rows of an item
constexpr int kSoftmax = 128;           // threads
constexpr int kThreads = 256;
constexpr int kSoftmaxRegisters = 184, kOtherRegisters = 72;   // 128 threads each; launched with 128 a thread
constexpr int kKeys = 128;              // keys of a tile
constexpr float kRescaleAt = 8.0f;
constexpr uint32_t kTileBytes = 128 * 128;     // 128 rows of 64 bf16

struct FwdArgs {
    Operand q, k, v, o;
    Shape shape;
    Bias bias;
    float* lse;
    LutShape lut;
    int row_blocks, items;
};

// HALVES: 64-column halves of the head dimension (1 up to 64, 2 up to 128).  With one half there is room to keep P beside S,
// so the next tile's scores are computed while this tile's exponentials are, and for a second q; with two, P takes S's place.
// Heads of 64 at 2 x 4096 tokens: 114 us with one half, 141 us with the plan for two.
template <int HALVES>
struct FwdPlan {
    static constexpr int stages = HALVES == 1 ? 2 : 1, q_bufs = HALVES == 1 ? 2 : 1;
    static constexpr bool p_apart = HALVES == 1;
    static constexpr uint32_t columns = 256;
    static constexpr uint32_t s_col = 0, p_col = p_apart ? 128 : 0, o_col = p_apart ? 192 : 128;
    static constexpr uint32_t q_bytes = HALVES * kTileBytes, kv_bytes = HALVES * kTileBytes;
    static constexpr uint32_t tiles_bytes = q_bufs * q_bytes + 2 * stages * kv_bytes;
    static constexpr uint32_t bars = 7 + 4 * q_bufs + 4 * stages;
    static constexpr uint32_t fixed_bytes = tiles_bytes + 256 + sizeof(Ranks);
};

template <int HALVES>
size_t fwd_smem(const LutShape& l, bool lut) {
    return 1024 + FwdPlan<HALVES>::fixed_bytes + (lut ? FwdPlan<HALVES>::q_bufs * l.floats * sizeof(float) + 2 * l.pad + 1 : 0);
}

struct Item {
    int b, h, q0, len, keys, n;        // sequence, head, first row, valid keys, keys any row sees, tiles
};

template <typename RANKS>
__device__ __forceinline__ Item item_at(const FwdArgs& a, const RANKS& ranks, int i) {
    const Shape& sh = a.shape;
    Item t;
    int block;
    query_item(sh, ranks, a.row_blocks, i, block, t.b, t.h, t.len);
    t.q0 = block * kRows;
    t.keys = t.len;
    if (sh.causal) t.keys = min(t.keys, min(t.q0 + kRows, sh.len_q) + sh.q_pos);
    t.n = t.keys > 0 ? (t.keys + kKeys - 1) / kKeys : 0;
    return t;
}

template <int HALVES, bool LUT, typename RANKS>
__global__ void __launch_bounds__(kThreads, 2) attn_fwd_kernel(const __grid_constant__ FwdArgs a) {
    using Plan = FwdPlan<HALVES>;
    constexpr int ST = Plan::stages, QB = Plan::q_bufs;
    extern __shared__ uint8_t raw[];
    uint8_t* smem = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);     // the tiles want 1024-byte lines; still seen to be shared memory
    const uint32_t base = smem_u32(smem);
    const uint32_t sq = base, sk = sq + QB * Plan::q_bytes, sv = sk + ST * Plan::kv_bytes;
    const uint32_t bars = base + Plan::tiles_bytes;
    const uint32_t s_full = bars, s_free = bars + 8, p_ready = bars + 16, pv_done = bars + 24, o_free = bars + 32, drained = bars + 40;
    const uint32_t q_full = bars + 56, q_empty = q_full + 8 * QB;
    const uint32_t k_full = q_empty + 8 * QB, k_empty = k_full + 8 * ST, v_full = k_empty + 8 * ST, v_empty = v_full + 8 * ST;
    const uint32_t lut_full = v_empty + 8 * ST, lut_empty = lut_full + 8 * QB;
    uint32_t* words = reinterpret_cast<uint32_t*>(smem + Plan::tiles_bytes + 8 * Plan::bars);
    volatile uint32_t* dead = words + 1;
    RANKS& ranks = *reinterpret_cast<RANKS*>(smem + Plan::tiles_bytes + 256);
    float* luts = reinterpret_cast<float*>(smem + Plan::fixed_bytes);
    uint8_t* lut_bucket = reinterpret_cast<uint8_t*>(luts + QB * a.lut.floats);

    const Shape& sh = a.shape;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        bar_init(s_full, 1);
        bar_init(s_free, 4);
        bar_init(p_ready, 4);
        bar_init(pv_done, 1);
        bar_init(o_free, 4);
        bar_init(drained, 1);
        bar_init(drained + 8, 1);
        for (int i = 0; i < QB; ++i) {
            bar_init(q_full + 8 * i, 1);
            bar_init(q_empty + 8 * i, 4);
            bar_init(lut_full + 8 * i, 1);
            bar_init(lut_empty + 8 * i, 4);
        }
        for (int i = 0; i < ST; ++i) {
            bar_init(k_full + 8 * i, 1);
            bar_init(k_empty + 8 * i, 1);
            bar_init(v_full + 8 * i, 1);
            bar_init(v_empty + 8 * i, 1);
        }
        words[1] = 0;
        bar_init_fence();
    }
    if (warp == 5) tmem_alloc(smem_u32(words), Plan::columns);
    if (threadIdx.x == kSoftmax) {
        tma_prefetch(&a.q.map);
        tma_prefetch(&a.k.map);
        tma_prefetch(&a.v.map);
        tma_prefetch(&a.o.map);
    }
    if (LUT && warp < 4) {
        if (a.bias.table) fill_buckets(a.bias, lut_bucket, a.lut.pad, threadIdx.x, kSoftmax);
        if (sh.causal)
            for (int i = 0; i < QB; ++i) mask_ahead(luts + i * a.lut.floats, a.lut, threadIdx.x, kSoftmax);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = words[0];
    grid_dependency_sync();
    if constexpr (RANKS::on) rank_sequences(sh, ranks);

    if (warp >= 4) give_registers<kOtherRegisters>();
    if (warp == 4) {
        int ordinal = 0, tile = 0;                             // items and tiles whose copies have been started
        Item t;
        for (int round = 0; next_item(a, ranks, round, t);) {
            if (t.n == 0) continue;
            if (*dead) break;
            const int hk = sh.by_group(t.h), buf = ordinal % QB;
            auto copy_tile = [&](int j) {
                const int st = tile % ST;
                const uint32_t free_parity = ((tile / ST) & 1) ^ 1;
                wait(k_empty + 8 * st, free_parity, dead, 2);
                bar_expect(k_full + 8 * st, Plan::kv_bytes);
                for (int c = 0; c < HALVES; ++c)
                    tma_load4(sk + st * Plan::kv_bytes + c * kTileBytes, &a.k.map, k_full + 8 * st, 64 * c, j * kKeys, hk * a.k.head_mul, t.b * a.k.batch_mul);
                wait(v_empty + 8 * st, free_parity, dead, 4);
                bar_expect(v_full + 8 * st, Plan::kv_bytes);
                for (int c = 0; c < HALVES; ++c)
                    tma_load4(sv + st * Plan::kv_bytes + c * kTileBytes, &a.v.map, v_full + 8 * st, 64 * c, j * kKeys, hk * a.v.head_mul, t.b * a.v.batch_mul);
                ++tile;
            };
            if (lane == 0) {
                wait(q_empty + 8 * buf, ((ordinal / QB) & 1) ^ 1, dead, 1);
                bar_expect(q_full + 8 * buf, Plan::q_bytes);
                for (int c = 0; c < HALVES; ++c)
                    tma_load4(sq + buf * Plan::q_bytes + c * kTileBytes, &a.q.map, q_full + 8 * buf, 64 * c, t.q0, t.h * a.q.head_mul, t.b * a.q.batch_mul);
                for (int j = 0; j < t.n && !*dead; ++j) copy_tile(j);
            }
            ++ordinal;
        }
        // every copy has landed before the block may leave, whoever else has given up
        if (lane == 0) {
            for (int i = max(0, ordinal - QB); i < ordinal; ++i) drain(q_full + 8 * (i % QB), (i / QB) & 1);
            for (int i = max(0, tile - ST); i < tile; ++i) {
                drain(k_full + 8 * (i % ST), (i / ST) & 1);
                drain(v_full + 8 * (i % ST), (i / ST) & 1);
            }
        }
    } else if (warp == 5) {
        // The warp walks together and one lane issues: what a product is given stays the same for all lanes.
        constexpr uint32_t desc = mma_desc(kKeys, false);
        const bool leader = elect_one();
        const uint64_t q_desc = desc_k_major(sq), k_desc = desc_k_major(sk);
        Cursor<FwdArgs, Item> at;
        for (at.start(a, ranks); at.more; at.next(a, ranks)) {
            const int st = at.tile % ST, buf = at.ordinal % QB;
            if (at.j == 0) wait_warp(q_full + 8 * buf, (at.ordinal / QB) & 1, dead, 8);
            wait_warp(k_full + 8 * st, (at.tile / ST) & 1, dead, 16);
            // the last tile's scores have been read, or (P in their place) used
            if (at.tile > 0) wait_warp(Plan::p_apart ? s_free : pv_done, (at.tile - 1) & 1, dead, 32);
            tc_fence_after();
            const uint64_t qd = q_desc + buf * (Plan::q_bytes >> 4), kd = k_desc + st * (Plan::kv_bytes >> 4);
            if (leader) {
#pragma unroll
                for (int i = 0; i < 4 * HALVES; ++i) {         // 16 elements of the head each; behind dim they are zeros
                    const uint32_t off = ((i >> 2) * kTileBytes + (i & 3) * 32) >> 4;
                    mma_ss(tmem + Plan::s_col, qd + off, kd + off, desc, i > 0);
                }
                mma_commit(s_full);
                mma_commit(k_empty + 8 * st);
            }
            __syncwarp();
        }
        if (leader) {
            mma_commit(drained);
            drain(drained, 0);
        }
    } else if (warp == 6) {
        constexpr uint32_t desc = mma_desc(64 * HALVES, true);
        const bool leader = elect_one();
        const uint64_t v_desc = desc_n_major(sv, kTileBytes);
        Cursor<FwdArgs, Item> at;
        for (at.start(a, ranks); at.more; at.next(a, ranks)) {
            const int st = at.tile % ST;
            if (at.j == 0) wait_warp(o_free, (at.ordinal & 1) ^ 1, dead, 64);  // the last item's O has been read
            wait_warp(v_full + 8 * st, (at.tile / ST) & 1, dead, 256);
            wait_warp(p_ready, at.tile & 1, dead, 128);
            tc_fence_after();
            const int keys = at.item.keys - at.j * kKeys;      // groups of 16 that nobody sees are left out
            const uint64_t vd = v_desc + st * (Plan::kv_bytes >> 4);
            const bool more = at.j > 0;
            if (leader) {
#pragma unroll
                for (int i = 0; i < kKeys / 16; ++i)
                    if (16 * i < keys) mma_ts(tmem + Plan::o_col, tmem + Plan::p_col + i * 8, vd + i * 128, desc, more || i > 0);
                mma_commit(pv_done);
                mma_commit(v_empty + 8 * st);
            }
            __syncwarp();
        }
        if (leader) {
            mma_commit(drained + 8);
            drain(drained + 8, 0);
        }
    } else if (warp == 7) {
        int ordinal = 0;
        Item t;
        for (int round = 0; LUT && next_item(a, ranks, round, t);) {
            if (t.n == 0) continue;
            const int buf = ordinal % QB, first = t.q0 + sh.q_pos;     // distances from the last row's first key to the first row's last
            wait_warp(lut_empty + 8 * buf, ((ordinal / QB) & 1) ^ 1, dead, 1 << 14);
            fill_lut(a.bias, t.h, lut_bucket, luts + buf * a.lut.floats, a.lut, -(first + kRows - 1), sh.causal ? 0 : t.keys - 1 - first, 1, lane, 32);
            __syncwarp();
            if (lane == 0) bar_arrive(lut_full + 8 * buf);
            ++ordinal;
        }
    } else if (warp < 4) {
        take_registers<kSoftmaxRegisters>();
        const int row = threadIdx.x;
        const uint32_t lanes = tmem + ((uint32_t)warp << 21);
        int ordinal = 0, tile = 0;
        bool leaving = false;          // this warp's rows of the last item are on their way out of that item's q
        auto release_q = [&](int buf) {
            if (lane == 0) {
                tma_store_wait_read();
                bar_arrive(q_empty + 8 * buf);
            }
        };
        Item t;
        for (int round = 0; next_item(a, ranks, round, t);) {
            if (t.n == 0) {
                if (t.q0 + row < sh.len_q) {
                    zero_row(a.o, sh.dim, t.b, t.h, t.q0 + row);
                    a.lse[((size_t)t.b * sh.heads_q + t.h) * sh.len_q + t.q0 + row] = -INFINITY;
                }
                continue;
            }
            const int pos = t.q0 + row + sh.q_pos;             // the row's position among the keys
            // rows whose every key up to the sequence's end lies within the causal mask need no other, unless what lies behind may be NaN
            const bool cut = t.len < sh.len_kv || !(sh.causal && min(t.q0 + kRows, sh.len_q) + sh.q_pos <= t.len);
            const int buf = ordinal % QB;
            const float* lut = luts + buf * a.lut.floats;
            float ref = -INFINITY, sum = 0.0f, left = 0.0f, right = 0.0f;      // left, right: the far keys' bias
            if (LUT) {
                wait_warp(lut_full + 8 * buf, (ordinal / QB) & 1, dead, 1 << 15);
                left = lut_far(lut, a.lut, false);
                right = lut_far(lut, a.lut, true);
            }
            for (int j = 0; j < t.n; ++j, ++tile) {
                const int k0 = j * kKeys;
                wait_warp(s_full, tile & 1, dead, 1024);
                tc_fence_after();
                uint32_t v[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(v[c], lanes + Plan::s_col + 32 * c);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_use(v[c]);
                if (Plan::p_apart) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(s_free);
                }

                // x = v * mul + add, in base 2
                float mul = sh.scale_log2, add = 0.0f, top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                auto cut_off = [&] {
#pragma unroll
                    for (int c = 0; c < kKeys; ++c)
                        if (k0 + c >= t.len) v[c >> 5][c & 31] = 0xFF800000u;
                };
                auto highest = [&] {
#pragma unroll
                    for (int c = 0; c < kKeys; c += 2)
                        top[(c >> 1) & 3] = max3(top[(c >> 1) & 3], __uint_as_float(v[c >> 5][c & 31]), __uint_as_float(v[c >> 5][(c & 31) + 1]));
                };
                const Span span = LUT ? span_of(a.bias, k0 - (t.q0 + kRows - 1 + sh.q_pos), k0 + kKeys - 1 - (t.q0 + sh.q_pos)) : kSpanFarLeft;
                if (LUT && span == kSpanMixed) {
                    const float* at = lut_at(lut, a.lut, k0 - pos);
                    const uint64_t mul2v = pack2(mul, mul);
#pragma unroll
                    for (int c = 0; c < kKeys; c += 2) {
                        const float2 b = *reinterpret_cast<const float2*>(at + c);
                        float x, y;
                        unpack2(fma2(pack2(__uint_as_float(v[c >> 5][c & 31]), __uint_as_float(v[c >> 5][(c & 31) + 1])), mul2v, pack2(b.x, b.y)), x, y);
                        v[c >> 5][c & 31] = __float_as_uint(x);
                        v[c >> 5][(c & 31) + 1] = __float_as_uint(y);
                    }
                    mul = 1.0f;
                } else if (LUT) {
                    add = span == kSpanFarRight ? right : left;
                }
                if (cut && k0 + kKeys > t.len) cut_off();
                highest();
                float high = fmaf(max3(max3(top[0], top[1], top[2]), top[3], top[3]), mul, add);
                if (LUT && __any_sync(0xFFFFFFFFu, !(high < INFINITY))) {
                    // a mask was added: an infinite score or a NaN that it should have covered is taken out here
                    if (span == kSpanMixed) {
                        const float* at = lut_at(lut, a.lut, k0 - pos);
#pragma unroll
                        for (int c = 0; c < kKeys; ++c)
                            if (at[c] == -INFINITY) v[c >> 5][c & 31] = 0xFF800000u;
                    } else if (add == -INFINITY) {
#pragma unroll
                        for (int c = 0; c < kKeys; ++c) v[c >> 5][c & 31] = 0xFF800000u;
                    }
                    top[0] = top[1] = top[2] = top[3] = -INFINITY;
                    highest();
                    high = fmaf(max3(max3(top[0], top[1], top[2]), top[3], top[3]), mul, add);
                }

                wait_warp(pv_done, (tile - 1) & 1, dead, 2048);        // O and P of the last tile are free
                tc_fence_after();
                const bool grown = high > ref + kRescaleAt || (ref == -INFINITY && high > -INFINITY);
                if (__any_sync(0xFFFFFFFFu, grown)) {
                    const float next = grown ? high : ref;
                    const float factor = next == -INFINITY ? 1.0f : exp2_fast(ref - next);
                    ref = next;
                    sum *= factor;
                    if (j > 0) {
                        // eight columns at a time: the scores hold the registers
#pragma unroll 1
                        for (int c = 0; c < 64 * HALVES; c += 8) {
                            uint32_t o[8];
                            tmem_ld8(o, lanes + Plan::o_col + c);
                            tmem_wait_ld();
                            tmem_use(o);
#pragma unroll
                            for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                            tmem_st8(lanes + Plan::o_col + c, o);
                        }
                    }
                }
                if (!(high < INFINITY)) ref = NAN;             // an infinite score or a NaN: the row's result is NaN
                const float off = add - (ref == -INFINITY ? 0.0f : ref);
                const uint64_t mul2v = pack2(mul, mul), off2 = pack2(off, off);
                uint64_t part[2] = {0, 0};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t p[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float x, y;
                        unpack2(fma2(pack2(__uint_as_float(v[c][2 * e]), __uint_as_float(v[c][2 * e + 1])), mul2v, off2), x, y);
                        x = exp2_fast(x);
                        y = exp2_fast(y);
                        part[e & 1] = add2(part[e & 1], pack2(x, y));
                        p[e] = pack_bf16(x, y);
                    }
                    tmem_st16(lanes + Plan::p_col + 16 * c, p);
                }
                float s0, s1;
                unpack2(add2(part[0], part[1]), s0, s1);
                sum += s0 + s1;
                if (k0 + kKeys > t.len && t.len < sh.len_kv) {
                    // v rows behind the sequence's end are whatever the caller has there; 0 * NaN must not reach O
                    const int st = tile % ST;
                    wait_warp(v_full + 8 * st, (tile / ST) & 1, dead, 4096);
                    if (k0 + row >= t.len) {
#pragma unroll
                        for (int c = 0; c < HALVES; ++c)
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                *reinterpret_cast<uint4*>(smem + (sv - base) + st * Plan::kv_bytes + c * kTileBytes + row * 128 + 16 * e) = make_uint4(0, 0, 0, 0);
                    }
                    fence_async_smem();
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_ready);
                if (QB > 1 && leaving) {
                    release_q((ordinal - 1) % QB);
                    leaving = false;
                }
            }
            if (LUT) {
                __syncwarp();
                if (lane == 0) bar_arrive(lut_empty + 8 * buf);
            }
            // O goes out through q's place in shared memory, which is free: q's last product has completed
            wait_warp(pv_done, (tile - 1) & 1, dead, 8192);
            tc_fence_after();
            if (*dead) ref = NAN;                              // a wait has run out: the item's results show it
            const bool none = ref == -INFINITY;                // no allowed key
            const float inv = none ? 0.0f : 1.0f / sum + (ref - ref);
            uint8_t* staging = smem + buf * Plan::q_bytes + warp * 2 * HALVES * 2048;
#pragma unroll
            for (int c = 0; c < 2 * HALVES; ++c) {
                uint32_t o[32];
                tmem_ld32(o, lanes + Plan::o_col + 32 * c);
                tmem_wait_ld();
                tmem_use(o);
                stage_box(o, inv, staging + c * 2048, lane);
            }
            tc_fence_before();
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                bar_arrive(o_free);
                if (t.q0 + 32 * warp < sh.len_q) {
                    for (int c = 0; c < 2 * HALVES; ++c)
                        if (32 * c < sh.dim)
                            tma_store4(&a.o.map, smem_u32(staging) + c * 2048, 32 * c, t.q0 + 32 * warp, t.h * a.o.head_mul, t.b * a.o.batch_mul);
                    tma_store_commit();
                }
            }
            if (t.q0 + row < sh.len_q)
                a.lse[((size_t)t.b * sh.heads_q + t.h) * sh.len_q + t.q0 + row] = none ? -INFINITY : (ref + log2_fast(sum)) * kLn2;
            if (QB > 1) leaving = true;                        // another q is ready: this one's place may wait
            else release_q(buf);
            ++ordinal;
        }
        if (leaving) release_q((ordinal - 1) % QB);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        tmem_free(tmem, Plan::columns);
    }
}

template <int HALVES, bool LUT, typename RANKS>
int launch_fwd(FwdArgs& a, cudaStream_t s) {
    const size_t smem = fwd_smem<HALVES>(a.lut, LUT);
    static SmemLimit limit;
    if (!limit.raise(attn_fwd_kernel<HALVES, LUT, RANKS>, a.shape.device, smem)) return ALSGD_E_CUDA;
    const int wave = blocks_at_once(smem, 2);
    return launch_dependent(attn_fwd_kernel<HALVES, LUT, RANKS>, dim3(a.items < wave ? a.items : wave), dim3(kThreads), smem, s, a) == cudaSuccess ? ALSGD_OK
                                                                                                                                             : ALSGD_E_CUDA;
}

template <typename RANKS>
int launch_fwd(FwdArgs& a, bool wide, bool lut, cudaStream_t s) {
    if (wide) return lut ? launch_fwd<2, true, RANKS>(a, s) : launch_fwd<2, false, RANKS>(a, s);
    return lut ? launch_fwd<1, true, RANKS>(a, s) : launch_fwd<1, false, RANKS>(a, s);
}

}  // namespace

extern "C" int alsgd_attn_fwd(const alsgd_attn_desc* desc, const alsgd_attn_tensor* q, const alsgd_attn_tensor* k, const alsgd_attn_tensor* v,
                              const void* table, const int32_t* kv_len, const alsgd_attn_tensor* o, float* lse, void* stream) {
    int rc = check_desc(desc);
    if (rc != ALSGD_OK) return rc;
    const alsgd_attn_desc& d = *desc;
    if ((d.buckets != 0) != (table != nullptr) || !table_aligned(d, table) || reinterpret_cast<uintptr_t>(kv_len) % 4) return ALSGD_E_ARG;
    if (d.len_q && (!lse || reinterpret_cast<uintptr_t>(lse) % 4)) return ALSGD_E_ARG;
    if ((rc = check_tensor(q, d.batch, d.len_q, d.heads_q, false)) != ALSGD_OK) return rc;
    if ((rc = check_tensor(k, d.batch, d.len_kv, d.heads_kv, false)) != ALSGD_OK) return rc;
    if ((rc = check_tensor(v, d.batch, d.len_kv, d.heads_kv, false)) != ALSGD_OK) return rc;
    if ((rc = check_tensor(o, d.batch, d.len_q, d.heads_q, true)) != ALSGD_OK) return rc;
    if (d.len_q == 0) return ALSGD_OK;

    const uint64_t row_blocks = (d.len_q + kRows - 1) / kRows, items = (uint64_t)d.batch * d.heads_q * row_blocks;
    if (items > 0x7FFFFFFFull - 2 * kSMs) return ALSGD_E_RANGE;
    UseDevice use(d.device);
    if (!use.ok) return ALSGD_E_CUDA;
    FwdArgs a;
    a.shape = make_shape(d, kv_len, kRows);
    make_bias(d, table, &a.bias);
    a.lse = lse;
    a.lut = lut_shape(a.bias.far, kRows, kKeys, a.shape.causal);
    a.row_blocks = (int)row_blocks;
    a.items = (int)items;
    if ((rc = make_operand(*q, d.batch, d.len_q, d.heads_q, d.dim, kRows, 64, &a.q)) != ALSGD_OK) return rc;
    if ((rc = make_operand(*o, d.batch, d.len_q, d.heads_q, d.dim, 32, 32, &a.o)) != ALSGD_OK) return rc;
    // without keys the kernel touches neither map
    if ((rc = make_operand(d.len_kv ? *k : *q, d.batch, d.len_kv ? d.len_kv : d.len_q, d.len_kv ? d.heads_kv : d.heads_q, d.dim, kKeys, 64, &a.k)) != ALSGD_OK) return rc;
    if ((rc = make_operand(d.len_kv ? *v : *q, d.batch, d.len_kv ? d.len_kv : d.len_q, d.len_kv ? d.heads_kv : d.heads_q, d.dim, kKeys, 64, &a.v)) != ALSGD_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool lut = d.buckets || a.shape.causal;
    if (by_rank(a.shape)) return launch_fwd<Ranks>(a, d.dim > 64, lut, s);
    return launch_fwd<NoRanks>(a, d.dim > 64, lut, s);
}

extern "C" int alsgd_attn_status(int32_t device, uint32_t* waits_out) {
    if (!waits_out) return ALSGD_E_ARG;
    if (device < 0 || device >= kMaxDevices) return ALSGD_E_RANGE;
    UseDevice use(device);
    if (!use.ok) return ALSGD_E_CUDA;
    unsigned fwd = 0, bwd = 0;
    // the copies alone would wait for the default stream, but not for streams that are independent of it
    if (cudaDeviceSynchronize() != cudaSuccess) return ALSGD_E_CUDA;
    if (cudaMemcpyFromSymbol(&fwd, g_wait_error, sizeof fwd) != cudaSuccess || !bwd_wait_word(&bwd)) return ALSGD_E_CUDA;
    *waits_out = fwd | bwd;
    return ALSGD_OK;
}

extern "C" int alsgd_attn_bucket(const alsgd_attn_desc* desc, int32_t distance, uint32_t* bucket_out) {
    if (!bucket_out) return ALSGD_E_ARG;
    const int rc = check_desc(desc);
    if (rc != ALSGD_OK) return rc;
    if (desc->buckets == 0) return ALSGD_E_ARG;
    Bias s;
    make_bias(*desc, nullptr, &s);
    const int64_t r = distance, a = s.two_sided ? (r < 0 ? -r : r) : (r < 0 ? -r : 0);
    int64_t at = a;
    if (a >= s.near) {
        at = s.near;
        for (int i = 0; i < s.n_limits; ++i) at += a >= s.limits[i];
    }
    *bucket_out = (uint32_t)(at + (s.two_sided && r > 0 ? s.per_side : 0));
    return ALSGD_OK;
}
