// alsgd_attn_bwd: gradients of attention with a learned relative position bias.  The probabilities are formed again
// from the scores and the forward pass's log-sum-exp:
//
//   p_ij = e^(x_ij - lse_i)      dv_j = sum_i p_ij do_i                  dp_ij = do_i . v_j
//   delta_i = do_i . o_i         ds_ij = p_ij (dp_ij - delta_i)          dT[bucket] = sum of ds_ij over its distances
//   dq_i = scale sum_j ds_ij k_j                                         dk_j = scale sum_i ds_ij q_i
//
// Two kernels, each with its sums in tensor memory, so that nothing is added by atomics and a result's bits do not
// depend on the order in which blocks finish:
//   attn_dq_kernel    128 query rows against tiles of 64 keys:    S, dP, dQ += dS K; also delta and the bias' gradient
//   attn_dkv_kernel   128 keys against tiles of 64 query rows:    S', dP', dV += P' dO, dK += dS' Q (transposed tiles:
//                     a lane holds one key); the query heads that share a key head are walked by the same block
// One kernel that forms S and dP once would save two of the seven products and half of the exponentials, but has to
// add dQ across blocks: 32 KB of binary32 for every 128 x 128 scores, which at a head of 64 costs the L2 more than the
// second pass costs the tensor cores.
//
// Both are built like the forward kernel: blocks walk work items sorted by their tiles; groups of four warps do the
// arithmetic, one thread to a row of a tile; warps of their own copy tiles, issue S and dP, issue the sums, and lay out
// the next item's bias by distance (with it the causal mask).  dq: two blocks per SM with one such group each.  dkv: one
// block per SM with two groups that take the item's tiles in turn, because dV, dK and two tiles fill tensor memory.
//
// Everything is binary32 but the operands of the second products: p and ds are rounded to bf16 (the type of do, q and
// k), as the forward pass rounds p.
//
// Bound: the arithmetic warps, as in the forward kernel, with the exponentials taken twice (122 us of them at 2 x 4096 tokens,
// 16 heads of 64).  Measured (B200), causal with 32 buckets, dq / dkv / dtable one after the other without overlap:
//   2 x 4096 tokens, 16 heads of 64:    180 / 183 / 4 us, 372 to 385 together (the higher at the power limit): 0.46 PFLOP/s,
//                                       tensor cores busy for 26 and 35 %; 337 us without a bias
//   64 x 256 tokens, 16 heads of 64:    95 / 85 / 7 us, 184 together: 1.5 TB/s.  Every tile lies across the diagonal: the bias'
//                                       gradient by distance is 16 us of it, delta 15 us, the look for masked pairs whose
//                                       scores overflow 10 us, the rest items that begin and end; 151 us without a bias
//   1000 x 511 to 1531, heads of 128 in groups of 4: 108 / 83 / 3 us, 199 together, 0.47 PFLOP/s
#include "alsgd_attn.cuh"

using namespace alsgd_attn;
using namespace alsgd_ops;
using namespace alsgd_tc;

namespace {

constexpr int kOwn = 128;               // rows of an item
constexpr int kStep = 64;               // rows of a streamed tile
constexpr uint32_t kOwnBytes = 128 * 128;      // 128 rows of 64 bf16
constexpr uint32_t kStepBytes = 64 * 128;
constexpr int kGroup = 16, kGroups = kStep / kGroup;   // columns whose diagonals are summed in one chain, chains
constexpr int kChain = kGroup + 32;     // sums a chain leaves, padded
constexpr int kDiagonals = kGroups * kChain;            // of a warp; lanes that have none to leave write as many beside them

constexpr int kDqMath = 128, kDqThreads = 256;  // the threads that do the arithmetic of attn_dq_kernel, all of them

// =============================================================================================== dq

struct DqArgs {
    Operand q, k, v, dout, dq;
    Shape shape;
    Bias bias;
    const float* lse;
    const uint16_t* o;
    int64_t o_batch, o_pos, o_head;     // steps of o
    float* delta;                       // out: [batch][heads_q][len_q]
    float* partial;                     // out: [batch * heads_q][row blocks][4 warps][buckets]
    LutShape lut;
    int row_blocks, items;
};

struct DqItem {
    int b, h, block, q0, len, keys, n;  // sequence, head, row block, first row, valid keys, keys any row sees, tiles
};

template <typename RANKS>
__device__ __forceinline__ DqItem item_at(const DqArgs& a, const RANKS& ranks, int i) {
    const Shape& sh = a.shape;
    DqItem t;
    query_item(sh, ranks, a.row_blocks, i, t.block, t.b, t.h, t.len);
    t.q0 = t.block * kOwn;
    t.keys = t.len;
    if (sh.causal) t.keys = min(t.keys, min(t.q0 + kOwn, sh.len_q) + sh.q_pos);
    t.n = t.keys > 0 ? (t.keys + kStep - 1) / kStep : 0;
    return t;
}

template <int HALVES>
struct DqPlan {
    static constexpr int stages = HALVES == 1 ? 2 : 1, own_bufs = HALVES == 1 ? 2 : 1;
    static constexpr bool apart = HALVES == 1;         // dS beside S, so that the next tile's scores need not wait for dQ
    static constexpr int math_registers = HALVES == 1 ? 200 : 184, other_registers = 256 - math_registers; // 128 threads each; launched with 128 a thread
    static constexpr uint32_t columns = 256;
    static constexpr uint32_t s_col = 0, dp_col = 64, dq_col = 128, ds_col = apart ? 192 : 0;
    static constexpr uint32_t own_bytes = HALVES * kOwnBytes, step_bytes = HALVES * kStepBytes;
    static constexpr uint32_t tiles_bytes = own_bufs * 2 * own_bytes + 2 * stages * step_bytes;
    static constexpr uint32_t bars = 7 + 4 * own_bufs + 2 * stages;
    static constexpr uint32_t fixed_bytes = tiles_bytes + 256 + sizeof(Ranks);
};

template <int HALVES>
size_t dq_smem(const LutShape& l, bool lut, int buckets) {
    return 1024 + DqPlan<HALVES>::fixed_bytes + (lut ? DqPlan<HALVES>::own_bufs * l.floats * sizeof(float) + 2 * l.pad + 16 : 0) +
           (buckets ? 4 * (kDiagonals + kGroups * kGroup + buckets) * sizeof(float) + buckets * sizeof(short2) : 0);
}

// LUT: there is a bias or a causal mask.  BIAS: there is a bias, and its gradient.
template <int HALVES, bool LUT, bool BIAS, typename RANKS>
__global__ void __launch_bounds__(kDqThreads, 2) attn_dq_kernel(const __grid_constant__ DqArgs a) {
    using Plan = DqPlan<HALVES>;
    constexpr int ST = Plan::stages, OB = Plan::own_bufs;
    extern __shared__ uint8_t raw[];
    uint8_t* smem = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);     // the tiles want 1024-byte lines; still seen to be shared memory
    const uint32_t base = smem_u32(smem);
    const uint32_t sq = base, sdo = sq + OB * Plan::own_bytes, sk = sdo + OB * Plan::own_bytes, sv = sk + ST * Plan::step_bytes;
    const uint32_t bars = base + Plan::tiles_bytes;
    const uint32_t s_full = bars, s_free = bars + 8, ds_ready = bars + 16, dq_done = bars + 24, dq_free = bars + 32, drained = bars + 40;
    const uint32_t own_full = bars + 56, own_empty = own_full + 8 * OB, lut_full = own_empty + 8 * OB, lut_empty = lut_full + 8 * OB;
    const uint32_t full = lut_empty + 8 * OB, empty = full + 8 * ST;
    uint32_t* words = reinterpret_cast<uint32_t*>(smem + Plan::tiles_bytes + 8 * Plan::bars);
    volatile uint32_t* dead = words + 1;
    constexpr int kSums = kDiagonals + kGroups * kGroup;
    RANKS& ranks = *reinterpret_cast<RANKS*>(smem + Plan::tiles_bytes + 256);
    float* diagonals = reinterpret_cast<float*>(smem + Plan::fixed_bytes);             // [4 warps][kSums]
    float* by_bucket = diagonals + (BIAS ? 4 * kSums : 0);                             // [4 warps][buckets]
    short2* spans = reinterpret_cast<short2*>(by_bucket + (BIAS ? 4 * a.bias.buckets : 0));       // distances of a bucket
    float* luts = reinterpret_cast<float*>(spans) + (BIAS ? (a.bias.buckets + 3) / 4 * 4 : 0);
    uint8_t* lut_bucket = reinterpret_cast<uint8_t*>(luts + OB * a.lut.floats);

    const Shape& sh = a.shape;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        bar_init(s_full, 1);
        bar_init(s_free, 4);
        bar_init(ds_ready, 4);
        bar_init(dq_done, 1);
        bar_init(dq_free, 4);
        bar_init(drained, 1);
        bar_init(drained + 8, 1);
        for (int i = 0; i < OB; ++i) {
            bar_init(own_full + 8 * i, 1);
            bar_init(own_empty + 8 * i, 4);
            bar_init(lut_full + 8 * i, 1);
            bar_init(lut_empty + 8 * i, 4);
        }
        for (int i = 0; i < ST; ++i) {
            bar_init(full + 8 * i, 1);
            bar_init(empty + 8 * i, 1);
        }
        words[1] = 0;
        bar_init_fence();
    }
    if (warp == 5) tmem_alloc(smem_u32(words), Plan::columns);
    if (threadIdx.x == kDqMath) {
        tma_prefetch(&a.q.map);
        tma_prefetch(&a.dout.map);
        tma_prefetch(&a.k.map);
        tma_prefetch(&a.v.map);
        tma_prefetch(&a.dq.map);
    }
    if (LUT && warp < 4) {
        if (BIAS) {
            fill_buckets(a.bias, lut_bucket, a.lut.pad, threadIdx.x, kDqMath);
            for (int e = threadIdx.x; e < a.bias.buckets; e += kDqMath) {
                int first, last;
                bucket_span(a.bias, e, first, last);
                spans[e] = make_short2((short)first, (short)last);
            }
        }
        if (sh.causal)
            for (int i = 0; i < OB; ++i) mask_ahead(luts + i * a.lut.floats, a.lut, threadIdx.x, kDqMath);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = words[0];
    grid_dependency_sync();
    if constexpr (RANKS::on) rank_sequences(sh, ranks);

    if (warp >= 4) give_registers<Plan::other_registers>();
    if (warp == 4) {
        if (lane == 0) {
            int ordinal = 0, tile = 0;                         // items and tiles whose copies have been started
            DqItem t;
            for (int round = 0; next_item(a, ranks, round, t);) {
                if (t.n == 0) continue;
                if (*dead) break;
                const int hk = sh.by_group(t.h), buf = ordinal % OB;
                wait(own_empty + 8 * buf, ((ordinal / OB) & 1) ^ 1, dead, 1 << 16);
                bar_expect(own_full + 8 * buf, 2 * Plan::own_bytes);
                for (int c = 0; c < HALVES; ++c) {
                    const uint32_t at = buf * Plan::own_bytes + c * kOwnBytes;
                    tma_load4(sq + at, &a.q.map, own_full + 8 * buf, 64 * c, t.q0, t.h * a.q.head_mul, t.b * a.q.batch_mul);
                    tma_load4(sdo + at, &a.dout.map, own_full + 8 * buf, 64 * c, t.q0, t.h * a.dout.head_mul, t.b * a.dout.batch_mul);
                }
                ++ordinal;
                const int pos = t.q0 + sh.q_pos;               // of the first row
                for (int j = 0; j < t.n && !*dead; ++j, ++tile) {
                    const int st = tile % ST;
                    const int from = BIAS && far_out(a.bias, t.h, j * kStep - (pos + kOwn - 1), (j + 1) * kStep - 1 - pos) ? sh.len_kv : j * kStep;
                    wait(empty + 8 * st, ((tile / ST) & 1) ^ 1, dead, 2 << 16);
                    bar_expect(full + 8 * st, 2 * Plan::step_bytes);
                    for (int c = 0; c < HALVES; ++c) {
                        const uint32_t at = st * Plan::step_bytes + c * kStepBytes;
                        tma_load4(sk + at, &a.k.map, full + 8 * st, 64 * c, from, hk * a.k.head_mul, t.b * a.k.batch_mul);
                        tma_load4(sv + at, &a.v.map, full + 8 * st, 64 * c, from, hk * a.v.head_mul, t.b * a.v.batch_mul);
                    }
                }
            }
            // every copy has landed before the block may leave, whoever else has given up
            for (int i = max(0, ordinal - OB); i < ordinal; ++i) drain(own_full + 8 * (i % OB), (i / OB) & 1);
            for (int i = max(0, tile - ST); i < tile; ++i) drain(full + 8 * (i % ST), (i / ST) & 1);
        }
    } else if (warp == 5) {
        // The warp walks together and one lane issues: what a product is given stays the same for all lanes.
        constexpr uint32_t desc = mma_desc(kStep, false);
        const bool leader = elect_one();
        const uint64_t q_desc = desc_k_major(sq), do_desc = desc_k_major(sdo), k_desc = desc_k_major(sk), v_desc = desc_k_major(sv);
        Cursor<DqArgs, DqItem> at;
        for (at.start(a, ranks); at.more; at.next(a, ranks)) {
            const int st = at.tile % ST, buf = at.ordinal % OB;
            if (at.j == 0) wait_warp(own_full + 8 * buf, (at.ordinal / OB) & 1, dead, 4 << 16);
            wait_warp(full + 8 * st, (at.tile / ST) & 1, dead, 8 << 16);
            // the last tile's S and dP have been read, or (dS in their place) used
            if (at.tile > 0) wait_warp(Plan::apart ? s_free : dq_done, (at.tile - 1) & 1, dead, 16 << 16);
            tc_fence_after();
            const uint32_t own = buf * (Plan::own_bytes >> 4), step = st * (Plan::step_bytes >> 4);
            if (leader) {
#pragma unroll
                for (int i = 0; i < 4 * HALVES; ++i) {         // 16 elements of the head each; behind dim they are zeros
                    const uint32_t o = own + (((i >> 2) * kOwnBytes + (i & 3) * 32) >> 4), s = step + (((i >> 2) * kStepBytes + (i & 3) * 32) >> 4);
                    mma_ss(tmem + Plan::s_col, q_desc + o, k_desc + s, desc, i > 0);
                    mma_ss(tmem + Plan::dp_col, do_desc + o, v_desc + s, desc, i > 0);
                }
                mma_commit(s_full);
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
        const uint64_t k_desc = desc_n_major(sk, kStepBytes);
        Cursor<DqArgs, DqItem> at;
        for (at.start(a, ranks); at.more; at.next(a, ranks)) {
            const int st = at.tile % ST;
            if (at.j == 0) wait_warp(dq_free, (at.ordinal & 1) ^ 1, dead, 32 << 16);   // the last item's dQ has been read
            wait_warp(ds_ready, at.tile & 1, dead, 64 << 16);
            tc_fence_after();
            const uint64_t kd = k_desc + st * (Plan::step_bytes >> 4);
            const bool more = at.j > 0;
            if (leader) {
#pragma unroll
                for (int i = 0; i < kStep / 16; ++i) mma_ts(tmem + Plan::dq_col, tmem + Plan::ds_col + i * 8, kd + i * 128, desc, more || i > 0);
                mma_commit(dq_done);
                mma_commit(empty + 8 * st);
            }
            __syncwarp();
        }
        if (leader) {
            mma_commit(drained + 8);
            drain(drained + 8, 0);
        }
    } else if (warp == 7) {
        int ordinal = 0;
        DqItem t;
        for (int round = 0; LUT && next_item(a, ranks, round, t);) {
            if (t.n == 0) continue;
            const int buf = ordinal % OB, first = t.q0 + sh.q_pos;     // distances from the last row's first key to the first row's last
            wait_warp(lut_empty + 8 * buf, ((ordinal / OB) & 1) ^ 1, dead, 128 << 16);
            const bool out = fill_lut(a.bias, t.h, lut_bucket, luts + buf * a.lut.floats, a.lut, -(first + kOwn - 1), sh.causal ? 0 : t.keys - 1 - first, 1, lane, 32);
            const bool outs = __any_sync(0xFFFFFFFFu, out);
            if (lane == 0) lut_set_outs(luts + buf * a.lut.floats, a.lut, outs);
            __syncwarp();
            if (lane == 0) bar_arrive(lut_full + 8 * buf);
            ++ordinal;
        }
    } else if (warp < 4) {
        take_registers<Plan::math_registers>();
        const int row = threadIdx.x;
        const uint32_t lanes = tmem + ((uint32_t)warp << 21);
        float* sums = diagonals + warp * kSums;
        float* leaves = lane == 31 ? sums : sums + kDiagonals;         // a chain's end, and a place nobody reads
        const int leave_step = lane == 31 ? kChain : kGroup;
        const float not_first = lane == 0 ? 0.0f : 1.0f;               // nothing comes into lane 0
        float* bucket_sums = by_bucket + warp * a.bias.buckets;
        int ordinal = 0, tile = 0;
        bool leaving = false;          // this warp's rows of the last item are on their way out of that item's q
        auto release_own = [&](int buf) {
            if (lane == 0) {
                tma_store_wait_read();
                bar_arrive(own_empty + 8 * buf);
            }
        };
        // The warp's rows of o, which delta wants, and lse, asked for one item ahead (rows of 64; twice that would hold too many
        // registers).  Eight lanes to a row, four rows at a time: o[i] is 16 bytes of row 4 i + lane / 8.
        uint4 o[8 * HALVES];
        float next_lse = -INFINITY;
        auto ask_for_o = [&](const DqItem& t) {
            const uint16_t* p = a.o + (int64_t)t.b * a.o_batch + (int64_t)t.h * a.o_head + 8 * (lane & 7);
            next_lse = t.q0 + row < sh.len_q ? a.lse[((size_t)t.b * sh.heads_q + t.h) * sh.len_q + t.q0 + row] : -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = t.q0 + 32 * warp + 4 * i + (lane >> 3);
#pragma unroll
                for (int c = 0; c < HALVES; ++c)
                    o[c * 8 + i] = r < sh.len_q && 64 * c + 8 * (lane & 7) < sh.dim ? *reinterpret_cast<const uint4*>(p + (int64_t)r * a.o_pos + 64 * c)
                                                                                : make_uint4(0, 0, 0, 0);
            }
        };
        // this thread's row of do . o
        auto delta_of = [&](const uint8_t* dout) {
            float part[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = 32 * warp + 4 * i + (lane >> 3);
                float acc[2] = {0.0f, 0.0f};
#pragma unroll
                for (int c = 0; c < HALVES; ++c) {
                    const uint4 x = o[c * 8 + i], y = *reinterpret_cast<const uint4*>(dout + c * kOwnBytes + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
                    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        acc[0] = fmaf(bf16_lo(xs[e]), bf16_lo(ys[e]), acc[0]);
                        acc[1] = fmaf(bf16_hi(xs[e]), bf16_hi(ys[e]), acc[1]);
                    }
                }
                part[i] = acc[0] + acc[1];
            }
            // sums over the eight lanes, halving what each lane still carries: lane 8 q + k ends with row 4 k + q
#pragma unroll
            for (int step = 4; step > 0; step >>= 1) {
                const bool upper = lane & step;
#pragma unroll
                for (int i = 0; i < step; ++i) {
                    const float give = upper ? part[i] : part[i + step], keep = upper ? part[i + step] : part[i];
                    part[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, step);
                }
            }
            return __shfl_sync(0xFFFFFFFFu, part[0], (lane & 3) * 8 + (lane >> 2));
        };
        int round = 0;
        DqItem t;
        bool more = next_item(a, ranks, round, t);
        if (more && HALVES == 1) ask_for_o(t);
        while (more) {
            if (HALVES == 2) ask_for_o(t);
            const int buf = ordinal % OB;
            const bool inside = t.q0 + row < sh.len_q;
            const size_t stat = ((size_t)t.b * sh.heads_q + t.h) * sh.len_q + t.q0 + row;
            float* partial = a.partial + ((((size_t)t.b * sh.heads_q + t.h) * a.row_blocks + t.block) * 4 + warp) * a.bias.buckets;
            if (t.n == 0) {
                if (inside) {
                    zero_row(a.dq, sh.dim, t.b, t.h, t.q0 + row);
                    a.delta[stat] = 0.0f;
                }
                if (BIAS)
                    for (int e = lane; e < a.bias.buckets; e += 32) partial[e] = 0.0f;
                more = next_item(a, ranks, round, t);
                if (more && HALVES == 1) ask_for_o(t);
                continue;
            }
            const float lse = next_lse;
            const bool live = lse != -INFINITY;
            const int pos = t.q0 + row + sh.q_pos;
            const float* lut = luts + buf * a.lut.floats;
            if (BIAS) {
                for (int e = lane; e < a.bias.buckets; e += 32) bucket_sums[e] = 0.0f;
                __syncwarp();
            }
            wait_warp(own_full + 8 * buf, (ordinal / OB) & 1, dead, 256 << 16);
            float delta = delta_of(smem + (sdo - base) + buf * Plan::own_bytes);
            if (!live) delta = 0.0f;                           // whatever do holds
            if (*dead) delta = NAN;
            if (inside) a.delta[stat] = delta;

            // A row with one allowed key has p = 1 whatever its score: ds = 0, where dp - delta would leave two sums' noise.
            const int seen = sh.causal ? min(t.len, pos + 1) : t.len;
            const bool used = live && seen > 1;
            // rows whose every key up to the sequence's end lies within the causal mask need no other, unless what lies behind may be NaN
            const bool cut = t.len < sh.len_kv || !(sh.causal && min(t.q0 + kOwn, sh.len_q) + sh.q_pos <= t.len);
            const bool some_idle = __any_sync(0xFFFFFFFFu, !used);
            const float lse2 = live ? lse * kLog2e : 0.0f;
            float far_left = 0.0f, far_right = 0.0f, left = 0.0f, right = 0.0f;        // left, right: the far keys' bias
            if (LUT) {
                wait_warp(lut_full + 8 * buf, (ordinal / OB) & 1, dead, 1024 << 16);
                left = lut_far(lut, a.lut, false);
                right = lut_far(lut, a.lut, true);
            }
            for (int j = 0; j < t.n; ++j, ++tile) {
                const int k0 = j * kStep;
                wait_warp(s_full, tile & 1, dead, 512 << 16);
                tc_fence_after();
                uint32_t s[2][32], d[2][32];
                tmem_ld32(s[0], lanes + Plan::s_col);
                tmem_ld32(s[1], lanes + Plan::s_col + 32);
                tmem_ld32(d[0], lanes + Plan::dp_col);
                tmem_ld32(d[1], lanes + Plan::dp_col + 32);
                tmem_wait_ld();
                tmem_use(s[0]);
                tmem_use(s[1]);
                tmem_use(d[0]);
                tmem_use(d[1]);
                if (Plan::apart) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(s_free);
                }
                const Span span = LUT ? span_of(a.bias, k0 - (t.q0 + kOwn - 1 + sh.q_pos), k0 + kStep - 1 - (t.q0 + sh.q_pos)) : kSpanFarLeft;
                const bool mixed = LUT && span == kSpanMixed;
                const uint64_t mul2v = pack2(sh.scale_log2, sh.scale_log2), nd2 = pack2(-delta, -delta);
                // ds from x - lse = s * mul + off, in base 2
                auto gradient = [&](auto off2) {
#pragma unroll
                    for (int c = 0; c < kStep; c += 2) {
                        float x, y;
                        unpack2(fma2(pack2(__uint_as_float(s[c >> 5][c & 31]), __uint_as_float(s[c >> 5][(c & 31) + 1])), mul2v, off2(c)), x, y);
                        const uint64_t p = pack2(exp2_fast(x), exp2_fast(y));
                        unpack2(mul2(p, add2(pack2(__uint_as_float(d[c >> 5][c & 31]), __uint_as_float(d[c >> 5][(c & 31) + 1])), nd2)), x, y);
                        d[c >> 5][c & 31] = __float_as_uint(x);
                        d[c >> 5][(c & 31) + 1] = __float_as_uint(y);
                    }
                };
                if (mixed) {
                    const float* at = lut_at(lut, a.lut, k0 - pos);
                    const uint64_t lse2v = pack2(-lse2, -lse2);
                    gradient([&](int c) {
                        const float2 b = *reinterpret_cast<const float2*>(at + c);
                        return add2(pack2(b.x, b.y), lse2v);
                    });
                    // the warp's part of the tile may hold masked pairs
                    if ((sh.causal && k0 + kStep - 1 > t.q0 + 32 * warp + sh.q_pos) || (BIAS && lut_outs(lut, a.lut))) {
                        float top[2] = {0.0f, 0.0f};
#pragma unroll
                        for (int c = 0; c < kStep; c += 2)
                            top[(c >> 1) & 1] = max3(top[(c >> 1) & 1], __uint_as_float(d[c >> 5][c & 31]), __uint_as_float(d[c >> 5][(c & 31) + 1]));
                        if (__builtin_expect(__any_sync(0xFFFFFFFFu, isnan(top[0]) || isnan(top[1])), 0)) {
#pragma unroll
                            for (int c = 0; c < kStep; ++c)
                                if (lut_at(lut, a.lut, k0 - pos)[c] == -INFINITY) d[c >> 5][c & 31] = 0;
                        }
                    }
                } else {
                    const float off = (LUT ? (span == kSpanFarRight ? right : left) : 0.0f) - lse2;
                    const uint64_t off2v = pack2(off, off);
                    gradient([&](int) { return off2v; });
                }
                if (some_idle || (cut && k0 + kStep > t.len)) {
                    const int end = used ? t.len - k0 : 0;
#pragma unroll
                    for (int c = 0; c < kStep; ++c)
                        if (c >= end) d[c >> 5][c & 31] = 0;
                }
                if (Plan::apart) {                             // dS of the last tile has been used
                    wait_warp(dq_done, (tile - 1) & 1, dead, 2048 << 16);
                    tc_fence_after();
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e] = pack_bf16(__uint_as_float(d[c][2 * e]), __uint_as_float(d[c][2 * e + 1]));
                    tmem_st16(lanes + Plan::ds_col + 16 * c, w);
                }
                if (k0 + kStep > t.len && t.len < sh.len_kv) {
                    // keys behind the sequence's end may hold anything; 0 * NaN must not reach dq
                    const int st = tile % ST, r = row & (kStep - 1), part = row >> 6;
                    if (k0 + r >= t.len) {
#pragma unroll
                        for (int c = 0; c < HALVES; ++c)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                *reinterpret_cast<uint4*>(smem + (sk - base) + st * Plan::step_bytes + c * kStepBytes + r * 128 + 64 * part + 16 * e) = make_uint4(0, 0, 0, 0);
                    }
                    fence_async_smem();
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(ds_ready);
                if (BIAS) {
                    if (!mixed) {
                        uint64_t both[2] = {0, 0};
#pragma unroll
                        for (int c = 0; c < kStep; c += 2)
                            both[(c >> 1) & 1] = add2(both[(c >> 1) & 1], pack2(__uint_as_float(d[c >> 5][c & 31]), __uint_as_float(d[c >> 5][(c & 31) + 1])));
                        float x, y;
                        unpack2(add2(both[0], both[1]), x, y);
                        if (span == kSpanFarLeft) far_left += x + y; else far_right += x + y;
                    } else {
                        // Sums along the diagonals of the warp's 32 x 64 part: a running sum moves one lane down per column and
                        // leaves at lane 31, complete.  Four groups of 16 columns, whose chains of shuffles overlap.
                        float run[kGroups][4];
#pragma unroll
                        for (int g = 0; g < kGroups; ++g) run[g][3] = 0.0f;
#pragma unroll
                        for (int c = 0; c < kGroup; ++c) {
#pragma unroll
                            for (int g = 0; g < kGroups; ++g) {
                                const float moved = __shfl_up_sync(0xFFFFFFFFu, run[g][(c + 3) & 3], 1);
                                run[g][c & 3] = fmaf(moved, not_first, __uint_as_float(d[(kGroup * g + c) >> 5][(kGroup * g + c) & 31]));
                                if ((c & 3) == 3)
                                    *reinterpret_cast<float4*>(leaves + leave_step * g + c - 3) = make_float4(run[g][0], run[g][1], run[g][2], run[g][3]);
                            }
                        }
#pragma unroll
                        for (int g = 0; g < kGroups; ++g) sums[kChain * g + (lane == 31 ? kChain - 1 : kChain - 2 - lane)] = lane == 31 ? 0.0f : run[g][3];
                        __syncwarp();
                        // A bucket is a run of distances: sums within runs, 32 diagonals at a time, and the last lane of each run
                        // adds to its bucket
                        const int first = k0 - (t.q0 + 32 * warp + 31 + sh.q_pos);     // distance of diagonal 0
                        float x[3];
                        int bucket[3], from[3], to[3];
#pragma unroll
                        for (int e = 0; e < 3; ++e) {
                            const int at = 32 * e + lane;
                            bucket[e] = lut_bucket[a.lut.pad + first + at];
                            const short2 span = spans[bucket[e]];
                            from[e] = max(span.x - first - 32 * e, 0);
                            to[e] = min(span.y - first - 32 * e, 31);
                            x[e] = 0.0f;
#pragma unroll
                            for (int g = 0; g < kGroups; ++g) {
                                const int local = at - kGroup * g;
                                if (local >= 0 && local < kChain) x[e] += sums[kChain * g + local];
                            }
                        }
#pragma unroll
                        for (int o = 1; o < 32; o <<= 1) {
#pragma unroll
                            for (int e = 0; e < 3; ++e) {
                                const float y = __shfl_up_sync(0xFFFFFFFFu, x[e], o);
                                if (lane - o >= from[e]) x[e] += y;
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 3; ++e) {
                            if (lane == to[e]) bucket_sums[bucket[e]] += x[e];
                            __syncwarp();
                        }
                    }
                }
                if (OB > 1 && leaving) {
                    release_own((ordinal - 1) % OB);
                    leaving = false;
                }
            }
            if (LUT) {
                __syncwarp();
                if (lane == 0) bar_arrive(lut_empty + 8 * buf);
            }
            const DqItem last = t;
            more = next_item(a, ranks, round, t);
            if (more && HALVES == 1) ask_for_o(t);
            wait_warp(dq_done, (tile - 1) & 1, dead, 4096 << 16);
            tc_fence_after();
            const bool lost = *dead;                           // a wait has run out: the item's results show it
            if (BIAS) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    far_left += __shfl_down_sync(0xFFFFFFFFu, far_left, o);
                    far_right += __shfl_down_sync(0xFFFFFFFFu, far_right, o);
                }
                if (lane == 0) {
                    bucket_sums[lut_bucket[0]] += far_left;
                    bucket_sums[lut_bucket[2 * a.lut.pad]] += far_right;
                }
                __syncwarp();
                for (int e = lane; e < a.bias.buckets; e += 32) partial[e] = lost ? NAN : bucket_sums[e];
            }
            // dq goes out through q's place, which is free: its last product has completed
            uint8_t* staging = smem + buf * Plan::own_bytes + warp * 2 * HALVES * 2048;
#pragma unroll
            for (int c = 0; c < 2 * HALVES; ++c) {
                uint32_t r[32];
                tmem_ld32(r, lanes + Plan::dq_col + 32 * c);
                tmem_wait_ld();
                tmem_use(r);
                stage_box(r, lost ? NAN : sh.scale, staging + c * 2048, lane);
            }
            tc_fence_before();
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                bar_arrive(dq_free);
                if (last.q0 + 32 * warp < sh.len_q) {
                    for (int c = 0; c < 2 * HALVES; ++c)
                        if (32 * c < sh.dim)
                            tma_store4(&a.dq.map, smem_u32(staging) + c * 2048, 32 * c, last.q0 + 32 * warp, last.h * a.dq.head_mul, last.b * a.dq.batch_mul);
                    tma_store_commit();
                }
            }
            if (OB > 1) leaving = true;                        // another q is ready: this one's place may wait
            else release_own(buf);
            ++ordinal;
        }
        if (leaving) release_own((ordinal - 1) % OB);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        tmem_free(tmem, Plan::columns);
    }
}

// =============================================================================================== dk, dv

struct DkvArgs {
    Operand q, k, v, dout, dk, dv;
    Shape shape;
    Bias bias;
    const float* lse;
    const float* delta;
    LutShape lut;
    int items;
};

struct DkvItem {
    int b, hk, k0, len, q_first, per_head, n;  // sequence, key head, first key, valid keys, first query tile, tiles per query head, tiles
};

template <typename RANKS>
__device__ __forceinline__ DkvItem item_at(const DkvArgs& a, const RANKS& ranks, int i) {
    const Shape& sh = a.shape;
    DkvItem t;
    int block;                                                 // the first keys see the most queries: they come first
    if constexpr (RANKS::on) {
        const int pair = sh.by_heads_kv(i);
        int rank;
        ranked_pair(sh, ranks, kOwn, pair, block, rank);
        t.hk = i - pair * sh.heads_kv;
        t.b = ranks.seq[rank];
        t.len = ranks.len[rank];
    } else {
        block = sh.by_all_kv(i);
        const int bh = i - block * sh.batch * sh.heads_kv;
        t.b = sh.by_heads_kv(bh);
        t.hk = bh - t.b * sh.heads_kv;
        t.len = clamped_len(sh, t.b);
    }
    t.k0 = block * kOwn;
    const int q_tiles = (sh.len_q + kStep - 1) / kStep;
    t.q_first = 0;                                             // the first tile with a row that sees one of the keys
    if (sh.causal && t.k0 > sh.q_pos) t.q_first = min((t.k0 - sh.q_pos) / kStep, q_tiles);
    t.per_head = q_tiles - t.q_first;
    t.n = t.k0 < t.len ? t.per_head * sh.group : 0;
    return t;
}

constexpr int kDkvMath = 256, kDkvThreads = 384;
constexpr int kDkvMathRegisters = 208, kDkvOtherRegisters = 88;   // 256 and 128 threads; launched with 168 a thread

template <int HALVES, int STAGES>
struct DkvPlan {
    static constexpr int stages = STAGES, own_bufs = HALVES == 1 ? 2 : 1;
    static constexpr bool apart = HALVES == 1;         // P and dS beside S and dP, so that the scores two tiles on need not wait for the sums
    static constexpr uint32_t columns = 512;
    static constexpr uint32_t s_col = 0, dp_col = 64, group_cols = 128;                // a group's S and dP; the other group's follow
    static constexpr uint32_t dv_col = 256, dk_col = 256 + 64 * HALVES;
    static constexpr uint32_t p_col = apart ? 384 : s_col, ds_col = apart ? 416 : dp_col, p_cols = apart ? 64 : 128;
    static constexpr uint32_t own_bytes = HALVES * kOwnBytes, step_bytes = HALVES * kStepBytes;
    static constexpr uint32_t tiles_bytes = own_bufs * 2 * own_bytes + 2 * stages * step_bytes;
    static constexpr uint32_t bars = 16 + 2 * own_bufs + 3 * stages;
    static constexpr uint32_t stat_floats = 2 * kStep + 4;     // (-lse in base 2)[64], (-delta)[64], whether the tile has holes
    static constexpr uint32_t ranks_bytes = sizeof(KeyRanks);
    static constexpr uint32_t fixed_bytes = tiles_bytes + 512 + ranks_bytes + stages * stat_floats * sizeof(float);
};

template <int HALVES, int STAGES>
size_t dkv_smem(const LutShape& l, bool lut) {
    return 1024 + DkvPlan<HALVES, STAGES>::fixed_bytes + (lut ? 2 * l.floats * sizeof(float) + 2 * l.pad + 1 : 0);
}

// LUT: there is a bias or a causal mask.  The table by distance is kept for each of the two groups' current query head: table
// (query head's ordinal) % 2, the axis turned round, since a thread's columns are queries.
template <int HALVES, int STAGES, bool LUT, typename RANKS>
__global__ void __launch_bounds__(kDkvThreads, 1) attn_dkv_kernel(const __grid_constant__ DkvArgs a) {
    using Plan = DkvPlan<HALVES, STAGES>;
    constexpr int ST = Plan::stages, OB = Plan::own_bufs;
    extern __shared__ uint8_t raw[];
    uint8_t* smem = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);     // the tiles want 1024-byte lines; still seen to be shared memory
    const uint32_t base = smem_u32(smem);
    const uint32_t sk = base, sv = sk + OB * Plan::own_bytes, sq = sv + OB * Plan::own_bytes, sdo = sq + ST * Plan::step_bytes;
    const uint32_t bars = base + Plan::tiles_bytes;
    const uint32_t s_full = bars, s_free = bars + 16, p_ready = bars + 32, sums_done = bars + 48;      // two each: a group's
    const uint32_t acc_free = bars + 64, acc_done = bars + 72, drained = bars + 80;
    const uint32_t own_full = bars + 96, own_empty = own_full + 8 * OB, lut_full = own_empty + 8 * OB, lut_empty = lut_full + 16;
    const uint32_t full = lut_empty + 16, empty = full + 8 * ST, stat_full = empty + 8 * ST;
    uint32_t* words = reinterpret_cast<uint32_t*>(smem + Plan::tiles_bytes + 8 * Plan::bars);
    volatile uint32_t* dead = words + 1;
    RANKS& ranks = *reinterpret_cast<RANKS*>(smem + Plan::tiles_bytes + 512);
    float* stats = reinterpret_cast<float*>(smem + Plan::tiles_bytes + 512 + Plan::ranks_bytes);
    float* luts = stats + ST * Plan::stat_floats;
    uint8_t* lut_bucket = reinterpret_cast<uint8_t*>(luts + 2 * a.lut.floats);

    const Shape& sh = a.shape;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            bar_init(s_full + 8 * i, 1);
            bar_init(s_free + 8 * i, 4);
            bar_init(p_ready + 8 * i, 4);
            bar_init(sums_done + 8 * i, 1);
            bar_init(lut_full + 8 * i, 1);
            bar_init(lut_empty + 8 * i, 8);
            bar_init(drained + 8 * i, 1);
        }
        bar_init(acc_free, 8);
        bar_init(acc_done, 1);
        for (int i = 0; i < OB; ++i) {
            bar_init(own_full + 8 * i, 1);
            bar_init(own_empty + 8 * i, 8);
        }
        for (int i = 0; i < ST; ++i) {
            bar_init(full + 8 * i, 1);
            bar_init(empty + 8 * i, 1);
            bar_init(stat_full + 8 * i, 1);
        }
        words[1] = 0;
        bar_init_fence();
    }
    if (warp == 9) tmem_alloc(smem_u32(words), Plan::columns);
    if (threadIdx.x == kDkvMath) {
        tma_prefetch(&a.q.map);
        tma_prefetch(&a.dout.map);
        tma_prefetch(&a.k.map);
        tma_prefetch(&a.v.map);
        tma_prefetch(&a.dk.map);
        tma_prefetch(&a.dv.map);
    }
    if (LUT && warp < 8) {
        if (a.bias.table) fill_buckets(a.bias, lut_bucket, a.lut.pad, threadIdx.x, kDkvMath);
        if (sh.causal)
            for (int i = 0; i < 2; ++i) mask_behind(luts + i * a.lut.floats, a.lut, threadIdx.x, kDkvMath);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = words[0];
    grid_dependency_sync();
    if constexpr (RANKS::on) rank_sequences(sh, kOwn, ranks);

    if (warp >= 8) give_registers<kDkvOtherRegisters>();
    if (warp == 8) {
        int ordinal = 0, tile = 0;                             // items and tiles whose copies have been started
        DkvItem t;
        for (int round = 0; next_item(a, ranks, round, t);) {
            if (t.n == 0) continue;
            if (__any_sync(0xFFFFFFFFu, *dead)) break;
            const int buf = ordinal % OB;
            wait_warp(own_empty + 8 * buf, ((ordinal / OB) & 1) ^ 1, dead, 1 << 16);
            if (lane == 0) {
                bar_expect(own_full + 8 * buf, 2 * Plan::own_bytes);
                for (int c = 0; c < HALVES; ++c) {
                    const uint32_t at = buf * Plan::own_bytes + c * kOwnBytes;
                    tma_load4(sk + at, &a.k.map, own_full + 8 * buf, 64 * c, t.k0, t.hk * a.k.head_mul, t.b * a.k.batch_mul);
                    tma_load4(sv + at, &a.v.map, own_full + 8 * buf, 64 * c, t.k0, t.hk * a.v.head_mul, t.b * a.v.batch_mul);
                }
            }
            ++ordinal;
            int head = t.hk * sh.group, q_tile = t.q_first;
            float lse[2], delta[2];                            // of the tile's rows, two per lane, asked for one tile ahead
            auto ask = [&](int head, int q_tile) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = q_tile * kStep + lane + 32 * e;
                    const size_t at = ((size_t)t.b * sh.heads_q + head) * sh.len_q + r;
                    lse[e] = r < sh.len_q ? a.lse[at] : INFINITY;      // behind len_q: p = 0
                    delta[e] = r < sh.len_q ? a.delta[at] : 0.0f;
                }
            };
            ask(head, q_tile);
            for (int j = 0; j < t.n; ++j, ++tile) {
                const int st = tile % ST, pos0 = q_tile * kStep + sh.q_pos;
                const int from = LUT && far_out(a.bias, head, t.k0 - (pos0 + kStep - 1), t.k0 + kOwn - 1 - pos0) ? sh.len_q : q_tile * kStep;
                wait_warp(empty + 8 * st, ((tile / ST) & 1) ^ 1, dead, 2 << 16);
                if (__any_sync(0xFFFFFFFFu, *dead)) break;
                if (lane == 0) {
                    bar_expect(full + 8 * st, 2 * Plan::step_bytes);
                    for (int c = 0; c < HALVES; ++c) {
                        const uint32_t at = st * Plan::step_bytes + c * kStepBytes;
                        tma_load4(sq + at, &a.q.map, full + 8 * st, 64 * c, from, head * a.q.head_mul, t.b * a.q.batch_mul);
                        tma_load4(sdo + at, &a.dout.map, full + 8 * st, 64 * c, from, head * a.dout.head_mul, t.b * a.dout.batch_mul);
                    }
                }
                float* stat = stats + st * Plan::stat_floats;
                bool hole = false;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    hole |= lse[e] == -INFINITY;               // a row without allowed keys: p = 0 too
                    stat[lane + 32 * e] = lse[e] == -INFINITY ? -INFINITY : -lse[e] * kLog2e;
                    stat[kStep + lane + 32 * e] = -delta[e];
                }
                if (++q_tile == t.q_first + t.per_head) {
                    q_tile = t.q_first;
                    ++head;
                }
                if (j + 1 < t.n) ask(head, q_tile);
                hole = __any_sync(0xFFFFFFFFu, hole);
                if (lane == 0) stat[2 * kStep] = hole ? 1.0f : 0.0f;
                __syncwarp();
                if (lane == 0) bar_arrive(stat_full + 8 * st);
            }
        }
        // every copy has landed before the block may leave, whoever else has given up
        for (int i = max(0, ordinal - OB); i < ordinal; ++i) drain(own_full + 8 * (i % OB), (i / OB) & 1);
        for (int i = max(0, tile - ST); i < tile; ++i) drain(full + 8 * (i % ST), (i / ST) & 1);
    } else if (warp == 9) {
        constexpr uint32_t desc = mma_desc(kStep, false);
        const bool leader = elect_one();
        const uint64_t q_desc = desc_k_major(sq), do_desc = desc_k_major(sdo), k_desc = desc_k_major(sk), v_desc = desc_k_major(sv);
        Cursor<DkvArgs, DkvItem> at;
        for (at.start(a, ranks); at.more; at.next(a, ranks)) {
            const int st = at.tile % ST, buf = at.ordinal % OB, g = at.tile & 1;
            if (at.j == 0) wait_warp(own_full + 8 * buf, (at.ordinal / OB) & 1, dead, 4 << 16);
            wait_warp(full + 8 * st, (at.tile / ST) & 1, dead, 8 << 16);
            // the group's last S and dP have been read, or (P and dS in their place) used
            if (at.tile > 1) wait_warp((Plan::apart ? s_free : sums_done) + 8 * g, ((at.tile >> 1) - 1) & 1, dead, 16 << 16);
            tc_fence_after();
            const uint32_t own = buf * (Plan::own_bytes >> 4), step = st * (Plan::step_bytes >> 4), to = tmem + g * Plan::group_cols;
            if (leader) {
#pragma unroll
                for (int i = 0; i < 4 * HALVES; ++i) {
                    const uint32_t o = own + (((i >> 2) * kOwnBytes + (i & 3) * 32) >> 4), s = step + (((i >> 2) * kStepBytes + (i & 3) * 32) >> 4);
                    mma_ss(to + Plan::s_col, k_desc + o, q_desc + s, desc, i > 0);
                    mma_ss(to + Plan::dp_col, v_desc + o, do_desc + s, desc, i > 0);
                }
                mma_commit(s_full + 8 * g);
            }
            __syncwarp();
        }
        if (leader) {
            mma_commit(drained);
            drain(drained, 0);
        }
    } else if (warp == 10) {
        constexpr uint32_t desc = mma_desc(64 * HALVES, true);
        const bool leader = elect_one();
        const uint64_t q_desc = desc_n_major(sq, kStepBytes), do_desc = desc_n_major(sdo, kStepBytes);
        Cursor<DkvArgs, DkvItem> at;
        for (at.start(a, ranks); at.more; at.next(a, ranks)) {
            const int st = at.tile % ST, g = at.tile & 1;
            if (at.j == 0) wait_warp(acc_free, (at.ordinal & 1) ^ 1, dead, 32 << 16);  // the last item's dV and dK have been read
            wait_warp(p_ready + 8 * g, (at.tile >> 1) & 1, dead, 64 << 16);
            tc_fence_after();
            const uint32_t step = st * (Plan::step_bytes >> 4), p = tmem + Plan::p_col + g * Plan::p_cols, ds = tmem + Plan::ds_col + g * Plan::p_cols;
            const bool more = at.j > 0, last = at.j + 1 == at.item.n;
            if (leader) {
#pragma unroll
                for (int i = 0; i < kStep / 16; ++i) {
                    mma_ts(tmem + Plan::dv_col, p + 8 * i, do_desc + step + i * 128, desc, more || i > 0);
                    mma_ts(tmem + Plan::dk_col, ds + 8 * i, q_desc + step + i * 128, desc, more || i > 0);
                }
                mma_commit(sums_done + 8 * g);
                mma_commit(empty + 8 * st);
                if (last) mma_commit(acc_done);
            }
            __syncwarp();
        }
        if (leader) {
            mma_commit(drained + 8);
            drain(drained + 8, 0);
        }
    } else if (warp == 11) {
        int heads = 0;                                         // query heads whose tables have been laid out
        DkvItem t;
        for (int round = 0; LUT && next_item(a, ranks, round, t);) {
            if (t.n == 0) continue;
            const int first = t.q_first * kStep + sh.q_pos;        // query positions, to the last tile's end: p = 0 there needs a finite bias
            const int last = (t.q_first + t.per_head) * kStep - 1 + sh.q_pos;
            for (int i = 0; i < sh.group; ++i, ++heads) {
                const int buf = heads & 1;
                wait_warp(lut_empty + 8 * buf, ((heads >> 1) & 1) ^ 1, dead, 128 << 16);
                const bool out = fill_lut(a.bias, t.hk * sh.group + i, lut_bucket, luts + buf * a.lut.floats, a.lut, sh.causal ? 0 : first - (t.k0 + kOwn - 1), last - t.k0, -1, lane, 32);
                const bool outs = __any_sync(0xFFFFFFFFu, out);
                if (lane == 0) lut_set_outs(luts + buf * a.lut.floats, a.lut, outs);
                __syncwarp();
                if (lane == 0) bar_arrive(lut_full + 8 * buf);
            }
        }
    } else if (warp < 8) {
        take_registers<kDkvMathRegisters>();
        const int g = warp >> 2, quad = warp & 3;
        const int row = quad * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)quad << 21);
        const uint32_t s_at = lanes + g * Plan::group_cols + Plan::s_col, dp_at = lanes + g * Plan::group_cols + Plan::dp_col;
        const uint32_t p_at = lanes + Plan::p_col + g * Plan::p_cols, ds_at = lanes + Plan::ds_col + g * Plan::p_cols;
        int ordinal = 0, tile = 0, heads = 0;
        bool leaving = false;          // this warp's rows of the last item are on their way out of that item's k or v
        auto release_own = [&](int buf) {
            if (lane == 0) {
                tma_store_wait_read();
                bar_arrive(own_empty + 8 * buf);
            }
        };
        DkvItem t;
        for (int round = 0; next_item(a, ranks, round, t);) {
            const int key = t.k0 + row, buf = ordinal % OB;
            if (t.n == 0) {
                if (key < sh.len_kv) {
                    if (g == 0) zero_row(a.dk, sh.dim, t.b, t.hk, key);
                    else zero_row(a.dv, sh.dim, t.b, t.hk, key);
                }
                continue;
            }
            int q_tile = t.q_first;
            bool head_starts_for_me = false;
            float left = 0.0f, right = 0.0f;                   // the bias of the head's far keys
            bool outs = false;                                 // whether a bucket of the head is taken out
            for (int j = 0; j < t.n; ++j, ++tile) {
                const int table = heads & 1;
                const bool head_starts = q_tile == t.q_first, head_ends = q_tile + 1 == t.q_first + t.per_head;
                const int st = tile % ST, pos0 = q_tile * kStep + sh.q_pos;
                if (LUT && head_starts) {
                    wait_warp(lut_full + 8 * table, (heads >> 1) & 1, dead, 256 << 16);
                    head_starts_for_me = true;
                }
                if ((tile & 1) == g) {
                    const uint32_t parity = (tile >> 1) & 1;
                    wait_warp(stat_full + 8 * st, (tile / ST) & 1, dead, 512 << 16);
                    const float* nl = stats + st * Plan::stat_floats;
                    const float* nd = nl + kStep;
                    wait_warp(s_full + 8 * g, parity, dead, 1024 << 16);
                    tc_fence_after();
                    if (LUT && head_starts_for_me) {
                        left = lut_far(luts + table * a.lut.floats, a.lut, false);
                        right = lut_far(luts + table * a.lut.floats, a.lut, true);
                        outs = lut_outs(luts + table * a.lut.floats, a.lut);
                        head_starts_for_me = false;
                    }
                    const Span span = LUT ? span_of(a.bias, t.k0 - (pos0 + kStep - 1), t.k0 + kOwn - 1 - pos0) : kSpanFarLeft;
                    const bool mixed = LUT && span == kSpanMixed;
                    const float* bias_at = LUT ? lut_at(luts + table * a.lut.floats, a.lut, pos0 - key) : nullptr;     // on the turned axis: query - key
                    const float add = LUT ? (span == kSpanFarRight ? right : left) : 0.0f;
                    const uint64_t mul2v = pack2(sh.scale_log2, sh.scale_log2), add2v = pack2(add, add);
                    const bool holes = nl[2 * kStep] != 0.0f;
                    const int alone = key - pos0;              // the column that sees this key alone, if it is the first key
                    const bool single = t.len == 1 || (sh.causal && key == 0 && alone >= 0 && alone < kStep);
                    // half a tile at a time: lse and delta of its columns need registers too
#pragma unroll
                    for (int c0 = 0; c0 < kStep; c0 += 32) {
                        uint32_t s[32], d[32];
                        tmem_ld32(s, s_at + c0);
                        tmem_ld32(d, dp_at + c0);
                        tmem_wait_ld();
                        tmem_use(s);
                        tmem_use(d);
                        if (Plan::apart && c0 == 32) {
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) bar_arrive(s_free + 8 * g);
                        }
                        uint32_t wp[16], wd[16];
                        auto probabilities = [&](auto bias2) {
#pragma unroll
                            for (int c = 0; c < 32; c += 4) {
                                const float4 l = *reinterpret_cast<const float4*>(nl + c0 + c);
                                const float4 m = *reinterpret_cast<const float4*>(nd + c0 + c);
                                const uint64_t ls[2] = {pack2(l.x, l.y), pack2(l.z, l.w)}, ms[2] = {pack2(m.x, m.y), pack2(m.z, m.w)};
#pragma unroll
                                for (int u = 0; u < 2; ++u) {
                                    const int e = c + 2 * u;
                                    float x, y;
                                    unpack2(fma2(pack2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), mul2v, add2(ls[u], bias2(e))), x, y);
                                    x = exp2_fast(x);
                                    y = exp2_fast(y);
                                    wp[e >> 1] = pack_bf16(x, y);
                                    unpack2(mul2(pack2(x, y), add2(pack2(__uint_as_float(d[e]), __uint_as_float(d[e + 1])), ms[u])), x, y);
                                    wd[e >> 1] = pack_bf16(x, y);
                                }
                            }
                        };
                        if (mixed) {
                            probabilities([&](int e) {
                                const float2 b = *reinterpret_cast<const float2*>(bias_at + c0 + e);
                                return pack2(b.x, b.y);
                            });
                            // the warp's part may hold masked pairs
                            if (outs || (sh.causal && t.k0 + 32 * quad + 31 > pos0 + c0)) {
                                uint32_t top = wd[0];
#pragma unroll
                                for (int e = 1; e < 16; ++e) top = max_bf16x2(top, wd[e]);
                                if (__builtin_expect(__any_sync(0xFFFFFFFFu, (top & 0x7FFFu) > 0x7F80u || (top & 0x7FFF0000u) > 0x7F800000u), 0)) {
#pragma unroll
                                    for (int c = 0; c < 32; ++c) {
                                        if (bias_at[c0 + c] != -INFINITY) continue;
                                        const uint32_t keep = c & 1 ? 0x0000FFFFu : 0xFFFF0000u;
                                        wp[c >> 1] &= keep;
                                        wd[c >> 1] &= keep;
                                    }
                                }
                            }
                        } else {
                            probabilities([&](int) { return add2v; });
                        }
                        if (single || holes) {
                            // rows that see one key alone: p = 1, ds = 0.  Rows inside len_q with nothing allowed: whatever do and q hold
#pragma unroll
                            for (int c = 0; c < 32; ++c) {
                                const uint32_t keep = c & 1 ? 0x0000FFFFu : 0xFFFF0000u;
                                const bool hole = holes && nl[c0 + c] == -INFINITY;
                                if (hole) wp[c >> 1] &= keep;
                                if (hole || (single && (t.len == 1 || c0 + c == alone))) wd[c >> 1] &= keep;
                            }
                        }
                        if (Plan::apart && tile > 1 && c0 == 0) {      // P and dS of the group's last tile have been used
                            wait_warp(sums_done + 8 * g, parity ^ 1, dead, 2048 << 16);
                            tc_fence_after();
                        }
                        tmem_st16(p_at + (c0 >> 1), wp);
                        tmem_st16(ds_at + (c0 >> 1), wd);
                    }
                    if (holes) {
                        // and must not reach a product: 0 * NaN
                        const int r = row & (kStep - 1), part = row >> 6;
                        if (nl[r] == -INFINITY) {
#pragma unroll
                            for (int c = 0; c < HALVES; ++c)
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const uint32_t at = st * Plan::step_bytes + c * kStepBytes + r * 128 + 64 * part + 16 * e;
                                    *reinterpret_cast<uint4*>(smem + (sq - base) + at) = make_uint4(0, 0, 0, 0);
                                    *reinterpret_cast<uint4*>(smem + (sdo - base) + at) = make_uint4(0, 0, 0, 0);
                                }
                        }
                        fence_async_smem();
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(p_ready + 8 * g);
                    if (OB > 1 && leaving) {
                        release_own((ordinal - 1) % OB);
                        leaving = false;
                    }
                }
                if (head_ends) {
                    if (LUT) {
                        __syncwarp();
                        if (lane == 0) bar_arrive(lut_empty + 8 * table);
                    }
                    ++heads;
                    q_tile = t.q_first;
                } else {
                    ++q_tile;
                }
            }
            if (OB > 1 && leaving) {                           // an item of one tile, which was the other group's
                release_own((ordinal - 1) % OB);
                leaving = false;
            }
            wait_warp(acc_done, ordinal & 1, dead, 4096 << 16);
            tc_fence_after();
            // dk (the first group) and dv go out through k's and v's places, which are free: every product has completed.  Keys
            // behind the sequence's end get zeros
            const float factor = *dead ? NAN : g == 0 ? sh.scale : 1.0f;       // a wait has run out: the item's results show it
            uint8_t* staging = smem + ((g == 0 ? sk : sv) - base) + buf * Plan::own_bytes + quad * 2 * HALVES * 2048;
#pragma unroll
            for (int c = 0; c < 2 * HALVES; ++c) {
                uint32_t r[32];
                tmem_ld32(r, lanes + (g == 0 ? Plan::dk_col : Plan::dv_col) + 32 * c);
                tmem_wait_ld();
                tmem_use(r);
                if (key >= t.len) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) r[e] = 0;
                }
                stage_box(r, factor, staging + c * 2048, lane);
            }
            tc_fence_before();
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                bar_arrive(acc_free);
                if (t.k0 + 32 * quad < sh.len_kv) {
                    for (int c = 0; c < 2 * HALVES; ++c) {
                        if (32 * c >= sh.dim) continue;
                        if (g == 0) tma_store4(&a.dk.map, smem_u32(staging) + c * 2048, 32 * c, t.k0 + 32 * quad, t.hk * a.dk.head_mul, t.b * a.dk.batch_mul);
                        else tma_store4(&a.dv.map, smem_u32(staging) + c * 2048, 32 * c, t.k0 + 32 * quad, t.hk * a.dv.head_mul, t.b * a.dv.batch_mul);
                    }
                    tma_store_commit();
                }
            }
            if (OB > 1) leaving = true;                        // other places are ready: these may wait
            else release_own(buf);
            ++ordinal;
        }
        if (leaving) release_own((ordinal - 1) % OB);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        tmem_free(tmem, Plan::columns);
    }
}

// =============================================================================================== bias

// dtable[h][n] = sum over the sequences and row blocks of one head, in that order.  A block per head and 32 buckets: 32 rows at
// a time, so that a training batch's thousand rows are a few loads a thread.
constexpr int kTableRows = 32;

__global__ void __launch_bounds__(32 * kTableRows) attn_dtable_kernel(const float* partial, int batch, int heads, int blocks, int buckets,
                                                                      float* out32, uint16_t* out16) {
    __shared__ double shared[kTableRows][32];
    grid_dependency_sync();
    const int h = blockIdx.x, bucket = blockIdx.y * 32 + threadIdx.x;
    double s = 0.0;
    if (bucket < buckets && blocks > 0) {                      // without queries there are no rows
        int b = threadIdx.y / blocks, block = threadIdx.y % blocks;
#pragma unroll 4
        for (int i = threadIdx.y; i < batch * blocks; i += kTableRows) {
            const float* row = partial + (((size_t)b * heads + h) * blocks + block) * 4 * buckets + bucket;
            s += (double)(row[0] + row[buckets]) + (double)(row[2 * buckets] + row[3 * buckets]);
            for (block += kTableRows; block >= blocks; block -= blocks) ++b;
        }
    }
    shared[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y == 0 && bucket < buckets) {
        for (int i = 1; i < kTableRows; ++i) s += shared[i][threadIdx.x];
        if (out32) out32[(size_t)h * buckets + bucket] = (float)s;
        else out16[(size_t)h * buckets + bucket] = (uint16_t)(pack_bf16((float)s, 0.0f) & 0xFFFFu);
    }
}

template <auto KERNEL, typename A>
int launch(int threads, int per_sm, size_t smem, const A& a, cudaStream_t s) {
    static SmemLimit limit;
    if (!limit.raise(KERNEL, a.shape.device, smem)) return ALSGD_E_CUDA;
    const int wave = blocks_at_once(smem, per_sm);
    return launch_dependent(KERNEL, dim3(a.items < wave ? a.items : wave), dim3(threads), smem, s, a) == cudaSuccess ? ALSGD_OK : ALSGD_E_CUDA;
}

template <int HALVES, typename RANKS>
int launch_dq(const DqArgs& a, cudaStream_t s) {
    const bool bias = a.bias.table != nullptr, lut = bias || a.shape.causal;
    const size_t smem = dq_smem<HALVES>(a.lut, lut, bias ? a.bias.buckets : 0);
    if (bias) return launch<attn_dq_kernel<HALVES, true, true, RANKS>>(kDqThreads, 2, smem, a, s);
    return lut ? launch<attn_dq_kernel<HALVES, true, false, RANKS>>(kDqThreads, 2, smem, a, s) : launch<attn_dq_kernel<HALVES, false, false, RANKS>>(kDqThreads, 2, smem, a, s);
}

template <int HALVES, int STAGES, typename RANKS>
int launch_dkv(const DkvArgs& a, cudaStream_t s) {
    const bool lut = a.bias.table != nullptr || a.shape.causal;
    const size_t smem = dkv_smem<HALVES, STAGES>(a.lut, lut);
    return lut ? launch<attn_dkv_kernel<HALVES, STAGES, true, RANKS>>(kDkvThreads, 1, smem, a, s)
               : launch<attn_dkv_kernel<HALVES, STAGES, false, RANKS>>(kDkvThreads, 1, smem, a, s);
}

// Four tiles on the way; two where wide heads and a table that reaches 703 or further leave no room for more (heads of 128 in
// groups of 4, 1000 queries, 511 to 1531 keys, all kernels: 199 us with four, 213 us with two).  Narrow heads have a plan of
// their own in both kernels: at 2 x 4096 tokens and heads of 64, 373 us, and 578 us with the plans for wide ones.
template <typename RANKS>
int launch_dkv(const DkvArgs& a, bool wide, cudaStream_t s) {
    if (!wide) return launch_dkv<1, 4, RANKS>(a, s);
    return dkv_smem<2, 4>(a.lut, a.bias.table != nullptr || a.shape.causal) <= SmemLimit::kMost ? launch_dkv<2, 4, RANKS>(a, s) : launch_dkv<2, 2, RANKS>(a, s);
}

uint64_t delta_bytes(const alsgd_attn_desc& d) { return ((uint64_t)d.batch * d.heads_q * d.len_q * 4 + 255) / 256 * 256; }
uint64_t partial_bytes(const alsgd_attn_desc& d) { return (uint64_t)d.batch * d.heads_q * ((d.len_q + kOwn - 1) / kOwn) * 4 * d.buckets * 4; }

}  // namespace

extern "C" int alsgd_attn_bwd_bytes(const alsgd_attn_desc* desc, uint64_t* bytes_out) {
    if (!bytes_out) return ALSGD_E_ARG;
    const int rc = check_desc(desc);
    if (rc != ALSGD_OK) return rc;
    *bytes_out = delta_bytes(*desc) + partial_bytes(*desc);
    return ALSGD_OK;
}

extern "C" int alsgd_attn_bwd(const alsgd_attn_desc* desc, const alsgd_attn_tensor* q, const alsgd_attn_tensor* k, const alsgd_attn_tensor* v,
                              const void* table, const int32_t* kv_len, const alsgd_attn_tensor* o, const float* lse,
                              const alsgd_attn_tensor* dout, const alsgd_attn_tensor* dq, const alsgd_attn_tensor* dk,
                              const alsgd_attn_tensor* dv, void* dtable, void* work, uint64_t work_bytes, void* stream) {
    int rc = check_desc(desc);
    if (rc != ALSGD_OK) return rc;
    const alsgd_attn_desc& d = *desc;
    if ((d.buckets != 0) != (table != nullptr) || (d.buckets != 0) != (dtable != nullptr)) return ALSGD_E_ARG;
    if (!table_aligned(d, table) || !table_aligned(d, dtable) || reinterpret_cast<uintptr_t>(kv_len) % 4) return ALSGD_E_ARG;
    if (d.len_q && (!lse || reinterpret_cast<uintptr_t>(lse) % 4)) return ALSGD_E_ARG;
    const struct { const alsgd_attn_tensor* t; bool query, output; } all[] = {
        {q, true, false}, {k, false, false}, {v, false, false}, {o, true, false}, {dout, true, false}, {dq, true, true}, {dk, false, true}, {dv, false, true}};
    for (const auto& x : all) {
        rc = check_tensor(x.t, d.batch, x.query ? d.len_q : d.len_kv, x.query ? d.heads_q : d.heads_kv, x.output);
        if (rc != ALSGD_OK) return rc;
    }
    const uint64_t need = delta_bytes(d) + partial_bytes(d);
    if (need && (!work || reinterpret_cast<uintptr_t>(work) % 256)) return ALSGD_E_ARG;
    if (work_bytes < need) return ALSGD_E_NOMEM;

    UseDevice use(d.device);
    if (!use.ok) return ALSGD_E_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    float* delta = static_cast<float*>(work);
    float* partial = reinterpret_cast<float*>(static_cast<char*>(work) + delta_bytes(d));
    const int blocks = (int)((d.len_q + kOwn - 1) / kOwn);
    // an operand without positions is never read: any map will do
    auto operand = [&](const alsgd_attn_tensor* t, bool query, uint32_t rows, uint32_t cols, Operand* out) {
        const bool swap = (query ? d.len_q : d.len_kv) == 0;
        const bool as_query = query != swap;
        return make_operand(swap ? (query ? *k : *q) : *t, d.batch, as_query ? d.len_q : d.len_kv, as_query ? d.heads_q : d.heads_kv, d.dim, rows, cols, out);
    };
    const uint64_t q_items = (uint64_t)d.batch * d.heads_q * blocks, kv_items = (uint64_t)d.batch * d.heads_kv * ((d.len_kv + kOwn - 1) / kOwn);
    if (q_items > 0x7FFFFFFFull - 2 * kSMs || kv_items > 0x7FFFFFFFull - 2 * kSMs) return ALSGD_E_RANGE;
    if (d.len_q) {
        DqArgs a;
        a.shape = make_shape(d, kv_len, kOwn);
        make_bias(d, table, &a.bias);
        a.lut = lut_shape(a.bias.far, kOwn, kStep, a.shape.causal);
        a.row_blocks = blocks;
        a.items = (int)q_items;
        a.lse = lse;
        a.o = static_cast<const uint16_t*>(o->data);
        a.o_batch = d.batch == 1 ? 0 : o->stride_batch;
        a.o_pos = d.len_q == 1 ? 0 : o->stride_pos;
        a.o_head = d.heads_q == 1 ? 0 : o->stride_head;
        a.delta = delta;
        a.partial = partial;
        if ((rc = operand(q, true, kOwn, 64, &a.q)) != ALSGD_OK || (rc = operand(dout, true, kOwn, 64, &a.dout)) != ALSGD_OK ||
            (rc = operand(dq, true, 32, 32, &a.dq)) != ALSGD_OK || (rc = operand(k, false, kStep, 64, &a.k)) != ALSGD_OK ||
            (rc = operand(v, false, kStep, 64, &a.v)) != ALSGD_OK)
            return rc;
        if (by_rank(a.shape)) rc = d.dim <= 64 ? launch_dq<1, Ranks>(a, s) : launch_dq<2, Ranks>(a, s);
        else rc = d.dim <= 64 ? launch_dq<1, NoRanks>(a, s) : launch_dq<2, NoRanks>(a, s);
        if (rc != ALSGD_OK) return rc;
    }
    if (d.len_kv) {
        DkvArgs a;
        a.shape = make_shape(d, kv_len, kOwn);
        make_bias(d, table, &a.bias);
        a.lut = lut_shape(a.bias.far, kOwn, kStep, false);     // on the turned axis the allowed keys lie ahead
        a.items = (int)kv_items;
        a.lse = lse;
        a.delta = delta;
        if ((rc = operand(q, true, kStep, 64, &a.q)) != ALSGD_OK || (rc = operand(dout, true, kStep, 64, &a.dout)) != ALSGD_OK ||
            (rc = operand(k, false, kOwn, 64, &a.k)) != ALSGD_OK || (rc = operand(v, false, kOwn, 64, &a.v)) != ALSGD_OK ||
            (rc = operand(dk, false, 32, 32, &a.dk)) != ALSGD_OK || (rc = operand(dv, false, 32, 32, &a.dv)) != ALSGD_OK)
            return rc;
        rc = by_rank(a.shape) ? launch_dkv<KeyRanks>(a, d.dim > 64, s) : launch_dkv<NoRanks>(a, d.dim > 64, s);
        if (rc != ALSGD_OK) return rc;
    }
    if (d.buckets) {
        const bool wide = d.table_dtype == ALSGD_F32;
        if (launch_dependent(attn_dtable_kernel, dim3(d.heads_q, (d.buckets + 31) / 32), dim3(32, kTableRows), 0, s, (const float*)partial, (int)d.batch,
                             (int)d.heads_q, blocks, (int)d.buckets, wide ? static_cast<float*>(dtable) : nullptr,
                             wide ? nullptr : static_cast<uint16_t*>(dtable)) != cudaSuccess)
            return ALSGD_E_CUDA;
    }
    return ALSGD_OK;
}

namespace alsgd_attn {
// The backward kernels' part of alsgd_attn_status; the caller has made the device current.
bool bwd_wait_word(unsigned* out) { return cudaMemcpyFromSymbol(out, g_wait_error, sizeof *out) == cudaSuccess; }
}  // namespace alsgd_attn
