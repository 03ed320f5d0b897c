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
// add dQ across blocks.
//
// Both are built like the forward kernel: blocks walk the work items, those with the most tiles first; warps 0-7 do the
// arithmetic on a tile (warps w and w + 4 share 32 rows and take 32 columns each), warp 8 copies tiles, warp 9 issues the
// products.
//
// Everything is binary32 but the operands of the second products: p and ds are rounded to bf16 (the type of do, q and
// k), as the forward pass rounds p.
#include "alsgd_attn.cuh"

using namespace alsgd_attn;
using namespace alsgd_ops;
using namespace alsgd_tc;

namespace {

constexpr int kOwn = 128;               // rows of an item
constexpr int kStep = 64;               // rows of a streamed tile
constexpr int kMath = 256;              // threads that do the arithmetic
constexpr int kThreads = kMath + 64;
constexpr int kAll = 5;                 // named barrier of those threads; 1 to 4 belong to the pairs of warps
constexpr uint32_t kOwnBytes = 128 * 128;      // 128 rows of 64 bf16
constexpr uint32_t kStepBytes = 64 * 128;
constexpr int kDiagonals = 2 * 48;      // sums a warp keeps of its 32 x 32 part, in two groups of 16 columns

// =============================================================================================== dq

struct DqArgs {
    Operand q, k, v, dout, dq;
    Shape shape;
    Bias bias;
    const float* lse;
    const uint16_t* o;
    int64_t o_batch, o_pos, o_head;     // steps of o
    float* delta;                       // out: [batch][heads_q][len_q]
    float* partial;                     // out: [batch * heads_q][row blocks][buckets]
    int pad, row_blocks, items;
};

struct DqItem {
    int b, h, block, q0, len, keys, n;  // sequence, head, row block, first row, valid keys, keys any row sees, tiles
};

__device__ __forceinline__ DqItem item_at(const DqArgs& a, int i) {
    const Shape& sh = a.shape;
    const int bh = sh.batch * sh.heads_q;
    DqItem t;
    t.block = a.row_blocks - 1 - i / bh;
    t.q0 = t.block * kOwn;
    t.b = i % bh / sh.heads_q;
    t.h = i % bh % sh.heads_q;
    t.len = sh.kv_len ? min(max(sh.kv_len[t.b], 0), sh.len_kv) : sh.len_kv;
    t.keys = t.len;
    if (sh.causal) t.keys = min(t.keys, min(t.q0 + kOwn, sh.len_q) + sh.q_pos);
    t.n = t.keys > 0 ? (t.keys + kStep - 1) / kStep : 0;
    return t;
}

template <int HALVES>
struct DqPlan {
    static constexpr int stages = HALVES == 1 ? 2 : 1, own_bufs = HALVES == 1 ? 2 : 1;
    static constexpr bool apart = HALVES == 1;         // dS beside S, so that the next tile's scores need not wait for dQ
    static constexpr uint32_t columns = 256;
    static constexpr uint32_t s_col = 0, dp_col = 64, dq_col = 128;
    static constexpr uint32_t ds_col = apart ? 192 : 0, ds_half = apart ? 16 : 32;     // dS of columns 32-63 lies ds_half further
    static constexpr uint32_t own_bytes = HALVES * kOwnBytes, step_bytes = HALVES * kStepBytes;
    static constexpr uint32_t tiles_bytes = own_bufs * 2 * own_bytes + 2 * stages * step_bytes;
    static constexpr uint32_t bars = 6 + 2 * own_bufs + 2 * stages;
    static constexpr uint32_t fixed_bytes = tiles_bytes + 256 + 4 * kOwn * sizeof(float);
};

template <int HALVES>
size_t dq_smem(int pad, int buckets) {
    return 1024 + DqPlan<HALVES>::fixed_bytes + (buckets ? 8 * (kDiagonals + buckets) * sizeof(float) + (2 * pad + 1) * (sizeof(float) + 1) : 0);
}

template <int HALVES, bool BIAS>
__global__ void __launch_bounds__(kThreads, 2) attn_dq_kernel(const __grid_constant__ DqArgs a) {
    using Plan = DqPlan<HALVES>;
    constexpr int ST = Plan::stages, OB = Plan::own_bufs;
    extern __shared__ uint8_t raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    const uint32_t base = smem_u32(smem);
    const uint32_t sq = base, sdo = sq + OB * Plan::own_bytes, sk = sdo + OB * Plan::own_bytes, sv = sk + ST * Plan::step_bytes;
    const uint32_t bars = base + Plan::tiles_bytes;
    const uint32_t s_full = bars, s_free = bars + 8, ds_ready = bars + 16, dq_done = bars + 24, dq_free = bars + 32, drained = bars + 40;
    const uint32_t own_full = bars + 48, own_empty = own_full + 8 * OB, full = own_empty + 8 * OB, empty = full + 8 * ST;
    uint32_t* words = reinterpret_cast<uint32_t*>(smem + Plan::tiles_bytes + 8 * Plan::bars);
    volatile uint32_t* dead = words + 1;
    float* shared_delta = reinterpret_cast<float*>(smem + Plan::tiles_bytes + 256);    // [2][2][kOwn]: items in turn
    float* diagonals = shared_delta + 4 * kOwn;
    float* by_bucket = diagonals + 8 * kDiagonals;             // [8 warps][buckets]
    float* lut = by_bucket + 8 * a.bias.buckets;
    uint8_t* lut_bucket = reinterpret_cast<uint8_t*>(lut + 2 * a.pad + 1);

    const Shape& sh = a.shape;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        bar_init(s_full, 1);
        bar_init(s_free, 8);
        bar_init(ds_ready, 8);
        bar_init(dq_done, 1);
        bar_init(dq_free, 8);
        bar_init(drained, 1);
        for (int i = 0; i < OB; ++i) {
            bar_init(own_full + 8 * i, 1);
            bar_init(own_empty + 8 * i, 8);
        }
        for (int i = 0; i < ST; ++i) {
            bar_init(full + 8 * i, 1);
            bar_init(empty + 8 * i, 1);
        }
        words[1] = 0;
        bar_init_fence();
    }
    if (warp == 9) tmem_alloc(smem_u32(words), Plan::columns);
    if (threadIdx.x == kMath) {
        tma_prefetch(&a.q.map);
        tma_prefetch(&a.dout.map);
        tma_prefetch(&a.k.map);
        tma_prefetch(&a.v.map);
        tma_prefetch(&a.dq.map);
    }
    if (BIAS && warp < 8) fill_buckets(a.bias, lut_bucket, a.pad, threadIdx.x, kMath);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = words[0];
    grid_dependency_sync();

    if (warp == 8) {
        if (lane == 0) {
            int ordinal = 0, tile = 0;                         // items and tiles whose copies have been started
            for (int i = blockIdx.x; i < a.items; i += gridDim.x) {
                const DqItem t = item_at(a, i);
                if (t.n == 0) continue;
                const int hk = t.h / sh.group, buf = ordinal % OB;
                wait(own_empty + 8 * buf, ((ordinal / OB) & 1) ^ 1, dead, 1 << 16);
                if (*dead) break;
                bar_expect(own_full + 8 * buf, 2 * Plan::own_bytes);
                for (int c = 0; c < HALVES; ++c) {
                    const uint32_t at = buf * Plan::own_bytes + c * kOwnBytes;
                    tma_load4(sq + at, &a.q.map, own_full + 8 * buf, 64 * c, t.q0, t.h * a.q.head_mul, t.b * a.q.batch_mul);
                    tma_load4(sdo + at, &a.dout.map, own_full + 8 * buf, 64 * c, t.q0, t.h * a.dout.head_mul, t.b * a.dout.batch_mul);
                }
                ++ordinal;
                for (int j = 0; j < t.n; ++j) {
                    const int st = tile % ST;
                    wait(empty + 8 * st, ((tile / ST) & 1) ^ 1, dead, 2 << 16);
                    if (*dead) break;
                    bar_expect(full + 8 * st, 2 * Plan::step_bytes);
                    for (int c = 0; c < HALVES; ++c) {
                        const uint32_t at = st * Plan::step_bytes + c * kStepBytes;
                        tma_load4(sk + at, &a.k.map, full + 8 * st, 64 * c, j * kStep, hk * a.k.head_mul, t.b * a.k.batch_mul);
                        tma_load4(sv + at, &a.v.map, full + 8 * st, 64 * c, j * kStep, hk * a.v.head_mul, t.b * a.v.batch_mul);
                    }
                    ++tile;
                }
            }
            // every copy has landed before the block may leave, whoever else has given up
            for (int i = max(0, ordinal - OB); i < ordinal; ++i) drain(own_full + 8 * (i % OB), (i / OB) & 1);
            for (int i = max(0, tile - ST); i < tile; ++i) drain(full + 8 * (i % ST), (i / ST) & 1);
        }
    } else if (warp == 9) {
        // The warp walks together and one lane issues: what a product is given stays the same for all lanes, which is what
        // its instruction wants, and a tile costs this warp little more than its products.
        constexpr uint32_t desc_s = mma_desc(kStep, false), desc_q = mma_desc(64 * HALVES, true);
        const bool leader = elect_one();
        const uint64_t q_desc = desc_k_major(sq), do_desc = desc_k_major(sdo), k_desc = desc_k_major(sk), v_desc = desc_k_major(sv);
        const uint64_t kn_desc = desc_n_major(sk, kStepBytes);
        Cursor<DqArgs, DqItem> ahead, at;                      // of S and dP, and of dQ
        ahead.start(a);
        at = ahead;
        auto scores = [&]() {
            const int st = ahead.tile % ST, buf = ahead.ordinal % OB;
            if (ahead.j == 0) wait_warp(own_full + 8 * buf, (ahead.ordinal / OB) & 1, dead, 4 << 16);
            wait_warp(full + 8 * st, (ahead.tile / ST) & 1, dead, 8 << 16);
            tc_fence_after();
            const uint32_t own = buf * (Plan::own_bytes >> 4), step = st * (Plan::step_bytes >> 4);
            if (leader) {
#pragma unroll
                for (int i = 0; i < 4 * HALVES; ++i) {         // 16 elements of the head each; behind dim they are zeros
                    const uint32_t o = own + (((i >> 2) * kOwnBytes + (i & 3) * 32) >> 4), s = step + (((i >> 2) * kStepBytes + (i & 3) * 32) >> 4);
                    mma_ss(tmem + Plan::s_col, q_desc + o, k_desc + s, desc_s, i > 0);
                    mma_ss(tmem + Plan::dp_col, do_desc + o, v_desc + s, desc_s, i > 0);
                }
                mma_commit(s_full);
            }
            __syncwarp();
            ahead.next(a);
        };
        if (ahead.more) scores();
        int items = 0;                                         // whose dQ has been started
        while (at.more) {
            const int st = at.tile % ST;
            const uint32_t parity = at.tile & 1;
            if (Plan::apart && ahead.more) {
                wait_warp(s_free, parity, dead, 16 << 16);
                scores();
            }
            if (at.j == 0) {                                   // the last item's dQ has been read
                wait_warp(dq_free, (items & 1) ^ 1, dead, 32 << 16);
                ++items;
            }
            wait_warp(ds_ready, parity, dead, 64 << 16);
            tc_fence_after();
            const uint64_t kd = kn_desc + st * (Plan::step_bytes >> 4);
            const bool more = at.j > 0;
            if (leader) {
#pragma unroll
                for (int i = 0; i < kStep / 16; ++i)
                    mma_ts(tmem + Plan::dq_col, tmem + Plan::ds_col + (i >> 1) * Plan::ds_half + (i & 1) * 8, kd + i * 128, desc_q, more || i > 0);
                mma_commit(empty + 8 * st);
                mma_commit(dq_done);
            }
            __syncwarp();
            if (!Plan::apart && ahead.more) {
                wait_warp(dq_done, parity, dead, 128 << 16);
                scores();
            }
            at.next(a);
        }
        if (leader) {
            mma_commit(drained);
            drain(drained, 0);
        }
    } else {
        const int half = warp >> 2, quad = warp & 3;
        const int row = quad * 32 + lane, pair = 1 + quad;
        const uint32_t lanes = tmem + ((uint32_t)quad << 21);
        float* sums = diagonals + warp * kDiagonals;
        float* bucket_sums = by_bucket + warp * a.bias.buckets;
        int ordinal = 0, tile = 0;
        for (int i = blockIdx.x; i < a.items; i += gridDim.x) {
            const DqItem t = item_at(a, i);
            const int buf = ordinal % OB;
            const bool inside = t.q0 + row < sh.len_q;
            const int pos = t.q0 + row + sh.q_pos;
            const size_t stat = ((size_t)t.b * sh.heads_q + t.h) * sh.len_q + t.q0 + row;
            float* partial = a.partial + (((size_t)t.b * sh.heads_q + t.h) * a.row_blocks + t.block) * a.bias.buckets;
            if (t.n == 0) {
                if (inside) {
                    if (half == 0) {
                        zero_row(a.dq, sh.dim, t.b, t.h, t.q0 + row);
                        a.delta[stat] = 0.0f;
                    }
                }
                if (BIAS)
                    for (int e = threadIdx.x; e < a.bias.buckets; e += kMath) partial[e] = 0.0f;
                continue;
            }
            const float lse = inside ? a.lse[stat] : -INFINITY;
            const bool live = lse != -INFINITY;
            // delta: this thread's half of the row's do . o
            uint4 o[4 * HALVES];
#pragma unroll
            for (int c = 0; c < 4 * HALVES; ++c) {
                const int x = 8 * (4 * HALVES * half + c);
                o[c] = live && x < sh.dim ? *reinterpret_cast<const uint4*>(a.o + (int64_t)t.b * a.o_batch + (int64_t)(t.q0 + row) * a.o_pos +
                                                                            (int64_t)t.h * a.o_head + x)
                                          : make_uint4(0, 0, 0, 0);
            }
            if (BIAS) {
                const int first = t.q0 + sh.q_pos;             // distances from the last row's first key to the first row's last
                sync_threads(kAll, kMath);
                fill_lut(a.bias, t.h, lut_bucket, lut, a.pad, -(first + kOwn - 1), sh.causal ? 0 : t.keys - 1 - first, threadIdx.x, kMath);
                for (int e = lane; e < a.bias.buckets; e += 32) bucket_sums[e] = 0.0f;
                sync_threads(kAll, kMath);
            }
            wait_warp(own_full + 8 * buf, (ordinal / OB) & 1, dead, 256 << 16);
            float delta = 0.0f;
            if (live) {
                float acc[2] = {0.0f, 0.0f};
#pragma unroll
                for (int c = 0; c < 4 * HALVES; ++c) {
                    const int chunk = 4 * HALVES * half + c;
                    const uint4 y = *reinterpret_cast<const uint4*>(smem + (sdo - base) + buf * Plan::own_bytes + (chunk >> 3) * kOwnBytes + row * 128 +
                                                                    (((chunk & 7) ^ (row & 7)) << 4));
                    const uint32_t xs[4] = {o[c].x, o[c].y, o[c].z, o[c].w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        acc[0] = fmaf(bf16_lo(xs[e]), bf16_lo(ys[e]), acc[0]);
                        acc[1] = fmaf(bf16_hi(xs[e]), bf16_hi(ys[e]), acc[1]);
                    }
                }
                delta = acc[0] + acc[1];
            }
            float* halves = shared_delta + (ordinal & 1) * 2 * kOwn;
            halves[half * kOwn + row] = delta;
            sync_threads(pair, 64);
            delta += halves[(half ^ 1) * kOwn + row];
            if (inside && half == 0) a.delta[stat] = delta;

            // A row with one allowed key has p = 1 whatever its score: ds = 0, where dp - delta would leave two sums' noise.
            const int seen = sh.causal ? min(t.len, pos + 1) : t.len;
            const int used = live && seen > 1 ? seen : 0;
            const bool some_cut = __any_sync(0xFFFFFFFFu, used == 0);
            const float lse2 = live ? lse * kLog2e : 0.0f;
            float far_left = 0.0f, far_right = 0.0f;
            for (int j = 0; j < t.n; ++j, ++tile) {
                const int k0 = j * kStep, col0 = k0 + 32 * half;
                wait_warp(s_full, tile & 1, dead, 512 << 16);
                tc_fence_after();
                uint32_t s[32], d[32];
                tmem_ld32(s, lanes + Plan::s_col + 32 * half);
                tmem_ld32(d, lanes + Plan::dp_col + 32 * half);
                tmem_wait_ld();
                tmem_use(s);
                tmem_use(d);
                if (Plan::apart) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(s_free);
                }
                // x - lse = s * mul + off in base 2
                float mul = sh.scale_log2, off = -lse2;
                Span span = kSpanMixed;
                if (BIAS) {
                    span = span_of(a.bias, k0 - (t.q0 + kOwn - 1 + sh.q_pos), k0 + kStep - 1 - (t.q0 + sh.q_pos));
                    if (span == kSpanMixed) {
                        const float* at = lut + a.pad + col0 - pos;
#pragma unroll
                        for (int c = 0; c < 32; ++c) s[c] = __float_as_uint(fmaf(__uint_as_float(s[c]), mul, at[c]));
                        mul = 1.0f;
                    } else {
                        off += lut[span == kSpanFarLeft ? 0 : 2 * a.pad];
                    }
                }
                const uint64_t mul2v = pack2(mul, mul), off2 = pack2(off, off), nd2 = pack2(-delta, -delta);
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    float x, y;
                    unpack2(fma2(pack2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), mul2v, off2), x, y);
                    const uint64_t p = pack2(exp2_fast(x), exp2_fast(y));
                    unpack2(mul2(p, add2(pack2(__uint_as_float(d[e]), __uint_as_float(d[e + 1])), nd2)), x, y);
                    d[e] = __float_as_uint(x);
                    d[e + 1] = __float_as_uint(y);
                }
                if (some_cut || k0 + kStep > t.len || (sh.causal && k0 + kStep - 1 > t.q0 + sh.q_pos)) {
                    const int allowed = used - col0;
#pragma unroll
                    for (int c = 0; c < 32; ++c)
                        if (c >= allowed) d[c] = 0;
                }
                if (j > 0 && Plan::apart) {                    // dS of the last tile has been used
                    wait_warp(dq_done, (tile - 1) & 1, dead, 1024 << 16);
                    tc_fence_after();
                }
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = pack_bf16(__uint_as_float(d[2 * e]), __uint_as_float(d[2 * e + 1]));
                tmem_st16(lanes + Plan::ds_col + Plan::ds_half * half, w);
                if (k0 + kStep > t.len && t.len < sh.len_kv) {
                    // keys behind the sequence's end may hold anything; 0 * NaN must not reach dq
                    const int st = tile % ST, r = threadIdx.x & (kStep - 1), part = threadIdx.x >> 6;
                    if (k0 + r >= t.len) {
#pragma unroll
                        for (int c = 0; c < HALVES; ++c)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                *reinterpret_cast<uint4*>(smem + (sk - base) + st * Plan::step_bytes + c * kStepBytes + r * 128 + 32 * part + 16 * e) = make_uint4(0, 0, 0, 0);
                    }
                    fence_async_smem();
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(ds_ready);
                if (BIAS) {
                    if (span != kSpanMixed) {
                        uint64_t both[2] = {0, 0};
#pragma unroll
                        for (int e = 0; e < 16; ++e) both[e & 1] = add2(both[e & 1], pack2(__uint_as_float(d[2 * e]), __uint_as_float(d[2 * e + 1])));
                        float x, y;
                        unpack2(add2(both[0], both[1]), x, y);
                        if (span == kSpanFarLeft) far_left += x + y; else far_right += x + y;
                    } else {
                        // Sums along the diagonals of the warp's 32 x 32 part: a running sum moves one lane down per column and
                        // leaves at lane 31, complete.  Two groups of 16 columns, whose chains of shuffles overlap.
                        float run[2] = {0.0f, 0.0f};
#pragma unroll
                        for (int c = 0; c < 16; ++c) {
#pragma unroll
                            for (int g = 0; g < 2; ++g) {
                                run[g] = __shfl_up_sync(0xFFFFFFFFu, run[g], 1);
                                run[g] = (lane == 0 ? 0.0f : run[g]) + __uint_as_float(d[16 * g + c]);
                                if (lane == 31) sums[48 * g + c] = run[g];
                            }
                        }
#pragma unroll
                        for (int g = 0; g < 2; ++g) sums[48 * g + (lane == 31 ? 47 : 46 - lane)] = lane == 31 ? 0.0f : run[g];
                        __syncwarp();
                        const int first = col0 - (t.q0 + 32 * quad + 31 + sh.q_pos);
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            // a bucket is a run of distances: sums within runs, and the last lane of each run adds to its bucket
                            const int at = 32 * e + lane;
                            const int bucket = lut_bucket[a.pad + first + at];
                            float x = (at < 47 ? sums[at] : 0.0f) + (at >= 16 ? sums[48 + at - 16] : 0.0f);
#pragma unroll
                            for (int o = 1; o < 32; o <<= 1) {
                                const float y = __shfl_up_sync(0xFFFFFFFFu, x, o);
                                const int other = __shfl_up_sync(0xFFFFFFFFu, bucket, o);
                                if (lane >= o && other == bucket) x += y;
                            }
                            const int next = __shfl_down_sync(0xFFFFFFFFu, bucket, 1);
                            if (lane == 31 || next != bucket) bucket_sums[bucket] += x;
                            __syncwarp();
                        }
                    }
                }
            }
            if (BIAS) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    far_left += __shfl_down_sync(0xFFFFFFFFu, far_left, o);
                    far_right += __shfl_down_sync(0xFFFFFFFFu, far_right, o);
                }
                if (lane == 0) {
                    bucket_sums[lut_bucket[0]] += far_left;
                    bucket_sums[lut_bucket[2 * a.pad]] += far_right;
                }
                sync_threads(kAll, kMath);
                for (int e = threadIdx.x; e < a.bias.buckets; e += kMath) {
                    float x = 0.0f;
#pragma unroll
                    for (int w = 0; w < 8; ++w) x += by_bucket[w * a.bias.buckets + e];
                    partial[e] = x;
                }
            }
            wait_warp(dq_done, (tile - 1) & 1, dead, 2048 << 16);
            tc_fence_after();
            // dq goes out through q's place, which is free: its last product has completed
#pragma unroll
            for (int c = 0; c < HALVES; ++c) {
                const int x = 32 * (HALVES * half + c);
                uint32_t r[32];
                tmem_ld32(r, lanes + Plan::dq_col + x);
                tmem_wait_ld();
                tmem_use(r);
                if (t.q0 + 32 * quad < sh.len_q && x < sh.dim)
                    store_box(&a.dq.map, r, sh.scale, smem + buf * Plan::own_bytes + (warp * HALVES + c) * 2048, lane, x, t.q0 + 32 * quad,
                              t.h * a.dq.head_mul, t.b * a.dq.batch_mul);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                bar_arrive(dq_free);
                tma_store_wait_read();
                bar_arrive(own_empty + 8 * buf);
            }
            ++ordinal;
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
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
    int pad, items;
};

struct DkvItem {
    int b, hk, k0, len, q_first, per_head, n;  // sequence, key head, first key, valid keys, first query tile, tiles per query head, tiles
};

__device__ __forceinline__ DkvItem item_at(const DkvArgs& a, int i) {
    const Shape& sh = a.shape;
    const int bh = sh.batch * sh.heads_kv;
    DkvItem t;
    t.k0 = i / bh * kOwn;                                      // the first keys see the most queries: they come first
    t.b = i % bh / sh.heads_kv;
    t.hk = i % bh % sh.heads_kv;
    t.len = sh.kv_len ? min(max(sh.kv_len[t.b], 0), sh.len_kv) : sh.len_kv;
    const int q_tiles = (sh.len_q + kStep - 1) / kStep;
    t.q_first = 0;                                             // the first tile with a row that sees one of the keys
    if (sh.causal && t.k0 > sh.q_pos) t.q_first = min((t.k0 - sh.q_pos) / kStep, q_tiles);
    t.per_head = q_tiles - t.q_first;
    t.n = t.k0 < t.len ? t.per_head * sh.group : 0;
    return t;
}

template <int HALVES>
struct DkvPlan {
    static constexpr int stages = 2, own_bufs = HALVES == 1 ? 2 : 1;
    static constexpr bool apart = HALVES == 2;         // P and dS beside S and dP; one block per SM has all 512 columns
    static constexpr int blocks = HALVES == 1 ? 2 : 1;
    static constexpr uint32_t columns = HALVES == 1 ? 256 : 512;
    static constexpr uint32_t s_col = 0, dp_col = 64, dv_col = 128, dk_col = 128 + 64 * HALVES;
    static constexpr uint32_t p_col = apart ? 384 : s_col, ds_col = apart ? 416 : dp_col, p_half = apart ? 16 : 32;
    static constexpr uint32_t own_bytes = HALVES * kOwnBytes, step_bytes = HALVES * kStepBytes;
    static constexpr uint32_t tiles_bytes = own_bufs * 2 * own_bytes + 2 * stages * step_bytes;
    static constexpr uint32_t bars = 6 + 2 * own_bufs + 3 * stages;
    static constexpr uint32_t stat_floats = 2 * kStep + 4;     // (-lse in base 2)[64], (-delta)[64], whether the tile has holes
    static constexpr uint32_t fixed_bytes = tiles_bytes + 256 + stages * stat_floats * sizeof(float);
};

template <int HALVES>
size_t dkv_smem(int pad, bool bias) {
    return 1024 + DkvPlan<HALVES>::fixed_bytes + (bias ? (2 * pad + 1) * (sizeof(float) + 1) : 0);
}

template <int HALVES, bool BIAS>
__global__ void __launch_bounds__(kThreads, DkvPlan<HALVES>::blocks) attn_dkv_kernel(const __grid_constant__ DkvArgs a) {
    using Plan = DkvPlan<HALVES>;
    constexpr int ST = Plan::stages, OB = Plan::own_bufs;
    extern __shared__ uint8_t raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    const uint32_t base = smem_u32(smem);
    const uint32_t sk = base, sv = sk + OB * Plan::own_bytes, sq = sv + OB * Plan::own_bytes, sdo = sq + ST * Plan::step_bytes;
    const uint32_t bars = base + Plan::tiles_bytes;
    const uint32_t s_full = bars, s_free = bars + 8, p_ready = bars + 16, acc_done = bars + 24, acc_free = bars + 32, drained = bars + 40;
    const uint32_t own_full = bars + 48, own_empty = own_full + 8 * OB, full = own_empty + 8 * OB, empty = full + 8 * ST, stat_full = empty + 8 * ST;
    uint32_t* words = reinterpret_cast<uint32_t*>(smem + Plan::tiles_bytes + 8 * Plan::bars);
    volatile uint32_t* dead = words + 1;
    float* stats = reinterpret_cast<float*>(smem + Plan::tiles_bytes + 256);
    float* lut = stats + ST * Plan::stat_floats;
    uint8_t* lut_bucket = reinterpret_cast<uint8_t*>(lut + 2 * a.pad + 1);

    const Shape& sh = a.shape;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        bar_init(s_full, 1);
        bar_init(s_free, 8);
        bar_init(p_ready, 8);
        bar_init(acc_done, 1);
        bar_init(acc_free, 8);
        bar_init(drained, 1);
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
    if (threadIdx.x == kMath) {
        tma_prefetch(&a.q.map);
        tma_prefetch(&a.dout.map);
        tma_prefetch(&a.k.map);
        tma_prefetch(&a.v.map);
        tma_prefetch(&a.dk.map);
        tma_prefetch(&a.dv.map);
    }
    if (BIAS && warp < 8) fill_buckets(a.bias, lut_bucket, a.pad, threadIdx.x, kMath);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = words[0];
    grid_dependency_sync();

    if (warp == 8) {
        int ordinal = 0, tile = 0;                             // items and tiles whose copies have been started
        for (int i = blockIdx.x; i < a.items; i += gridDim.x) {
            const DkvItem t = item_at(a, i);
            if (t.n == 0) continue;
            const int buf = ordinal % OB;
            wait_warp(own_empty + 8 * buf, ((ordinal / OB) & 1) ^ 1, dead, 1 << 16);
            if (__any_sync(0xFFFFFFFFu, *dead)) break;
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
            for (int j = 0; j < t.n; ++j) {
                const int st = tile % ST, q0 = q_tile * kStep;
                wait_warp(empty + 8 * st, ((tile / ST) & 1) ^ 1, dead, 2 << 16);
                if (__any_sync(0xFFFFFFFFu, *dead)) break;
                if (lane == 0) {
                    bar_expect(full + 8 * st, 2 * Plan::step_bytes);
                    for (int c = 0; c < HALVES; ++c) {
                        const uint32_t at = st * Plan::step_bytes + c * kStepBytes;
                        tma_load4(sq + at, &a.q.map, full + 8 * st, 64 * c, q0, head * a.q.head_mul, t.b * a.q.batch_mul);
                        tma_load4(sdo + at, &a.dout.map, full + 8 * st, 64 * c, q0, head * a.dout.head_mul, t.b * a.dout.batch_mul);
                    }
                }
                // lse and delta of the tile's rows, two per lane
                float* stat = stats + st * Plan::stat_floats;
                bool hole = false;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = lane + 32 * e;
                    float nl = -INFINITY, nd = 0.0f;           // a row behind len_q, or without allowed keys: p = 0
                    if (q0 + r < sh.len_q) {
                        const size_t at = ((size_t)t.b * sh.heads_q + head) * sh.len_q + q0 + r;
                        const float lse = a.lse[at];
                        if (lse == -INFINITY) hole = true; else nl = -lse * kLog2e;
                        nd = -a.delta[at];
                    }
                    stat[r] = nl;
                    stat[kStep + r] = nd;
                }
                hole = __any_sync(0xFFFFFFFFu, hole);
                if (lane == 0) {
                    stat[2 * kStep] = hole ? 1.0f : 0.0f;
                }
                __syncwarp();
                if (lane == 0) bar_arrive(stat_full + 8 * st);
                if (++q_tile == t.q_first + t.per_head) {
                    q_tile = t.q_first;
                    ++head;
                }
                ++tile;
            }
        }
        // every copy has landed before the block may leave, whoever else has given up
        for (int i = max(0, ordinal - OB); i < ordinal; ++i) drain(own_full + 8 * (i % OB), (i / OB) & 1);
        for (int i = max(0, tile - ST); i < tile; ++i) drain(full + 8 * (i % ST), (i / ST) & 1);
    } else if (warp == 9) {
        constexpr uint32_t desc_s = mma_desc(kStep, false), desc_acc = mma_desc(64 * HALVES, true);
        const bool leader = elect_one();
        const uint64_t q_desc = desc_k_major(sq), do_desc = desc_k_major(sdo), k_desc = desc_k_major(sk), v_desc = desc_k_major(sv);
        const uint64_t qn_desc = desc_n_major(sq, kStepBytes), don_desc = desc_n_major(sdo, kStepBytes);
        Cursor<DkvArgs, DkvItem> ahead, at;                    // of S' and dP', and of dV and dK
        ahead.start(a);
        at = ahead;
        auto scores = [&]() {
            const int st = ahead.tile % ST, buf = ahead.ordinal % OB;
            if (ahead.j == 0) wait_warp(own_full + 8 * buf, (ahead.ordinal / OB) & 1, dead, 4 << 16);
            wait_warp(full + 8 * st, (ahead.tile / ST) & 1, dead, 8 << 16);
            tc_fence_after();
            const uint32_t own = buf * (Plan::own_bytes >> 4), step = st * (Plan::step_bytes >> 4);
            if (leader) {
#pragma unroll
                for (int i = 0; i < 4 * HALVES; ++i) {
                    const uint32_t o = own + (((i >> 2) * kOwnBytes + (i & 3) * 32) >> 4), s = step + (((i >> 2) * kStepBytes + (i & 3) * 32) >> 4);
                    mma_ss(tmem + Plan::s_col, k_desc + o, q_desc + s, desc_s, i > 0);
                    mma_ss(tmem + Plan::dp_col, v_desc + o, do_desc + s, desc_s, i > 0);
                }
                mma_commit(s_full);
            }
            __syncwarp();
            ahead.next(a);
        };
        if (ahead.more) scores();
        int items = 0;                                         // whose dV and dK have been started
        while (at.more) {
            const int st = at.tile % ST;
            const uint32_t parity = at.tile & 1;
            // with one place for k and v, the next item's come only after this item's last products
            const bool early = Plan::apart && ahead.more && (OB > 1 || ahead.j > 0);
            if (early) {
                wait_warp(s_free, parity, dead, 16 << 16);
                scores();
            }
            if (at.j == 0) {                                   // the last item's dV and dK have been read
                wait_warp(acc_free, (items & 1) ^ 1, dead, 32 << 16);
                ++items;
            }
            wait_warp(p_ready, parity, dead, 64 << 16);
            tc_fence_after();
            const uint32_t step = st * (Plan::step_bytes >> 4);
            const bool more = at.j > 0;
            if (leader) {
#pragma unroll
                for (int i = 0; i < kStep / 16; ++i) {
                    const uint32_t p = (i >> 1) * Plan::p_half + (i & 1) * 8;
                    mma_ts(tmem + Plan::dv_col, tmem + Plan::p_col + p, don_desc + step + i * 128, desc_acc, more || i > 0);
                    mma_ts(tmem + Plan::dk_col, tmem + Plan::ds_col + p, qn_desc + step + i * 128, desc_acc, more || i > 0);
                }
                mma_commit(empty + 8 * st);
                mma_commit(acc_done);
            }
            __syncwarp();
            if (!early && ahead.more) {
                wait_warp(acc_done, parity, dead, 128 << 16);
                scores();
            }
            at.next(a);
        }
        if (leader) {
            mma_commit(drained);
            drain(drained, 0);
        }
    } else {
        const int half = warp >> 2, quad = warp & 3;
        const int row = quad * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)quad << 21);
        int ordinal = 0, tile = 0;
        for (int i = blockIdx.x; i < a.items; i += gridDim.x) {
            const DkvItem t = item_at(a, i);
            const int key = t.k0 + row, buf = ordinal % OB;
            if (t.n == 0) {
                if (key < sh.len_kv) {
                    if (half == 0) zero_row(a.dk, sh.dim, t.b, t.hk, key);
                    else zero_row(a.dv, sh.dim, t.b, t.hk, key);
                }
                continue;
            }
            int head = t.hk * sh.group, q_tile = t.q_first;
            for (int j = 0; j < t.n; ++j, ++tile) {
                const int st = tile % ST, q0 = q_tile * kStep, pos0 = q0 + sh.q_pos, col0 = 32 * half;
                if (BIAS && q_tile == t.q_first) {             // another query head: its table, once nobody uses the last one's
                    const int last = (t.q_first + t.per_head) * kStep - 1 + sh.q_pos;
                    sync_threads(kAll, kMath);
                    fill_lut(a.bias, head, lut_bucket, lut, a.pad, t.k0 - last, sh.causal ? 0 : t.k0 + kOwn - 1 - pos0, threadIdx.x, kMath);
                    sync_threads(kAll, kMath);
                }
                wait_warp(stat_full + 8 * st, (tile / ST) & 1, dead, 256 << 16);
                const float* nl = stats + st * Plan::stat_floats;
                const float* nd = nl + kStep;
                wait_warp(s_full, tile & 1, dead, 512 << 16);
                tc_fence_after();
                const Span span = BIAS ? span_of(a.bias, t.k0 - (pos0 + kStep - 1), t.k0 + kOwn - 1 - pos0) : kSpanFarLeft;
                const float mul = BIAS && span == kSpanMixed ? 1.0f : sh.scale_log2;
                const float add = BIAS && span != kSpanMixed ? lut[span == kSpanFarLeft ? 0 : 2 * a.pad] : 0.0f;
                const bool holes = nl[2 * kStep] != 0.0f;      // rows inside len_q with nothing allowed
                // 16 columns at a time, for the registers' sake
#pragma unroll 1
                for (int c0 = 0; c0 < 32; c0 += 16) {
                    const int col = col0 + c0;
                    uint32_t s[16], d[16];
                    tmem_ld16(s, lanes + Plan::s_col + col);
                    tmem_ld16(d, lanes + Plan::dp_col + col);
                    tmem_wait_ld();
                    tmem_use(s);
                    tmem_use(d);
                    if (Plan::apart && c0 == 16) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) bar_arrive(s_free);
                    }
                    if (BIAS && span == kSpanMixed) {
                        const float* at = lut + a.pad + key - (pos0 + col);
#pragma unroll
                        for (int c = 0; c < 16; ++c) s[c] = __float_as_uint(fmaf(__uint_as_float(s[c]), sh.scale_log2, at[-c]));
                    }
                    const int first = sh.causal ? key - (pos0 + col) : 0;      // rows before it do not see the key
                    if (sh.causal && t.k0 + kOwn - 1 > pos0) {
#pragma unroll
                        for (int c = 0; c < 16; ++c)
                            if (c < first) s[c] = 0xFF800000u;
                    }
                    const uint64_t mul2v = pack2(mul, mul), add2v = pack2(add, add);
                    uint32_t wp[8], wd[8];
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const float4 l = *reinterpret_cast<const float4*>(nl + col + e);
                        const float4 m = *reinterpret_cast<const float4*>(nd + col + e);
                        const uint64_t ls[2] = {pack2(l.x, l.y), pack2(l.z, l.w)}, ms[2] = {pack2(m.x, m.y), pack2(m.z, m.w)};
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const int at = e + 2 * u;
                            float x, y;
                            unpack2(fma2(pack2(__uint_as_float(s[at]), __uint_as_float(s[at + 1])), mul2v, add2(ls[u], add2v)), x, y);
                            x = exp2_fast(x);
                            y = exp2_fast(y);
                            wp[at >> 1] = pack_bf16(x, y);
                            unpack2(mul2(pack2(x, y), add2(pack2(__uint_as_float(d[at]), __uint_as_float(d[at + 1])), ms[u])), x, y);
                            wd[at >> 1] = pack_bf16(x, y);
                        }
                    }
                    if (t.len == 1 || (sh.causal && key == 0)) {       // rows that see one key alone: p = 1, ds = 0
#pragma unroll
                        for (int c = 0; c < 16; ++c)
                            if (t.len == 1 || c == first) wd[c >> 1] &= c & 1 ? 0x0000FFFFu : 0xFFFF0000u;
                    }
                    if (holes) {                               // whatever their do and q hold
#pragma unroll
                        for (int c = 0; c < 16; ++c)
                            if (nl[col + c] == -INFINITY) {
                                wp[c >> 1] &= c & 1 ? 0x0000FFFFu : 0xFFFF0000u;
                                wd[c >> 1] &= c & 1 ? 0x0000FFFFu : 0xFFFF0000u;
                            }
                    }
                    if (j > 0 && Plan::apart && c0 == 0) {     // P and dS of the last tile have been used
                        wait_warp(acc_done, (tile - 1) & 1, dead, 1024 << 16);
                        tc_fence_after();
                    }
                    tmem_st8(lanes + Plan::p_col + Plan::p_half * half + (c0 >> 1), wp);
                    tmem_st8(lanes + Plan::ds_col + Plan::p_half * half + (c0 >> 1), wd);
                }
                if (holes) {
                    // and must not reach a product: 0 * NaN
                    const int r = threadIdx.x & (kStep - 1), part = threadIdx.x >> 6;
                    if (nl[r] == -INFINITY) {
#pragma unroll
                        for (int c = 0; c < HALVES; ++c)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const uint32_t at = st * Plan::step_bytes + c * kStepBytes + r * 128 + 32 * part + 16 * e;
                                *reinterpret_cast<uint4*>(smem + (sq - base) + at) = make_uint4(0, 0, 0, 0);
                                *reinterpret_cast<uint4*>(smem + (sdo - base) + at) = make_uint4(0, 0, 0, 0);
                            }
                    }
                    fence_async_smem();
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_ready);
                if (++q_tile == t.q_first + t.per_head) {
                    q_tile = t.q_first;
                    ++head;
                }
            }
            wait_warp(acc_done, (tile - 1) & 1, dead, 2048 << 16);
            tc_fence_after();
            // dk (warps 0-3) and dv go out through k's and v's places, which are free: every product has completed.  Keys
            // behind the sequence's end get zeros
            const uint32_t col = half == 0 ? Plan::dk_col : Plan::dv_col;
            uint8_t* staging = smem + ((half == 0 ? sk : sv) - base) + buf * Plan::own_bytes + quad * 2 * HALVES * 2048;
#pragma unroll
            for (int c = 0; c < 2 * HALVES; ++c) {
                uint32_t r[32];
                tmem_ld32(r, lanes + col + 32 * c);
                tmem_wait_ld();
                tmem_use(r);
                if (key >= t.len) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) r[e] = 0;
                }
                if (t.k0 + 32 * quad >= sh.len_kv || 32 * c >= sh.dim) continue;
                if (half == 0) store_box(&a.dk.map, r, sh.scale, staging + c * 2048, lane, 32 * c, t.k0 + 32 * quad, t.hk * a.dk.head_mul, t.b * a.dk.batch_mul);
                else store_box(&a.dv.map, r, 1.0f, staging + c * 2048, lane, 32 * c, t.k0 + 32 * quad, t.hk * a.dv.head_mul, t.b * a.dv.batch_mul);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                bar_arrive(acc_free);
                tma_store_wait_read();
                bar_arrive(own_empty + 8 * buf);
            }
            ++ordinal;
        }
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

// dtable[h][n] = sum over the sequences and query blocks of one head, in that order.
__global__ void __launch_bounds__(256) attn_dtable_kernel(const float* partial, int batch, int heads, int blocks, int buckets,
                                                          float* out32, uint16_t* out16) {
    __shared__ double shared[8][32];
    grid_dependency_sync();
    const int h = blockIdx.x, bucket = blockIdx.y * 32 + threadIdx.x;
    double s = 0.0;
    if (bucket < buckets)
        for (int i = threadIdx.y; i < batch * blocks; i += 8) {
            const size_t row = ((size_t)(i / blocks) * heads + h) * blocks + i % blocks;
            s += partial[row * buckets + bucket];
        }
    shared[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y == 0 && bucket < buckets) {
        for (int i = 1; i < 8; ++i) s += shared[i][threadIdx.x];
        if (out32) out32[(size_t)h * buckets + bucket] = (float)s;
        else out16[(size_t)h * buckets + bucket] = (uint16_t)(pack_bf16((float)s, 0.0f) & 0xFFFFu);
    }
}

template <typename K, typename A>
int launch(K kernel, int per_sm, size_t smem, const A& a, cudaStream_t s) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return ALSGD_E_CUDA;
    const int wave = blocks_at_once(smem, per_sm);
    return launch_dependent(kernel, dim3(a.items < wave ? a.items : wave), dim3(kThreads), smem, s, a) == cudaSuccess ? ALSGD_OK : ALSGD_E_CUDA;
}

uint64_t delta_bytes(const alsgd_attn_desc& d) { return ((uint64_t)d.batch * d.heads_q * d.len_q * 4 + 255) / 256 * 256; }
uint64_t partial_bytes(const alsgd_attn_desc& d) { return (uint64_t)d.batch * d.heads_q * ((d.len_q + kOwn - 1) / kOwn) * d.buckets * 4; }

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
    if (reinterpret_cast<uintptr_t>(table) % 4 || reinterpret_cast<uintptr_t>(dtable) % 4 || reinterpret_cast<uintptr_t>(kv_len) % 4) return ALSGD_E_ARG;
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
        a.shape = make_shape(d, kv_len);
        make_bias(d, table, &a.bias);
        a.pad = a.bias.far + kOwn + kStep;
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
        if (d.dim <= 64) rc = d.buckets ? launch(attn_dq_kernel<1, true>, 2, dq_smem<1>(a.pad, (int)d.buckets), a, s)
                                        : launch(attn_dq_kernel<1, false>, 2, dq_smem<1>(a.pad, 0), a, s);
        else rc = d.buckets ? launch(attn_dq_kernel<2, true>, 2, dq_smem<2>(a.pad, (int)d.buckets), a, s)
                            : launch(attn_dq_kernel<2, false>, 2, dq_smem<2>(a.pad, 0), a, s);
        if (rc != ALSGD_OK) return rc;
    }
    if (d.len_kv) {
        DkvArgs a;
        a.shape = make_shape(d, kv_len);
        make_bias(d, table, &a.bias);
        a.pad = a.bias.far + kOwn + kStep;
        a.items = (int)kv_items;
        a.lse = lse;
        a.delta = delta;
        if ((rc = operand(q, true, kStep, 64, &a.q)) != ALSGD_OK || (rc = operand(dout, true, kStep, 64, &a.dout)) != ALSGD_OK ||
            (rc = operand(k, false, kOwn, 64, &a.k)) != ALSGD_OK || (rc = operand(v, false, kOwn, 64, &a.v)) != ALSGD_OK ||
            (rc = operand(dk, false, 32, 32, &a.dk)) != ALSGD_OK || (rc = operand(dv, false, 32, 32, &a.dv)) != ALSGD_OK)
            return rc;
        if (d.dim <= 64) rc = d.buckets ? launch(attn_dkv_kernel<1, true>, 2, dkv_smem<1>(a.pad, true), a, s)
                                        : launch(attn_dkv_kernel<1, false>, 2, dkv_smem<1>(a.pad, false), a, s);
        else rc = d.buckets ? launch(attn_dkv_kernel<2, true>, 1, dkv_smem<2>(a.pad, true), a, s)
                            : launch(attn_dkv_kernel<2, false>, 1, dkv_smem<2>(a.pad, false), a, s);
        if (rc != ALSGD_OK) return rc;
    }
    if (d.buckets) {
        const bool wide = d.table_dtype == ALSGD_F32;
        if (launch_dependent(attn_dtable_kernel, dim3(d.heads_q, (d.buckets + 31) / 32), dim3(32, 8), 0, s, (const float*)partial, (int)d.batch,
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
