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
//                     a thread holds one key); the query heads that share a key head are walked by the same block
// One kernel that forms S and dP once would save two of the seven products and half of the exponentials, but has to
// add dQ across blocks.
//
// Everything is binary32 but the operands of the second products: p and ds are rounded to bf16 (the type of do, q and
// k), as the forward pass rounds p.
#include "alsgd_attn.cuh"

using namespace alsgd_attn;
using namespace alsgd_ops;
using namespace alsgd_tc;

namespace {

constexpr int kOwn = 128;               // rows a block owns
constexpr int kStep = 64;               // rows of a streamed tile
constexpr int kThreads = 192;
constexpr uint32_t kOwnBytes = 128 * 128;      // 128 rows of 64 bf16
constexpr uint32_t kStepBytes = 64 * 128;
constexpr int kDiagonals = 96;          // of 32 rows x 64 columns, padded

// Whether `p` holds in any of the block's first 128 threads (all of which call it).
__device__ __forceinline__ bool any_of_128(bool p) {
    uint32_t r;
    asm volatile("{\n .reg .pred a, b;\n setp.ne.u32 a, %1, 0;\n barrier.cta.red.or.pred b, 1, 128, a;\n selp.u32 %0, 1, 0, b;\n}\n"
                 : "=r"(r) : "r"((uint32_t)p) : "memory");
    return r != 0;
}

__device__ __forceinline__ float* smem_f(uint8_t* p) { return reinterpret_cast<float*>(p); }

// =============================================================================================== dq

struct DqArgs {
    Operand q, k, v, dout, dq;
    Shape shape;
    Bias bias;
    const float* lse;
    const uint16_t* o;
    int64_t o_batch, o_pos, o_head;     // steps of o
    float* delta;                       // out: [batch][heads_q][len_q]
    float* partial;                     // out: [batch * heads_q][query blocks][buckets]
    int pad;
};

template <int HALVES>
struct DqPlan {
    static constexpr int stages = HALVES == 1 ? 3 : 1;
    static constexpr bool apart = HALVES == 1;         // dS beside S, so that the next tile's scores need not wait for dQ
    static constexpr uint32_t columns = 256;
    static constexpr uint32_t s_col = 0, dp_col = 64, ds_col = apart ? 192 : 0, dq_col = 128;
    static constexpr uint32_t own_bytes = HALVES * kOwnBytes, step_bytes = HALVES * kStepBytes;
    static constexpr uint32_t tiles_bytes = 2 * own_bytes + 2 * stages * step_bytes;
    static constexpr uint32_t bars = 6 + 2 * stages;
};

template <int HALVES>
size_t dq_smem(int pad, int buckets) {
    return 1024 + DqPlan<HALVES>::tiles_bytes + 256 +
           (buckets ? (4 * kDiagonals + 4 * buckets + 2 * pad + 1) * sizeof(float) + (2 * pad + 1) : 0);
}

template <int HALVES, bool BIAS>
__global__ void __launch_bounds__(kThreads, 2) attn_dq_kernel(const __grid_constant__ DqArgs a) {
    using Plan = DqPlan<HALVES>;
    constexpr int ST = Plan::stages;
    extern __shared__ uint8_t raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    const uint32_t base = smem_u32(smem);
    const uint32_t sq = base, sdo = sq + Plan::own_bytes, sk = sdo + Plan::own_bytes, sv = sk + ST * Plan::step_bytes;
    const uint32_t bars = base + Plan::tiles_bytes;
    const uint32_t own_full = bars, s_full = bars + 8, s_free = bars + 16, ds_ready = bars + 24, dq_done = bars + 32, drained = bars + 40;
    const uint32_t full = bars + 48, empty = full + 8 * ST;
    uint32_t* words = reinterpret_cast<uint32_t*>(smem + Plan::tiles_bytes + 8 * Plan::bars);
    volatile uint32_t* dead = words + 1;
    float* diag = smem_f(smem + Plan::tiles_bytes + 256);
    float* by_bucket = diag + 4 * kDiagonals;
    float* lut = by_bucket + 4 * a.bias.buckets;
    uint8_t* lut_bucket = reinterpret_cast<uint8_t*>(lut + 2 * a.pad + 1);

    const Shape& sh = a.shape;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int b = blockIdx.x / sh.heads_q, h = blockIdx.x % sh.heads_q, hk = h / sh.group;
    const int block = gridDim.y - 1 - blockIdx.y;              // the longest rows of a causal mask start first
    const int q0 = block * kOwn;

    if (threadIdx.x == 0) {
        bar_init(own_full, 1);
        bar_init(s_full, 1);
        bar_init(s_free, 4);
        bar_init(ds_ready, 4);
        bar_init(dq_done, 1);
        bar_init(drained, 1);
        for (int i = 0; i < ST; ++i) {
            bar_init(full + 8 * i, 1);
            bar_init(empty + 8 * i, 1);
        }
        words[1] = 0;
        bar_init_fence();
    }
    if (warp == 5) tmem_alloc(smem_u32(words), Plan::columns);
    if (threadIdx.x == 128) {
        tma_prefetch(&a.q.map);
        tma_prefetch(&a.dout.map);
        tma_prefetch(&a.k.map);
        tma_prefetch(&a.v.map);
        tma_prefetch(&a.dq.map);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = words[0];
    grid_dependency_sync();

    const int len = sh.kv_len ? min(max(sh.kv_len[b], 0), sh.len_kv) : sh.len_kv;
    int keys = len;
    if (sh.causal) keys = min(keys, min(q0 + kOwn, sh.len_q) + sh.q_pos);
    const int n = keys > 0 ? (keys + kStep - 1) / kStep : 0;

    if (warp == 4) {
        if (lane == 0) {                                       // do is wanted for delta even where no key is
            bar_expect(own_full, 2 * Plan::own_bytes);
            for (int c = 0; c < HALVES; ++c) {
                tma_load4(sq + c * kOwnBytes, &a.q.map, own_full, 64 * c, q0, h * a.q.head_mul, b * a.q.batch_mul);
                tma_load4(sdo + c * kOwnBytes, &a.dout.map, own_full, 64 * c, q0, h * a.dout.head_mul, b * a.dout.batch_mul);
            }
            int j = 0;
            for (; j < n; ++j) {
                const int st = j % ST;
                if (!wait(empty + 8 * st, ((j / ST) & 1) ^ 1, dead, 1)) break;
                bar_expect(full + 8 * st, 2 * Plan::step_bytes);
                for (int c = 0; c < HALVES; ++c) {
                    tma_load4(sk + st * Plan::step_bytes + c * kStepBytes, &a.k.map, full + 8 * st, 64 * c, j * kStep, hk * a.k.head_mul, b * a.k.batch_mul);
                    tma_load4(sv + st * Plan::step_bytes + c * kStepBytes, &a.v.map, full + 8 * st, 64 * c, j * kStep, hk * a.v.head_mul, b * a.v.batch_mul);
                }
            }
            drain(own_full, 0);
            for (int i = max(0, j - ST); i < j; ++i) drain(full + 8 * (i % ST), (i / ST) & 1);
        }
    } else if (warp == 5) {
        if (lane == 0 && n > 0) {
            constexpr uint32_t desc_s = mma_desc(kStep, false), desc_q = mma_desc(64 * HALVES, true);
            const int steps = (sh.dim + 15) / 16;
            auto scores = [&](int j) {
                const int st = j % ST;
                if (!wait(full + 8 * st, (j / ST) & 1, dead, 2)) return false;
                tc_fence_after();
                for (int i = 0; i < steps; ++i) {
                    const uint32_t own = (i >> 2) * kOwnBytes + (i & 3) * 32, step = st * Plan::step_bytes + (i >> 2) * kStepBytes + (i & 3) * 32;
                    mma_ss(tmem + Plan::s_col, desc_k_major(sq + own), desc_k_major(sk + step), desc_s, i > 0);
                }
                for (int i = 0; i < steps; ++i) {
                    const uint32_t own = (i >> 2) * kOwnBytes + (i & 3) * 32, step = st * Plan::step_bytes + (i >> 2) * kStepBytes + (i & 3) * 32;
                    mma_ss(tmem + Plan::dp_col, desc_k_major(sdo + own), desc_k_major(sv + step), desc_s, i > 0);
                }
                mma_commit(s_full);
                return true;
            };
            bool ok = wait(own_full, 0, dead, 4) && scores(0);
            for (int j = 0; j < n && ok; ++j) {
                const int st = j % ST;
                if (Plan::apart && j + 1 < n) {
                    ok = wait(s_free, j & 1, dead, 8) && scores(j + 1);
                    if (!ok) break;
                }
                ok = wait(ds_ready, j & 1, dead, 16);
                if (!ok) break;
                tc_fence_after();
                for (int i = 0; i < kStep / 16; ++i)
                    mma_ts(tmem + Plan::dq_col, tmem + Plan::ds_col + 8 * i, desc_n_major(sk + st * Plan::step_bytes + i * 2048, kStepBytes),
                           desc_q, j > 0 || i > 0);
                mma_commit(empty + 8 * st);
                mma_commit(dq_done);
                if (!Plan::apart && j + 1 < n) ok = wait(dq_done, j & 1, dead, 32) && scores(j + 1);
            }
            mma_commit(drained);
            drain(drained, 0);
        }
    } else {
        const int row = threadIdx.x;
        const bool inside = q0 + row < sh.len_q;
        const int pos = q0 + row + sh.q_pos;
        const uint32_t lanes = tmem + ((uint32_t)warp << 21);
        const size_t stat = ((size_t)b * sh.heads_q + h) * sh.len_q + q0 + row;
        const float lse = inside ? a.lse[stat] : -INFINITY;
        const bool live = lse != -INFINITY;
        if (BIAS) {
            fill_lut(a.bias, h, lut, a.pad, row, 128);
            for (int i = row; i <= 2 * a.pad; i += 128) lut_bucket[i] = (uint8_t)bucket_of(a.bias, i - a.pad);
            for (int i = row; i < 4 * a.bias.buckets; i += 128) by_bucket[i] = 0.0f;
            asm volatile("bar.sync 1, 128;" ::: "memory");
        }
        bool ok = wait_warp(own_full, 0, dead, 64);
        float delta = 0.0f;
        if (ok && live) {
            const uint16_t* o = a.o + (int64_t)b * a.o_batch + (int64_t)(q0 + row) * a.o_pos + (int64_t)h * a.o_head;
            float acc[2] = {0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < 8 * HALVES; ++c) {
                if (8 * c >= sh.dim) break;
                const uint4 x = *reinterpret_cast<const uint4*>(o + 8 * c);
                const uint4 y = *reinterpret_cast<const uint4*>(smem + (sdo - base) + (c >> 3) * kOwnBytes + row * 128 + (((c & 7) ^ (row & 7)) << 4));
                const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    acc[0] = fmaf(bf16_lo(xs[e]), bf16_lo(ys[e]), acc[0]);
                    acc[1] = fmaf(bf16_hi(xs[e]), bf16_hi(ys[e]), acc[1]);
                }
            }
            delta = acc[0] + acc[1];
        }
        if (inside) a.delta[stat] = delta;
        // A row with one allowed key has p = 1 whatever its score: ds = 0, where dp - delta would leave two sums' noise.
        const int seen = sh.causal ? min(len, pos + 1) : len;
        const int used = live && seen > 1 ? seen : 0;
        const bool some_cut = __any_sync(0xFFFFFFFFu, used == 0);
        // x - lse = s * mul + off in base 2; a row without any allowed key has ds = 0
        const float lse2 = live ? lse * kLog2e : 0.0f;
        float far_left = 0.0f, far_right = 0.0f;
        for (int j = 0; j < n && ok; ++j) {
            const int k0 = j * kStep;
            ok = wait_warp(s_full, j & 1, dead, 128);
            if (!ok) break;
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
            float mul = sh.scale_log2, off = -lse2;
            Span span = kSpanMixed;
            if (BIAS) {
                span = span_of(a.bias, k0 - (q0 + kOwn - 1 + sh.q_pos), k0 + kStep - 1 - (q0 + sh.q_pos));
                if (span == kSpanMixed) {
                    const float* at = lut + a.pad + k0 - pos;
#pragma unroll
                    for (int c = 0; c < kStep; ++c) s[c >> 5][c & 31] = __float_as_uint(fmaf(__uint_as_float(s[c >> 5][c & 31]), mul, at[c]));
                    mul = 1.0f;
                } else {
                    off += lut[span == kSpanFarLeft ? 0 : 2 * a.pad];
                }
            }
            const uint64_t mul2v = pack2(mul, mul), off2 = pack2(off, off), nd2 = pack2(-delta, -delta);
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float x, y;
                    unpack2(fma2(pack2(__uint_as_float(s[c][2 * i]), __uint_as_float(s[c][2 * i + 1])), mul2v, off2), x, y);
                    const uint64_t p = pack2(exp2_fast(x), exp2_fast(y));
                    unpack2(mul2(p, add2(pack2(__uint_as_float(d[c][2 * i]), __uint_as_float(d[c][2 * i + 1])), nd2)), x, y);
                    d[c][2 * i] = __float_as_uint(x);
                    d[c][2 * i + 1] = __float_as_uint(y);
                }
            if (some_cut || k0 + kStep > len || (sh.causal && k0 + kStep - 1 > q0 + sh.q_pos)) {
                const int allowed = used - k0;
#pragma unroll
                for (int c = 0; c < kStep; ++c)
                    if (c >= allowed) d[c >> 5][c & 31] = 0;
            }
            if (j > 0 && Plan::apart) {                        // dS of the last tile has been used
                ok = wait_warp(dq_done, (j - 1) & 1, dead, 256);
                if (!ok) break;
                tc_fence_after();
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = pack_bf16(__uint_as_float(d[c][2 * i]), __uint_as_float(d[c][2 * i + 1]));
                tmem_st16(lanes + Plan::ds_col + 16 * c, w);
            }
            if (k0 + kStep > len && len < sh.len_kv) {
                // keys behind the sequence's end may hold anything; 0 * NaN must not reach dq
                const int st = j % ST, r = row & (kStep - 1), part = row >> 6;
                if (k0 + r >= len) {
#pragma unroll
                    for (int c = 0; c < HALVES; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            *reinterpret_cast<uint4*>(smem + (sk - base) + st * Plan::step_bytes + c * kStepBytes + r * 128 + 64 * part + 16 * i) = make_uint4(0, 0, 0, 0);
                }
                fence_async_smem();
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(ds_ready);
            if (BIAS) {
                if (span != kSpanMixed) {
                    uint64_t t[2] = {0, 0};
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        t[i & 1] = add2(t[i & 1], pack2(__uint_as_float(d[i >> 4][2 * (i & 15)]), __uint_as_float(d[i >> 4][2 * (i & 15) + 1])));
                    float x, y;
                    unpack2(add2(t[0], t[1]), x, y);
                    if (span == kSpanFarLeft) far_left += x + y; else far_right += x + y;
                } else {
                    // Sums along the diagonals of the warp's 32 x 64 part: a running sum moves one lane down per column
                    // and leaves at lane 31, complete; diagonal c - lane + 31 has distance first + that.
                    float* sums = diag + warp * kDiagonals;
                    float run = 0.0f;
#pragma unroll
                    for (int c = 0; c < kStep; ++c) {
                        run = __shfl_up_sync(0xFFFFFFFFu, run, 1);
                        run = (lane == 0 ? 0.0f : run) + __uint_as_float(d[c >> 5][c & 31]);
                        if (lane == 31) sums[c] = run;
                    }
                    sums[lane == 31 ? 95 : 94 - lane] = lane == 31 ? 0.0f : run;
                    __syncwarp();
                    const int first = k0 - (q0 + 32 * warp + 31 + sh.q_pos);
#pragma unroll
                    for (int i = 0; i < 3; ++i) {
                        // a bucket is a run of distances: sums within runs, and the last lane of each run adds to its bucket
                        const int at = 32 * i + lane;
                        const int bucket = lut_bucket[a.pad + first + at];
                        float x = sums[at];
#pragma unroll
                        for (int o = 1; o < 32; o <<= 1) {
                            const float y = __shfl_up_sync(0xFFFFFFFFu, x, o);
                            const int other = __shfl_up_sync(0xFFFFFFFFu, bucket, o);
                            if (lane >= o && other == bucket) x += y;
                        }
                        const int next = __shfl_down_sync(0xFFFFFFFFu, bucket, 1);
                        if (lane == 31 || next != bucket) by_bucket[warp * a.bias.buckets + bucket] += x;
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
                by_bucket[warp * a.bias.buckets + lut_bucket[0]] += far_left;
                by_bucket[warp * a.bias.buckets + lut_bucket[2 * a.pad]] += far_right;
            }
            asm volatile("bar.sync 1, 128;" ::: "memory");
            float* out = a.partial + ((size_t)blockIdx.x * gridDim.y + block) * a.bias.buckets;
            for (int i = row; i < a.bias.buckets; i += 128)
                out[i] = (by_bucket[i] + by_bucket[a.bias.buckets + i]) + (by_bucket[2 * a.bias.buckets + i] + by_bucket[3 * a.bias.buckets + i]);
        }
        if (n > 0 && ok) ok = wait_warp(dq_done, (n - 1) & 1, dead, 512);
        if (ok && q0 + 32 * warp < sh.len_q) {
            tc_fence_after();
            // q's place is free: every product has completed.  Without keys nothing has been issued and the copy has landed
#pragma unroll
            for (int c = 0; c < 2 * HALVES; ++c) {
                uint32_t o[32];
                if (n > 0) {
                    tmem_ld32(o, lanes + Plan::dq_col + 32 * c);
                    tmem_wait_ld();
                    tmem_use(o);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = 0;
                }
                uint8_t* line = smem + (c >> 1) * kOwnBytes + row * 128;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        w[e] = pack_bf16(__uint_as_float(o[8 * i + 2 * e]) * sh.scale, __uint_as_float(o[8 * i + 2 * e + 1]) * sh.scale);
                    *reinterpret_cast<uint4*>(line + ((((c & 1) * 4 + i) ^ (row & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                for (int c = 0; c < HALVES; ++c)
                    if (64 * c < sh.dim)
                        tma_store4(&a.dq.map, sq + c * kOwnBytes + warp * 4096, 64 * c, q0 + 32 * warp, h * a.dq.head_mul, b * a.dq.batch_mul);
                tma_store_commit();
                tma_store_wait_read();
            }
        }
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
    int pad;
};

template <int HALVES>
struct DkvPlan {
    static constexpr int stages = HALVES == 1 ? 3 : 2;
    static constexpr bool apart = HALVES == 2;         // P and dS beside S and dP; one block per SM has all 512 columns
    static constexpr int blocks = HALVES == 1 ? 2 : 1;
    static constexpr uint32_t columns = HALVES == 1 ? 256 : 512;
    static constexpr uint32_t s_col = 0, dp_col = 64, dv_col = 128, dk_col = 128 + 64 * HALVES;
    static constexpr uint32_t p_col = apart ? 384 : s_col, ds_col = apart ? 416 : dp_col;
    static constexpr uint32_t own_bytes = HALVES * kOwnBytes, step_bytes = HALVES * kStepBytes;
    static constexpr uint32_t tiles_bytes = 2 * own_bytes + 2 * stages * step_bytes;
    static constexpr uint32_t bars = 6 + 2 * stages;
    static constexpr uint32_t stats_bytes = 2 * 2 * kStep * 4;
};

template <int HALVES>
size_t dkv_smem(int pad, bool bias) {
    return 1024 + DkvPlan<HALVES>::tiles_bytes + 256 + DkvPlan<HALVES>::stats_bytes + (bias ? (2 * pad + 1) * sizeof(float) : 0);
}

template <int HALVES, bool BIAS>
__global__ void __launch_bounds__(kThreads, DkvPlan<HALVES>::blocks) attn_dkv_kernel(const __grid_constant__ DkvArgs a) {
    using Plan = DkvPlan<HALVES>;
    constexpr int ST = Plan::stages;
    extern __shared__ uint8_t raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    const uint32_t base = smem_u32(smem);
    const uint32_t sk = base, sv = sk + Plan::own_bytes, sq = sv + Plan::own_bytes, sdo = sq + ST * Plan::step_bytes;
    const uint32_t bars = base + Plan::tiles_bytes;
    const uint32_t own_full = bars, s_full = bars + 8, s_free = bars + 16, p_ready = bars + 24, acc_done = bars + 32, drained = bars + 40;
    const uint32_t full = bars + 48, empty = full + 8 * ST;
    uint32_t* words = reinterpret_cast<uint32_t*>(smem + Plan::tiles_bytes + 8 * Plan::bars);
    volatile uint32_t* dead = words + 1;
    float* stats = smem_f(smem + Plan::tiles_bytes + 256);     // two buffers of (-lse in base 2)[64], (-delta)[64]
    float* lut = stats + Plan::stats_bytes / 4;

    const Shape& sh = a.shape;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int b = blockIdx.x / sh.heads_kv, hk = blockIdx.x % sh.heads_kv;
    const int k0 = blockIdx.y * kOwn;                          // the first keys see the most queries: they start first

    if (threadIdx.x == 0) {
        bar_init(own_full, 1);
        bar_init(s_full, 1);
        bar_init(s_free, 4);
        bar_init(p_ready, 4);
        bar_init(acc_done, 1);
        bar_init(drained, 1);
        for (int i = 0; i < ST; ++i) {
            bar_init(full + 8 * i, 1);
            bar_init(empty + 8 * i, 1);
        }
        words[1] = 0;
        bar_init_fence();
    }
    if (warp == 5) tmem_alloc(smem_u32(words), Plan::columns);
    if (threadIdx.x == 128) {
        tma_prefetch(&a.q.map);
        tma_prefetch(&a.dout.map);
        tma_prefetch(&a.k.map);
        tma_prefetch(&a.v.map);
        tma_prefetch(&a.dk.map);
        tma_prefetch(&a.dv.map);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = words[0];
    grid_dependency_sync();

    const int len = sh.kv_len ? min(max(sh.kv_len[b], 0), sh.len_kv) : sh.len_kv;
    const int q_tiles = (sh.len_q + kStep - 1) / kStep;
    int q_first = 0;                                           // the first tile with a row that sees one of the keys
    if (sh.causal && k0 > sh.q_pos) q_first = min((k0 - sh.q_pos) / kStep, q_tiles);
    const int per_head = q_tiles - q_first;
    const int n = k0 < len ? per_head * sh.group : 0;

    if (warp == 4) {
        if (lane == 0 && n > 0) {
            bar_expect(own_full, 2 * Plan::own_bytes);
            for (int c = 0; c < HALVES; ++c) {
                tma_load4(sk + c * kOwnBytes, &a.k.map, own_full, 64 * c, k0, hk * a.k.head_mul, b * a.k.batch_mul);
                tma_load4(sv + c * kOwnBytes, &a.v.map, own_full, 64 * c, k0, hk * a.v.head_mul, b * a.v.batch_mul);
            }
            int t = 0, head = hk * sh.group, tile = q_first;
            for (; t < n; ++t) {
                const int st = t % ST;
                if (!wait(empty + 8 * st, ((t / ST) & 1) ^ 1, dead, 1 << 16)) break;
                bar_expect(full + 8 * st, 2 * Plan::step_bytes);
                for (int c = 0; c < HALVES; ++c) {
                    tma_load4(sq + st * Plan::step_bytes + c * kStepBytes, &a.q.map, full + 8 * st, 64 * c, tile * kStep, head * a.q.head_mul, b * a.q.batch_mul);
                    tma_load4(sdo + st * Plan::step_bytes + c * kStepBytes, &a.dout.map, full + 8 * st, 64 * c, tile * kStep, head * a.dout.head_mul, b * a.dout.batch_mul);
                }
                if (++tile == q_tiles) {
                    tile = q_first;
                    ++head;
                }
            }
            drain(own_full, 0);
            for (int i = max(0, t - ST); i < t; ++i) drain(full + 8 * (i % ST), (i / ST) & 1);
        }
    } else if (warp == 5) {
        if (lane == 0 && n > 0) {
            constexpr uint32_t desc_s = mma_desc(kStep, false), desc_acc = mma_desc(64 * HALVES, true);
            const int steps = (sh.dim + 15) / 16;
            auto scores = [&](int t) {
                const int st = t % ST;
                if (!wait(full + 8 * st, (t / ST) & 1, dead, 2 << 16)) return false;
                tc_fence_after();
                for (int i = 0; i < steps; ++i) {
                    const uint32_t own = (i >> 2) * kOwnBytes + (i & 3) * 32, step = st * Plan::step_bytes + (i >> 2) * kStepBytes + (i & 3) * 32;
                    mma_ss(tmem + Plan::s_col, desc_k_major(sk + own), desc_k_major(sq + step), desc_s, i > 0);
                }
                for (int i = 0; i < steps; ++i) {
                    const uint32_t own = (i >> 2) * kOwnBytes + (i & 3) * 32, step = st * Plan::step_bytes + (i >> 2) * kStepBytes + (i & 3) * 32;
                    mma_ss(tmem + Plan::dp_col, desc_k_major(sv + own), desc_k_major(sdo + step), desc_s, i > 0);
                }
                mma_commit(s_full);
                return true;
            };
            bool ok = wait(own_full, 0, dead, 4 << 16) && scores(0);
            for (int t = 0; t < n && ok; ++t) {
                const int st = t % ST;
                if (Plan::apart && t + 1 < n) {
                    ok = wait(s_free, t & 1, dead, 8 << 16) && scores(t + 1);
                    if (!ok) break;
                }
                ok = wait(p_ready, t & 1, dead, 16 << 16);
                if (!ok) break;
                tc_fence_after();
                for (int i = 0; i < kStep / 16; ++i)
                    mma_ts(tmem + Plan::dv_col, tmem + Plan::p_col + 8 * i, desc_n_major(sdo + st * Plan::step_bytes + i * 2048, kStepBytes),
                           desc_acc, t > 0 || i > 0);
                for (int i = 0; i < kStep / 16; ++i)
                    mma_ts(tmem + Plan::dk_col, tmem + Plan::ds_col + 8 * i, desc_n_major(sq + st * Plan::step_bytes + i * 2048, kStepBytes),
                           desc_acc, t > 0 || i > 0);
                mma_commit(empty + 8 * st);
                mma_commit(acc_done);
                if (!Plan::apart && t + 1 < n) ok = wait(acc_done, t & 1, dead, 32 << 16) && scores(t + 1);
            }
            mma_commit(drained);
            drain(drained, 0);
        }
    } else {
        const int row = threadIdx.x;
        const int key = k0 + row;
        const uint32_t lanes = tmem + ((uint32_t)warp << 21);
        int head = hk * sh.group, tile = q_first;
        // thread t < 64 brings lse of the tile's row t, thread 64 + t its delta
        auto stat_of = [&](int head, int tile) {
            const int i = tile * kStep + (row & (kStep - 1));
            if (i >= sh.len_q) return row < kStep ? -INFINITY : 0.0f;
            const size_t at = ((size_t)b * sh.heads_q + head) * sh.len_q + i;
            if (row >= kStep) return -a.delta[at];
            const float lse = a.lse[at];
            return lse == -INFINITY ? -INFINITY : -lse * kLog2e;       // a row without allowed keys: p = 0
        };
        if (BIAS) {
            // the table of the first query head; the others' follow when the walk reaches them
            fill_lut(a.bias, head, lut, a.pad, row, 128);
        }
        // rows inside len_q with nothing allowed: their do and q may hold anything and must not reach a product
        auto is_hole = [&](int tile, float stat) { return row < kStep && tile * kStep + row < sh.len_q && stat == -INFINITY; };
        float stat = n > 0 ? stat_of(head, tile) : 0.0f;
        stats[row] = stat;
        bool hole = is_hole(tile, stat), holes = any_of_128(hole);
        // a wait that runs out does not leave the loop: the other warps still need this one at the barriers
        bool ok = true;
        for (int t = 0; t < n; ++t) {
            const int q0 = tile * kStep;
            int next_tile = tile + 1, next_head = head;
            if (next_tile == q_tiles) {
                next_tile = q_first;
                ++next_head;
            }
            stat = t + 1 < n ? stat_of(next_head, next_tile) : 0.0f;
            const float* nl = stats + (t & 1) * 2 * kStep;
            const float* nd = nl + kStep;
            ok = wait_warp(s_full, t & 1, dead, 64 << 16) && ok;
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
            float mul = sh.scale_log2, add = 0.0f;
            if (BIAS) {
                const Span span = span_of(a.bias, k0 - (q0 + kStep - 1 + sh.q_pos), k0 + kOwn - 1 - (q0 + sh.q_pos));
                if (span == kSpanMixed) {
                    const float* at = lut + a.pad + key - (q0 + sh.q_pos);
#pragma unroll
                    for (int c = 0; c < kStep; ++c) s[c >> 5][c & 31] = __float_as_uint(fmaf(__uint_as_float(s[c >> 5][c & 31]), mul, at[-c]));
                    mul = 1.0f;
                } else {
                    add = lut[span == kSpanFarLeft ? 0 : 2 * a.pad];
                }
            }
            const uint64_t mul2v = pack2(mul, mul), add2v = pack2(add, add);
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float4 l = *reinterpret_cast<const float4*>(nl + 32 * c + 2 * i);
                    const float4 e = *reinterpret_cast<const float4*>(nd + 32 * c + 2 * i);
                    const uint64_t ls[2] = {pack2(l.x, l.y), pack2(l.z, l.w)}, es[2] = {pack2(e.x, e.y), pack2(e.z, e.w)};
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int at = 2 * (i + u);
                        float x, y;
                        unpack2(fma2(pack2(__uint_as_float(s[c][at]), __uint_as_float(s[c][at + 1])), mul2v, add2(ls[u], add2v)), x, y);
                        x = exp2_fast(x);
                        y = exp2_fast(y);
                        s[c][at] = __float_as_uint(x);
                        s[c][at + 1] = __float_as_uint(y);
                        unpack2(mul2(pack2(x, y), add2(pack2(__uint_as_float(d[c][at]), __uint_as_float(d[c][at + 1])), es[u])), x, y);
                        d[c][at] = __float_as_uint(x);
                        d[c][at + 1] = __float_as_uint(y);
                    }
                }
            if (len == 1 || (sh.causal && k0 + kOwn - 1 > q0 + sh.q_pos)) {
                const int first = sh.causal ? key - (q0 + sh.q_pos) : 0;               // rows before it do not see the key
                const int first_d = len == 1 ? kStep : first + (key == 0);             // rows that see it alone: p = 1, ds = 0
#pragma unroll
                for (int c = 0; c < kStep; ++c) {
                    if (c < first) s[c >> 5][c & 31] = 0;
                    if (c < first_d) d[c >> 5][c & 31] = 0;
                }
            }
            if (holes) {
#pragma unroll
                for (int c = 0; c < kStep; ++c)
                    if (nl[c] == -INFINITY) s[c >> 5][c & 31] = d[c >> 5][c & 31] = 0;
                if (hole) {
                    const int st = t % ST;
#pragma unroll
                    for (int c = 0; c < HALVES; ++c)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            *reinterpret_cast<uint4*>(smem + (sq - base) + st * Plan::step_bytes + c * kStepBytes + row * 128 + 16 * i) = make_uint4(0, 0, 0, 0);
                            *reinterpret_cast<uint4*>(smem + (sdo - base) + st * Plan::step_bytes + c * kStepBytes + row * 128 + 16 * i) = make_uint4(0, 0, 0, 0);
                        }
                }
                fence_async_smem();
            }
            if (t > 0 && Plan::apart) {                        // P and dS of the last tile have been used
                ok = wait_warp(acc_done, (t - 1) & 1, dead, 128 << 16) && ok;
                tc_fence_after();
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = pack_bf16(__uint_as_float(s[c][2 * i]), __uint_as_float(s[c][2 * i + 1]));
                tmem_st16(lanes + Plan::p_col + 16 * c, w);
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = pack_bf16(__uint_as_float(d[c][2 * i]), __uint_as_float(d[c][2 * i + 1]));
                tmem_st16(lanes + Plan::ds_col + 16 * c, w);
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(p_ready);
            stats[((t + 1) & 1) * 2 * kStep + row] = stat;
            hole = is_hole(next_tile, stat);
            holes = any_of_128(hole);
            if (BIAS && next_head != head && t + 1 < n) {      // everyone is done with the last head's table
                fill_lut(a.bias, next_head, lut, a.pad, row, 128);
                asm volatile("bar.sync 1, 128;" ::: "memory");
            }
            tile = next_tile;
            head = next_head;
        }
        if (n > 0 && ok) ok = wait_warp(acc_done, (n - 1) & 1, dead, 256 << 16);
        if (ok && k0 + 32 * warp < sh.len_kv) {
            tc_fence_after();
            // k's and v's places are free: every product has completed.  Keys behind the sequence's end get zeros
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                const float scale = side == 0 ? sh.scale : 1.0f;
#pragma unroll
                for (int c = 0; c < 2 * HALVES; ++c) {
                    uint32_t o[32];
                    if (n > 0) {
                        tmem_ld32(o, lanes + (side == 0 ? Plan::dk_col : Plan::dv_col) + 32 * c);
                        tmem_wait_ld();
                        tmem_use(o);
                    }
                    if (n == 0 || key >= len) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = 0;
                    }
                    uint8_t* line = smem + side * Plan::own_bytes + (c >> 1) * kOwnBytes + row * 128;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            w[e] = pack_bf16(__uint_as_float(o[8 * i + 2 * e]) * scale, __uint_as_float(o[8 * i + 2 * e + 1]) * scale);
                        *reinterpret_cast<uint4*>(line + ((((c & 1) * 4 + i) ^ (row & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                for (int c = 0; c < HALVES; ++c)
                    if (64 * c < sh.dim) {
                        tma_store4(&a.dk.map, sk + c * kOwnBytes + warp * 4096, 64 * c, k0 + 32 * warp, hk * a.dk.head_mul, b * a.dk.batch_mul);
                        tma_store4(&a.dv.map, sv + c * kOwnBytes + warp * 4096, 64 * c, k0 + 32 * warp, hk * a.dv.head_mul, b * a.dv.batch_mul);
                    }
                tma_store_commit();
                tma_store_wait_read();
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 5) {
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
int launch(K kernel, dim3 grid, size_t smem, const A& a, cudaStream_t s) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return ALSGD_E_CUDA;
    return launch_dependent(kernel, grid, dim3(kThreads), smem, s, a) == cudaSuccess ? ALSGD_OK : ALSGD_E_CUDA;
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
    auto operand = [&](const alsgd_attn_tensor* t, bool query, uint32_t rows, Operand* out) {
        const bool swap = (query ? d.len_q : d.len_kv) == 0;
        const bool as_query = query != swap;
        return make_operand(swap ? (query ? *k : *q) : *t, d.batch, as_query ? d.len_q : d.len_kv, as_query ? d.heads_q : d.heads_kv, d.dim, rows, out);
    };
    if (d.len_q) {
        DqArgs a;
        a.shape = make_shape(d, kv_len);
        make_bias(d, table, &a.bias);
        a.pad = a.bias.far + kOwn + kStep;
        a.lse = lse;
        a.o = static_cast<const uint16_t*>(o->data);
        a.o_batch = d.batch == 1 ? 0 : o->stride_batch;
        a.o_pos = d.len_q == 1 ? 0 : o->stride_pos;
        a.o_head = d.heads_q == 1 ? 0 : o->stride_head;
        a.delta = delta;
        a.partial = partial;
        if ((rc = operand(q, true, kOwn, &a.q)) != ALSGD_OK || (rc = operand(dout, true, kOwn, &a.dout)) != ALSGD_OK ||
            (rc = operand(dq, true, 32, &a.dq)) != ALSGD_OK || (rc = operand(k, false, kStep, &a.k)) != ALSGD_OK ||
            (rc = operand(v, false, kStep, &a.v)) != ALSGD_OK)
            return rc;
        const dim3 grid(d.batch * d.heads_q, blocks);
        if (d.dim <= 64) rc = d.buckets ? launch(attn_dq_kernel<1, true>, grid, dq_smem<1>(a.pad, (int)d.buckets), a, s)
                                        : launch(attn_dq_kernel<1, false>, grid, dq_smem<1>(a.pad, 0), a, s);
        else rc = d.buckets ? launch(attn_dq_kernel<2, true>, grid, dq_smem<2>(a.pad, (int)d.buckets), a, s)
                            : launch(attn_dq_kernel<2, false>, grid, dq_smem<2>(a.pad, 0), a, s);
        if (rc != ALSGD_OK) return rc;
    }
    if (d.len_kv) {
        DkvArgs a;
        a.shape = make_shape(d, kv_len);
        make_bias(d, table, &a.bias);
        a.pad = a.bias.far + kOwn + kStep;
        a.lse = lse;
        a.delta = delta;
        if ((rc = operand(q, true, kStep, &a.q)) != ALSGD_OK || (rc = operand(dout, true, kStep, &a.dout)) != ALSGD_OK ||
            (rc = operand(k, false, kOwn, &a.k)) != ALSGD_OK || (rc = operand(v, false, kOwn, &a.v)) != ALSGD_OK ||
            (rc = operand(dk, false, 32, &a.dk)) != ALSGD_OK || (rc = operand(dv, false, 32, &a.dv)) != ALSGD_OK)
            return rc;
        const dim3 grid(d.batch * d.heads_kv, (d.len_kv + kOwn - 1) / kOwn);
        if (d.dim <= 64) rc = d.buckets ? launch(attn_dkv_kernel<1, true>, grid, dkv_smem<1>(a.pad, true), a, s)
                                        : launch(attn_dkv_kernel<1, false>, grid, dkv_smem<1>(a.pad, false), a, s);
        else rc = d.buckets ? launch(attn_dkv_kernel<2, true>, grid, dkv_smem<2>(a.pad, true), a, s)
                            : launch(attn_dkv_kernel<2, false>, grid, dkv_smem<2>(a.pad, false), a, s);
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
