// alsgd_attn_fwd: attention with a learned relative position bias.
//
//   x_ij = scale q_i.k_j + T[bucket(j - i)]  over the allowed j,   lse_i = log sum_j e^x_ij,   o_i = sum_j e^(x_ij - lse_i) v_j
//
// A work item is 128 query rows of one head; the resident blocks walk the items, those with the most keys first.  Keys come
// in tiles; a row's running maximum and sum are kept by one thread (the row's lane of tensor memory), so a tile is read
// once and nothing of size len_q x len_kv exists.
//   warps 0-3  softmax: scores from tensor memory, maximum, e^x, sum; probabilities (bf16) back to tensor memory, over the
//              scores they come from
//   warp 4     copies q, k and v tiles through tensor maps and issues the products  S = q k^T  (operands in shared memory)
//              and  O += P v  (P in tensor memory)
// Within a block a tile's steps follow one another: S, softmax, O.  What fills the machine is other blocks: with heads of
// up to 64, tiles of 64 keys take 128 columns of tensor memory and 52 KB, so four blocks share an SM and one's products,
// copies and waits run under the others' exponentials.  Wider heads take tiles of 128 keys, two blocks per SM.
//
// Exponents are taken in base 2 relative to a reference that follows the running maximum only when that has grown by
// more than 8: the sums then hold values up to 2^8, which binary32 and bf16 hold as well as values up to 1, and O in
// tensor memory is rescaled a few times per row instead of once per tile.  Scores, maximum, sum and O are binary32;
// the probabilities are rounded to bf16 for the second product (the operand type of v), the sum uses them unrounded.
#include "alsgd_attn.cuh"

using namespace alsgd_attn;
using namespace alsgd_ops;
using namespace alsgd_tc;

namespace {

constexpr int kRows = 128;              // query rows of an item
constexpr int kSoftmax = 128;           // threads
constexpr int kThreads = kSoftmax + 32;
constexpr int kAll = 1;                 // named barrier of the softmax threads
constexpr int kPolyOf4 = 0;             // of four pairs of exponentials, how many take the polynomial
constexpr float kRescaleAt = 8.0f;
constexpr uint32_t kRowsBytes = kRows * 128;   // 64 bf16 of each row

struct FwdArgs {
    Operand q, k, v, o;
    Shape shape;
    Bias bias;
    float* lse;
    int pad;                            // reach of the bias table by distance
    int row_blocks, items, keys;
};

// HALVES: 64-column halves of the head dimension (1 up to 64, 2 up to 128).
template <int HALVES>
struct FwdPlan {
    static constexpr int keys = HALVES == 1 ? 64 : 128, blocks = HALVES == 1 ? 4 : 2, stages = HALVES == 1 ? 2 : 1;
    static constexpr uint32_t columns = HALVES == 1 ? 128 : 256, s_col = 0, p_col = 0, o_col = keys;
    static constexpr uint32_t half_bytes = keys * 128;         // 64 columns of a k or v tile
    static constexpr uint32_t q_bytes = HALVES * kRowsBytes, kv_bytes = HALVES * half_bytes;
    static constexpr uint32_t tiles_bytes = q_bytes + 2 * stages * kv_bytes;
    static constexpr uint32_t bars = 6 + 2 * stages;
    static constexpr uint32_t fixed_bytes = tiles_bytes + 128;
};

template <int HALVES>
size_t fwd_smem(int pad, bool bias) {
    return 1024 + FwdPlan<HALVES>::fixed_bytes + (bias ? (2 * pad + 1) * (sizeof(float) + 1) : 0);
}

struct Item {
    int b, h, q0, len, keys, n;        // sequence, head, first row, valid keys, keys any row sees, tiles
};

__device__ __forceinline__ Item item_at(const FwdArgs& a, int i) {
    const Shape& sh = a.shape;
    const int bh = sh.batch * sh.heads_q;
    Item t;
    t.q0 = (a.row_blocks - 1 - i / bh) * kRows;
    t.b = i % bh / sh.heads_q;
    t.h = i % bh % sh.heads_q;
    t.len = sh.kv_len ? min(max(sh.kv_len[t.b], 0), sh.len_kv) : sh.len_kv;
    t.keys = t.len;
    if (sh.causal) t.keys = min(t.keys, min(t.q0 + kRows, sh.len_q) + sh.q_pos);
    t.n = t.keys > 0 ? (t.keys + a.keys - 1) / a.keys : 0;
    return t;
}

template <int HALVES, bool BIAS>
__global__ void __launch_bounds__(kThreads, FwdPlan<HALVES>::blocks) attn_fwd_kernel(const __grid_constant__ FwdArgs a) {
    using Plan = FwdPlan<HALVES>;
    constexpr int ST = Plan::stages, KEYS = Plan::keys;
    extern __shared__ uint8_t raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    const uint32_t base = smem_u32(smem);
    const uint32_t sq = base, sk = sq + Plan::q_bytes, sv = sk + ST * Plan::kv_bytes;
    const uint32_t bars = base + Plan::tiles_bytes;
    const uint32_t q_full = bars, s_full = bars + 8, p_ready = bars + 16, pv_done = bars + 24, o_free = bars + 32, drained = bars + 40;
    const uint32_t k_full = bars + 48, v_full = k_full + 8 * ST;
    uint32_t* words = reinterpret_cast<uint32_t*>(smem + Plan::tiles_bytes + 8 * Plan::bars);
    volatile uint32_t* dead = words + 1;
    float* lut = reinterpret_cast<float*>(smem + Plan::fixed_bytes);
    uint8_t* lut_bucket = reinterpret_cast<uint8_t*>(lut + 2 * a.pad + 1);

    const Shape& sh = a.shape;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        bar_init(q_full, 1);
        bar_init(s_full, 1);
        bar_init(p_ready, 4);
        bar_init(pv_done, 1);
        bar_init(o_free, 4);
        bar_init(drained, 1);
        for (int i = 0; i < ST; ++i) {
            bar_init(k_full + 8 * i, 1);
            bar_init(v_full + 8 * i, 1);
        }
        words[1] = 0;
        bar_init_fence();
    }
    if (warp == 4) {
        tmem_alloc(smem_u32(words), Plan::columns);
        if (lane == 0) {
            tma_prefetch(&a.q.map);
            tma_prefetch(&a.k.map);
            tma_prefetch(&a.v.map);
        }
    } else if (BIAS) {
        fill_buckets(a.bias, lut_bucket, a.pad, threadIdx.x, kSoftmax);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = words[0];
    grid_dependency_sync();

    if (warp == 4) {
        // The warp walks together and one lane issues: what a product is given stays the same for all lanes.
        constexpr uint32_t desc_s = mma_desc(KEYS, false), desc_o = mma_desc(64 * HALVES, true);
        const bool leader = elect_one();
        const uint64_t q_desc = desc_k_major(sq), k_desc = desc_k_major(sk), v_desc = desc_n_major(sv, Plan::half_bytes);
        auto fetch_q = [&](const Item& t) {
            if (leader) {
                bar_expect(q_full, Plan::q_bytes);
                for (int c = 0; c < HALVES; ++c)
                    tma_load4(sq + c * kRowsBytes, &a.q.map, q_full, 64 * c, t.q0, t.h * a.q.head_mul, t.b * a.q.batch_mul);
            }
        };
        auto fetch = [&](const Operand& x, uint32_t full, uint32_t to, const Item& t, int j, int st) {
            if (leader) {
                bar_expect(full + 8 * st, Plan::kv_bytes);
                for (int c = 0; c < HALVES; ++c)
                    tma_load4(to + st * Plan::kv_bytes + c * Plan::half_bytes, &x.map, full + 8 * st, 64 * c, j * KEYS, t.h / sh.group * x.head_mul, t.b * x.batch_mul);
            }
        };
        Cursor<FwdArgs, Item> at, load;                        // of the products, and of the k and v copies, ST tiles ahead
        at.start(a);
        load = at;
        if (at.more) fetch_q(at.item);
        for (int st = 0; st < ST && load.more; ++st) {
            fetch(a.k, k_full, sk, load.item, load.j, st);
            fetch(a.v, v_full, sv, load.item, load.j, st);
            load.next(a);
        }
        int items = 0;                                         // whose O has been started
        bool v_due = false;                                    // a v copy may start now that the place of the last tile's is free
        while (at.more) {
            const int st = at.tile % ST;
            const uint32_t full_parity = (at.tile / ST) & 1, parity = at.tile & 1;
            if (at.j == 0) wait_warp(q_full, at.ordinal & 1, dead, 1);
            wait_warp(k_full + 8 * st, full_parity, dead, 2);
            tc_fence_after();
            const uint64_t kd = k_desc + st * (Plan::kv_bytes >> 4);
            if (leader) {
#pragma unroll
                for (int i = 0; i < 4 * HALVES; ++i)           // 16 elements of the head each; behind dim they are zeros
                    mma_ss(tmem + Plan::s_col, q_desc + (((i >> 2) * kRowsBytes + (i & 3) * 32) >> 4),
                           kd + (((i >> 2) * Plan::half_bytes + (i & 3) * 32) >> 4), desc_s, i > 0);
                mma_commit(s_full);
            }
            if (v_due) {
                fetch(a.v, v_full, sv, load.item, load.j, load.tile % ST);
                load.next(a);
                v_due = false;
            }
            if (at.j == 0) {                                   // the last item's O has been read
                wait_warp(o_free, (items & 1) ^ 1, dead, 4);
                ++items;
            }
            wait_warp(v_full + 8 * st, full_parity, dead, 8);
            wait_warp(p_ready, parity, dead, 16);
            if (__any_sync(0xFFFFFFFFu, *dead)) break;
            tc_fence_after();
            const int keys = at.item.keys - at.j * KEYS;       // groups of 16 that nobody sees are left out
            const uint64_t vd = v_desc + st * (Plan::kv_bytes >> 4);
            const bool more = at.j > 0;
            if (leader) {
#pragma unroll
                for (int i = 0; i < KEYS / 16; ++i)
                    if (16 * i < keys) mma_ts(tmem + Plan::o_col, tmem + Plan::p_col + i * 8, vd + i * 128, desc_o, more || i > 0);
                mma_commit(pv_done);
            }
            // the scores of this tile have been formed: its k's place is free, and behind the item's last tile q's
            if (load.more) {
                fetch(a.k, k_full, sk, load.item, load.j, st);
                v_due = true;
            }
            at.next(a);
            if (at.more && at.j == 0) fetch_q(at.item);
            wait_warp(pv_done, parity, dead, 32);
        }
        // everything in flight lands before the block may leave, whoever has given up
        if (leader) {
            mma_commit(drained);
            drain(drained, 0);
            if (*dead) {
                drain(q_full, 0);
                drain(q_full, 1);
                for (int i = 0; i < ST; ++i) {
                    drain(k_full + 8 * i, 0);
                    drain(k_full + 8 * i, 1);
                    drain(v_full + 8 * i, 0);
                    drain(v_full + 8 * i, 1);
                }
            }
        }
    } else {
        const int row = threadIdx.x;
        const uint32_t lanes = tmem + ((uint32_t)warp << 21);
        int tile = 0;
        for (int i = blockIdx.x; i < a.items; i += gridDim.x) {
            const Item t = item_at(a, i);
            const bool inside = t.q0 + row < sh.len_q;
            float* lse = a.lse + ((size_t)t.b * sh.heads_q + t.h) * sh.len_q + t.q0 + row;
            if (t.n == 0) {
                if (inside) {
                    zero_row(a.o, sh.dim, t.b, t.h, t.q0 + row);
                    *lse = -INFINITY;
                }
                continue;
            }
            const int pos = t.q0 + row + sh.q_pos;             // the row's position among the keys
            if (BIAS) {
                const int first = t.q0 + sh.q_pos;             // distances from the last row's first key to the first row's last
                sync_threads(kAll, kSoftmax);
                fill_lut(a.bias, t.h, lut_bucket, lut, a.pad, -(first + kRows - 1), sh.causal ? 0 : t.keys - 1 - first, threadIdx.x, kSoftmax);
                sync_threads(kAll, kSoftmax);
            }
            float ref = -INFINITY, sum = 0.0f;
            for (int j = 0; j < t.n; ++j, ++tile) {
                const int k0 = j * KEYS;
                wait_warp(s_full, tile & 1, dead, 64);         // also: O holds the tiles before, P's place is free
                tc_fence_after();
                uint32_t v[KEYS / 32][32];
#pragma unroll
                for (int c = 0; c < KEYS / 32; ++c) tmem_ld32(v[c], lanes + Plan::s_col + 32 * c);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < KEYS / 32; ++c) tmem_use(v[c]);

                // x = v * mul + add, in base 2
                float mul = sh.scale_log2, add = 0.0f;
                if (BIAS) {
                    const Span span = span_of(a.bias, k0 - (t.q0 + kRows - 1 + sh.q_pos), k0 + KEYS - 1 - (t.q0 + sh.q_pos));
                    if (span == kSpanMixed) {
                        const float* at = lut + a.pad + k0 - pos;
#pragma unroll
                        for (int c = 0; c < KEYS; ++c) v[c >> 5][c & 31] = __float_as_uint(fmaf(__uint_as_float(v[c >> 5][c & 31]), mul, at[c]));
                        mul = 1.0f;
                    } else {
                        add = lut[span == kSpanFarLeft ? 0 : 2 * a.pad];
                    }
                }
                if (k0 + KEYS > t.len || (sh.causal && k0 + KEYS - 1 > t.q0 + sh.q_pos)) {
                    const int allowed = (sh.causal ? min(t.len, pos + 1) : t.len) - k0;
#pragma unroll
                    for (int c = 0; c < KEYS; ++c)
                        if (c >= allowed) v[c >> 5][c & 31] = 0xFF800000u;
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < KEYS; c += 2)
                    top[(c >> 1) & 3] = max3(top[(c >> 1) & 3], __uint_as_float(v[c >> 5][c & 31]), __uint_as_float(v[c >> 5][(c & 31) + 1]));
                const float high = fmaf(max3(max3(top[0], top[1], top[2]), top[3], top[3]), mul, add);

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
                for (int c = 0; c < KEYS / 32; ++c) {
                    uint32_t p[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const uint64_t xy = fma2(pack2(__uint_as_float(v[c][2 * e]), __uint_as_float(v[c][2 * e + 1])), mul2v, off2);
                        float x, y;
                        if ((e & 3) < kPolyOf4) {
                            exp2_poly(xy, x, y);
                        } else {
                            unpack2(xy, x, y);
                            x = exp2_fast(x);
                            y = exp2_fast(y);
                        }
                        part[e & 1] = add2(part[e & 1], pack2(x, y));
                        p[e] = pack_bf16(x, y);
                    }
                    tmem_st16(lanes + Plan::p_col + 16 * c, p);
                }
                float s0, s1;
                unpack2(add2(part[0], part[1]), s0, s1);
                sum += s0 + s1;
                if (k0 + KEYS > t.len && t.len < sh.len_kv) {
                    // v rows behind the sequence's end are whatever the caller has there; 0 * NaN must not reach O
                    const int st = tile % ST;
                    wait_warp(v_full + 8 * st, (tile / ST) & 1, dead, 128);
                    if (row < KEYS && k0 + row >= t.len) {
#pragma unroll
                        for (int c = 0; c < HALVES; ++c)
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                *reinterpret_cast<uint4*>(smem + (sv - base) + st * Plan::kv_bytes + c * Plan::half_bytes + row * 128 + 16 * e) = make_uint4(0, 0, 0, 0);
                    }
                    fence_async_smem();
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(p_ready);
            }
            wait_warp(pv_done, (tile - 1) & 1, dead, 256);
            tc_fence_after();
            const bool none = ref == -INFINITY;                // no allowed key
            const float inv = none ? 0.0f : 1.0f / sum + (ref - ref);
            uint32_t o[HALVES * 2][32];
#pragma unroll
            for (int c = 0; c < 2 * HALVES; ++c) tmem_ld32(o[c], lanes + Plan::o_col + 32 * c);
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < 2 * HALVES; ++c) tmem_use(o[c]);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(o_free);
            if (inside) {
#pragma unroll
                for (int c = 0; c < 2 * HALVES; ++c) store_columns(a.o, sh.dim, t.b, t.h, t.q0 + row, 32 * c, o[c], inv);
                *lse = none ? -INFINITY : (ref + log2f(sum)) * kLn2;
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 4) {
        tc_fence_after();
        tmem_free(tmem, Plan::columns);
    }
}

template <int HALVES, bool BIAS>
int launch_fwd(FwdArgs& a, cudaStream_t s) {
    const size_t smem = fwd_smem<HALVES>(a.pad, BIAS);
    if (cudaFuncSetAttribute(attn_fwd_kernel<HALVES, BIAS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return ALSGD_E_CUDA;
    const int wave = blocks_at_once(smem, FwdPlan<HALVES>::blocks);
    return launch_dependent(attn_fwd_kernel<HALVES, BIAS>, dim3(a.items < wave ? a.items : wave), dim3(kThreads), smem, s, a) == cudaSuccess ? ALSGD_OK
                                                                                                                                             : ALSGD_E_CUDA;
}

}  // namespace

extern "C" int alsgd_attn_fwd(const alsgd_attn_desc* desc, const alsgd_attn_tensor* q, const alsgd_attn_tensor* k, const alsgd_attn_tensor* v,
                              const void* table, const int32_t* kv_len, const alsgd_attn_tensor* o, float* lse, void* stream) {
    int rc = check_desc(desc);
    if (rc != ALSGD_OK) return rc;
    const alsgd_attn_desc& d = *desc;
    if ((d.buckets != 0) != (table != nullptr) || reinterpret_cast<uintptr_t>(table) % 4 || reinterpret_cast<uintptr_t>(kv_len) % 4) return ALSGD_E_ARG;
    if (d.len_q && (!lse || reinterpret_cast<uintptr_t>(lse) % 4)) return ALSGD_E_ARG;
    if ((rc = check_tensor(q, d.batch, d.len_q, d.heads_q, false)) != ALSGD_OK) return rc;
    if ((rc = check_tensor(k, d.batch, d.len_kv, d.heads_kv, false)) != ALSGD_OK) return rc;
    if ((rc = check_tensor(v, d.batch, d.len_kv, d.heads_kv, false)) != ALSGD_OK) return rc;
    if ((rc = check_tensor(o, d.batch, d.len_q, d.heads_q, true)) != ALSGD_OK) return rc;
    if (d.len_q == 0) return ALSGD_OK;

    UseDevice use(d.device);
    if (!use.ok) return ALSGD_E_CUDA;
    FwdArgs a;
    a.shape = make_shape(d, kv_len);
    make_bias(d, table, &a.bias);
    a.lse = lse;
    a.keys = d.dim <= 64 ? FwdPlan<1>::keys : FwdPlan<2>::keys;
    a.pad = a.bias.far + kRows + a.keys;
    a.row_blocks = (int)((d.len_q + kRows - 1) / kRows);
    const uint64_t items = (uint64_t)d.batch * d.heads_q * a.row_blocks;
    if (items > 0x7FFFFFFFull - 2 * kSMs) return ALSGD_E_RANGE;
    a.items = (int)items;
    if ((rc = make_operand(*q, d.batch, d.len_q, d.heads_q, d.dim, kRows, 64, &a.q)) != ALSGD_OK) return rc;
    if ((rc = make_operand(*o, d.batch, d.len_q, d.heads_q, d.dim, 32, 64, &a.o)) != ALSGD_OK) return rc;
    // without keys the kernel touches neither map
    if ((rc = make_operand(d.len_kv ? *k : *q, d.batch, d.len_kv ? d.len_kv : d.len_q, d.len_kv ? d.heads_kv : d.heads_q, d.dim, a.keys, 64, &a.k)) != ALSGD_OK) return rc;
    if ((rc = make_operand(d.len_kv ? *v : *q, d.batch, d.len_kv ? d.len_kv : d.len_q, d.len_kv ? d.heads_kv : d.heads_q, d.dim, a.keys, 64, &a.v)) != ALSGD_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (d.dim <= 64) return d.buckets ? launch_fwd<1, true>(a, s) : launch_fwd<1, false>(a, s);
    return d.buckets ? launch_fwd<2, true>(a, s) : launch_fwd<2, false>(a, s);
}

extern "C" int alsgd_attn_status(int32_t device, uint32_t* waits_out) {
    if (!waits_out) return ALSGD_E_ARG;
    if (device < 0 || device >= kMaxDevices) return ALSGD_E_RANGE;
    UseDevice use(device);
    if (!use.ok) return ALSGD_E_CUDA;
    unsigned fwd = 0, bwd = 0;
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
