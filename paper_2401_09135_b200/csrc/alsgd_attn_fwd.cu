// alsgd_attn_fwd: attention with a learned relative position bias.
//
//   x_ij = scale q_i.k_j + T[bucket(j - i)]  over the allowed j,   lse_i = log sum_j e^x_ij,   o_i = sum_j e^(x_ij - lse_i) v_j
//
// One block per 128 query rows of one head.  Keys come in tiles of 128; a row's running maximum and sum are kept by
// one thread (the row's lane of tensor memory), so a tile is read once and nothing of size len_q x len_kv exists.
//   warps 0-3  softmax: scores from tensor memory, maximum, e^x, sum; probabilities (bf16) back to tensor memory
//   warp 4     copies q, then k and v tiles, through tensor maps
//   warp 5     issues the products  S = q k^T  (operands in shared memory)  and  O += P v  (P in tensor memory)
// Two blocks share an SM (256 tensor memory columns and about 100 KB each): one block's products and its start and
// end run under the other's exponentials.
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

constexpr int kRows = 128;              // query rows of a block
constexpr int kKeys = 128;              // keys of a tile
constexpr int kThreads = 192;
constexpr float kRescaleAt = 8.0f;
constexpr uint32_t kTileBytes = 128 * 128;     // 128 rows of 64 bf16

struct FwdArgs {
    Operand q, k, v, o;
    Shape shape;
    Bias bias;
    float* lse;
    int pad;                            // reach of the bias table by distance
};

// HALVES: 64-column halves of the head dimension (1 up to 64, 2 up to 128).  With one half there is room to keep P beside S,
// so the next tile's scores are computed while this tile's exponentials are; with two P takes S's place.
template <int HALVES>
struct FwdPlan {
    static constexpr int stages = HALVES == 1 ? 2 : 1;
    static constexpr bool p_apart = HALVES == 1;
    static constexpr uint32_t columns = 256;
    static constexpr uint32_t s_col = 0, p_col = p_apart ? 128 : 0, o_col = p_apart ? 192 : 128;
    static constexpr uint32_t q_bytes = HALVES * kTileBytes, kv_bytes = HALVES * kTileBytes;
    static constexpr uint32_t tiles_bytes = q_bytes + 2 * stages * kv_bytes;
    static constexpr uint32_t bars = 6 + 4 * stages;
};

template <int HALVES>
size_t fwd_smem(int pad, bool bias) {
    return 1024 + FwdPlan<HALVES>::tiles_bytes + 256 + (bias ? (2 * pad + 1) * sizeof(float) : 0);
}

template <int HALVES, bool BIAS>
__global__ void __launch_bounds__(kThreads, 2) attn_fwd_kernel(const __grid_constant__ FwdArgs a) {
    using Plan = FwdPlan<HALVES>;
    constexpr int ST = Plan::stages;
    extern __shared__ uint8_t raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    const uint32_t base = smem_u32(smem);
    const uint32_t sq = base, sk = sq + Plan::q_bytes, sv = sk + ST * Plan::kv_bytes;
    const uint32_t bars = base + Plan::tiles_bytes;
    const uint32_t q_full = bars, s_full = bars + 8, s_free = bars + 16, p_ready = bars + 24, pv_done = bars + 32, drained = bars + 40;
    const uint32_t k_full = bars + 48, k_empty = k_full + 8 * ST, v_full = k_empty + 8 * ST, v_empty = v_full + 8 * ST;
    uint32_t* words = reinterpret_cast<uint32_t*>(smem + Plan::tiles_bytes + 8 * Plan::bars);
    volatile uint32_t* dead = words + 1;
    float* lut = reinterpret_cast<float*>(smem + Plan::tiles_bytes + 256);

    const Shape& sh = a.shape;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int b = blockIdx.x / sh.heads_q, h = blockIdx.x % sh.heads_q, hk = h / sh.group;
    const int q0 = (gridDim.y - 1 - blockIdx.y) * kRows;       // the longest rows of a causal mask start first

    if (threadIdx.x == 0) {
        bar_init(q_full, 1);
        bar_init(s_full, 1);
        bar_init(s_free, 4);
        bar_init(p_ready, 4);
        bar_init(pv_done, 1);
        bar_init(drained, 1);
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
    if (threadIdx.x == 128) {
        tma_prefetch(&a.q.map);
        tma_prefetch(&a.k.map);
        tma_prefetch(&a.v.map);
        tma_prefetch(&a.o.map);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = words[0];
    grid_dependency_sync();

    const int len = sh.kv_len ? min(max(sh.kv_len[b], 0), sh.len_kv) : sh.len_kv;
    int keys = len;                                            // keys that any row of the block sees
    if (sh.causal) keys = min(keys, min(q0 + kRows, sh.len_q) + sh.q_pos);
    const int n = keys > 0 ? (keys + kKeys - 1) / kKeys : 0;

    if (warp == 4) {
        if (lane == 0 && n > 0) {
            bar_expect(q_full, Plan::q_bytes);
            for (int c = 0; c < HALVES; ++c) tma_load4(sq + c * kTileBytes, &a.q.map, q_full, 64 * c, q0, h * a.q.head_mul, b * a.q.batch_mul);
            int j = 0;
            bool ok = true;
            for (; j < n && ok; ++j) {
                const int st = j % ST;
                const uint32_t free_parity = ((j / ST) & 1) ^ 1;
                ok = wait(k_empty + 8 * st, free_parity, dead, 1);
                if (!ok) break;
                bar_expect(k_full + 8 * st, Plan::kv_bytes);
                for (int c = 0; c < HALVES; ++c)
                    tma_load4(sk + st * Plan::kv_bytes + c * kTileBytes, &a.k.map, k_full + 8 * st, 64 * c, j * kKeys, hk * a.k.head_mul, b * a.k.batch_mul);
                ok = wait(v_empty + 8 * st, free_parity, dead, 2);
                if (!ok) {                                     // this tile's k copy is in flight
                    drain(k_full + 8 * st, (j / ST) & 1);
                    break;
                }
                bar_expect(v_full + 8 * st, Plan::kv_bytes);
                for (int c = 0; c < HALVES; ++c)
                    tma_load4(sv + st * Plan::kv_bytes + c * kTileBytes, &a.v.map, v_full + 8 * st, 64 * c, j * kKeys, hk * a.v.head_mul, b * a.v.batch_mul);
            }
            // every copy has landed before the block may leave, whoever else has given up
            drain(q_full, 0);
            for (int i = max(0, j - ST); i < j; ++i) {
                drain(k_full + 8 * (i % ST), (i / ST) & 1);
                drain(v_full + 8 * (i % ST), (i / ST) & 1);
            }
        }
    } else if (warp == 5) {
        if (lane == 0 && n > 0) {
            constexpr uint32_t desc_s = mma_desc(kKeys, false), desc_o = mma_desc(64 * HALVES, true);
            const int steps = (sh.dim + 15) / 16;
            auto scores = [&](int j) {
                const int st = j % ST;
                if (!wait(k_full + 8 * st, (j / ST) & 1, dead, 4)) return false;
                tc_fence_after();
                for (int i = 0; i < steps; ++i) {
                    const uint32_t at = (i >> 2) * kTileBytes + (i & 3) * 32;
                    mma_ss(tmem + Plan::s_col, desc_k_major(sq + at), desc_k_major(sk + st * Plan::kv_bytes + at), desc_s, i > 0);
                }
                mma_commit(k_empty + 8 * st);
                mma_commit(s_full);
                return true;
            };
            bool ok = wait(q_full, 0, dead, 8) && scores(0);
            for (int j = 0; j < n && ok; ++j) {
                const int st = j % ST;
                if (Plan::p_apart && j + 1 < n) {
                    ok = wait(s_free, j & 1, dead, 16) && scores(j + 1);
                    if (!ok) break;
                }
                ok = wait(p_ready, j & 1, dead, 32) && wait(v_full + 8 * st, (j / ST) & 1, dead, 64);
                if (!ok) break;
                tc_fence_after();
                const int k_steps = min(kKeys, keys - j * kKeys + 15) / 16;      // 16 keys each; those nobody sees are left out
                for (int i = 0; i < k_steps; ++i)
                    mma_ts(tmem + Plan::o_col, tmem + Plan::p_col + 8 * i, desc_n_major(sv + st * Plan::kv_bytes + i * 2048, kTileBytes),
                           desc_o, j > 0 || i > 0);
                mma_commit(v_empty + 8 * st);
                mma_commit(pv_done);
                if (!Plan::p_apart && j + 1 < n) ok = wait(pv_done, j & 1, dead, 128) && scores(j + 1);
            }
            mma_commit(drained);
            drain(drained, 0);
        }
    } else {
        const int row = threadIdx.x;
        const int pos = q0 + row + sh.q_pos;                   // the row's position among the keys
        const uint32_t lanes = tmem + ((uint32_t)warp << 21);
        if (BIAS) {
            fill_lut(a.bias, h, lut, a.pad, row, 128);
            asm volatile("bar.sync 1, 128;" ::: "memory");
        }
        float ref = -INFINITY, sum = 0.0f;
        bool ok = true;
        for (int j = 0; j < n; ++j) {
            const int k0 = j * kKeys;
            ok = wait_warp(s_full, j & 1, dead, 256);
            if (!ok) break;
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
            float mul = sh.scale_log2, add = 0.0f;
            if (BIAS) {
                const Span span = span_of(a.bias, k0 - (q0 + kRows - 1 + sh.q_pos), k0 + kKeys - 1 - (q0 + sh.q_pos));
                if (span == kSpanMixed) {
                    const float* at = lut + a.pad + k0 - pos;
#pragma unroll
                    for (int c = 0; c < 128; ++c) v[c >> 5][c & 31] = __float_as_uint(fmaf(__uint_as_float(v[c >> 5][c & 31]), mul, at[c]));
                    mul = 1.0f;
                } else {
                    add = lut[span == kSpanFarLeft ? 0 : 2 * a.pad];
                }
            }
            if (k0 + kKeys > len || (sh.causal && k0 + kKeys - 1 > q0 + sh.q_pos)) {
                const int allowed = (sh.causal ? min(len, pos + 1) : len) - k0;
#pragma unroll
                for (int c = 0; c < 128; ++c)
                    if (c >= allowed) v[c >> 5][c & 31] = 0xFF800000u;
            }
            float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < 128; ++c) top[c & 3] = fmaxf(top[c & 3], __uint_as_float(v[c >> 5][c & 31]));
            const float high = fmaf(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), mul, add);

            if (j > 0) {                                       // O and P of the last tile are free
                ok = wait_warp(pv_done, (j - 1) & 1, dead, 512);
                if (!ok) break;
                tc_fence_after();
            }
            const bool grown = high > ref + kRescaleAt || (ref == -INFINITY && high > -INFINITY);
            if (__any_sync(0xFFFFFFFFu, grown)) {
                const float next = grown ? high : ref;
                const float factor = next == -INFINITY ? 1.0f : exp2_fast(ref - next);
                ref = next;
                sum *= factor;
                if (j > 0) {
#pragma unroll
                    for (int c = 0; c < 2 * HALVES; ++c) {
                        uint32_t o[32];
                        tmem_ld32(o, lanes + Plan::o_col + 32 * c);
                        tmem_wait_ld();
                        tmem_use(o);
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * factor);
                        tmem_st32(lanes + Plan::o_col + 32 * c, o);
                    }
                }
            }
            const float off = add - (ref == -INFINITY ? 0.0f : ref);
            const uint64_t mul2v = pack2(mul, mul), off2 = pack2(off, off);
            uint64_t part[2] = {0, 0};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t p[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float x, y;
                    unpack2(fma2(pack2(__uint_as_float(v[c][2 * i]), __uint_as_float(v[c][2 * i + 1])), mul2v, off2), x, y);
                    x = exp2_fast(x);
                    y = exp2_fast(y);
                    part[i & 1] = add2(part[i & 1], pack2(x, y));
                    p[i] = pack_bf16(x, y);
                }
                tmem_st16(lanes + Plan::p_col + 16 * c, p);
            }
            float s0, s1;
            unpack2(add2(part[0], part[1]), s0, s1);
            sum += s0 + s1;
            if (k0 + kKeys > len && len < sh.len_kv) {
                // v rows behind the sequence's end are whatever the caller has there; 0 * NaN must not reach O
                const int st = j % ST;
                ok = wait_warp(v_full + 8 * st, (j / ST) & 1, dead, 1024);
                if (!ok) break;
                if (k0 + row >= len) {
#pragma unroll
                    for (int c = 0; c < HALVES; ++c)
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            *reinterpret_cast<uint4*>(smem + (sv - base) + st * Plan::kv_bytes + c * kTileBytes + row * 128 + 16 * i) = make_uint4(0, 0, 0, 0);
                }
                fence_async_smem();
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(p_ready);
        }
        if (n > 0 && ok) ok = wait_warp(pv_done, (n - 1) & 1, dead, 2048);
        if (ok && q0 + 32 * warp < sh.len_q) {
            tc_fence_after();
            const float inv = sum > 0.0f ? 1.0f / sum : (sum == 0.0f ? 0.0f : sum);      // a NaN stays one
            // q's place in shared memory is free (its last product has completed): the rows go out through it
#pragma unroll
            for (int c = 0; c < 2 * HALVES; ++c) {
                uint32_t o[32];
                if (n > 0) {
                    tmem_ld32(o, lanes + Plan::o_col + 32 * c);
                    tmem_wait_ld();
                    tmem_use(o);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = 0;
                }
                uint8_t* line = smem + (c >> 1) * kTileBytes + row * 128;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        w[e] = pack_bf16(__uint_as_float(o[8 * i + 2 * e]) * inv, __uint_as_float(o[8 * i + 2 * e + 1]) * inv);
                    *reinterpret_cast<uint4*>(line + ((((c & 1) * 4 + i) ^ (row & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                for (int c = 0; c < HALVES; ++c)
                    if (64 * c < sh.dim)
                        tma_store4(&a.o.map, sq + c * kTileBytes + warp * 4096, 64 * c, q0 + 32 * warp, h * a.o.head_mul, b * a.o.batch_mul);
                tma_store_commit();
            }
            if (q0 + row < sh.len_q)
                a.lse[((size_t)b * sh.heads_q + h) * sh.len_q + q0 + row] = sum == 0.0f ? -INFINITY : (ref + log2f(sum)) * kLn2;
            if (lane == 0) tma_store_wait_read();
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

template <int HALVES, bool BIAS>
int launch_fwd(const FwdArgs& a, cudaStream_t s) {
    const size_t smem = fwd_smem<HALVES>(a.pad, BIAS);
    if (cudaFuncSetAttribute(attn_fwd_kernel<HALVES, BIAS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return ALSGD_E_CUDA;
    const dim3 grid(a.shape.batch * a.shape.heads_q, (a.shape.len_q + kRows - 1) / kRows);
    return launch_dependent(attn_fwd_kernel<HALVES, BIAS>, grid, dim3(kThreads), smem, s, a) == cudaSuccess ? ALSGD_OK : ALSGD_E_CUDA;
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
    a.pad = a.bias.far + kRows + kKeys;
    if ((rc = make_operand(*q, d.batch, d.len_q, d.heads_q, d.dim, kRows, &a.q)) != ALSGD_OK) return rc;
    if ((rc = make_operand(*o, d.batch, d.len_q, d.heads_q, d.dim, 32, &a.o)) != ALSGD_OK) return rc;
    // without keys the kernel touches neither map
    if ((rc = make_operand(d.len_kv ? *k : *q, d.batch, d.len_kv ? d.len_kv : d.len_q, d.len_kv ? d.heads_kv : d.heads_q, d.dim, kKeys, &a.k)) != ALSGD_OK) return rc;
    if ((rc = make_operand(d.len_kv ? *v : *q, d.batch, d.len_kv ? d.len_kv : d.len_q, d.len_kv ? d.heads_kv : d.heads_q, d.dim, kKeys, &a.v)) != ALSGD_OK) return rc;
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
