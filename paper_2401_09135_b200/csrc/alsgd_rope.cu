// Rotary positions: every head of q and k turned, pair by pair, by an angle that grows with the token's position.
//
//     (a, b) -> amplitude (a cos t - b sin t, a sin t + b cos t),   t = position * f_i,   f_i = base^(-2i / rot), scaled
//
// Bytes bound it: q and k are read once and written once.  A block takes a few tokens, whose cosines and sines all heads
// share: they are formed once, in binary64 up to the reduced angle (a position of 2^20 times a frequency has no fraction
// worth using in binary32), while the block's first loads are on their way.  A thread holds both elements of every pair that
// it turns, so results may overwrite operands.
#include "../../include/alsgd.h"
#include "alsgd_ops.cuh"

#include <cfloat>
#include <cmath>
#include <cstring>

namespace {

using namespace alsgd_ops;

constexpr int kThreads = 256;
constexpr int kMaxDim = 256;
// Units of two groups that a thread has in flight, with five blocks per SM: 21.6 us at 64 x 256 tokens and 32 heads of 64, 28.8 at
// 4 x 4099 tokens and 20 heads of 128, of calls captured in a loop over one set of tensors, part of which stays in the L2; 24.0 to 24.6
// and 30.6 to 31.3 (5.5 and 5.4 TB/s) of calls on tensors that change.  Instructions count here as much as memory (70 % of the issue
// slots): with four blocks, or six and spilled registers, both were 5 to 15 % slower, and with four units.
constexpr int kUnits = 2;
constexpr int kMaxTokens = 16;         // of a block

// From one sequence, position, head to the next.
struct Steps {
    int64_t batch;
    int pos, head;
};

// An operand and its result.
struct Side {
    const void* in;
    void* out;
    Steps from, to;
};

struct RopeArgs {
    Side side[2];                      // q, k
    const void* positions;             // may be null
    int wide_positions;                // of 64 bits
    int64_t pos0;
    int len, heads_q, heads, dim, rot, interleaved, tokens, per_block;
    int units, turned, angles;         // of a head; turned: units that begin the two halves
    int angle_step;                    // angles, to an even number
    Divide by_token, by_units, by_len, by_angles;                  // units of a token, of a head; tokens of a sequence; angles
    float amplitude, turn;             // turn: 1, or -1 for the inverse
    double turns[kMaxDim / 2];         // f_i / (2 pi)
};

// N elements in a row, as they lie and as 32-bit floats.
template <typename T, int N>
struct Group {
    static constexpr int kBytes = N * sizeof(T);
    uint32_t w[(kBytes + 3) / 4];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (kBytes >= 16) {
#pragma unroll
            for (int i = 0; i < kBytes / 16; ++i) {
                const uint4 x = reinterpret_cast<const uint4*>(p)[i];
                w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
            }
        } else if constexpr (kBytes == 8) {
            const uint2 x = *reinterpret_cast<const uint2*>(p);
            w[0] = x.x, w[1] = x.y;
        } else if constexpr (kBytes == 4) {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        } else {
            w[0] = *reinterpret_cast<const uint16_t*>(p);
        }
    }
    __device__ __forceinline__ void widen(float (&v)[N]) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(w[i]);
            else v[i] = i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
        }
    }
    __device__ __forceinline__ static void store(T* p, const float (&v)[N]) {
        Group g;
#pragma unroll
        for (int i = 0; i < (kBytes + 3) / 4; ++i) {
            if constexpr (sizeof(T) == 4) g.w[i] = __float_as_uint(v[i]);
            else if constexpr (N > 1) g.w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
            else g.w[i] = pack_bf16(v[0], 0.0f);
        }
        if constexpr (kBytes >= 16) {
#pragma unroll
            for (int i = 0; i < kBytes / 16; ++i) reinterpret_cast<uint4*>(p)[i] = make_uint4(g.w[4 * i], g.w[4 * i + 1], g.w[4 * i + 2], g.w[4 * i + 3]);
        } else if constexpr (kBytes == 8) {
            *reinterpret_cast<uint2*>(p) = make_uint2(g.w[0], g.w[1]);
        } else if constexpr (kBytes == 4) {
            *reinterpret_cast<uint32_t*>(p) = g.w[0];
        } else {
            *reinterpret_cast<uint16_t*>(p) = (uint16_t)g.w[0];
        }
    }
};

__device__ __forceinline__ void turn_pair(float c, float s, float& a, float& b) {
    const float x = a, y = b;
    a = fmaf(x, c, -(y * s));
    b = fmaf(x, s, y * c);
}

// Cosine and sine (times the amplitude) of the block's tokens, [token][angle].  A token's begin on 16 bytes.
__device__ __forceinline__ void fill_angles(const RopeArgs& a, float2* table, int token0, int tokens) {
    for (int i = threadIdx.x; i < tokens * a.angles; i += kThreads) {
        const int t = a.by_angles(i), n = i - t * a.angles, token = token0 + t;
        int64_t pos;
        if (!a.positions) pos = a.pos0 + token - a.by_len(token) * a.len;
        else pos = a.wide_positions ? static_cast<const int64_t*>(a.positions)[token] : static_cast<const int32_t*>(a.positions)[token];
        const double turns = (double)pos * a.turns[n];
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        table[t * a.angle_step + n] = make_float2(c * a.amplitude, s * (a.amplitude * a.turn));
    }
}

// Where a unit's two groups of N elements start; one that starts at dim or beyond does not exist.
//   half: a group of either half of the turned part, then of either half of the rest.  interleaved: of either half of the
//   head.  Neighbouring threads take neighbouring groups: 32 bytes a thread in a row took 39 us in place of 35.5 (4 x 4099
//   tokens, 20 heads of 128, half of each turned).
struct Unit {
    int batch, pos, head;
    int at[2];
    int token, n;                      // token of the block, unit of the head
    int side;
    __device__ __forceinline__ int64_t offset(const Steps& s) const { return batch * s.batch + (int64_t)pos * s.pos + (int64_t)head * s.head; }
};
// (Plain divisions and remainders here bounded the kernel by its instructions: 33 us at 64 x 256 tokens against 26 with
// reciprocals.)
template <int N>
__device__ __forceinline__ Unit unit_of(const RopeArgs& a, int token0, int i) {
    Unit u;
    u.token = a.by_token(i);
    const int rest = i - u.token * (a.heads * a.units), head = a.by_units(rest);
    u.n = rest - head * a.units;
    const int token = token0 + u.token, b = a.by_len(token);
    u.batch = b;
    u.pos = token - b * a.len;
    u.side = head >= a.heads_q;
    u.head = head - (u.side ? a.heads_q : 0);
    if (u.n < a.turned) {
        u.at[0] = N * u.n;
        u.at[1] = a.rot / 2 + u.at[0];
    } else {
        u.at[0] = N * (u.n + a.turned);                            // behind 2 * turned groups
        u.at[1] = u.at[0] + N * (a.units - a.turned);
    }
    return u;
}

// N: 8, or what divides half of the turned part where the halves are apart (every group then lies where a load of its size may).
template <typename T, int N>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 5 : 3) rope_kernel(const __grid_constant__ RopeArgs a) {
    extern __shared__ __align__(16) float2 table[];
    grid_dependency_sync();
    const int token0 = blockIdx.x * a.per_block, tokens = min(a.per_block, a.tokens - token0);
    const int units = tokens * a.heads * a.units;
    const bool copies = a.side[0].in != a.side[0].out || a.side[1].in != a.side[1].out;      // in place, what is not turned stays
    bool angles = false;
    for (int u0 = threadIdx.x; u0 < units || !angles; u0 += kThreads * kUnits) {
        Group<T, N> raw[kUnits][2];
#pragma unroll
        for (int j = 0; j < kUnits; ++j) {
            const int i = u0 + j * kThreads;
            if (i >= units) continue;
            const Unit u = unit_of<N>(a, token0, i);
            const T* p = static_cast<const T*>(a.side[u.side].in) + u.offset(a.side[u.side].from);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (u.at[h] < a.dim) raw[j][h].load(p + u.at[h]);
        }
        if (!angles) {
            fill_angles(a, table, token0, tokens);
            __syncthreads();
            angles = true;
        }
#pragma unroll
        for (int j = 0; j < kUnits; ++j) {
            const int i = u0 + j * kThreads;
            if (i >= units) continue;
            const Unit u = unit_of<N>(a, token0, i);
            T* p = static_cast<T*>(a.side[u.side].out) + u.offset(a.side[u.side].to);
            const float2* cs = table + u.token * a.angle_step;
            float e[2][N];
            raw[j][0].widen(e[0]);
            raw[j][1].widen(e[1]);
            if (u.n < a.turned) {
                if constexpr (N == 1) {
                    turn_pair(cs[u.n].x, cs[u.n].y, e[0][0], e[1][0]);
                } else {
#pragma unroll
                    for (int x = 0; x < N; x += 2) {
                        const float4 two = *reinterpret_cast<const float4*>(cs + N * u.n + x);
                        turn_pair(two.x, two.y, e[0][x], e[1][x]);
                        turn_pair(two.z, two.w, e[0][x + 1], e[1][x + 1]);
                    }
                }
            } else if (N == 8 && a.interleaved) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int pair = u.at[h] / 2;
#pragma unroll
                    for (int x = 0; x < N / 2; x += 2) {
                        if (pair + x >= a.angles) break;
                        const float4 two = *reinterpret_cast<const float4*>(cs + pair + x);
                        turn_pair(two.x, two.y, e[h][2 * x], e[h][2 * x + 1]);
                        if (pair + x + 1 < a.angles) turn_pair(two.z, two.w, e[h][2 * x + 2], e[h][2 * x + 3]);
                    }
                }
            } else if (!copies) {
                continue;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (u.at[h] < a.dim) Group<T, N>::store(p + u.at[h], e[h]);
        }
    }
}

int check_rope_tensor(const alsgd_attn_tensor* t, const alsgd_rope_desc& d, uint32_t heads, bool output) {
    if (!t) return ALSGD_E_ARG;
    if (!t->data || reinterpret_cast<uintptr_t>(t->data) % 16) return ALSGD_E_ARG;
    const int64_t step[3] = {t->stride_pos, t->stride_head, t->stride_batch};
    const uint64_t extent[3] = {d.len, heads, d.batch};
    const int64_t unit = d.dtype == ALSGD_F32 ? 4 : 8;
    for (int i = 0; i < 3; ++i) {
        if (extent[i] == 1) continue;
        if (step[i] < 0 || step[i] % unit || step[i] >= (1ll << 39)) return ALSGD_E_ARG;
        if (step[i] == 0 && output) return ALSGD_E_ARG;
        if (i < 2 && step[i] > INT32_MAX) return ALSGD_E_RANGE;
    }
    return ALSGD_OK;
}

Steps steps_of(const alsgd_attn_tensor& t, const alsgd_rope_desc& d, uint32_t heads) {
    return {d.batch > 1 ? t.stride_batch : 0, d.len > 1 ? (int)t.stride_pos : 0, heads > 1 ? (int)t.stride_head : 0};
}

int check_rope(const alsgd_rope_desc* d) {
    if (!d) return ALSGD_E_ARG;
    if (d->batch == 0 || d->heads_q == 0 || d->dim == 0 || d->dim % 8 || d->rot == 0 || d->rot % 2 || d->rot > d->dim) return ALSGD_E_ARG;
    if (d->flags & ~(ALSGD_ROPE_INTERLEAVED | ALSGD_ROPE_INVERSE)) return ALSGD_E_ARG;
    if (d->dtype != ALSGD_F32 && d->dtype != ALSGD_BF16) return ALSGD_E_ARG;
    if (d->position_dtype != ALSGD_I32 && d->position_dtype != ALSGD_I64) return ALSGD_E_ARG;
    if (!(d->base > 1.0) || !std::isfinite(d->base) || !(d->factor >= 1.0) || !std::isfinite(d->factor)) return ALSGD_E_ARG;
    if (!(std::fabs(d->amplitude) <= FLT_MAX) || (float)d->amplitude == 0.0f) return ALSGD_E_ARG;      // the kernel has it in binary32
    if (!(d->context >= 0.0) || !std::isfinite(d->context) || !(d->turns_low >= 0.0) || !std::isfinite(d->turns_high)) return ALSGD_E_ARG;
    if (d->turns_high != 0.0 && !(d->turns_high > d->turns_low)) return ALSGD_E_ARG;
    if (d->dim > kMaxDim) return ALSGD_E_UNSUPPORTED;
    if (d->len > 1u << 22 || (uint64_t)d->heads_q + d->heads_k > 1u << 16) return ALSGD_E_RANGE;
    // a block's units are counted in 32 bits; kMaxTokens * 2^16 heads * 256 elements stay below 2^31, tokens must as well
    if ((uint64_t)d->batch * d->len > 0x7FFFFFFFull - kMaxTokens) return ALSGD_E_RANGE;
    if (d->device < 0 || d->device >= kMaxDevices) return ALSGD_E_RANGE;
    return ALSGD_OK;
}

void frequencies(const alsgd_rope_desc& d, double* f) {
    const double two_pi = 6.283185307179586476925;
    for (uint32_t i = 0; i < d.rot / 2; ++i) {
        double v = std::pow(d.base, -2.0 * i / d.rot);
        if (d.factor != 1.0) {
            double keep = 0.0;
            if (d.turns_high != 0.0) {
                keep = (d.context * v / two_pi - d.turns_low) / (d.turns_high - d.turns_low);
                keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            }
            v = v * keep + v / d.factor * (1.0 - keep);
        }
        f[i] = v;
    }
}

template <typename T>
cudaError_t launch(int group, dim3 grid, dim3 block, size_t smem, cudaStream_t s, const RopeArgs& a) {
    switch (group) {
        case 8: return launch_dependent(rope_kernel<T, 8>, grid, block, smem, s, a);
        case 4: return launch_dependent(rope_kernel<T, 4>, grid, block, smem, s, a);
        case 2: return launch_dependent(rope_kernel<T, 2>, grid, block, smem, s, a);
        default: return launch_dependent(rope_kernel<T, 1>, grid, block, smem, s, a);
    }
}

}  // namespace

extern "C" int alsgd_rope_frequencies(const alsgd_rope_desc* desc, double* out) {
    const int rc = check_rope(desc);
    if (rc != ALSGD_OK) return rc;
    if (!out) return ALSGD_E_ARG;
    frequencies(*desc, out);
    return ALSGD_OK;
}

extern "C" int alsgd_rope(const alsgd_rope_desc* desc, const alsgd_attn_tensor* q, const alsgd_attn_tensor* k, const void* positions,
                          const alsgd_attn_tensor* q_out, const alsgd_attn_tensor* k_out, void* stream) {
    int rc = check_rope(desc);
    if (rc != ALSGD_OK) return rc;
    const alsgd_rope_desc& d = *desc;
    if (reinterpret_cast<uintptr_t>(positions) % (d.position_dtype == ALSGD_I64 ? 8 : 4)) return ALSGD_E_ARG;
    if (d.len == 0) return ALSGD_OK;
    if ((rc = check_rope_tensor(q, d, d.heads_q, false)) != ALSGD_OK) return rc;
    if ((rc = check_rope_tensor(q_out, d, d.heads_q, true)) != ALSGD_OK) return rc;
    if (d.heads_k) {
        if ((rc = check_rope_tensor(k, d, d.heads_k, false)) != ALSGD_OK) return rc;
        if ((rc = check_rope_tensor(k_out, d, d.heads_k, true)) != ALSGD_OK) return rc;
    }
    UseDevice use(d.device);
    if (!use.ok) return ALSGD_E_CUDA;

    RopeArgs a;
    std::memset(&a, 0, sizeof a);
    a.side[0] = {q->data, q_out->data, steps_of(*q, d, d.heads_q), steps_of(*q_out, d, d.heads_q)};
    if (d.heads_k) a.side[1] = {k->data, k_out->data, steps_of(*k, d, d.heads_k), steps_of(*k_out, d, d.heads_k)};
    a.positions = positions;
    a.wide_positions = d.position_dtype == ALSGD_I64;
    a.pos0 = d.pos0;
    a.len = (int)d.len;
    a.heads_q = (int)d.heads_q;
    a.heads = (int)(d.heads_q + d.heads_k);
    a.dim = (int)d.dim;
    a.rot = (int)d.rot;
    a.interleaved = (d.flags & ALSGD_ROPE_INTERLEAVED) != 0;
    a.tokens = (int)(d.batch * d.len);
    a.angles = a.rot / 2;
    a.angle_step = (a.angles + 1) / 2 * 2;
    a.amplitude = (float)d.amplitude;
    a.turn = d.flags & ALSGD_ROPE_INVERSE ? -1.0f : 1.0f;
    frequencies(d, a.turns);
    for (int i = 0; i < a.angles; ++i) a.turns[i] *= 1.0 / 6.283185307179586476925;
    int group = 8;
    if (!a.interleaved)
        while (a.angles % group) group /= 2;
    a.turned = a.interleaved ? 0 : a.angles / group;
    a.units = a.turned + ((a.interleaved ? a.dim : a.dim - a.rot) / group + 1) / 2;
    a.by_token = divide_by(a.heads * a.units);
    a.by_units = divide_by(a.units);
    a.by_len = divide_by(a.len);
    a.by_angles = divide_by(a.angles);
    // enough tokens for every thread's kUnits, but no fewer than two blocks per SM as long as there are tokens for them
    const int per_token = a.heads * a.units;
    a.per_block = kThreads * kUnits / per_token;
    if (a.per_block > a.tokens / (2 * kSMs)) a.per_block = a.tokens / (2 * kSMs);
    if (a.per_block > kMaxTokens) a.per_block = kMaxTokens;
    if (a.per_block < 1) a.per_block = 1;
    const dim3 grid((a.tokens + a.per_block - 1) / a.per_block), block(kThreads);
    const size_t smem = (size_t)a.per_block * a.angle_step * sizeof(float2);   // at most 16 KB
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = d.dtype == ALSGD_F32 ? launch<float>(group, grid, block, smem, s, a) : launch<uint16_t>(group, grid, block, smem, s, a);
    return e == cudaSuccess ? ALSGD_OK : ALSGD_E_CUDA;
}
