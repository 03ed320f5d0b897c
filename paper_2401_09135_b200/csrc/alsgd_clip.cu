// alsgd_clip_grads: global norm of a list of gradient tensors, and the clipped gradient as one flat vector.
//
//   n = sqrt(sum over all tensors of g^2),  c = 1 if n <= max_norm else max_norm / n,  out[offset_t + i] = c * g_t[i]
//
// Two launches.  norm_kernel reads every tensor once: a thread adds 4 or 8 squares at a time in binary32 and
// everything above in binary64, blocks leave one partial each, and the block that takes the last ticket adds the
// partials in index order, so the same inputs give the same bits on every call.  A group of squares that leaves the
// binary32 range (overflow, or everything below 2^-100) is formed again in binary64, and so is the quotient by a norm
// beyond it: no non-zero list has a zero norm, and a finite one whose norm is reported as infinite is clipped by its
// value.  scale_kernel reads the tensors a second time, walking the tiles from the last to the first because the first
// pass left the end of the list in the 126 MB L2.
//
// Bound: memory.  The floor reads every gradient once and writes the flat vector once; a list beyond the L2 is read
// again from HBM for all but the last ~100 MB.  Measured (B200): 22.9M fp32 elements 45 us, 109.5M bf16 to bf16 106 us,
// 149.8M fp32 277 us, which is 6.5 TB/s over the three passes.
#include "../../include/alsgd.h"
#include "alsgd_ops.cuh"

#include <cmath>

using namespace alsgd_ops;

namespace {

constexpr int kBlock = 256;
constexpr int kLoads = 8;                                   // 16-byte loads per thread per tile
constexpr uint32_t kTileVecs = kBlock * kLoads;             // 16-byte vectors per tile: 8192 fp32 or 16384 bf16 elements
constexpr int kNormPerSm = 4;                               // blocks that walk the tiles; 3 to 5 of them are alike, 8 with 4 loads cost 2-6 %
constexpr uint32_t kNormBlocks = kSMs * kNormPerSm;
constexpr size_t kWorkHead = 256;                           // Head, padded
constexpr int kMaxGroup = 512;                              // tensors per launch

// In front of the partials.  The factor that the elements are multiplied by is parts[0] * parts[1]: one that is below the
// normal range goes as parts of its own size and 2^-64, so that its 24 bits stay.  One load brings both: every warp of the
// scale pass asks for them, and a second request to their one line cost 2.5 us.
struct Head {
    unsigned ticket;
    alignas(8) float2 parts;
};

template <int CAP>
struct Tensors {
    const void* src[CAP];
    uint64_t numel[CAP];
    uint64_t offset[CAP];
    uint32_t tile_end[CAP];      // tiles of the tensors up to and including this one
    uint8_t bf16[CAP];
    uint32_t n;
};

__device__ __forceinline__ uint64_t tile_elems(bool bf16) { return (uint64_t)kTileVecs * (bf16 ? 8 : 4); }

// Tensor of a tile: the first whose tile_end exceeds it, `from` on (tiles are visited in ascending order).
template <int CAP>
__device__ __forceinline__ uint32_t walk(const Tensors<CAP>& t, uint32_t from, uint32_t tile) {
    while (t.tile_end[from] <= tile) ++from;
    return from;
}

// The same without a starting point, by halving.
template <int CAP>
__device__ __forceinline__ uint32_t find(const Tensors<CAP>& t, uint32_t tile) {
    uint32_t lo = 0, hi = t.n - 1;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) >> 1;
        if (t.tile_end[mid] <= tile) lo = mid + 1; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ void widen(const uint4& w, bool bf16, float (&x)[8]) {
    if (bf16) {
        x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
        x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
    } else {
        x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
        x[4] = x[5] = x[6] = x[7] = 0.0f;
    }
}

// Elements [e, e + count) of a tensor, count <= 4 or 8, zeros behind them; one 16-byte load where it is allowed.
__device__ __forceinline__ uint4 load_vec(const void* src, bool bf16, uint64_t e, uint64_t numel, bool aligned) {
    const uint32_t per = bf16 ? 8 : 4;
    if (aligned && e + per <= numel) return *reinterpret_cast<const uint4*>(static_cast<const char*>(src) + e * (bf16 ? 2 : 4));
    uint32_t w[4] = {0, 0, 0, 0};
    if (bf16) {
        const uint16_t* p = static_cast<const uint16_t*>(src);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (e + i < numel) w[i >> 1] |= (uint32_t)p[e + i] << (16 * (i & 1));
    } else {
        const uint32_t* p = static_cast<const uint32_t*>(src);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (e + i < numel) w[i] = p[e + i];
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Squares of one group in binary64, for groups whose binary32 sum is not trusted.
__device__ __noinline__ double squares_wide(uint4 w, bool bf16) {
    float x[8];
    widen(w, bf16, x);
    double s = 0.0;
    for (int i = 0; i < 8; ++i) s += (double)x[i] * (double)x[i];
    return s;
}

__device__ __forceinline__ double squares(const uint4& w, bool bf16) {
    float x[8];
    widen(w, bf16, x);
    float s = x[0] * x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) s = fmaf(x[i], x[i], s);
    if (s >= 0x1p-100f && s < INFINITY) return (double)s;
    if (((w.x | w.y | w.z | w.w) & (bf16 ? 0x7FFF7FFFu : 0x7FFFFFFFu)) == 0) return 0.0;   // nothing but zeros: the usual reason
    return squares_wide(w, bf16);
}

__device__ __forceinline__ double block_sum(double v, double* shared) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xFFFFFFFFu, v, o);
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x == 0)
        for (int i = 0; i < kBlock / 32; ++i) s += shared[i];
    return s;
}

// last: partials of all launches of the call, or 0 where another norm launch follows this one.
template <int CAP>
__global__ void __launch_bounds__(kBlock, kNormPerSm) norm_kernel(const __grid_constant__ Tensors<CAP> t, double* partial, uint32_t first,
                                                      uint32_t last, Head* head, float max_norm, float* stats) {
    __shared__ double shared[kBlock / 32];
    __shared__ bool closing;
    grid_dependency_sync();
    double acc = 0.0;
    const uint32_t tiles = t.n ? t.tile_end[t.n - 1] : 0;
    uint32_t at = 0;
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        at = walk(t, at, tile);
        const bool bf16 = t.bf16[at];
        const void* src = t.src[at];
        const uint64_t numel = t.numel[at];
        const bool aligned = (reinterpret_cast<uintptr_t>(src) & 15) == 0;
        const uint64_t e0 = (uint64_t)(tile - (at ? t.tile_end[at - 1] : 0)) * tile_elems(bf16);
        uint4 w[kLoads];
        if (aligned && e0 + tile_elems(bf16) <= numel) {
            const uint4* p = reinterpret_cast<const uint4*>(static_cast<const char*>(src) + e0 * (bf16 ? 2 : 4)) + threadIdx.x;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) w[i] = p[i * kBlock];
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                w[i] = load_vec(src, bf16, e0 + (uint64_t)(i * kBlock + threadIdx.x) * (bf16 ? 8 : 4), numel, aligned);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) acc += squares(w[i], bf16);
    }
    const double s = block_sum(acc, shared);
    if (threadIdx.x == 0) {
        partial[first + blockIdx.x] = s;
        __threadfence();
        closing = last != 0 && atomicAdd(&head->ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!closing) return;
    __threadfence();
    acc = 0.0;
    for (uint32_t i = threadIdx.x; i < last; i += kBlock) acc += __ldcg(partial + i);
    __syncthreads();
    const double total = block_sum(acc, shared);
    if (threadIdx.x == 0) {
        head->ticket = 0;
        const double root = sqrt(total);
        const float norm = (float)root;
        float factor = norm <= max_norm ? 1.0f : max_norm / norm;      // a norm that is NaN makes the factor NaN
        float2 parts = make_float2(factor, 1.0f);
        if (norm == INFINITY && factor == 0.0f) {              // beyond binary32 at least: by its 2^-64th
            parts.x = max_norm / (float)(root * 0x1p-64);
            factor = parts.x * 0x1p-64f;
            if (factor < 0x1p-126f) parts.y = 0x1p-64f;
            else parts.x = factor;
        }
        stats[0] = norm;
        stats[1] = factor;
        head->parts = parts;
    }
}

template <typename OUT>
__device__ __forceinline__ void store_vec(OUT* out, uint64_t e, uint64_t numel, const float (&y)[8], uint32_t per, bool aligned) {
    if (aligned && e + per <= numel) {
        if constexpr (sizeof(OUT) == 4) {
            *reinterpret_cast<float4*>(out + e) = make_float4(y[0], y[1], y[2], y[3]);
            if (per == 8) *reinterpret_cast<float4*>(out + e + 4) = make_float4(y[4], y[5], y[6], y[7]);
        } else if (per == 8) {
            *reinterpret_cast<uint4*>(out + e) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]),
                                                            pack_bf16(y[6], y[7]));
        } else {
            *reinterpret_cast<uint2*>(out + e) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i < (int)per && e + i < numel) {
            if constexpr (sizeof(OUT) == 4) out[e + i] = y[i];
            else out[e + i] = (OUT)(pack_bf16(y[i], 0.0f) & 0xFFFFu);
        }
    }
}

template <int CAP, typename OUT>
__global__ void __launch_bounds__(kBlock) scale_kernel(const __grid_constant__ Tensors<CAP> t, OUT* out, const Head* head) {
    const uint32_t tile = gridDim.x - 1 - blockIdx.x;
    const uint32_t at = find(t, tile);
    const bool bf16 = t.bf16[at];
    const uint32_t per = bf16 ? 8 : 4;
    const void* src = t.src[at];
    const uint64_t numel = t.numel[at];
    OUT* dst = out + t.offset[at];
    const bool aligned = (reinterpret_cast<uintptr_t>(src) & 15) == 0;
    const bool out_aligned = (reinterpret_cast<uintptr_t>(dst) & 15) == 0;
    const uint64_t e0 = (uint64_t)(tile - (at ? t.tile_end[at - 1] : 0)) * tile_elems(bf16);
    grid_dependency_sync();
    const float2 c = __ldcg(&head->parts);
    uint4 w[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) w[i] = load_vec(src, bf16, e0 + (uint64_t)(i * kBlock + threadIdx.x) * per, numel, aligned);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const uint64_t e = e0 + (uint64_t)(i * kBlock + threadIdx.x) * per;
        float x[8];
        widen(w[i], bf16, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = x[j] * c.x * c.y;
        store_vec(dst, e, numel, x, per, out_aligned);
    }
}

uint32_t tiles_of(const alsgd_grad_desc& g) {
    const uint64_t per = (uint64_t)kTileVecs * (g.dtype == ALSGD_BF16 ? 8 : 4);
    return (uint32_t)((g.numel + per - 1) / per);
}

template <int CAP>
void fill(Tensors<CAP>& t, const alsgd_grad_desc* g, uint32_t n) {
    uint32_t tiles = 0;
    t.n = n;
    for (uint32_t i = 0; i < n; ++i) {
        tiles += tiles_of(g[i]);
        t.src[i] = g[i].data;
        t.numel[i] = g[i].numel;
        t.offset[i] = g[i].offset;
        t.tile_end[i] = tiles;
        t.bf16[i] = g[i].dtype == ALSGD_BF16;
    }
}

// One group of tensors: its norm launch (out == nullptr) or its scaling launch.
template <int CAP>
cudaError_t launch_group(const alsgd_grad_desc* g, uint32_t n, double* partial, uint32_t first, uint32_t last, Head* head,
                         float max_norm, float* stats, void* out, uint32_t out_dtype, uint32_t grid, cudaStream_t s) {
    Tensors<CAP> t;
    fill(t, g, n);
    if (!out) return launch_dependent(norm_kernel<CAP>, dim3(grid), dim3(kBlock), 0, s, t, partial, first, last, head, max_norm, stats);
    if (out_dtype == ALSGD_BF16)
        return launch_dependent(scale_kernel<CAP, uint16_t>, dim3(grid), dim3(kBlock), 0, s, t, static_cast<uint16_t*>(out), head);
    return launch_dependent(scale_kernel<CAP, float>, dim3(grid), dim3(kBlock), 0, s, t, static_cast<float*>(out), head);
}

// The table travels as a kernel argument; short lists take the short one (copying 14 KB of arguments costs a launch
// about a microsecond).
cudaError_t launch_any(const alsgd_grad_desc* g, uint32_t n, double* partial, uint32_t first, uint32_t last, Head* head,
                       float max_norm, float* stats, void* out, uint32_t out_dtype, uint32_t grid, cudaStream_t s) {
    if (n <= 16) return launch_group<16>(g, n, partial, first, last, head, max_norm, stats, out, out_dtype, grid, s);
    if (n <= 128) return launch_group<128>(g, n, partial, first, last, head, max_norm, stats, out, out_dtype, grid, s);
    return launch_group<kMaxGroup>(g, n, partial, first, last, head, max_norm, stats, out, out_dtype, grid, s);
}

int group_tiles(const alsgd_grad_desc* g, uint32_t n, uint64_t* tiles) {
    *tiles = 0;
    for (uint32_t i = 0; i < n; ++i) {
        const uint64_t per = (uint64_t)kTileVecs * (g[i].dtype == ALSGD_BF16 ? 8 : 4);
        *tiles += g[i].numel / per + (g[i].numel % per != 0);
        if (*tiles >= 1ull << 30) return ALSGD_E_RANGE;
    }
    return ALSGD_OK;
}

}  // namespace

extern "C" int alsgd_clip_grads_bytes(uint32_t n, uint64_t* bytes_out) {
    if (n == 0 || !bytes_out) return ALSGD_E_ARG;
    const uint64_t groups = ((uint64_t)n + kMaxGroup - 1) / kMaxGroup;
    *bytes_out = kWorkHead + groups * kNormBlocks * sizeof(double);
    return ALSGD_OK;
}

extern "C" int alsgd_clip_grads(const alsgd_grad_desc* grads, uint32_t n, float max_norm, void* out, uint32_t out_dtype,
                                uint64_t out_elems, float* stats, void* work, uint64_t work_bytes, int32_t device, void* stream) {
    if (!grads || n == 0 || !stats || !work || !(max_norm > 0.0f)) return ALSGD_E_ARG;
    if (out_dtype != ALSGD_F32 && out_dtype != ALSGD_BF16) return ALSGD_E_ARG;
    if (device < 0 || device >= kMaxDevices) return ALSGD_E_RANGE;
    const uintptr_t out_size = out_dtype == ALSGD_BF16 ? 2 : 4;
    if (reinterpret_cast<uintptr_t>(out) % out_size || reinterpret_cast<uintptr_t>(work) % 256 ||
        reinterpret_cast<uintptr_t>(stats) % 4)
        return ALSGD_E_ARG;
    for (uint32_t i = 0; i < n; ++i) {
        const alsgd_grad_desc& g = grads[i];
        if (g.dtype != ALSGD_F32 && g.dtype != ALSGD_BF16) return ALSGD_E_ARG;
        if (g.numel && (!g.data || reinterpret_cast<uintptr_t>(g.data) % (g.dtype == ALSGD_BF16 ? 2 : 4))) return ALSGD_E_ARG;
        if (out && (g.numel > out_elems || g.offset > out_elems - g.numel)) return ALSGD_E_RANGE;
        uint64_t tiles;
        if (group_tiles(&g, 1, &tiles) != ALSGD_OK) return ALSGD_E_RANGE;
    }
    for (uint32_t at = 0; at < n; at += kMaxGroup) {
        uint64_t tiles;
        if (group_tiles(grads + at, n - at < kMaxGroup ? n - at : kMaxGroup, &tiles) != ALSGD_OK) return ALSGD_E_RANGE;
    }
    uint64_t need = 0;
    alsgd_clip_grads_bytes(n, &need);
    if (work_bytes < need) return ALSGD_E_NOMEM;

    UseDevice use(device);
    if (!use.ok) return ALSGD_E_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    Head* head = static_cast<Head*>(work);
    double* partial = reinterpret_cast<double*>(static_cast<char*>(work) + kWorkHead);
    uint32_t first = 0;
    for (uint32_t at = 0; at < n; at += kMaxGroup) {
        const uint32_t m = n - at < kMaxGroup ? n - at : kMaxGroup;
        uint64_t tiles;
        group_tiles(grads + at, m, &tiles);
        // an empty list still gets one block: it writes its zero partial and, as the last launch, the results
        const uint32_t grid = tiles == 0 ? 1 : tiles < kNormBlocks ? (uint32_t)tiles : kNormBlocks;
        const uint32_t last = at + m == n ? first + grid : 0;
        if (launch_any(grads + at, m, partial, first, last, head, max_norm, stats, nullptr, 0, grid, s) != cudaSuccess) return ALSGD_E_CUDA;
        first += grid;
    }
    if (!out) return ALSGD_OK;
    const uint32_t groups = (n + kMaxGroup - 1) / kMaxGroup;
    for (uint32_t k = groups; k-- > 0;) {
        const uint32_t at = k * kMaxGroup, m = n - at < kMaxGroup ? n - at : kMaxGroup;
        uint64_t tiles;
        group_tiles(grads + at, m, &tiles);
        if (tiles == 0) continue;
        if (launch_any(grads + at, m, partial, 0, 0, head, max_norm, stats, out, out_dtype, (uint32_t)tiles, s) != cudaSuccess) return ALSGD_E_CUDA;
    }
    return ALSGD_OK;
}
