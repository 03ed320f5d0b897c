// Two blocks of a cluster, one of which waits for what nothing brings, with few tries: prints both blocks' marks and what the
// wait reported, for a wait of either block and for one that finds its phase complete.
#include "../paper_2401_09135_b200/csrc/alsgd_pair.cuh"

#include <cstdio>

using namespace alsgd_tc;

__global__ void __cluster_dims__(2, 1, 1) marks_kernel(int who, bool arrives, uint32_t* out) {
    __shared__ __align__(8) uint64_t bar;
    __shared__ uint32_t dead;
    if (threadIdx.x == 0) {
        dead = 0;
        bar_init(smem_u32(&bar), 1);
        bar_init_fence();
    }
    __syncthreads();
    cluster_sync();
    if ((int)cluster_rank() == who && threadIdx.x == 0) {
        if (arrives) bar_arrive(smem_u32(&bar));
        wait_pair(smem_u32(&bar), 0, &dead, 4, 1 << 10);
    }
    __syncwarp();
    cluster_sync();
    if (threadIdx.x == 0) {
        out[cluster_rank()] = *(volatile uint32_t*)&dead;
        if (cluster_rank() == 0) out[2] = atomicExch(&g_wait_error, 0u);
    }
}

int main() {
    uint32_t* out;
    if (cudaMallocManaged(&out, 12) != cudaSuccess) return 1;
    for (int i = 0; i < 3; ++i) {
        marks_kernel<<<2, 32>>>(i & 1, i == 2, out);
        if (cudaDeviceSynchronize() != cudaSuccess) return 1;
        std::printf("%u %u %u\n", out[0], out[1], out[2]);
    }
    return 0;
}
