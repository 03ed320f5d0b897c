// dz as the backward pass's logits hand it out, of 32 rows x 32 words whose probabilities are all 1: prints how many entries are
// NaN, 0 and 1, for a block whose wait ran out and one whose did not, with every other row and the words behind `words` left out.
#include "../paper_2401_09135_b200/csrc/alsgd_vocab.cu"

#include <cstdio>

__global__ void settle_kernel(bool lost, bool some, int words, int* out) {
    uint32_t z[32];
    for (int j = 0; j < 32; ++j) z[j] = 0;
    const bool used = !some || threadIdx.x % 2 == 0;
    exponentials(z, 1.0f, 0.0f);
    times(z, factor_of(1.0f, lost));
    settle(z, used, __all_sync(~0u, used), words);
    for (int j = 0; j < 32; ++j) {
        const float v = __uint_as_float(z[j]);
        atomicAdd(out + (v != v ? 0 : v == 0.0f ? 1 : v == 1.0f ? 2 : 3), 1);
    }
}

int main() {
    int* out;
    if (cudaMallocManaged(&out, 16) != cudaSuccess) return 1;
    for (int i = 0; i < 8; ++i) {
        for (int k = 0; k < 4; ++k) out[k] = 0;
        settle_kernel<<<1, 32>>>(i & 1, i & 2, i & 4 ? 20 : 500, out);
        if (cudaDeviceSynchronize() != cudaSuccess) return 1;
        std::printf("%d %d %d %d\n", out[0], out[1], out[2], out[3]);
    }
    return 0;
}
