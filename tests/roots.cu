// The square root and the reciprocal of the AdamW kernels next to CUDA's correctly rounded ones, for every number of a range.
#include <cuda_runtime.h>

#include "../paper_1908_06077_b200/csrc/nuq_adamw.cuh"

// counts[0], counts[1]: how many numbers differ; last[0], last[1]: the bits of one of them
__global__ void compare(unsigned from, unsigned to, unsigned long long* counts, unsigned* last) {
    const unsigned long long step = (unsigned long long)gridDim.x * blockDim.x;
    unsigned long long differ[2] = {0, 0};
    for (unsigned long long i = from + (unsigned long long)blockIdx.x * blockDim.x + threadIdx.x; i <= to; i += step) {
        const float x = __uint_as_float((unsigned)i);
        const bool wrong[2] = {__float_as_uint(nuq::ordinary_root(x)) != __float_as_uint(__fsqrt_rn(x)), __float_as_uint(nuq::reciprocal(x)) != __float_as_uint(__frcp_rn(x))};
        for (int k = 0; k < 2; ++k) {
            if (!wrong[k]) continue;
            ++differ[k];
            last[k] = (unsigned)i;
        }
    }
    for (int k = 0; k < 2; ++k)
        if (differ[k]) atomicAdd(counts + k, differ[k]);
}

// counts, last: device, two each, zeroed.  Returns a CUDA error.
extern "C" int compare_range(unsigned from, unsigned to, unsigned long long* counts, unsigned* last) {
    compare<<<148 * 8, 256>>>(from, to, counts, last);
    const cudaError_t e = cudaGetLastError();
    return e != cudaSuccess ? (int)e : (int)cudaDeviceSynchronize();
}
