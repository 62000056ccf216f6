// The bounded wait of the matrix products (csrc/a2sgd_tcgen05.cuh): a barrier that nothing completes is given up after
// its limit, by every lane, the CTA's other warps follow, and the context stays usable; a barrier that completes
// lets every lane through, late arrivals included.
#include "a2sgd_tcgen05.cuh"

#include <cstdio>

using namespace a2sgd_tc;

// Warp 0 waits on a barrier that completes (warp 3's first lane arrives after a while), warps 1 and 2 on one that does not.
__global__ void waits(int *answers, unsigned long long *waited)
{
    __shared__ __align__(8) uint64_t bars[2];
    __shared__ volatile int gave_up;
    const uint32_t warp = threadIdx.x / 32;
    if (threadIdx.x == 0) {
        bar_init(smem_u32(bars), 1);
        bar_init(smem_u32(bars + 1), 1);
        gave_up = 0;
        bar_init_fence();
    }
    __syncthreads();
    const uint64_t begin = now_ns();
    if (warp < 3) answers[threadIdx.x] = bar_wait(smem_u32(bars + (warp ? 1 : 0)), 0, &gave_up);
    else if (threadIdx.x == 96) {
        __nanosleep(100000);
        bar_arrive_cluster(map_to(smem_u32(bars), 0)); // a CTA on its own is a cluster of one
    }
    __syncthreads();
    if (threadIdx.x == 0) *waited = now_ns() - begin, answers[96] = gave_up;
}

int main()
{
    int *answers, host[97];
    unsigned long long *waited, ns = 0;
    if (cudaMalloc(&answers, sizeof host) != cudaSuccess || cudaMalloc(&waited, sizeof ns) != cudaSuccess) return 2;
    waits<<<1, 128>>>(answers, waited);
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(host, answers, sizeof host, cudaMemcpyDeviceToHost) != cudaSuccess ||
        cudaMemcpy(&ns, waited, sizeof ns, cudaMemcpyDeviceToHost) != cudaSuccess) {
        std::printf("%s\n", cudaGetErrorString(cudaGetLastError()));
        return 2;
    }
    int good = host[96] == 1;
    for (int i = 0; i < 96; ++i) good &= host[i] == (i < 32);
    const double limits = (double)ns / (double)kWaitLimitNs;
    std::printf("%s after %.2f limits\n", good ? "as it should be" : "WRONG", limits);
    return good && limits > 0.99 && limits < 1.5 ? 0 : 1;
}
