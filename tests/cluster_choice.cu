// choose_cluster and launch_cluster over several devices, on the runtime of fake_cudart.cpp.
#include <cstdio>

#include "cluster.cuh"

extern "C" void fake_device(int device);
extern "C" void fake_reset();

__global__ void kernel(int) {}

static ipotk::ClusterFit fit;

static void call(int device, long long items, size_t smem)
{
    fake_device(device);
    const int c = ipotk::choose_cluster(fit, kernel, dim3(128), smem, items, 16);
    const cudaError_t e = ipotk::launch_cluster(kernel, dim3(c), dim3(128), smem, c, (cudaStream_t) nullptr, 1);
    printf("call device %d items %lld smem %zu cluster %d status %d\n", device, items, smem, c, (int)e);
}

int main()
{
    for (int device : {0, 1, 0, 1, 70, 1}) call(device, 5, 50000);   // 128 / 5: 16, 64 / 5: 12; 70: beyond any table
    call(0, 5, 120000);                                             // half as many side by side: 12
    call(0, 5, 50000);
    fake_reset();                                                   // the process has reset its devices
    call(0, 5, 50000);
    call(1, 5, 50000);
}
