// A stand-in for the few CUDA runtime calls that cluster.cuh makes, with several devices: no GPU and no driver.  Prints what is asked and launched.  A launch of more than 8 blocks
// a cluster is refused on a device where the kernel has not been allowed them, as the runtime does.
#include <cstdio>
#include <map>
#include <set>

#include <cuda_runtime_api.h>

static int current = 0;
static std::map<int, std::set<const void *>> allowed;

extern "C" {
void fake_device(int device) { current = device; }
void fake_reset() { allowed.clear(); }

cudaError_t cudaGetDevice(int *d) { *d = current; return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void *f, cudaFuncAttribute a, int value)
{
    if (a == cudaFuncAttributeNonPortableClusterSizeAllowed && value) allowed[current].insert(f);
    return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveClusters(int *n, const void *f, const cudaLaunchConfig_t *c)
{
    const int cluster = c->attrs[0].val.clusterDim.x;
    if (cluster > 8 && !allowed[current].count(f)) return cudaErrorInvalidClusterSize;
    // device 1 has half the multiprocessors, and more shared memory a block leaves room for half as many
    *n = (current == 1 ? 64 : 128) / cluster / (c->dynamicSmemBytes > 100000 ? 2 : 1);
    printf("asked device %d cluster %d smem %zu\n", current, cluster, c->dynamicSmemBytes);
    return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *f, void **)
{
    const int cluster = c->attrs[0].val.clusterDim.x;
    const bool refused = cluster > 8 && !allowed[current].count(f);
    printf("launch device %d cluster %d %s\n", current, cluster, refused ? "refused" : "ok");
    return refused ? cudaErrorInvalidClusterSize : cudaSuccess;
}
cudaError_t cudaLaunchKernel(const void *, dim3, dim3, void **, size_t, cudaStream_t) { return cudaSuccess; }

// what a kernel's registration and its host stub call
void **__cudaRegisterFatBinary(void *) { static void *h; return &h; }
void __cudaRegisterFatBinaryEnd(void **) {}
void __cudaUnregisterFatBinary(void **) {}
void __cudaRegisterFunction(void **, const char *, char *, const char *, int, void *, void *, void *, void *, void *) {}
char __cudaInitModule(void **) { return 0; }
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, void *) { return 0; }
cudaError_t __cudaPopCallConfiguration(dim3 *, dim3 *, size_t *, void *) { return cudaSuccess; }
cudaError_t __cudaGetKernel(cudaKernel_t *k, const void *f) { *k = (cudaKernel_t)f; return cudaSuccess; }
cudaError_t __cudaLaunchKernel(cudaKernel_t, dim3, dim3, void **, size_t, cudaStream_t) { return cudaSuccess; }
}
