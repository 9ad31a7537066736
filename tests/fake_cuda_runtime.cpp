// A stand-in for the CUDA runtime that launches nothing: the library's objects
// link against it, so that the host side of an entry point (checks, kernel
// attributes, launch shapes) runs without a GPU, on as many devices as a test
// wants.  It keeps what the runtime would refuse: dynamic shared memory past
// 48 KB that was not asked for on the current device.
#include <cuda_runtime_api.h>

#include <cstdio>
#include <cstring>
#include <map>
#include <utility>
#include <vector>

namespace {

constexpr int kDevices = 4;
int device = 0;
int sms[kDevices] = {152, 76, 152, 152};
std::map<std::pair<int, const void *>, int> most_smem;     // by device and kernel
struct Launch {
    unsigned x, y, z, threads, cluster;
    unsigned long long smem;
};
std::vector<Launch> launches;

cudaError_t launch(const void *kern, const Launch &l)
{
    auto at = most_smem.find({device, kern});
    if (l.smem > 48 * 1024 && (at == most_smem.end() || l.smem > (unsigned long long)at->second))
        return cudaErrorInvalidValue;
    launches.push_back(l);
    return cudaSuccess;
}

int encode(...) { return 0; }

} // namespace

extern "C" {

// ---- the test's side
void fake_device(int d) { device = d; }
int fake_launches() { return (int)launches.size(); }
void fake_launch(int i, unsigned *out) // grid x, y, z, threads, cluster, shared bytes
{
    const Launch &l = launches[i];
    const unsigned v[6] = {l.x, l.y, l.z, l.threads, l.cluster, (unsigned)l.smem};
    memcpy(out, v, sizeof v);
}

// ---- the runtime's side
cudaError_t cudaGetDevice(int *d)
{
    *d = device;
    return cudaSuccess;
}
cudaError_t cudaDeviceGetAttribute(int *v, cudaDeviceAttr a, int d)
{
    *v = a == cudaDevAttrComputeCapabilityMajor ? 10 : a == cudaDevAttrComputeCapabilityMinor ? 3
         : a == cudaDevAttrMultiProcessorCount  ? sms[d]
                                                : 0;
    return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void *kern, cudaFuncAttribute a, int v)
{
    if (a == cudaFuncAttributeMaxDynamicSharedMemorySize)
        most_smem[{device, kern}] = v;
    return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *kern, void **)
{
    unsigned cluster = 1;
    for (unsigned i = 0; i < c->numAttrs; ++i)
        if (c->attrs[i].id == cudaLaunchAttributeClusterDimension)
            cluster = c->attrs[i].val.clusterDim.x;
    return launch(kern, {c->gridDim.x, c->gridDim.y, c->gridDim.z, c->blockDim.x, cluster, c->dynamicSmemBytes});
}
cudaError_t cudaOccupancyMaxActiveClusters(int *n, const void *, const cudaLaunchConfig_t *c)
{
    *n = sms[device] / (int)c->gridDim.x - 1;               // (the last group of SMs holds no whole cluster)
    return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessor(int *n, const void *, int, size_t)
{
    *n = 1;
    return cudaSuccess;
}
cudaError_t cudaGetDriverEntryPointByVersion(const char *, void **p, unsigned, unsigned long long, cudaDriverEntryPointQueryResult *q)
{
    *p = reinterpret_cast<void *>(&encode);
    *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaMemcpyAsync(void *, const void *, size_t, cudaMemcpyKind, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaMemsetAsync(void *, int, size_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamWaitEvent(cudaStream_t, cudaEvent_t, unsigned) { return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamCreateWithFlags(cudaStream_t *, unsigned) { return cudaSuccess; }
cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaEventDestroy(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaEventCreateWithFlags(cudaEvent_t *, unsigned) { return cudaSuccess; }
cudaError_t cudaGetSymbolAddress(void **, const void *) { return cudaErrorInvalidSymbol; }

// ---- what nvcc's host code calls
void **__cudaRegisterFatBinary(void *) { return nullptr; }
void __cudaRegisterFatBinaryEnd(void **) {}
void __cudaUnregisterFatBinary(void **) {}
void __cudaRegisterFunction(void **, const char *, char *, const char *, int, uint3 *, uint3 *, dim3 *, dim3 *, int *) {}
void __cudaRegisterVar(void **, char *, char *, const char *, int, size_t, int, int) {}
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, void *) { return 0; }
cudaError_t __cudaPopCallConfiguration(dim3 *, dim3 *, size_t *, void *) { return cudaSuccess; }
cudaError_t __cudaGetKernel(cudaKernel_t *, const void *) { return cudaSuccess; }
cudaError_t __cudaLaunchKernel(cudaKernel_t, dim3 g, dim3 b, void **, size_t smem, cudaStream_t)
{
    launches.push_back({g.x, g.y, g.z, b.x, 1, smem});
    return cudaSuccess;
}

} // extern "C"
