// fake_cuda_runtime.cpp that also keeps the names of the kernels that the
// library holds and of those that it launched.
#include <cuda_runtime_api.h>

#define cudaLaunchKernelExC plain_launch
#define __cudaRegisterFunction plain_register
#include "fake_cuda_runtime.cpp"
#undef cudaLaunchKernelExC
#undef __cudaRegisterFunction

#include <string>

namespace {

// (registered before main, whatever the order of the objects)
std::map<const void *, std::string> &kernels()
{
    static std::map<const void *, std::string> k;
    return k;
}
std::vector<const void *> &launched()
{
    static std::vector<const void *> l;
    return l;
}

} // namespace

extern "C" {

int fake_kernels() { return (int)kernels().size(); }
const char *fake_kernel(int i)
{
    auto it = kernels().begin();
    std::advance(it, i);
    return it->second.c_str();
}
int fake_launched() { return (int)launched().size(); }
const char *fake_launched_kernel(int i) { return kernels()[launched()[i]].c_str(); }

cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *kern, void **args)
{
    const cudaError_t e = plain_launch(c, kern, args);
    if (e == cudaSuccess)
        launched().push_back(kern);
    return e;
}
void __cudaRegisterFunction(void **, const char *host, char *, const char *name, int, uint3 *, uint3 *, dim3 *, dim3 *, int *)
{
    kernels()[host] = name;
}

} // extern "C"
