// A CUDA runtime on the host for tests of the orthogonaliser's C entries: device memory is the
// host's, kernels are recorded instead of run (fake_kernels.cu), and a named call can be told to fail.
#include <cstdint>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>

#include <cuda.h>
#include <cuda_runtime.h>

// fake_kernels.cu: keep the kernels' counters as the kernels do
extern "C" bool fake_prepare(const void* args, unsigned grid);    // whether it found them at zero
extern "C" void fake_iterate(const void* args);

namespace {
std::map<const void*, std::string> kernels;
std::string events, failing;
int fail_after = -1, device = 0;

cudaError_t step(const char* call) {
    if (failing == call && fail_after >= 0 && fail_after-- == 0) return cudaErrorUnknown;
    return cudaSuccess;
}

CUresult encode_tiled(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                      const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                      CUtensorMapL2promotion, CUtensorMapFloatOOBfill) {
    return CUDA_SUCCESS;
}
}  // namespace

extern "C" {

// The call `name` fails once, after `skip` that succeed.
void fake_fail(const char* name, int skip) { failing = name; fail_after = skip; }
// What happened since this was last asked.
const char* fake_events() {
    static std::string out;
    out = events;
    events.clear();
    return out.c_str();
}
int fake_device() { return device; }

void** __cudaRegisterFatBinary(void*) { static void* h; return &h; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char* host, char*, const char* name, int, uint3*, uint3*, dim3*, dim3*, int*) {
    kernels[host] = name;
}
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, CUstream_st*) { return 0; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaSuccess; }
cudaError_t cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { return cudaErrorUnknown; }

cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* cfg, const void* func, void** args) {
    if (kernels[func].find("muon_prepare") != std::string::npos) {
        if (step("prepare")) return cudaErrorUnknown;
        if (!fake_prepare(args[0], cfg->gridDim.x)) events += "stale ";
        events += "prepare ";
    } else {
        if (step("iterate")) return cudaErrorUnknown;
        fake_iterate(args[0]);
        events += "iterate ";
    }
    return cudaSuccess;
}

cudaError_t cudaMalloc(void** p, size_t n) { *p = calloc(1, n); return step("malloc"); }
cudaError_t cudaFree(void* p) { free(p); return cudaSuccess; }
cudaError_t cudaHostAlloc(void** p, size_t n, unsigned) { *p = calloc(1, n); return cudaSuccess; }
cudaError_t cudaFreeHost(void* p) { free(p); return cudaSuccess; }
cudaError_t cudaMemcpy(void* to, const void* from, size_t n, cudaMemcpyKind) { memcpy(to, from, n); return cudaSuccess; }
cudaError_t cudaMemcpyAsync(void* to, const void* from, size_t n, cudaMemcpyKind, cudaStream_t) {
    memcpy(to, from, n);
    return cudaSuccess;
}
cudaError_t cudaMemsetAsync(void* to, int v, size_t n, cudaStream_t) {
    if (step("memset")) return cudaErrorUnknown;
    memset(to, v, n);
    events += "memset ";
    return cudaSuccess;
}
cudaError_t cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaGetDevice(int* d) { *d = device; return cudaSuccess; }
cudaError_t cudaSetDevice(int d) { device = d; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int) { *v = 148; return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return step("attribute"); }
cudaError_t cudaOccupancyMaxActiveClusters(int* n, const void*, const cudaLaunchConfig_t*) { *n = 70; return step("occupancy"); }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaGetDriverEntryPoint(const char*, void** p, unsigned long long, cudaDriverEntryPointQueryResult* q) {
    *p = reinterpret_cast<void*>(encode_tiled);
    *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}

}  // extern "C"
