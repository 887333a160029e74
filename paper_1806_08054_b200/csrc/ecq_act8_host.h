// Checks and launches that the entry points on matrices in 8 bits share.
#pragma once

#include <atomic>
#include <cstdint>
#include <mutex>

#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/ecq.h"
#include "ecq_act8.cuh"
#include "ecq_host.h"

namespace ecq {

// Polls of a wait inside a kernel (ecq_act8_set_wait_limit).
inline std::atomic<uint32_t> g_act8_wait_limit{kWaitLimit};

constexpr uint64_t kActMaxSide = 1ull << 28;
constexpr uint64_t kActMaxStride = 1ull << 36;                        // entries

enum { kPlain = 1, kCoded = 2, kAny = 3 };

// Rows and columns that a call takes: tiles of 128 x 128 are counted in 31 bits.
inline bool bad_size(uint64_t rows, uint64_t cols) {
    return rows > kActMaxSide || cols == 0 || cols > kActMaxSide || ((rows + 127) / 128) * ((cols + 127) / 128) > 0x7FFFFFFFull;
}

// A matrix of a call.  Rows of one in 8 bits begin on 16-byte boundaries, as the tensor cores' copies
// take them.  No rows: only the type counts.
inline bool bad_matrix(const ecq_act8_matrix* m, uint64_t rows, uint64_t cols, int kinds) {
    if (!m) return true;
    const bool coded = m->dtype == ECQ_E4M3 || m->dtype == ECQ_E5M2;
    const uint32_t es = coded ? 1u : dtype_bytes(m->dtype);
    if (!es || !(kinds & (coded ? kCoded : kPlain))) return true;
    if (rows == 0 || cols == 0) return false;
    if (!m->data || m->stride > kActMaxStride || (rows > 1 && m->stride < cols)) return true;
    if (!coded) return !aligned_to(m->data, es);
    return !m->scales || !aligned_to(m->data, 16) || !aligned_to(m->scales, 16) || m->stride < cols || (m->stride & 15);
}

inline Act8Mat act8_mat(const ecq_act8_matrix* m, uint64_t rows, uint64_t cols) {
    Act8Mat r = {};
    if (!m) return r;
    const bool coded = m->dtype >= 3;
    r.data = static_cast<unsigned char*>(m->data);
    r.stride = m->stride * (coded ? 1u : dtype_bytes(m->dtype));
    r.end = r.data + (rows - 1) * r.stride + cols * (coded ? 1u : dtype_bytes(m->dtype));
    r.scales = static_cast<uint8_t*>(m->scales);
    r.groups = (uint32_t)((cols + 511) / 512);
    r.dtype = m->dtype;
    r.wide = aligned_to(m->data, 16) && r.stride % 16 == 0;
    return r;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn tensor_map_encoder() {
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    });
    return fn;
}

// Kernels that take more shared memory than the default say so once a device.
inline bool allow_smem(const void* kernel, size_t bytes, std::atomic<bool>* done) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev >= kMaxDevices) return false;
    if (done[dev].load(std::memory_order_acquire)) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    done[dev].store(true, std::memory_order_release);
    return true;
}

// A launch whose CTAs may be placed while the work ahead of it in the stream is finishing (they touch
// no global memory before it has), in clusters where `cluster` is more than 1.
template <typename... KArgs, typename... Args>
int launch_act8(void (*kernel)(KArgs...), uint32_t grid, uint32_t block, size_t smem, uint32_t cluster, cudaStream_t st,
                Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...) != cudaSuccess) {
        cudaGetLastError();
        return ECQ_ERR_CUDA;
    }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return ECQ_OK;
}

}  // namespace ecq
