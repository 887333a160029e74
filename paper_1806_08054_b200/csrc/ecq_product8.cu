// C ABI of the products of matrices in 8 bits: argument checks, tensor maps, choice of the kernel.
#include <algorithm>
#include <atomic>
#include <cstdint>
#include <mutex>

#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/ecq.h"
#include "ecq_act8_host.h"
#include "ecq_product8.cuh"

using namespace ecq;

namespace {

std::atomic<uint32_t> g_wait_limit{kWaitLimit};

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn tensor_map_encoder() {
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

// Boxes of 128 bytes along K and `box` rows; what is beyond the matrix arrives as zeros.
bool entries_map(CUtensorMap* tm, const ecq_act8_matrix* m, uint64_t rows, uint64_t k, uint32_t box) {
    const cuuint64_t dims[2] = {k, rows}, strides[1] = {m->stride};
    const cuuint32_t boxes[2] = {kProdRow, box}, unit[2] = {1, 1};
    return tensor_map_encoder()(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, m->data, dims, strides, boxes, unit,
                                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Groups of 512 scale bytes.
bool scales_map(CUtensorMap* tm, const ecq_act8_matrix* m, uint64_t rows, uint64_t k) {
    const cuuint64_t dims[2] = {128, (rows + 127) / 128 * ((k + 511) / 512)}, strides[1] = {512};
    const cuuint32_t boxes[2] = {128, 1}, unit[2] = {1, 1};
    return tensor_map_encoder()(tm, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, m->scales, dims, strides, boxes, unit,
                                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Kernels that take more shared memory than the default say so once a device.
bool allow_smem(const void* kernel, size_t bytes, std::atomic<bool>* done) {
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

template <int TN, bool SWAP>
int launch_part(Product8& P, uint32_t parts, cudaStream_t st) {
    static std::atomic<bool> done[kMaxDevices];
    auto kernel = act8_product_part_kernel<TN, SWAP>;
    using S = ProdPart<TN, SWAP>;
    if (!allow_smem(reinterpret_cast<const void*>(kernel), S::kSmem, done)) return ECQ_ERR_CUDA;
    return launch_act8(kernel, P.tiles * parts, S::kThreads, S::kSmem, parts, st, P);
}

int launch_pair(Product8& P, uint32_t pairs, cudaStream_t st) {
    static std::atomic<bool> done[kMaxDevices];
    if (!allow_smem(reinterpret_cast<const void*>(act8_product_pair_kernel), ProdPair::kSmem, done)) return ECQ_ERR_CUDA;
    return launch_act8(act8_product_pair_kernel, 2 * std::min(pairs, P.tiles), ProdPair::kThreads, ProdPair::kSmem, 2, st, P);
}

uint32_t up(uint64_t x, uint32_t by) { return (uint32_t)((x + by - 1) / by); }

}  // namespace

extern "C" {

int ecq_act8_set_wait_limit(uint32_t polls) {
    g_wait_limit.store(polls, std::memory_order_relaxed);
    return ECQ_OK;
}

int ecq_act8_product(uint64_t m, uint64_t n, uint64_t k, const ecq_act8_matrix* a, const ecq_act8_matrix* b,
                     const ecq_act8_matrix* c, const ecq_act8_matrix* d, uint32_t* status, void* cuda_stream) {
    if (!n || !k || bad_size(m, n) || bad_size(m, k) || bad_size(n, k) || bad_matrix(a, m, k, kCoded) || bad_matrix(b, n, k, kCoded) ||
        (c && bad_matrix(c, m, n, kPlain)) || bad_matrix(d, m, n, kAny) || (c && d->dtype >= 3) || !aligned_to(status, 4))
        return ECQ_ERR_ARG;
    if (m == 0) return ECQ_OK;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || !tensor_map_encoder())
        return ECQ_ERR_CUDA;
    Product8 P = {};
    P.out = act8_mat(d, n);
    if (c) {
        const Act8Mat add = act8_mat(c, n);
        P.add = add.data;
        P.add_stride = add.stride;
        P.add_dtype = add.dtype;
        P.add_wide = add.wide;
    }
    P.status = status;
    P.rows = (uint32_t)m;
    P.cols = (uint32_t)n;
    P.steps = up(k, 128);
    P.tail = up(k - (uint64_t)(P.steps - 1) * 128, 32);
    P.left_groups = P.right_groups = up(k, 512);
    P.wait_limit = g_wait_limit.load(std::memory_order_relaxed);

    const bool swap = m <= 64;
    const uint32_t fa = a->dtype == ECQ_E5M2 ? 1u : 0u, fb = b->dtype == ECQ_E5M2 ? 1u : 0u;
    P.formats = swap ? fb << 7 | fa << 10 : fa << 7 | fb << 10;
    const uint64_t tiles256 = (uint64_t)up(m, 256) * up(n, 256);
    const bool pair = !swap && tiles256 >= 40;
    uint32_t right_box = 128;
    if (swap) right_box = m <= 16 ? 16 : m <= 32 ? 32 : 64;
    const ecq_act8_matrix *left = swap ? b : a, *right = swap ? a : b;
    const uint64_t left_rows = swap ? n : m, right_rows = swap ? m : n;
    if (!entries_map(&P.left, left, left_rows, k, 128) || !entries_map(&P.right, right, right_rows, k, right_box) ||
        !scales_map(&P.left_scales, left, left_rows, k) || !scales_map(&P.right_scales, right, right_rows, k))
        return ECQ_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (pair) {
        P.across = up(n, 256);
        P.tiles = (uint32_t)tiles256;
        return launch_pair(P, (uint32_t)sms / 2, st);
    }
    P.across = swap ? 1 : up(n, 128);
    P.tiles = up(left_rows, 128) * P.across;
    uint32_t parts = 1;
    while (parts < 8 && 2 * parts <= P.steps && (uint64_t)P.tiles * parts * 2 <= (uint64_t)sms) parts *= 2;
    if (!swap) return launch_part<128, false>(P, parts, st);
    return right_box == 16 ? launch_part<16, true>(P, parts, st)
         : right_box == 32 ? launch_part<32, true>(P, parts, st) : launch_part<64, true>(P, parts, st);
}

}  // extern "C"
