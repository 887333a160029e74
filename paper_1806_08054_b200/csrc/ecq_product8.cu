// C ABI of the products of matrices in 8 bits: argument checks, tensor maps, choice of the kernel.
#include <algorithm>
#include <atomic>
#include <cstdint>

#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/ecq.h"
#include "ecq_act8_host.h"
#include "ecq_product8.cuh"

using namespace ecq;

namespace {

// Boxes of 128 bytes along K and `box` rows; what is beyond the matrix arrives as zeros.
bool entries_map(CUtensorMap* tm, const ecq_act8_matrix* m, uint64_t rows, uint64_t k, uint32_t box) {
    const cuuint64_t dims[2] = {k, rows}, strides[1] = {m->stride};
    const cuuint32_t boxes[2] = {kProdRow, box}, unit[2] = {1, 1};
    return tensor_map_encoder()(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, m->data, dims, strides, boxes, unit,
                                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The result, in boxes of 32 rows of 64 bytes.
bool result_map(CUtensorMap* tm, const Act8Mat& d, uint64_t rows, uint64_t cols) {
    static const CUtensorMapDataType types[] = {CU_TENSOR_MAP_DATA_TYPE_FLOAT32, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                                                CU_TENSOR_MAP_DATA_TYPE_UINT8, CU_TENSOR_MAP_DATA_TYPE_UINT8};
    const uint32_t es = d.dtype == 0 ? 4 : d.dtype < 3 ? 2 : 1;
    const cuuint64_t dims[2] = {cols, rows}, strides[1] = {rows > 1 ? d.stride : (cols * es + 15) / 16 * 16};
    const cuuint32_t boxes[2] = {64 / es, 32}, unit[2] = {1, 1};
    return tensor_map_encoder()(tm, types[d.dtype], 2, d.data, dims, strides, boxes, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Groups of 512 scale bytes.
bool scales_map(CUtensorMap* tm, const ecq_act8_matrix* m, uint64_t rows, uint64_t k) {
    const cuuint64_t dims[2] = {128, (rows + 127) / 128 * ((k + 511) / 512)}, strides[1] = {512};
    const cuuint32_t boxes[2] = {128, 1}, unit[2] = {1, 1};
    return tensor_map_encoder()(tm, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, m->scales, dims, strides, boxes, unit,
                                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int CG, int TN, bool SWAP>
int launch_part(Product8& P, uint32_t parts, cudaStream_t st) {
    static std::atomic<bool> done[kMaxDevices];
    auto kernel = act8_product_part_kernel<CG, TN, SWAP>;
    using S = ProdPart<CG, TN, SWAP>;
    if (!allow_smem(reinterpret_cast<const void*>(kernel), S::kSmem, done)) return ECQ_ERR_CUDA;
    return launch_act8(kernel, P.tiles * parts * CG, S::kThreads, S::kSmem, parts * CG, st, P);
}

// Clusters of `parts` CTAs (pairs) that the current device holds at once: a cluster stays in a group of SMs, so
// that there may be fewer than SMs would be enough for.
template <int CG>
uint32_t clusters_at_once(uint32_t parts, int dev, int sms) {
    if (parts * CG == 1) return (uint32_t)sms;
    static std::atomic<uint32_t> known[kMaxDevices][4];
    const int at = parts == 1 ? 0 : parts == 2 ? 1 : parts == 4 ? 2 : 3;
    uint32_t have = known[dev][at].load(std::memory_order_acquire);
    if (have) return have;
    using S = ProdPart<CG, 128, false>;
    auto kernel = act8_product_part_kernel<CG, 128, false>;
    static std::atomic<bool> done[kMaxDevices];
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute size;
    size.id = cudaLaunchAttributeClusterDimension;
    size.val.clusterDim.x = parts * CG;
    size.val.clusterDim.y = size.val.clusterDim.z = 1;
    cfg.gridDim = dim3(parts * CG);
    cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.attrs = &size;
    cfg.numAttrs = 1;
    int n = 0;
    if (!allow_smem(reinterpret_cast<const void*>(kernel), S::kSmem, done) || cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
        cudaGetLastError();
        return 0;                                                     // not known: asked again
    }
    have = (uint32_t)std::max(0, n);
    known[dev][at].store(have, std::memory_order_release);
    return have;
}

int launch_pair(Product8& P, uint32_t pairs, cudaStream_t st) {
    static std::atomic<bool> done[kMaxDevices];
    if (!allow_smem(reinterpret_cast<const void*>(act8_product_pair_kernel), ProdPair::kSmem, done)) return ECQ_ERR_CUDA;
    return launch_act8(act8_product_pair_kernel, 2 * std::min(pairs, P.tiles), ProdPair::kThreads, ProdPair::kSmem, 2, st, P);
}

uint32_t up(uint64_t x, uint32_t by) { return (uint32_t)((x + by - 1) / by); }

// Tiles of 256 x 256 by pairs of CTAs that stay (cg 0); or a tile of 128 x 128 a CTA (cg 1) or of 256 x 128 a pair (cg
// 2), K shared out over `parts` of them.  By an estimate of the time in us: a launch, with its first loads and last results; steps of 128
// along K, 0.28 us each where a CTA takes 32 KB (64 bytes a clock), 0.27 in tiles of 256 x 128, for pairs up to 0.48 when all
// SMs load; the sums' way between CTAs; and results that do not go out by TMA (`slow`) or are added to what is there.
// Measured, cg 0, then cg 1 in 1, 2, 4, 8 parts, then cg 2 in 1, 2, 4:
//     1024 x 1024 x 8192   23.7   23.3  15.6  23.1  45.3   22.2  15.3  31.8      300 x 504 x 1000    8.4   7.0  6.3  6.3  7.2   6.6  5.9  6.3
//     128 x 4096 x 4096    14.7   14.0  10.6   9.9  23.8   13.6  11.1  25.5      512 x 4096 x 1024   7.9   7.1 13.7 27.9 62.0   7.8 14.1 33.8
//     the first, added     26.1   29.9  18.8  26.2  51.8   28.8  18.5  36.4      1000 x 2049 x 1537 15.7  13.4 19.8 38.1 74.2  13.3 25.0 40.3
struct Way { uint32_t cg, parts; };

Way choose(uint64_t m, uint64_t n, uint32_t steps, int dev, int sms, bool slow, bool in_place) {
    const uint64_t pairs = (uint64_t)sms / 2, tiles256 = (uint64_t)up(m, 256) * up(n, 256);
    double best = 4.8 + (slow ? 5.0 : in_place ? 2.4 : 0.0) +
                  (double)((tiles256 + pairs - 1) / pairs) * steps * (0.28 + 0.2 * std::min(1.0, (double)tiles256 / (double)pairs));
    Way way = {0, 1};
    for (uint32_t cg = 1; cg <= 2; ++cg)
        for (uint32_t p = 1; p <= (cg == 1 ? 8u : 4u) && p <= steps; p *= 2) {
            const uint64_t clusters = (uint64_t)up(m, 128 * cg) * up(n, 128), ctas = clusters * p * cg;
            if (ctas > (uint64_t)sms || clusters > (cg == 1 ? clusters_at_once<1>(p, dev, sms) : clusters_at_once<2>(p, dev, sms))) break;
            const double t = (p == 1 ? 4.5 : 5.5 + 1.5 * (double)ctas / sms) + (slow ? 4.0 / p : in_place ? 5.0 / p : 0.0) +
                             (double)((steps + p - 1) / p) * (cg == 1 ? 0.28 : 0.27);
            if (t < best) { best = t; way = {cg, p}; }
        }
    return way;
}

}  // namespace

extern "C" {

int ecq_act8_set_wait_limit(uint32_t polls) {
    g_act8_wait_limit.store(polls, std::memory_order_relaxed);
    return ECQ_OK;
}

int ecq_act8_product(uint64_t m, uint64_t n, uint64_t k, const ecq_act8_matrix* a, const ecq_act8_matrix* b,
                     const ecq_act8_matrix* c, const ecq_act8_matrix* d, uint32_t* status, void* cuda_stream) {
    if (!n || !k || bad_size(m, n) || bad_size(m, k) || bad_size(n, k) || bad_matrix(a, m, k, kCoded) || bad_matrix(b, n, k, kCoded) ||
        (c && bad_matrix(c, m, n, kPlain)) || bad_matrix(d, m, n, kAny) || (c && d->dtype >= 3) || !aligned_to(status, 4))
        return ECQ_ERR_ARG;
    if (m == 0) return ECQ_OK;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev >= kMaxDevices ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || !tensor_map_encoder())
        return ECQ_ERR_CUDA;
    Product8 P = {};
    P.out = act8_mat(d, m, n);
    const auto quad = [](const Act8Mat& x) { return aligned_to(x.data, x.dtype ? 8 : 16) && x.stride % (x.dtype ? 8 : 16) == 0; };
    P.out_quad = quad(P.out);
    if (c) {
        const Act8Mat add = act8_mat(c, m, n);
        P.add = add.data;
        P.add_stride = add.stride;
        P.add_dtype = add.dtype;
        P.add_wide = add.wide;
        P.add_quad = quad(add);
    }
    P.status = status;
    P.rows = (uint32_t)m;
    P.cols = (uint32_t)n;
    P.steps = up(k, 128);
    P.tail = up(k - (uint64_t)(P.steps - 1) * 128, 32);
    P.left_groups = P.right_groups = up(k, 512);
    P.wait_limit = g_act8_wait_limit.load(std::memory_order_relaxed);

    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (m == 1 && n * k <= 1u << 23 && d->dtype < 3) {
        Product8Few F = {act8_mat(a, m, k), act8_mat(b, n, k), P.out, P.add, P.add_stride, P.cols, (uint32_t)k, 1, P.add_dtype};
        const uint64_t warps = up(n, kFewRows);
        while (F.split < 8 && F.split * 512u < k && warps * F.split < (uint64_t)sms * 8) F.split *= 2;
        const uint32_t grid = up(warps * F.split, kFewThreads / 32);
        return launch_act8(act8_product_few_kernel, grid, kFewThreads, 0, 0, st, F);
    }
    const bool swap = m <= 64;
    const uint32_t fa = a->dtype == ECQ_E5M2 ? 1u : 0u, fb = b->dtype == ECQ_E5M2 ? 1u : 0u;
    P.formats = swap ? fb << 7 | fa << 10 : fa << 7 | fb << 10;
    uint32_t right_box = 128;
    if (swap) right_box = m <= 16 ? 16 : m <= 32 ? 32 : 64;
    const ecq_act8_matrix *left = swap ? b : a, *right = swap ? a : b;
    const uint64_t left_rows = swap ? n : m, right_rows = swap ? m : n;
    if (!entries_map(&P.left, left, left_rows, k, 128) || !entries_map(&P.right, right, right_rows, k, right_box) ||
        !scales_map(&P.left_scales, left, left_rows, k) || !scales_map(&P.right_scales, right, right_rows, k))
        return ECQ_ERR_CUDA;
    if (swap) {
        P.across = 1;
        P.tiles = up(n, 128);
        uint32_t parts = 1;
        while (parts < 8 && 2 * parts <= P.steps && (uint64_t)P.tiles * parts * 2 <= (uint64_t)sms) parts *= 2;
        return right_box == 16 ? launch_part<1, 16, true>(P, parts, st)
             : right_box == 32 ? launch_part<1, 32, true>(P, parts, st) : launch_part<1, 64, true>(P, parts, st);
    }
    const bool in_place = P.add && P.out.wide && P.add == P.out.data && P.add_stride == P.out.stride && P.add_dtype == 0 && P.out.dtype == 0;
    Way way = {0, 1};
    if (d->dtype < 3) way = choose(m, n, P.steps, dev, sms, !P.out.wide || (P.add && !in_place), in_place);
    P.in_place = in_place && way.cg == 0;
    P.across = up(n, way.cg ? 128 : 256);
    P.tiles = up(m, way.cg == 1 ? 128 : 256) * P.across;
    if (way.cg == 1) return launch_part<1, 128, false>(P, way.parts, st);
    if (way.cg == 2) {
        if (!entries_map(&P.right, b, n, k, 64)) return ECQ_ERR_CUDA;
        return launch_part<2, 128, false>(P, way.parts, st);
    }
    if (P.out.wide && !result_map(&P.result, P.out, m, n)) return ECQ_ERR_CUDA;
    return launch_pair(P, (uint32_t)sms / 2, st);
}

}  // extern "C"
