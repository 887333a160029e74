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

std::atomic<uint32_t> g_wait_limit{kWaitLimit};

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

int launch_pair(Product8& P, uint32_t pairs, cudaStream_t st) {
    static std::atomic<bool> done[kMaxDevices];
    if (!allow_smem(reinterpret_cast<const void*>(act8_product_pair_kernel), ProdPair::kSmem, done)) return ECQ_ERR_CUDA;
    return launch_act8(act8_product_pair_kernel, 2 * std::min(pairs, P.tiles), ProdPair::kThreads, ProdPair::kSmem, 2, st, P);
}

uint32_t up(uint64_t x, uint32_t by) { return (uint32_t)((x + by - 1) / by); }

// Tiles of 256 x 256 by pairs of CTAs with all of K (cg 0), or K shared out over `parts` CTAs (cg 1, tiles of 128
// x 128) or pairs (cg 2), by an estimate of the time in us.  A launch; steps of 128 along K, 32 KB a CTA: 0.28 us each
// (the 64 bytes a clock that an SM takes), up to 0.48 where all SMs load; where K is shared the sums'
// way through shared memory; and results that do not go out by TMA (`slow`), or that are added to what is there.  Measured (pairs, 128 x 128
// in 2, 4, 8 parts, pairs in 2):
//     1024 x 1024 x 8192     24.0   16.9   25.7   51.4   18.5       128 x 4096 x 1024    6.9    7.1    7.4   20.0    9.2
//     300 x 500 x 1000, slow 10.3    9.4    7.9    8.4   13.6       128 x 4096 x 4096   15.2   11.9   11.4   26.4   14.2
void choose(uint64_t tiles256, uint64_t tiles128, uint32_t steps, int sms, bool slow, bool in_place, int& cg, uint32_t& parts) {
    const uint64_t pairs = (uint64_t)sms / 2;
    double best = 3.9 + (slow ? 4.0 : in_place ? 2.0 : 0.0) +
                  (double)((tiles256 + pairs - 1) / pairs) * steps * (0.28 + 0.2 * std::min(1.0, (double)tiles256 / (double)pairs));
    for (int way = 1; way <= 2; ++way)
        for (uint32_t p = 2; p <= (way == 1 ? 8u : 2u) && 2 * p <= steps; p *= 2) {
            const uint64_t ctas = way == 1 ? tiles128 * p : tiles256 * p * 2;
            if (ctas > (uint64_t)sms) break;
            const double t = (way == 1 ? 6.7 : 8.5) + (slow ? (way == 1 ? 10.0 / p : 14.0) : in_place ? 1.3 : 0.0) + (double)((steps + p - 1) / p) * (0.28 + 0.04 * (double)ctas / sms);
            if (t < best) { best = t; cg = way; parts = p; }
        }
}

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
    P.wait_limit = g_wait_limit.load(std::memory_order_relaxed);

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
    const uint64_t tiles256 = (uint64_t)up(m, 256) * up(n, 256), tiles128 = (uint64_t)up(m, 128) * up(n, 128);
    int cg = 0;
    uint32_t parts = 1;
    const bool in_place = P.add && P.out.wide && P.add == P.out.data && P.add_stride == P.out.stride && P.add_dtype == 0 && P.out.dtype == 0;
    if (d->dtype < 3) choose(tiles256, tiles128, P.steps, sms, !P.out.wide || (P.add && !in_place), in_place, cg, parts);
    P.in_place = in_place;
    const uint32_t side = cg == 1 ? 128 : 256;
    P.across = up(n, side);
    P.tiles = (uint32_t)(cg == 1 ? tiles128 : tiles256);
    if (cg == 0 && P.out.wide && !result_map(&P.result, P.out, m, n)) return ECQ_ERR_CUDA;
    return cg == 0 ? launch_pair(P, (uint32_t)sms / 2, st) : cg == 1 ? launch_part<1, 128, false>(P, parts, st) : launch_part<2, 256, false>(P, parts, st);
}

}  // extern "C"
