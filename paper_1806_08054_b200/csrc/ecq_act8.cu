// C ABI of the operators on matrices in 8 bits, the products apart: argument checks and launches.
#include <atomic>
#include <cfloat>
#include <cstdint>

#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/ecq.h"
#include "ecq_act8_host.h"
#include "ecq_act8_kernels.cuh"

using namespace ecq;

namespace {

int sm_count(int& sms) {
    int dev = 0;
    return cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess
               ? ECQ_OK : ECQ_ERR_CUDA;
}

// ---- tiles
// Boxes of 128 x 128.
bool tile_map(CUtensorMap* tm, const Act8Mat& m, uint64_t rows, uint64_t cols) {
    static const CUtensorMapDataType types[] = {CU_TENSOR_MAP_DATA_TYPE_FLOAT32, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                                                CU_TENSOR_MAP_DATA_TYPE_UINT8, CU_TENSOR_MAP_DATA_TYPE_UINT8};
    const cuuint64_t dims[2] = {cols, rows}, strides[1] = {m.stride};
    const cuuint32_t boxes[2] = {128, 128}, unit[2] = {1, 1};
    return tensor_map_encoder()(tm, types[m.dtype], 2, m.data, dims, strides, boxes, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int OP, typename S, typename T>
int launch_tiles(Act8Tiles& P, cudaStream_t st) {
    using R = Act8Ring<OP, S, T>;
    int sms = 0;
    if (sm_count(sms) != ECQ_OK) return ECQ_ERR_CUDA;
    // Tiles ahead of their turn where a CTA has several.  A tile a CTA, and that, in us: 8192 x 4096 from 8 to 8 bits transposed 24.8, 21.5;
    // restored 19.7, 18.7; gate gradient 59, 46.5.  8192 x 1024: 7.0, 7.8; 6.3, 7.2; 18.2, 17.2.
    const uint32_t ctas = (uint32_t)sms * R::kCtas;
    if constexpr (R::kStages > 0) {
        static std::atomic<bool> done[kMaxDevices];
        auto kernel = act8_tiles_kernel<OP, S, T>;
        Act8Maps maps = {};
        // With room for one alone: where results are in 8 bits, two or more, and work is long: transposed, or four tiles a CTA.  Without and
        // with, in us, 8192 x 4096 and 8192 x 1024 (3.5 tiles a CTA): gradient from bf16, both results both ways 82.5, 66.7; 25.0, 22.8, in 8
        // bits 55.0, 49.3; 17.6, 17.9, to bf16 54.5, 55.5; 16.6, 18.9, to bf16 and transposed 78.2, 75.2; 23.4, 23.6; gradient to 32 bits from
        // 8, both ways 92.2, 79.6; 28.6, 26.1, plain 95.9, 95.4; 28.4, 31.6; gate in 32 bits, inputs kept 73.6, 67.6; 23.7, 23.8, and
        // transposed 89.9, 75.5; 27.6, 26.0, to 8 bits alone 55.6, 65.9; 18.4, 21.2.
        const int turned = (P.qt[0].data != nullptr) + (P.qt[1].data != nullptr);
        const int coded = turned + (P.q[0].data != nullptr) + (P.q[1].data != nullptr) + (P.kept[0].data != nullptr) + (P.kept[1].data != nullptr);
        const bool ahead = R::kStages > 1 || (coded >= 2 && !P.plain[0].data && !P.plain[1].data);
        const uint32_t least = R::kCtas == 1 && (R::kStages > 1 || turned) ? 2 : 4;
        if (ahead && P.wide && P.rows >= 128 && P.cols >= 128 && P.tiles >= least * ctas) {
            if (!tensor_map_encoder() || !tile_map(&maps.of[0], P.in[0], P.rows, P.cols) ||
                (OP != kActCopy && !tile_map(&maps.of[1], P.in[1], P.rows, P.cols)) ||
                (OP == kActGateGrad && !tile_map(&maps.of[2], P.d, P.rows, P.cols)) ||
                !allow_smem(reinterpret_cast<const void*>(kernel), R::kSmem, done))
                return ECQ_ERR_CUDA;
            return launch_act8(kernel, ctas, kActThreads, R::kSmem, 0, st, P, maps);
        }
    }
    // Parts of tiles where there are few (a row of 4096 restored 2.4 -> 2.0 us, gate gradient of 777 x 2816 8.4 -> 7.3; gate of 8192 x
    // 1024 in 512 tiles 16.6 -> 18.8).
    if (!P.qt[0].data && !P.qt[1].data && P.tiles <= 2 * (uint32_t)sms)
        return launch_act8(act8_tile_kernel<OP, S, T>, (P.rows + 31) / 32 * P.tiles_across, kActThreads / 4, 0, 0, st, P);
    return launch_act8(act8_tile_kernel<OP, S, T>, P.tiles, kActThreads, 0, 0, st, P);
}
template <int OP, typename T>
int launch_tiles(Act8Tiles& P, bool coded, cudaStream_t st) {
    return coded ? launch_tiles<OP, uint8_t, T>(P, st) : launch_tiles<OP, T, T>(P, st);
}
// `plain`: the type of the plain matrices (16 bits where there are none, as nothing needs 32 then).
template <int OP>
int launch_tiles(Act8Tiles& P, uint64_t rows, uint64_t cols, int plain, bool coded, void* stream) {
    P.rows = (uint32_t)rows;
    P.cols = (uint32_t)cols;
    P.tiles_across = (uint32_t)((cols + 127) / 128);
    P.tiles = (P.rows + 127) / 128 * P.tiles_across;
    P.wait_limit = g_act8_wait_limit.load(std::memory_order_relaxed);
    P.wide = 1;
    for (const Act8Mat* m : {&P.in[0], &P.in[1], &P.d, &P.plain[0], &P.plain[1]}) P.wide &= !m->data || m->wide;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    switch (plain) {
        case ECQ_F32: return launch_tiles<OP, float>(P, coded, st);
        case ECQ_BF16: return launch_tiles<OP, __nv_bfloat16>(P, coded, st);
        default: return launch_tiles<OP, __half>(P, coded, st);
    }
}

// ---- norm: threads of a row, whole warps up to 512, and vectors of eight columns of each
struct RowShape { uint32_t per_row, per_cta; int vectors; };
RowShape row_shape(uint64_t rows, uint64_t cols, int sms) {
    const uint32_t eights = (uint32_t)((cols + 7) / 8);
    // few rows: one vector a thread, and more threads; many: two
    RowShape s = {0, 0, rows * eights <= (uint64_t)sms * 512 ? 1 : 2};
    while (512 * (uint32_t)s.vectors < eights) s.vectors *= 2;
    s.per_row = (eights + 32 * (uint32_t)s.vectors - 1) / (32 * (uint32_t)s.vectors) * 32;
    s.per_cta = s.per_row > 128 || rows == 1 ? s.per_row : 256 / s.per_row * s.per_row;
    return s;
}

template <typename T, int NV>
int launch_norm(Act8Norm& P, const RowShape& s, int sms, cudaStream_t st) {
    const uint64_t slots = s.per_cta / s.per_row, need = (P.rows + slots - 1) / slots;
    uint64_t most = (uint64_t)sms * (1024 / s.per_cta);
    // Two rows ahead where a CTA has several: of 16-bit entries, where rows are so long that
    // few are worked on at a time, or where no time goes into 8 bits.  Without and with, in us, x and residual to sum and 8 bits:
    // 2048 x 16384 50.7, 39.7, 4096 x 8192 43.2, 40.4, 8192 x 4096 41.2, 41.9; x alone to 16 bits: 2048 x 16384 40.6, 25.9,
    // 8192 x 4096 30.5, 26.2, 8192 x 1024 10.6, 9.4, 8192 x 512 6.1, 6.4.  8192 x 4096 in 32 bits with a residual 73, 103 (half
    // the threads have room).
    if constexpr (sizeof(T) == 2 && NV > 1) {
        if (P.full && need > most && (s.per_row > 256 || (s.per_row >= 64 && !P.y8.data && !P.sum8.data))) {
            constexpr uint32_t kRoom = 192u * 1024u;                  // what an SM's CTAs take at most
            static std::atomic<bool> done[kMaxDevices];
            auto kernel = act8_norm_ahead_kernel<T, NV>;
            const uint32_t ctas = (NV == 4 ? 512 : 1024) / s.per_cta, row = s.per_cta * NV * 16 * (P.residual.data ? 2 : 1);
            most = (uint64_t)sms * ctas;
            if (!allow_smem(reinterpret_cast<const void*>(kernel), kRoom, done)) return ECQ_ERR_CUDA;
            return launch_act8(kernel, (uint32_t)(need < most ? need : most), s.per_cta, kNormStages * row, 0, st, P);
        }
    }
    return launch_act8(act8_norm_kernel<T, NV>, (uint32_t)(need < most ? need : most), s.per_cta, 0, 0, st, P);
}
template <typename T>
int launch_norm(Act8Norm& P, const RowShape& s, int sms, cudaStream_t st) {
    return s.vectors == 1 ? launch_norm<T, 1>(P, s, sms, st) : s.vectors == 2 ? launch_norm<T, 2>(P, s, sms, st) : launch_norm<T, 4>(P, s, sms, st);
}

uint32_t grad_grid(uint64_t rows, const RowShape& s, int sms) {
    const uint64_t slots = s.per_cta / s.per_row, need = (rows + slots - 1) / slots, most = (uint64_t)sms * (512 / s.per_cta);
    return (uint32_t)(need < most ? need : most);
}

template <typename S, typename T, int NV>
int launch_norm_grad(Act8NormGrad& P, const RowShape& s, uint32_t grid, cudaStream_t st) {
    static std::atomic<bool> done[kMaxDevices];
    auto kernel = act8_norm_grad_kernel<S, T, NV>;
    constexpr uint32_t kRoom = 208u * 1024u;                          // an SM's, for 512 threads
    const uint32_t ahead = 2 * s.per_cta * NormRead<S, T, NV>::kBytes, sums = s.per_cta > s.per_row ? s.per_cta * NV * 32 : 0;
    P.full &= ahead * (512 / s.per_cta) <= kRoom;
    const uint32_t smem = P.full && ahead > sums ? ahead : sums;
    if (!allow_smem(reinterpret_cast<const void*>(kernel), kRoom, done)) return ECQ_ERR_CUDA;
    return launch_act8(kernel, grid, s.per_cta, smem, 0, st, P);
}
template <typename S, typename T>
int launch_norm_grad(Act8NormGrad& P, const RowShape& s, uint32_t grid, cudaStream_t st) {
    return s.vectors == 1 ? launch_norm_grad<S, T, 1>(P, s, grid, st)
         : s.vectors == 2 ? launch_norm_grad<S, T, 2>(P, s, grid, st) : launch_norm_grad<S, T, 4>(P, s, grid, st);
}
template <typename T>
int launch_norm_grad(Act8NormGrad& P, const RowShape& s, uint32_t grid, bool coded, cudaStream_t st) {
    return coded ? launch_norm_grad<uint8_t, T>(P, s, grid, st) : launch_norm_grad<T, T>(P, s, grid, st);
}

// Plain matrices of a call have one type.
bool same_type(int& type, const ecq_act8_matrix* m) {
    if (!m || m->dtype >= 3) return true;
    if (type >= 0 && type != m->dtype) return false;
    type = m->dtype;
    return true;
}

bool bad_weight(const void* w, int dtype) { return w && (!dtype_bytes(dtype) || !aligned_to(w, dtype_bytes(dtype))); }

}  // namespace

extern "C" {

uint64_t ecq_act8_scale_bytes(uint64_t rows, uint64_t cols) {
    if (rows > kActMaxSide || cols > kActMaxSide) return 0;
    return (rows + 127) / 128 * ((cols + 511) / 512) * 512;
}

int ecq_act8_store(uint64_t rows, uint64_t cols, const ecq_act8_matrix* x, const ecq_act8_matrix* q, const ecq_act8_matrix* q_t,
                   void* cuda_stream) {
    if (bad_size(rows, cols) || (!q && !q_t) || bad_matrix(x, rows, cols, kAny) || (q && bad_matrix(q, rows, cols, kCoded)) ||
        (q_t && bad_matrix(q_t, cols, rows, kCoded)))
        return ECQ_ERR_ARG;
    if (rows == 0) return ECQ_OK;
    Act8Tiles P = {};
    P.in[0] = act8_mat(x, rows, cols);
    P.q[0] = act8_mat(q, rows, cols);
    P.qt[0] = act8_mat(q_t, cols, rows);
    return launch_tiles<kActCopy>(P, rows, cols, x->dtype < 3 ? x->dtype : ECQ_BF16, x->dtype >= 3, cuda_stream);
}

int ecq_act8_load(uint64_t rows, uint64_t cols, const ecq_act8_matrix* q, const ecq_act8_matrix* x, void* cuda_stream) {
    if (bad_size(rows, cols) || bad_matrix(q, rows, cols, kCoded) || bad_matrix(x, rows, cols, kPlain)) return ECQ_ERR_ARG;
    if (rows == 0) return ECQ_OK;
    Act8Tiles P = {};
    P.in[0] = act8_mat(q, rows, cols);
    P.plain[0] = act8_mat(x, rows, cols);
    return launch_tiles<kActCopy>(P, rows, cols, x->dtype, true, cuda_stream);
}

int ecq_act8_gate(uint64_t rows, uint64_t cols, const ecq_act8_matrix* gate, const ecq_act8_matrix* up, const ecq_act8_matrix* out,
                  const ecq_act8_matrix* out8, const ecq_act8_matrix* out8_t, const ecq_act8_matrix* gate8,
                  const ecq_act8_matrix* up8, void* cuda_stream) {
    if (bad_size(rows, cols) || bad_matrix(gate, rows, cols, kAny) || bad_matrix(up, rows, cols, kAny) || gate->dtype != up->dtype)
        return ECQ_ERR_ARG;
    if ((out && bad_matrix(out, rows, cols, kPlain)) || (out8 && bad_matrix(out8, rows, cols, kCoded)) ||
        (out8_t && bad_matrix(out8_t, cols, rows, kCoded)) || (gate8 && bad_matrix(gate8, rows, cols, kCoded)) ||
        (up8 && bad_matrix(up8, rows, cols, kCoded)) || (!out && !out8 && !out8_t && !gate8 && !up8))
        return ECQ_ERR_ARG;
    int type = -1;
    if (!same_type(type, gate) || !same_type(type, out)) return ECQ_ERR_ARG;
    if (rows == 0) return ECQ_OK;
    Act8Tiles P = {};
    P.in[0] = act8_mat(gate, rows, cols);
    P.in[1] = act8_mat(up, rows, cols);
    P.plain[0] = act8_mat(out, rows, cols);
    P.q[0] = act8_mat(out8, rows, cols);
    P.qt[0] = act8_mat(out8_t, cols, rows);
    P.kept[0] = act8_mat(gate8, rows, cols);
    P.kept[1] = act8_mat(up8, rows, cols);
    return launch_tiles<kActGate>(P, rows, cols, type < 0 ? ECQ_BF16 : type, gate->dtype >= 3, cuda_stream);
}

int ecq_act8_gate_grad(uint64_t rows, uint64_t cols, const ecq_act8_matrix* gate, const ecq_act8_matrix* up,
                       const ecq_act8_matrix* d_out, const ecq_act8_matrix* d_gate, const ecq_act8_matrix* d_up,
                       const ecq_act8_matrix* d_gate8, const ecq_act8_matrix* d_gate8_t, const ecq_act8_matrix* d_up8,
                       const ecq_act8_matrix* d_up8_t, void* cuda_stream) {
    if (bad_size(rows, cols) || bad_matrix(gate, rows, cols, kAny) || bad_matrix(up, rows, cols, kAny) ||
        gate->dtype != up->dtype || bad_matrix(d_out, rows, cols, kPlain))
        return ECQ_ERR_ARG;
    if ((d_gate && bad_matrix(d_gate, rows, cols, kPlain)) || (d_up && bad_matrix(d_up, rows, cols, kPlain)) ||
        (d_gate8 && bad_matrix(d_gate8, rows, cols, kCoded)) || (d_gate8_t && bad_matrix(d_gate8_t, cols, rows, kCoded)) ||
        (d_up8 && bad_matrix(d_up8, rows, cols, kCoded)) || (d_up8_t && bad_matrix(d_up8_t, cols, rows, kCoded)) ||
        (!d_gate && !d_up && !d_gate8 && !d_gate8_t && !d_up8 && !d_up8_t))
        return ECQ_ERR_ARG;
    int type = d_out->dtype;
    if (!same_type(type, gate) || !same_type(type, d_gate) || !same_type(type, d_up)) return ECQ_ERR_ARG;
    if (rows == 0) return ECQ_OK;
    Act8Tiles P = {};
    P.in[0] = act8_mat(gate, rows, cols);
    P.in[1] = act8_mat(up, rows, cols);
    P.d = act8_mat(d_out, rows, cols);
    P.plain[0] = act8_mat(d_gate, rows, cols);
    P.plain[1] = act8_mat(d_up, rows, cols);
    P.q[0] = act8_mat(d_gate8, rows, cols);
    P.q[1] = act8_mat(d_up8, rows, cols);
    P.qt[0] = act8_mat(d_gate8_t, cols, rows);
    P.qt[1] = act8_mat(d_up8_t, cols, rows);
    return launch_tiles<kActGateGrad>(P, rows, cols, type, gate->dtype >= 3, cuda_stream);
}

int ecq_act8_norm(uint64_t rows, uint64_t cols, const ecq_act8_matrix* x, const ecq_act8_matrix* residual, const void* weight,
                  int weight_dtype, float eps, const ecq_act8_matrix* sum, const ecq_act8_matrix* out, const ecq_act8_matrix* out8,
                  const ecq_act8_matrix* sum8, float* rstd, void* cuda_stream) {
    if (bad_size(rows, cols) || cols > ECQ_ACT8_NORM_MAX_COLS || bad_matrix(x, rows, cols, kPlain) ||
        (residual && bad_matrix(residual, rows, cols, kPlain)) || bad_weight(weight, weight_dtype) || !(eps >= 0.f && eps <= FLT_MAX))
        return ECQ_ERR_ARG;
    if ((sum && bad_matrix(sum, rows, cols, kPlain)) || (out && bad_matrix(out, rows, cols, kPlain)) ||
        (out8 && bad_matrix(out8, rows, cols, kCoded)) || (sum8 && bad_matrix(sum8, rows, cols, kCoded)) || !aligned_to(rstd, 4) ||
        (!sum && !out && !out8 && !sum8 && !rstd))
        return ECQ_ERR_ARG;
    int type = x->dtype;
    if (!same_type(type, residual) || !same_type(type, sum) || !same_type(type, out)) return ECQ_ERR_ARG;
    if (rows == 0) return ECQ_OK;
    int sms = 0;
    if (sm_count(sms) != ECQ_OK) return ECQ_ERR_CUDA;
    const RowShape s = row_shape(rows, cols, sms);
    Act8Norm P = {};
    P.x = act8_mat(x, rows, cols);
    P.residual = act8_mat(residual, rows, cols);
    P.sum = act8_mat(sum, rows, cols);
    P.y = act8_mat(out, rows, cols);
    P.y8 = act8_mat(out8, rows, cols);
    P.sum8 = act8_mat(sum8, rows, cols);
    P.weight = weight;
    P.weight_dtype = weight_dtype;
    P.rstd = rstd;
    P.rows = (uint32_t)rows;
    P.cols = (uint32_t)cols;
    P.per_row = s.per_row;
    P.eps = eps;
    P.inv_cols = (float)(1.0 / (double)cols);
    P.full = cols % 8 == 0;
    for (const Act8Mat* m : {&P.x, &P.residual, &P.sum, &P.y}) P.full &= !m->data || m->wide;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    switch (type) {
        case ECQ_F32: return launch_norm<float>(P, s, sms, st);
        case ECQ_BF16: return launch_norm<__nv_bfloat16>(P, s, sms, st);
        default: return launch_norm<__half>(P, s, sms, st);
    }
}

uint64_t ecq_act8_norm_grad_workspace_bytes(uint64_t rows, uint64_t cols) {
    int sms = 0;
    if (bad_size(rows, cols) || cols > ECQ_ACT8_NORM_MAX_COLS || sm_count(sms) != ECQ_OK) return 0;
    const RowShape s = row_shape(rows, cols, sms);
    return (uint64_t)grad_grid(rows, s, sms) * ((cols + 7) / 8 * 8) * sizeof(float);
}

int ecq_act8_norm_grad(uint64_t rows, uint64_t cols, const ecq_act8_matrix* sum, const void* weight, int weight_dtype,
                       const float* rstd, const ecq_act8_matrix* d_out, const ecq_act8_matrix* d_sum, const ecq_act8_matrix* d_x,
                       float* d_weight, void* workspace, uint64_t workspace_bytes, void* cuda_stream) {
    if (bad_size(rows, cols) || cols > ECQ_ACT8_NORM_MAX_COLS || bad_matrix(sum, rows, cols, kAny) || bad_weight(weight, weight_dtype) ||
        (rows && !rstd) || !aligned_to(rstd, 4) || bad_matrix(d_out, rows, cols, kPlain) || (d_sum && bad_matrix(d_sum, rows, cols, kPlain)) ||
        (d_x && bad_matrix(d_x, rows, cols, kPlain)) || !aligned_to(d_weight, 4) || (!d_x && !d_weight) ||
        (d_weight && rows && (!workspace || !aligned_to(workspace, 16))))
        return ECQ_ERR_ARG;
    int type = d_out->dtype;
    if (!same_type(type, sum) || !same_type(type, d_sum) || !same_type(type, d_x)) return ECQ_ERR_ARG;
    int sms = 0;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (rows == 0) {
        if (!d_weight) return ECQ_OK;
        return launch_act8(act8_add_kernel, (uint32_t)((cols + 31) / 32), 1024, 0, 0, st, (const float*)nullptr, 0u, 0u, (uint32_t)cols, d_weight);
    }
    if (sm_count(sms) != ECQ_OK) return ECQ_ERR_CUDA;
    const RowShape s = row_shape(rows, cols, sms);
    const uint32_t grid = grad_grid(rows, s, sms), pitch = (uint32_t)((cols + 7) / 8 * 8);
    if (d_weight && workspace_bytes < (uint64_t)grid * pitch * sizeof(float)) return ECQ_ERR_ARG;
    Act8NormGrad P = {};
    P.s = act8_mat(sum, rows, cols);
    P.d_out = act8_mat(d_out, rows, cols);
    P.d_sum = act8_mat(d_sum, rows, cols);
    P.d_x = act8_mat(d_x, rows, cols);
    P.weight = weight;
    P.weight_dtype = weight_dtype;
    P.rstd = rstd;
    P.sums = d_weight ? static_cast<float*>(workspace) : nullptr;
    P.rows = (uint32_t)rows;
    P.cols = (uint32_t)cols;
    P.per_row = s.per_row;
    P.pitch = pitch;
    P.inv_cols = (float)(1.0 / (double)cols);
    P.full = cols % 8 == 0;
    for (const Act8Mat* m : {&P.s, &P.d_out, &P.d_sum, &P.d_x}) P.full &= !m->data || m->wide;
    const bool coded = sum->dtype >= 3;
    int rc;
    switch (type) {
        case ECQ_F32: rc = launch_norm_grad<float>(P, s, grid, coded, st); break;
        case ECQ_BF16: rc = launch_norm_grad<__nv_bfloat16>(P, s, grid, coded, st); break;
        default: rc = launch_norm_grad<__half>(P, s, grid, coded, st); break;
    }
    if (rc != ECQ_OK || !d_weight) return rc;
    return launch_act8(act8_add_kernel, (uint32_t)((cols + 31) / 32), 1024, 0, 0, st, (const float*)P.sums, grid, pitch, (uint32_t)cols, d_weight);
}

}  // extern "C"
