// Matrices in 8 bits: storing and restoring them, and the operators of a language model's layer that
// write and read them (root-mean-square norm, gated activation, and their gradients).
#pragma once

#include <cstdint>

#include "ecq_act8.cuh"

namespace ecq {

// ---- storing, restoring and the gated activation: tiles of 128 x 128 -----------------------------
//
// Whatever is written in 8 bits transposed has its blocks along the tile's columns, so a CTA has a
// whole tile: a thread four rows of eight columns, 16 lanes a row's block.  All of it is bound by
// memory: each input is read once and each output written once.

enum { kActCopy = 0, kActGate = 1, kActGateGrad = 2 };
constexpr uint32_t kActThreads = 512;

struct Act8Tiles {
    Act8Mat in[2];                       // x; gate and up
    Act8Mat d;                           // gradient of the activation's output
    Act8Mat plain[2], q[2], qt[2];       // results (data NULL: not wanted): h, or d_gate and d_up
    Act8Mat kept[2];                     // gate and up in 8 bits
    uint32_t rows, cols, tiles_across;
};

// 1 / (1 + exp(-x)); WIDE: the rounding of x log2(e) is added back, which shows in 32 bits alone.
template <bool WIDE>
__device__ __forceinline__ float act8_sigmoid(float x) {
    const float t = __fmul_rn(x, -1.44269504088896f);
    float e = ex2(t);
    if (WIDE) {
        float lo = __fmaf_rn(x, -1.44269504088896f, -t);
        lo = __fmaf_rn(x, -1.925963033e-8f, lo);               // log2(e) beyond 24 bits
        e = t > -126.f && t < 126.f ? __fmaf_rn(e, __fmul_rn(lo, 0.693147181f), e) : e;
    }
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(__fadd_rn(1.f, e)));
    return y;
}

// Writes a thread's 4 x 8 results of a tile.
template <typename T>
__device__ __forceinline__ void act8_finish(const Act8Mat& plain, const Act8Mat& q, const Act8Mat& qt, uint32_t rows, uint32_t cols,
                                            uint32_t row0, uint32_t col0, const float (&v)[4][8], unsigned char* turned,
                                            uint32_t (*part)[128], uint32_t* top) {
    const uint32_t tid = threadIdx.x, cg = tid & 15u, rg = tid >> 4, col = col0 + 8 * cg, n = inside(col, cols);
    if (plain.data || q.data) {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const uint32_t row = row0 + 4 * rg + j, m = row < rows ? n : 0;
            if (plain.data && m) put8<T>(plain, row, col, m, v[j]);
            if (q.data) put8_coded(q, row, col, m, v[j], act8_block_max(act8_largest(v[j], 0)));
        }
    }
    if (!qt.data) return;
    // the columns' largest magnitudes: four rows in registers, two groups of rows a warp, 16 warps
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        uint32_t m = 0;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) m = max(m, __float_as_uint(v[j][i]) & 0x7FFFFFFFu);
        m = max(m, __shfl_xor_sync(~0u, m, 16));
        if ((tid & 16u) == 0) part[tid >> 5][8 * cg + i] = m;
    }
    __syncthreads();
    if (tid < 128) {
        uint32_t m = 0;
#pragma unroll
        for (uint32_t w = 0; w < kActThreads / 32; ++w) m = max(m, part[w][tid]);
        const uint32_t byte = act8_byte(m, qt.dtype);
        top[tid] = byte;
        if (col0 + tid < cols) qt.scales[act8_scale_at(col0 + tid, row0 >> 7, qt.groups)] = (uint8_t)byte;
    }
    __syncthreads();
    // The tile turned in shared memory: column c has 128 bytes, its four-byte words exchanged by the
    // group of eight columns so that neither a warp's words nor its 16-byte reads meet in a bank.
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        const uint32_t c = 8 * cg + i;
        const float x[4] = {v[0][i], v[1][i], v[2][i], v[3][i]};
        *reinterpret_cast<uint32_t*>(turned + c * 128u + ((rg ^ (2 * cg)) << 2)) = act8_quad(x, act8_down(top[c]), qt.dtype);
    }
    __syncthreads();
#pragma unroll
    for (uint32_t p = 0; p < 2; ++p) {
        const uint32_t c = (tid >> 3) + 64 * p, piece = tid & 7u, group = c >> 3;
        if (col0 + c >= cols || row0 + 16 * piece >= rows) continue;
        uint4 w = *reinterpret_cast<const uint4*>(turned + c * 128u + ((piece ^ (group >> 1)) << 4));
        if (group & 1u) w = make_uint4(w.z, w.w, w.x, w.y);
        unsigned char* to = qt.data + (uint64_t)(col0 + c) * qt.stride + row0 + 16 * piece;
        const uint32_t left = rows - (row0 + 16 * piece);
        if (left >= 16) {
            *reinterpret_cast<uint4*>(to) = w;
        } else {
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i)
                if (i < left) to[i] = (unsigned char)(u[i >> 2] >> (8 * (i & 3)));
        }
    }
    __syncthreads();                                                 // before the next results come here
}

// S: type of the inputs (uint8_t: either of 8 bits), T: of the plain results and of the gradient.
template <int OP, typename S, typename T>
__global__ void __launch_bounds__(kActThreads, OP == kActGateGrad ? 1 : 2) act8_tile_kernel(const __grid_constant__ Act8Tiles P) {
    __shared__ __align__(16) unsigned char turned[128 * 128];
    __shared__ uint32_t part[kActThreads / 32][128];
    __shared__ uint32_t top[128];
    const uint32_t tile_row = blockIdx.x / P.tiles_across, tile_col = blockIdx.x - tile_row * P.tiles_across;
    const uint32_t row0 = tile_row * 128u, col0 = tile_col * 128u;
    const uint32_t tid = threadIdx.x, cg = tid & 15u, rg = tid >> 4, col = col0 + 8 * cg, n = inside(col, P.cols);
    constexpr bool wide = sizeof(T) == 4;
    griddep_launch();
    griddep_wait();
    Raw8<S> a[4], b[4];
    Raw8<T> d[4];
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
        const uint32_t row = row0 + 4 * rg + j, m = row < P.rows ? n : 0;
        get8<S>(P.in[0], row, col, m, a[j]);
        if (OP != kActCopy) get8<S>(P.in[1], row, col, m, b[j]);
        if (OP == kActGateGrad) get8<T>(P.d, row, col, m, d[j]);
    }
    float v[4][8], u[OP == kActGateGrad ? 4 : 1][8];
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
        widen8<S>(a[j], P.in[0].dtype, v[j]);
        if (OP == kActCopy) continue;
        float x[8], y[8];
        widen8<S>(b[j], P.in[1].dtype, x);
        if (OP == kActGate) {
            const uint32_t row = row0 + 4 * rg + j, m = row < P.rows ? n : 0;
            if (P.kept[0].data) put8_coded(P.kept[0], row, col, m, v[j], act8_block_max(act8_largest(v[j], 0)));
            if (P.kept[1].data) put8_coded(P.kept[1], row, col, m, x, act8_block_max(act8_largest(x, 0)));
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = __fmul_rn(__fmul_rn(v[j][i], act8_sigmoid<wide>(v[j][i])), x[i]);
        } else {
            widen8<T>(d[j], 0, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float g = v[j][i], s = act8_sigmoid<wide>(g), ds = __fmul_rn(y[i], s);
                u[OP == kActGateGrad ? j : 0][i] = __fmul_rn(ds, g);
                v[j][i] = __fmul_rn(__fmul_rn(ds, x[i]), __fmaf_rn(g, __fsub_rn(1.f, s), 1.f));
            }
        }
    }
    act8_finish<T>(P.plain[0], P.q[0], P.qt[0], P.rows, P.cols, row0, col0, v, turned, part, top);
    if constexpr (OP == kActGateGrad) act8_finish<T>(P.plain[1], P.q[1], P.qt[1], P.rows, P.cols, row0, col0, u, turned, part, top);
}

// ---- norm -----------------------------------------------------------------------------------------
//
// A row belongs to `per_row` threads (whole warps, a power of two), NV times eight columns each, and
// stays in their registers: every entry is read once.  CTAs go over the rows with the grid's step, so
// that the weight is read once a CTA.

struct Act8Norm {
    Act8Mat x, residual, sum, y, y8, sum8;
    const void* weight;                  // NULL: ones
    float* rstd;
    int weight_dtype;
    uint32_t rows, cols, per_row;
    float eps, inv_cols;
};

__device__ __forceinline__ void act8_weight(const void* w, int dtype, uint32_t col, uint32_t n, float* x) {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        x[i] = 1.f;
        if (w && i < n)
            x[i] = dtype == 0 ? static_cast<const float*>(w)[col + i]
                 : dtype == 1 ? __bfloat162float(static_cast<const __nv_bfloat16*>(w)[col + i])
                              : __half2float(static_cast<const __half*>(w)[col + i]);
    }
}

// Sum over the threads of a row; `part` has room for a CTA's warps twice, taken in turn.
__device__ __forceinline__ float act8_row_sum(float v, uint32_t per_row, float* part, uint32_t turn) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = __fadd_rn(v, __shfl_xor_sync(~0u, v, o));
    if (per_row == 32) return v;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = per_row >> 5;
    float* mine = part + (turn & 1) * 32;
    if (lane == 0) mine[warp] = v;
    __syncthreads();
    v = lane < warps ? mine[(warp & ~(warps - 1)) + lane] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = __fadd_rn(v, __shfl_xor_sync(~0u, v, o));
    return v;
}

template <typename T, int NV>
__global__ void __launch_bounds__(512) act8_norm_kernel(const __grid_constant__ Act8Norm P) {
    __shared__ float part[64];
    const uint32_t slot = threadIdx.x / P.per_row, t = threadIdx.x - slot * P.per_row, slots = blockDim.x / P.per_row;
    griddep_launch();
    griddep_wait();
    float w[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const uint32_t col = (k * P.per_row + t) * 8;
        act8_weight(P.weight, P.weight_dtype, col, inside(col, P.cols), w[k]);
    }
    uint32_t turn = 0;
    for (uint64_t first = (uint64_t)blockIdx.x * slots; first < P.rows; first += (uint64_t)gridDim.x * slots, ++turn) {
        const uint32_t row = (uint32_t)first + slot;
        const bool real = row < P.rows;
        Raw8<T> a[NV], b[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const uint32_t col = (k * P.per_row + t) * 8, n = real ? inside(col, P.cols) : 0;
            get8<T>(P.x, row, col, n, a[k]);
            if (P.residual.data) get8<T>(P.residual, row, col, n, b[k]);
        }
        float s[NV][8], squares = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            widen8<T>(a[k], 0, s[k]);
            if (P.residual.data) {
                float r[8];
                widen8<T>(b[k], 0, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[k][i] = __fadd_rn(s[k][i], r[i]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) squares = __fmaf_rn(s[k][i], s[k][i], squares);
        }
        squares = act8_row_sum(squares, P.per_row, part, turn);
        const float rstd = __fdiv_rn(1.f, __fsqrt_rn(__fmaf_rn(squares, P.inv_cols, P.eps)));
        if (real && t == 0 && P.rstd) P.rstd[row] = rstd;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const uint32_t col = (k * P.per_row + t) * 8, n = real ? inside(col, P.cols) : 0;
            if (P.sum.data && n) put8<T>(P.sum, row, col, n, s[k]);
            if (P.sum8.data) put8_coded(P.sum8, row, col, n, s[k], act8_block_max(act8_largest(s[k], 0)));
#pragma unroll
            for (int i = 0; i < 8; ++i) s[k][i] = __fmul_rn(__fmul_rn(s[k][i], rstd), w[k][i]);
            if (P.y.data && n) put8<T>(P.y, row, col, n, s[k]);
            if (P.y8.data) put8_coded(P.y8, row, col, n, s[k], act8_block_max(act8_largest(s[k], 0)));
        }
    }
}

// Its gradient.  With n = s rstd and g = d_out w:  d_x = rstd (g - n mean(g n)) + d_sum, and the weight's
// gradient is the sum over the rows of d_out n: each thread adds its columns' in registers over the
// rows that it has, and a second launch adds these sums in a fixed order.
struct Act8NormGrad {
    Act8Mat s, d_out, d_sum, d_x;
    const void* weight;
    const float* rstd;
    float* sums;                         // [grid x rows at a time][cols], or NULL
    int weight_dtype;
    uint32_t rows, cols, per_row;
    float inv_cols;
};

template <typename S, typename T, int NV>
__global__ void __launch_bounds__(512) act8_norm_grad_kernel(const __grid_constant__ Act8NormGrad P) {
    __shared__ float part[64];
    const uint32_t slot = threadIdx.x / P.per_row, t = threadIdx.x - slot * P.per_row, slots = blockDim.x / P.per_row;
    griddep_launch();
    griddep_wait();
    float w[NV][8], dw[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const uint32_t col = (k * P.per_row + t) * 8;
        act8_weight(P.weight, P.weight_dtype, col, inside(col, P.cols), w[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[k][i] = 0.f;
    }
    uint32_t turn = 0;
    for (uint64_t first = (uint64_t)blockIdx.x * slots; first < P.rows; first += (uint64_t)gridDim.x * slots, ++turn) {
        const uint32_t row = (uint32_t)first + slot;
        const bool real = row < P.rows;
        Raw8<S> a[NV];
        Raw8<T> b[NV], c[NV];
        const float rstd = real ? P.rstd[row] : 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const uint32_t col = (k * P.per_row + t) * 8, n = real ? inside(col, P.cols) : 0;
            get8<S>(P.s, row, col, n, a[k]);
            get8<T>(P.d_out, row, col, n, b[k]);
            if (P.d_sum.data) get8<T>(P.d_sum, row, col, n, c[k]);
        }
        float normed[NV][8], g[NV][8], dot = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            widen8<S>(a[k], P.s.dtype, normed[k]);
            widen8<T>(b[k], 0, g[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                normed[k][i] = __fmul_rn(normed[k][i], rstd);
                dw[k][i] = __fmaf_rn(g[k][i], normed[k][i], dw[k][i]);
                g[k][i] = __fmul_rn(g[k][i], w[k][i]);
                dot = __fmaf_rn(g[k][i], normed[k][i], dot);
            }
        }
        const float mean = __fmul_rn(act8_row_sum(dot, P.per_row, part, turn), P.inv_cols);
        if (!P.d_x.data) continue;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const uint32_t col = (k * P.per_row + t) * 8, n = real ? inside(col, P.cols) : 0;
            float x[8];
            if (P.d_sum.data) widen8<T>(c[k], 0, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = __fmaf_rn(-normed[k][i], mean, g[k][i]);
                x[i] = P.d_sum.data ? __fmaf_rn(rstd, d, x[i]) : __fmul_rn(rstd, d);
            }
            if (n) put8<T>(P.d_x, row, col, n, x);
        }
    }
    if (!P.sums) return;
    float* to = P.sums + ((uint64_t)blockIdx.x * slots + slot) * P.cols;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const uint32_t col = (k * P.per_row + t) * 8;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (col + i < P.cols) to[col + i] = dw[k][i];
    }
}

// Columns of `count` vectors added: 32 columns a CTA, 16 threads a column.
__global__ void __launch_bounds__(512) act8_add_kernel(const float* sums, uint32_t count, uint32_t cols, float* out) {
    __shared__ float part[16][33];
    const uint32_t col = blockIdx.x * 32u + (threadIdx.x & 31u), lane = threadIdx.x & 31u, row = threadIdx.x >> 5;
    griddep_wait();
    float v = 0.f;
    if (col < cols)
#pragma unroll 4
        for (uint32_t i = row; i < count; i += 16) v = __fadd_rn(v, sums[(uint64_t)i * cols + col]);
    part[row][lane] = v;
    __syncthreads();
    if (row || col >= cols) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) v = __fadd_rn(v, part[i][lane]);
    out[col] = v;
}

}  // namespace ecq
