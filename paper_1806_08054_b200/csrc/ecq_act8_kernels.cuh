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
    int wide;                            // rows of all plain matrices begin on 16-byte boundaries
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

// A thread's place in a tile of a matrix: four rows, eight columns.
struct Act8Place {
    uint32_t rows, n;                    // rows and columns that are inside
    uint32_t row, col;                   // the first
};

template <bool FULL, typename T>
__device__ __forceinline__ void act8_put_plain(const Act8Mat& m, const Act8Place& at, const float (&v)[4][8]) {
    unsigned char* p = m.data + at.row * m.stride + (uint64_t)at.col * sizeof(T);
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j, p += m.stride)
        if (FULL || j < at.rows) put8<FULL, T>(p, at.n, m.wide, v[j]);
}

// Two of a thread's rows, the j-th and the next.
template <bool FULL>
__device__ __forceinline__ void act8_put_coded(const Act8Mat& m, const Act8Place& at, uint32_t j, const float* v, const float* w) {
    const uint32_t bytes = act8_agree(act8_byte(act8_largest(v), m.dtype) | act8_byte(act8_largest(w), m.dtype) << 16);
    unsigned char* p = m.data + (at.row + j) * m.stride + at.col;
    uint8_t* s = m.scales + act8_scale_at(at.row, at.col >> 7, m.groups) + 16 * j;   // four rows never leave a group of 32
    const bool first = (at.col & 127u) == 0;
    if (FULL || j < at.rows) put8_coded<FULL>(p, s, at.n, first, m.dtype, bytes & 255u, v);
    if (FULL || j + 1 < at.rows) put8_coded<FULL>(p + m.stride, s + 16, at.n, first, m.dtype, bytes >> 16, w);
}

template <bool FULL, typename T>
__device__ __forceinline__ void act8_get(const Act8Mat& m, const Act8Place& at, Raw8<T> (&r)[4]) {
    const unsigned char* p = m.data + at.row * m.stride + (uint64_t)at.col * sizeof(T);
    const uint8_t* s = sizeof(T) == 1 ? m.scales + act8_scale_at(at.row, at.col >> 7, m.groups) : nullptr;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j, p += m.stride, s += 16) get8<FULL>(p, s, FULL || j < at.rows ? at.n : 0, m.wide, r[j]);
}

// A thread's 4 x 8 results in 8 bits transposed; the whole CTA.
struct Act8Turn {
    unsigned char turned[128 * 128];
    uint32_t part[kActThreads / 32][128];
    float down[128];
};
template <bool FULL>
__device__ __forceinline__ void act8_put_turned(const Act8Mat& m, const Act8Place& at, uint32_t rows, uint32_t cols,
                                                const float (&v)[4][8], Act8Turn& t) {
    const uint32_t tid = threadIdx.x, cg = tid & 15u, rg = tid >> 4, row0 = at.row - 4 * rg, col0 = at.col - 8 * cg;
    // the columns' largest magnitudes: four rows in registers, two groups of rows a warp, 16 warps
    uint32_t big[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        const float x = top3(top3(v[0][i], v[1][i], v[2][i]), v[3][i], 0.f);
        big[i] = __float_as_uint(top3(x, __shfl_xor_sync(~0u, x, 16), 0.f));
    }
    if ((tid & 16u) == 0) {
        uint4* to = reinterpret_cast<uint4*>(&t.part[tid >> 5][8 * cg]);
        to[0] = make_uint4(big[0], big[1], big[2], big[3]);
        to[1] = make_uint4(big[4], big[5], big[6], big[7]);
    }
    __syncthreads();
    if (tid < 128) {
        uint32_t top = 0;
#pragma unroll
        for (uint32_t w = 0; w < kActThreads / 32; ++w) top = max(top, t.part[w][tid]);
        const uint32_t byte = act8_byte(top, m.dtype);
        t.down[tid] = act8_down(byte);
        if (FULL || col0 + tid < cols) m.scales[act8_scale_at(col0 + tid, row0 >> 7, m.groups)] = (uint8_t)byte;
    }
    __syncthreads();
    // The tile turned in shared memory: column c has 128 bytes, its four-byte words exchanged by the
    // group of eight columns so that neither a warp's words nor its 16-byte reads meet in a bank.
    float down[8];
    Elem<float>::widen(*reinterpret_cast<const uint4*>(t.down + 8 * cg), down);
    Elem<float>::widen(*reinterpret_cast<const uint4*>(t.down + 8 * cg + 4), down + 4);
    uint32_t* to = reinterpret_cast<uint32_t*>(t.turned + 8 * cg * 128u + ((rg ^ (2 * cg)) << 2));
    float y[8][4];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        const uint64_t by2 = pack2(down[i], down[i]);
        unpack2(mul2(pack2(v[0][i], v[1][i]), by2), y[i][0], y[i][1]);
        unpack2(mul2(pack2(v[2][i], v[3][i]), by2), y[i][2], y[i][3]);
    }
    if (m.dtype == 3) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) to[32 * i] = act8_e4m3(y[i][0], y[i][1]) | (uint32_t)act8_e4m3(y[i][2], y[i][3]) << 16;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) to[32 * i] = act8_e5m2(y[i][0], y[i][1]) | (uint32_t)act8_e5m2(y[i][2], y[i][3]) << 16;
    }
    __syncthreads();
    const uint32_t piece = tid & 7u, left = FULL ? 128u : row0 + 16 * piece < rows ? rows - (row0 + 16 * piece) : 0;
#pragma unroll
    for (uint32_t p = 0; p < 2; ++p) {
        const uint32_t c = (tid >> 3) + 64 * p, group = c >> 3;
        if (!FULL && (col0 + c >= cols || !left)) continue;
        uint4 w = *reinterpret_cast<const uint4*>(t.turned + c * 128u + ((piece ^ (group >> 1)) << 4));
        if (group & 1u) w = make_uint4(w.z, w.w, w.x, w.y);
        unsigned char* out = m.data + (uint64_t)(col0 + c) * m.stride + row0 + 16 * piece;
        if (left >= 16) {
            *reinterpret_cast<uint4*>(out) = w;
        } else {
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i)
                if (i < left) out[i] = (unsigned char)(u[i >> 2] >> (8 * (i & 3)));
        }
    }
}

// S: type of the inputs (uint8_t: either of 8 bits), T: of the plain results and of the gradient.
template <int OP, typename S, typename T, bool FULL>
__device__ __forceinline__ void act8_tile(const Act8Tiles& P, const Act8Place& at, Act8Turn& turn) {
    constexpr bool wide = sizeof(T) == 4;
    Raw8<S> a[4], b[4];
    Raw8<T> d[4];
    act8_get<FULL>(P.in[0], at, a);
    if (OP != kActCopy) act8_get<FULL>(P.in[1], at, b);
    if (OP == kActGateGrad) act8_get<FULL>(P.d, at, d);
    float v[4][8], u[OP == kActGateGrad ? 4 : 1][8];
    if constexpr (OP == kActCopy) {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) widen8(a[j], P.in[0].dtype, v[j]);
    }
    if constexpr (OP == kActGate) {
#pragma unroll
        for (uint32_t j = 0; j < 4; j += 2) {
            float x[2][8];
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
                widen8(a[j + h], P.in[0].dtype, v[j + h]);
                widen8(b[j + h], P.in[1].dtype, x[h]);
            }
            if (P.kept[0].data) act8_put_coded<FULL>(P.kept[0], at, j, v[j], v[j + 1]);
            if (P.kept[1].data) act8_put_coded<FULL>(P.kept[1], at, j, x[0], x[1]);
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float g = v[j + h][i];
                    v[j + h][i] = __fmul_rn(__fmul_rn(g, act8_sigmoid<wide>(g)), x[h][i]);
                }
        }
    }
    if constexpr (OP == kActGateGrad) {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            float y[8];
            widen8(a[j], P.in[0].dtype, v[j]);
            widen8(b[j], P.in[1].dtype, u[j]);
            widen8(d[j], 0, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float g = v[j][i], s = act8_sigmoid<wide>(g), ds = __fmul_rn(y[i], s);
                v[j][i] = __fmul_rn(__fmul_rn(ds, u[j][i]), __fmaf_rn(g, __fsub_rn(1.f, s), 1.f));
                u[j][i] = __fmul_rn(ds, g);
            }
        }
    }
    if (P.plain[0].data) act8_put_plain<FULL, T>(P.plain[0], at, v);
    if (P.q[0].data) {
        act8_put_coded<FULL>(P.q[0], at, 0, v[0], v[1]);
        act8_put_coded<FULL>(P.q[0], at, 2, v[2], v[3]);
    }
    if (P.qt[0].data) act8_put_turned<FULL>(P.qt[0], at, P.rows, P.cols, v, turn);
    if constexpr (OP == kActGateGrad) {
        if (P.plain[1].data) act8_put_plain<FULL, T>(P.plain[1], at, u);
        if (P.q[1].data) {
        act8_put_coded<FULL>(P.q[1], at, 0, u[0], u[1]);
        act8_put_coded<FULL>(P.q[1], at, 2, u[2], u[3]);
    }
        if (P.qt[1].data) {
            __syncthreads();                                         // the first is out of shared memory
            act8_put_turned<FULL>(P.qt[1], at, P.rows, P.cols, u, turn);
        }
    }
}

template <int OP, typename S, typename T>
__global__ void __launch_bounds__(kActThreads, OP == kActGateGrad ? 1 : 2) act8_tile_kernel(const __grid_constant__ Act8Tiles P) {
    __shared__ __align__(16) Act8Turn turn;
    const uint32_t tile_row = blockIdx.x / P.tiles_across, tile_col = blockIdx.x - tile_row * P.tiles_across;
    const uint32_t row0 = tile_row * 128u, col0 = tile_col * 128u;
    Act8Place at;
    at.row = row0 + 4 * (threadIdx.x >> 4);
    at.col = col0 + 8 * (threadIdx.x & 15u);
    at.n = inside(at.col, P.cols);
    at.rows = at.row < P.rows ? min(4u, P.rows - at.row) : 0;
    griddep_launch();
    griddep_wait();
    if (P.wide && row0 + 128 <= P.rows && col0 + 128 <= P.cols) act8_tile<OP, S, T, true>(P, at, turn);
    else act8_tile<OP, S, T, false>(P, at, turn);
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
    int full;                            // whole vectors: columns in eights, all rows on 16-byte boundaries
    uint32_t rows, cols, per_row;
    float eps, inv_cols;
};

// Where a row's vectors are.
__device__ __forceinline__ unsigned char* act8_row(const Act8Mat& m, uint32_t row) { return m.data + row * m.stride; }
// A row's scale bytes; block b's lies act8_scale_at(0, b, .) further.
__device__ __forceinline__ uint8_t* act8_row_scales(const Act8Mat& m, uint32_t row) { return m.scales + act8_scale_at(row, 0, m.groups); }
__device__ __forceinline__ uint32_t act8_block_at(uint32_t block) { return (block >> 2) * 512u + (block & 3u); }

// Vectors of a row in 8 bits, two blocks' scales at a time.
template <bool FULL, int NV>
__device__ __forceinline__ void act8_put_row(const Act8Mat& m, uint32_t row, uint32_t t, uint32_t per_row, uint32_t cols, bool real,
                                             const float (&v)[NV][8]) {
    uint32_t bytes[(NV + 1) / 2];
#pragma unroll
    for (int k = 0; k < NV; k += 2) {
        const uint32_t low = act8_byte(act8_largest(v[k]), m.dtype), high = k + 1 < NV ? act8_byte(act8_largest(v[k + 1 < NV ? k + 1 : k]), m.dtype) : 0;
        bytes[k / 2] = act8_agree(low | high << 16);
    }
    unsigned char* p = act8_row(m, row) + 8 * t;
    uint8_t* s = act8_row_scales(m, row);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const uint32_t col = (k * per_row + t) * 8, n = !real ? 0 : FULL ? (col < cols ? 8 : 0) : inside(col, cols);
        if (n) put8_coded<FULL>(p + k * per_row * 8, s + act8_block_at(col >> 7), n, (t & 15u) == 0, m.dtype, (bytes[k / 2] >> (16 * (k & 1))) & 255u, v[k]);
    }
}

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

template <typename T, int NV, bool FULL>
__device__ __forceinline__ void act8_norm_rows(const Act8Norm& P, float* part) {
    const uint32_t slot = threadIdx.x / P.per_row, t = threadIdx.x - slot * P.per_row, slots = blockDim.x / P.per_row;
    float w[NV][8];
    uint32_t cols[NV];                                               // entries of each vector that are inside
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const uint32_t col = (k * P.per_row + t) * 8;
        cols[k] = FULL ? (col < P.cols ? 8 : 0) : inside(col, P.cols);
        act8_weight(P.weight, P.weight_dtype, col, cols[k], w[k]);
    }
    const uint32_t step = P.per_row * 8 * (uint32_t)sizeof(T), at = 8 * t * (uint32_t)sizeof(T);
    uint32_t turn = 0;
    for (uint64_t first = (uint64_t)blockIdx.x * slots; first < P.rows; first += (uint64_t)gridDim.x * slots, ++turn) {
        const uint32_t row = (uint32_t)first + slot;
        const bool real = row < P.rows;
        Raw8<T> a[NV], b[NV];
        const unsigned char *x = act8_row(P.x, row) + at, *r = act8_row(P.residual, row) + at;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            a[k] = {};
            b[k] = {};
            if (real && cols[k]) {
                get8<FULL>(x + k * step, nullptr, cols[k], P.x.wide, a[k]);
                if (P.residual.data) get8<FULL>(r + k * step, nullptr, cols[k], P.residual.wide, b[k]);
            }
        }
        float s[NV][8], squares = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float y[8];
            widen8(a[k], 0, s[k]);
            widen8(b[k], 0, y);
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                if (P.residual.data) unpack2(add2(pack2(s[k][i], s[k][i + 1]), pack2(y[i], y[i + 1])), s[k][i], s[k][i + 1]);
                squares = __fmaf_rn(s[k][i], s[k][i], squares);
                squares = __fmaf_rn(s[k][i + 1], s[k][i + 1], squares);
            }
        }
        // what does not need the row's sum is written while the threads wait for each other
        if (P.sum.data) {
            unsigned char* to = act8_row(P.sum, row) + at;
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (real && cols[k]) put8<FULL, T>(to + k * step, cols[k], P.sum.wide, s[k]);
        }
        if (P.sum8.data) act8_put_row<FULL, NV>(P.sum8, row, t, P.per_row, P.cols, real, s);
        squares = act8_row_sum(squares, P.per_row, part, turn);
        const float rstd = __fdiv_rn(1.f, __fsqrt_rn(__fmaf_rn(squares, P.inv_cols, P.eps)));
        if (real && t == 0 && P.rstd) P.rstd[row] = rstd;
        if (!P.y.data && !P.y8.data) continue;
        const uint64_t by = pack2(rstd, rstd);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < 8; i += 2)
                unpack2(mul2(mul2(pack2(s[k][i], s[k][i + 1]), by), pack2(w[k][i], w[k][i + 1])), s[k][i], s[k][i + 1]);
        if (P.y.data) {
            unsigned char* to = act8_row(P.y, row) + at;
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (real && cols[k]) put8<FULL, T>(to + k * step, cols[k], P.y.wide, s[k]);
        }
        if (P.y8.data) act8_put_row<FULL, NV>(P.y8, row, t, P.per_row, P.cols, real, s);
    }
}

template <typename T, int NV>
__global__ void __launch_bounds__(512) act8_norm_kernel(const __grid_constant__ Act8Norm P) {
    __shared__ float part[64];
    griddep_launch();
    griddep_wait();
    if (P.full) act8_norm_rows<T, NV, true>(P, part);
    else act8_norm_rows<T, NV, false>(P, part);
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
    int full;
    uint32_t rows, cols, per_row;
    float inv_cols;
};

template <typename S, typename T, int NV, bool FULL>
__device__ __forceinline__ void act8_norm_grad_rows(const Act8NormGrad& P, float* part) {
    const uint32_t slot = threadIdx.x / P.per_row, t = threadIdx.x - slot * P.per_row, slots = blockDim.x / P.per_row;
    float w[NV][8], dw[NV][8];
    uint32_t cols[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const uint32_t col = (k * P.per_row + t) * 8;
        cols[k] = FULL ? (col < P.cols ? 8 : 0) : inside(col, P.cols);
        act8_weight(P.weight, P.weight_dtype, col, cols[k], w[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[k][i] = 0.f;
    }
    const uint32_t step = P.per_row * 8 * (uint32_t)sizeof(T), at = 8 * t * (uint32_t)sizeof(T);
    uint32_t turn = 0;
    for (uint64_t first = (uint64_t)blockIdx.x * slots; first < P.rows; first += (uint64_t)gridDim.x * slots, ++turn) {
        const uint32_t row = (uint32_t)first + slot;
        const bool real = row < P.rows;
        Raw8<S> a[NV];
        Raw8<T> b[NV], c[NV];
        const float rstd = real ? P.rstd[row] : 0.f;
        const unsigned char* s = act8_row(P.s, row) + 8 * t * sizeof(S);
        const uint8_t* scales = sizeof(S) == 1 ? act8_row_scales(P.s, row) : nullptr;
        const unsigned char *d = act8_row(P.d_out, row) + at, *e = act8_row(P.d_sum, row) + at;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            a[k] = {};
            b[k] = {};
            c[k] = {};
            if (real && cols[k]) {
                const uint8_t* scale = sizeof(S) == 1 ? scales + act8_block_at((k * P.per_row + t) >> 4) : nullptr;
                get8<FULL>(s + k * P.per_row * 8 * sizeof(S), scale, cols[k], P.s.wide, a[k]);
                get8<FULL>(d + k * step, nullptr, cols[k], P.d_out.wide, b[k]);
                if (P.d_sum.data) get8<FULL>(e + k * step, nullptr, cols[k], P.d_sum.wide, c[k]);
            }
        }
        float normed[NV][8], g[NV][8], dot = 0.f;
        const uint64_t by = pack2(rstd, rstd);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            widen8(a[k], P.s.dtype, normed[k]);
            widen8(b[k], 0, g[k]);
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const uint64_t n = mul2(pack2(normed[k][i], normed[k][i + 1]), by), o = pack2(g[k][i], g[k][i + 1]);
                unpack2(n, normed[k][i], normed[k][i + 1]);
                unpack2(fma2(o, n, pack2(dw[k][i], dw[k][i + 1])), dw[k][i], dw[k][i + 1]);
                unpack2(mul2(o, pack2(w[k][i], w[k][i + 1])), g[k][i], g[k][i + 1]);
                dot = __fmaf_rn(g[k][i], normed[k][i], dot);
                dot = __fmaf_rn(g[k][i + 1], normed[k][i + 1], dot);
            }
        }
        const float mean = __fmul_rn(act8_row_sum(dot, P.per_row, part, turn), P.inv_cols);
        if (!P.d_x.data) continue;
        unsigned char* to = act8_row(P.d_x, row) + at;
        const uint64_t less = pack2(-mean, -mean);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (!real || !cols[k]) continue;
            float x[8];
            widen8(c[k], 0, x);
#pragma unroll
            for (int i = 0; i < 8; i += 2)
                unpack2(fma2(by, fma2(pack2(normed[k][i], normed[k][i + 1]), less, pack2(g[k][i], g[k][i + 1])), pack2(x[i], x[i + 1])),
                        x[i], x[i + 1]);
            put8<FULL, T>(to + k * step, cols[k], P.d_x.wide, x);
        }
    }
    if (!P.sums) return;
    float* to = P.sums + ((uint64_t)blockIdx.x * slots + slot) * P.cols;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const uint32_t col = (k * P.per_row + t) * 8;
        if (FULL && cols[k]) {
            *reinterpret_cast<uint4*>(to + col) = Elem<float>::narrow(dw[k]);
            *reinterpret_cast<uint4*>(to + col + 4) = Elem<float>::narrow(dw[k] + 4);
            continue;
        }
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < cols[k]) to[col + i] = dw[k][i];
    }
}

template <typename S, typename T, int NV>
__global__ void __launch_bounds__(512) act8_norm_grad_kernel(const __grid_constant__ Act8NormGrad P) {
    __shared__ float part[64];
    griddep_launch();
    griddep_wait();
    if (P.full) act8_norm_grad_rows<S, T, NV, true>(P, part);
    else act8_norm_grad_rows<S, T, NV, false>(P, part);
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
