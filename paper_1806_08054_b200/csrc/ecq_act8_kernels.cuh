// Matrices in 8 bits: storing and restoring them, and the operators of a language model's layer that
// write and read them (root-mean-square norm, gated activation, and their gradients).
#pragma once

#include <cstdint>

#include <cuda.h>

#include "ecq_act8.cuh"
#include "ecq_tensor.cuh"

namespace ecq {

// ---- storing, restoring and the gated activation: tiles of 128 x 128 -----------------------------
//
// Whatever is written in 8 bits transposed has its blocks along the tile's columns, so a CTA has a
// whole tile: a thread four rows of eight columns, 16 lanes a row's block.  Each input is read once and each output written
// once.  Bound by memory where nothing is written transposed (8192 x 4096 bf16: stored 18.0 us, 5.6 TB/s, restored 18.4, the gate with
// both inputs kept 45.2, 5.2, its gradient to bf16 from 8 bits 44.6, 6.0, from bf16 54.5, 6.2), else by instructions: 130 for eight entries of
// a lane stored both ways (27.2 us), 314 for the gradient with both results both ways from 8 bits (71.3), 271 from bf16 (66.7), at 0.4 to
// 0.6 a cycle and scheduler.  The gate's 64 registers, for two CTAs an SM, keep 84 to 256 bytes a thread in local memory.

enum { kActCopy = 0, kActGate = 1, kActGateGrad = 2 };
constexpr uint32_t kActThreads = 512;

struct Act8Tiles {
    Act8Mat in[2];                       // x; gate and up
    Act8Mat d;                           // gradient of the activation's output
    Act8Mat plain[2], q[2], qt[2];       // results (data NULL: not wanted): h, or d_gate and d_up
    Act8Mat kept[2];                     // gate and up in 8 bits
    uint32_t rows, cols, tiles_across, tiles;
    int wide;                            // rows of all plain matrices begin on 16-byte boundaries
    uint32_t wait_limit;
};

// 1 / (1 + exp(-x)) of two entries; WIDE: the rounding of x log2(e) is added back, which shows in 32 bits alone.
template <bool WIDE>
__device__ __forceinline__ uint64_t act8_sigmoid2(uint64_t x) {
    const uint64_t by = pack2(-1.44269504088896f, -1.44269504088896f), t = mul2(x, by);
    float t0, t1;
    unpack2(t, t0, t1);
    uint64_t e = pack2(ex2(t0), ex2(t1));
    if (WIDE) {
        uint64_t lo = fma2(x, by, t ^ 0x8000000080000000ull);
        lo = fma2(x, pack2(-1.925963033e-8f, -1.925963033e-8f), lo);   // log2(e) beyond 24 bits
        lo = fma2(e, mul2(lo, pack2(0.693147181f, 0.693147181f)), e);
        float e0, e1, l0, l1;
        unpack2(e, e0, e1);
        unpack2(lo, l0, l1);
        e = pack2(t0 > -126.f && t0 < 126.f ? l0 : e0, t1 > -126.f && t1 < 126.f ? l1 : e1);
    }
    float y0, y1;
    unpack2(add2(e, pack2(1.f, 1.f)), y0, y1);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(y0));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(y1));
    return pack2(y0, y1);
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
        put8<FULL, 16, T>(m, p, FULL || j < at.rows ? at.n : 0, v[j]);
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
    for (uint32_t j = 0; j < 4; ++j, p += m.stride, s += 16) get8<FULL>(m, p, s, FULL || j < at.rows ? at.n : 0, r[j]);
}

// A thread's 4 x 8 entries of N results in 8 bits transposed, those that are wanted; the whole CTA.  Two together, as
// each step ends in a barrier that they then share.  Calls may follow each other: each part of shared memory is written a
// barrier after its last reader.
template <int N> struct Act8Turn {
    unsigned char turned[N][128 * 128];
    uint32_t part[N][kActThreads / 32][128];
    float down[N][128];
};
template <> struct Act8Turn<2> {         // the second lies in the first, for want of room
    union {
        unsigned char turned[2][128 * 128];
        uint32_t part[2][kActThreads / 32][128];
    };
    float down[2][128];
};
template <bool FULL, int N>
__device__ __forceinline__ void act8_put_turned(const Act8Mat (&m)[2], const Act8Place& at, uint32_t rows, uint32_t cols,
                                                const float (&v)[4][8], const float (&u)[4][8], Act8Turn<N>& t) {
    const uint32_t tid = threadIdx.x, cg = tid & 15u, rg = tid >> 4, row0 = at.row - 4 * rg, col0 = at.col - 8 * cg;
    if (N == 2) __syncthreads();
    // the columns' largest magnitudes: four rows in registers, two groups of rows a warp, 16 warps
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (!m[n].data) continue;
        const float (&x)[4][8] = n ? u : v;
        uint32_t big[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const float y = top3(top3(x[0][i], x[1][i], x[2][i]), x[3][i], 0.f);
            big[i] = __float_as_uint(top3(y, __shfl_xor_sync(~0u, y, 16), 0.f));
        }
        if ((tid & 16u) == 0) {
            uint4* to = reinterpret_cast<uint4*>(&t.part[n][tid >> 5][8 * cg]);
            to[0] = make_uint4(big[0], big[1], big[2], big[3]);
            to[1] = make_uint4(big[4], big[5], big[6], big[7]);
        }
    }
    __syncthreads();
    if (tid < 128 * N) {
        const uint32_t n = tid >> 7, c = tid & 127u;
        const Act8Mat& to = N == 2 && n ? m[1] : m[0];
        if (to.data) {
            uint32_t top = 0;
#pragma unroll
            for (uint32_t w = 0; w < kActThreads / 32; ++w) top = max(top, t.part[n][w][c]);
            const uint32_t byte = act8_byte(top, to.dtype);
            t.down[n][c] = act8_down(byte);
            if (FULL || col0 + c < cols) to.scales[act8_scale_at(col0 + c, row0 >> 7, to.groups)] = (uint8_t)byte;
        }
    }
    __syncthreads();
    // The tile turned in shared memory: column c has 128 bytes, its four-byte words exchanged by the
    // group of eight columns so that neither a warp's words nor its 16-byte reads meet in a bank.
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (!m[n].data) continue;
        const float (&x)[4][8] = n ? u : v;
        float down[8];
        Elem<float>::widen(*reinterpret_cast<const uint4*>(t.down[n] + 8 * cg), down);
        Elem<float>::widen(*reinterpret_cast<const uint4*>(t.down[n] + 8 * cg + 4), down + 4);
        uint32_t* to = reinterpret_cast<uint32_t*>(t.turned[n] + 8 * cg * 128u + ((rg ^ (2 * cg)) << 2));
        float y[8][4];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) y[i][j] = __fmul_rn(x[j][i], down[i]);   // not in pairs: rows are none
        if (m[n].dtype == 3) {
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) to[32 * i] = act8_e4m3(y[i][0], y[i][1]) | (uint32_t)act8_e4m3(y[i][2], y[i][3]) << 16;
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) to[32 * i] = act8_e5m2(y[i][0], y[i][1]) | (uint32_t)act8_e5m2(y[i][2], y[i][3]) << 16;
        }
    }
    __syncthreads();
    const uint32_t piece = tid & 7u, left = FULL ? 128u : row0 + 16 * piece < rows ? rows - (row0 + 16 * piece) : 0;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (!m[n].data) continue;
#pragma unroll
        for (uint32_t p = 0; p < 2; ++p) {
            const uint32_t c = (tid >> 3) + 64 * p, group = c >> 3;
            if (!FULL && (col0 + c >= cols || !left)) continue;
            uint4 w = *reinterpret_cast<const uint4*>(t.turned[n] + c * 128u + ((piece ^ (group >> 1)) << 4));
            if (group & 1u) w = make_uint4(w.z, w.w, w.x, w.y);
            unsigned char* out = m[n].data + (uint64_t)(col0 + c) * m[n].stride + row0 + 16 * piece;
            if (left >= 16) {
                *reinterpret_cast<uint4*>(out) = w;
            } else {
                const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (uint32_t i = 0; i < 16; ++i)
                    if (i < left) out[i] = (unsigned char)(q[i >> 2] >> (8 * (i & 3)));
            }
        }
    }
}

// What a thread reads of a tile.  S: type of the inputs (uint8_t: either of 8 bits), T: of the plain results and of
// the gradient.
template <int OP, typename S, typename T>
struct Act8Read {
    Raw8<S> a[4], b[OP == kActCopy ? 1 : 4];
    Raw8<T> d[OP == kActGateGrad ? 4 : 1];
};
template <int OP, typename S, typename T, bool FULL>
__device__ __forceinline__ void act8_read(const Act8Tiles& P, const Act8Place& at, Act8Read<OP, S, T>& r) {
    act8_get<FULL>(P.in[0], at, r.a);
    if constexpr (OP != kActCopy) act8_get<FULL>(P.in[1], at, r.b);
    if constexpr (OP == kActGateGrad) act8_get<FULL>(P.d, at, r.d);
}

// Tiles on their way in shared memory: each matrix's 128 rows of 128 entries, and of one in 8 bits the
// 512 scale bytes that its blocks are among.
template <int OP, typename S, typename T>
struct Act8Ring {
    static constexpr uint32_t kIn = 128 * 128 * sizeof(S) + (sizeof(S) == 1 ? 512 : 0);
    static constexpr uint32_t kBytes = kIn * (OP == kActCopy ? 1 : 2) + (OP == kActGateGrad ? 128 * 128 * sizeof(T) : 0);
    // an SM; 64 registers a thread are too few for a gradient, and for two inputs in 32 bits
    static constexpr uint32_t kCtas = OP == kActGateGrad || (OP == kActGate && sizeof(S) == 4) ? 1 : 2;
    static constexpr uint32_t kRoom = 226u * 1024u / kCtas - (OP == kActGateGrad ? 35u : 27u) * 1024u;
    // Restoring to 32 bits is bound by its stores (8192 x 4096 with and without, us: 40.5, 36.5).  Room for one alone, which comes while
    // the one before it is worked on, is used by launches whose work is long (`launch_tiles`); never of two CTAs an SM.
    static constexpr uint32_t kFit = kRoom / kBytes;
    static constexpr uint32_t kStages = OP == kActCopy && sizeof(S) == 1 && sizeof(T) == 4 ? 0 : kFit >= 2 ? kFit < 4 ? kFit : 4 : kCtas == 1 ? kFit : 0;
    static constexpr uint32_t kSmem = kStages * kBytes + 128;
};

// A thread's entries of a matrix of a tile in shared memory.
template <typename T>
__device__ __forceinline__ void act8_take(uint32_t from, uint32_t block, Raw8<T> (&r)[4]) {
    const uint32_t at = from + (threadIdx.x >> 4) * 4 * 128 * (uint32_t)sizeof(T) + (threadIdx.x & 15u) * 8 * (uint32_t)sizeof(T);
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) r[j].w[i] = lds16(at + j * 128 * (uint32_t)sizeof(T) + 16 * i);
}
template <>
__device__ __forceinline__ void act8_take<uint8_t>(uint32_t from, uint32_t block, Raw8<uint8_t> (&r)[4]) {
    const uint32_t row = (threadIdx.x >> 4) * 4, at = from + row * 128 + (threadIdx.x & 15u) * 8;
    const uint32_t scale = from + 128 * 128 + (uint32_t)act8_scale_at(row, block & 3u, 1);
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
        asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(r[j].w.x), "=r"(r[j].w.y) : "r"(at + j * 128));
        asm volatile("ld.shared.u8 %0, [%1];" : "=r"(r[j].byte) : "r"(scale + 16 * j));
    }
}

template <int OP, typename S, typename T, bool FULL>
__device__ __forceinline__ void act8_tile(const Act8Tiles& P, const Act8Place& at, const Act8Read<OP, S, T>& in,
                                          Act8Turn<OP == kActGateGrad ? 2 : 1>& turn) {
    constexpr bool wide = sizeof(T) == 4;
    const auto& a = in.a;
    const auto& b = in.b;
    const auto& d = in.d;
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
                for (int i = 0; i < 8; i += 2) {
                    const uint64_t g = pack2(v[j + h][i], v[j + h][i + 1]);
                    unpack2(mul2(mul2(g, act8_sigmoid2<wide>(g)), pack2(x[h][i], x[h][i + 1])), v[j + h][i], v[j + h][i + 1]);
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
            for (int i = 0; i < 8; i += 2) {
                const uint64_t one = pack2(1.f, 1.f), g = pack2(v[j][i], v[j][i + 1]), s = act8_sigmoid2<wide>(g);
                const uint64_t ds = mul2(pack2(y[i], y[i + 1]), s), slope = fma2(g, sub2(one, s), one);
                unpack2(mul2(mul2(ds, pack2(u[j][i], u[j][i + 1])), slope), v[j][i], v[j][i + 1]);
                unpack2(mul2(ds, g), u[j][i], u[j][i + 1]);
            }
        }
    }
    if (P.plain[0].data) act8_put_plain<FULL, T>(P.plain[0], at, v);
    if (P.q[0].data) {
        act8_put_coded<FULL>(P.q[0], at, 0, v[0], v[1]);
        act8_put_coded<FULL>(P.q[0], at, 2, v[2], v[3]);
    }
    if constexpr (OP == kActGateGrad) {
        if (P.plain[1].data) act8_put_plain<FULL, T>(P.plain[1], at, u);
        if (P.q[1].data) {
            act8_put_coded<FULL>(P.q[1], at, 0, u[0], u[1]);
            act8_put_coded<FULL>(P.q[1], at, 2, u[2], u[3]);
        }
        if (P.qt[0].data || P.qt[1].data) act8_put_turned<FULL, 2>(P.qt, at, P.rows, P.cols, v, u, turn);
    } else {
        if (P.qt[0].data) act8_put_turned<FULL, 1>(P.qt, at, P.rows, P.cols, v, v, turn);
    }
}

__device__ __forceinline__ Act8Place act8_place(const Act8Tiles& P, uint32_t row0, uint32_t col0) {
    Act8Place at;
    at.row = row0 + 4 * (threadIdx.x >> 4);
    at.col = col0 + 8 * (threadIdx.x & 15u);
    at.n = inside(at.col, P.cols);
    at.rows = at.row < P.rows ? min(4u, P.rows - at.row) : 0;
    return at;
}

// A tile a CTA; a part of one, of 32 rows, where nothing is written transposed.
template <int OP, typename S, typename T>
__global__ void __launch_bounds__(kActThreads, Act8Ring<OP, S, T>::kCtas) act8_tile_kernel(const __grid_constant__ Act8Tiles P) {
    __shared__ __align__(16) Act8Turn<OP == kActGateGrad ? 2 : 1> turn;
    const uint32_t rows = blockDim.x / 4, row0 = blockIdx.x / P.tiles_across * rows, col0 = blockIdx.x % P.tiles_across * 128u;
    const Act8Place at = act8_place(P, row0, col0);
    griddep_launch();
    griddep_wait();
    Act8Read<OP, S, T> in;
    if (P.wide && row0 + rows <= P.rows && col0 + 128 <= P.cols) {
        act8_read<OP, S, T, true>(P, at, in);
        act8_tile<OP, S, T, true>(P, at, in, turn);
    } else {
        act8_read<OP, S, T, false>(P, at, in);
        act8_tile<OP, S, T, false>(P, at, in, turn);
    }
}

struct Act8Maps { CUtensorMap of[3]; };  // in[0], in[1] and d in boxes of 128 x 128

// CTAs stay on the GPU and take every n-th tile.  Whole tiles come by TMA as many ahead as there is room for: a
// thread's four rows alone are too little on their way to memory, in 8 bits above all, and registers have
// no room for the next tile's.  After a wait that ran out tiles are read from memory, and none is asked for any more.
template <int OP, typename S, typename T>
__global__ void __launch_bounds__(kActThreads, Act8Ring<OP, S, T>::kCtas)
    act8_tiles_kernel(const __grid_constant__ Act8Tiles P, const __grid_constant__ Act8Maps maps) {
    using R = Act8Ring<OP, S, T>;
    constexpr uint32_t kStages = R::kStages;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(16) Act8Turn<OP == kActGateGrad ? 2 : 1> turn;
    __shared__ __align__(8) uint64_t bars[kStages];
    __shared__ volatile uint32_t late, asked;
    const uint32_t ring = (smem_u32(raw) + 127u) & ~127u, full = smem_u32(bars), tid = threadIdx.x;
    auto whole = [&](uint32_t tile) {
        return (tile / P.tiles_across + 1) * 128u <= P.rows && (tile % P.tiles_across + 1) * 128u <= P.cols && P.wide;
    };
    if (tid == 0) {
        for (uint32_t s = 0; s < kStages; ++s) mbar_init(full + 8 * s, 1);
        late = asked = 0;
        fence_mbar_init();
    }
    griddep_launch();
    __syncthreads();
    griddep_wait();
    // by one thread: the next whole tile from `coming` on
    uint32_t coming = blockIdx.x;
    auto ask = [&](uint32_t s) {
        while (coming < P.tiles && !whole(coming)) coming += gridDim.x;
        if (coming >= P.tiles) return;
        const uint32_t tr = coming / P.tiles_across, tc = coming % P.tiles_across, bar = full + 8 * s;
        uint32_t to = ring + s * R::kBytes;
        mbar_arrive_expect_tx(bar, R::kBytes);
#pragma unroll
        for (int m = 0; m < (OP == kActCopy ? 1 : 2); ++m, to += R::kIn) {
            tma_load_2d(to, &maps.of[m], (int)(tc * 128), (int)(tr * 128), bar);
            if (sizeof(S) == 1)
                asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to + 128 * 128),
                             "l"(P.in[m].scales + ((uint64_t)tr * P.in[m].groups + (tc >> 2)) * 512), "r"(512u), "r"(bar)
                             : "memory");
        }
        if (OP == kActGateGrad) tma_load_2d(to, &maps.of[2], (int)(tc * 128), (int)(tr * 128), bar);
        coming += gridDim.x;
        asked = asked + 1;
    };
    if (tid == 0)
        for (uint32_t s = 0; s < kStages; ++s) ask(s);
    uint32_t it = 0;                                                 // whole tiles so far
    for (uint32_t tile = blockIdx.x; tile < P.tiles; tile += gridDim.x) {
        const uint32_t row0 = tile / P.tiles_across * 128u, col0 = tile % P.tiles_across * 128u;
        const Act8Place at = act8_place(P, row0, col0);
        Act8Read<OP, S, T> in;
        if (!whole(tile)) {
            act8_read<OP, S, T, false>(P, at, in);
            act8_tile<OP, S, T, false>(P, at, in, turn);
            continue;
        }
        const uint32_t s = it % kStages, from = ring + s * R::kBytes;
        if (!late && mbar_wait_n(full + 8 * s, (it / kStages) & 1, P.wait_limit)) {
            act8_take(from, col0 >> 7, in.a);
            if constexpr (OP != kActCopy) act8_take(from + R::kIn, col0 >> 7, in.b);
            if constexpr (OP == kActGateGrad) act8_take(from + 2 * R::kIn, 0, in.d);
        } else {
            late = 1;
            act8_read<OP, S, T, true>(P, at, in);
        }
        ++it;
        __syncthreads();                                             // everyone has read the stage
        if (tid == 0 && !late) ask(s);
        act8_tile<OP, S, T, true>(P, at, in, turn);
    }
    // nothing is in flight when this CTA leaves
    if (tid == 0 && late)
        for (uint32_t n = asked, j = n > kStages ? n - kStages : 0; j < n; ++j) mbar_wait(full + 8 * (j % kStages), (j / kStages) & 1);
}

// ---- norm -----------------------------------------------------------------------------------------
//
// A row belongs to `per_row` threads (whole warps), NV times eight columns each, and
// stays in their registers: every entry is read once.  CTAs go over the rows with the grid's step, so
// that the weight is read once a CTA.  Bound by memory (8192 x 4096 bf16 to bf16 25.3 us, 5.3 TB/s; with the residual to the sum
// and 8 bits 41.2, 5.7), with few rows by latency (1 x 4096: 2.7, of which a launch is 2).

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
__device__ __forceinline__ float act8_row_sum(float v, uint32_t slot, uint32_t per_row, float* part, uint32_t turn) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = __fadd_rn(v, __shfl_xor_sync(~0u, v, o));
    if (per_row == 32) return v;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = per_row >> 5;
    float* mine = part + (turn & 1) * 32;
    if (lane == 0) mine[warp] = v;
    __syncthreads();
    v = lane < warps ? mine[slot * warps + lane] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = __fadd_rn(v, __shfl_xor_sync(~0u, v, o));
    return v;
}

// 16 bytes of a row (8 of one in 8 bits), E an entry's.  A lane's eight entries of 32 bits are two of these, halves of what comes
// from L2 as one, so it stays in L1 for the second.
template <uint32_t E>
__device__ __forceinline__ void copy_ahead(uint32_t to, const void* from) {
    if (E == 4) asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else if (E == 2) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}

constexpr uint32_t kNormStages = 3;

// AHEAD: the parts of the next two rows are on their way to shared memory meanwhile, in places of the thread's own, so that
// nobody waits for anybody.
template <typename T, int NV, bool FULL, bool AHEAD>
__device__ __forceinline__ void act8_norm_rows(const Act8Norm& P, float* part, unsigned char* raw) {
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
    const uint64_t stride = (uint64_t)gridDim.x * slots;
    constexpr int kVecs = (int)sizeof(T) / 2;                        // 16 bytes of all threads lie together
    const uint32_t piece = blockDim.x * 16u, stage = NV * kVecs * piece * (P.residual.data ? 2 : 1);
    const uint32_t ring = smem_u32(raw) + threadIdx.x * 16u, rings = kNormStages * stage;
    auto ask = [&](uint64_t row, uint32_t to) {
        if (row < P.rows) {
            const unsigned char *x = act8_row(P.x, (uint32_t)row) + at, *r = act8_row(P.residual, (uint32_t)row) + at;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < kVecs; ++i) {
                    if (!cols[k]) continue;
                    copy_ahead<sizeof(T)>(to + (k * kVecs + i) * piece, x + k * step + 16 * i);
                    if (P.residual.data) copy_ahead<sizeof(T)>(to + ((NV + k) * kVecs + i) * piece, r + k * step + 16 * i);
                }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    uint64_t coming = (uint64_t)blockIdx.x * slots + slot;           // the next row to ask for, and where to
    uint32_t into = 0, from = 0;
    if (AHEAD)
        for (; into + stage < rings; into += stage, coming += stride) ask(coming, ring + into);
    uint32_t turn = 0;
    for (uint64_t first = (uint64_t)blockIdx.x * slots; first < P.rows; first += stride, ++turn) {
        const uint32_t row = (uint32_t)first + slot;
        const bool real = row < P.rows;
        Raw8<T> a[NV], b[NV];
        const unsigned char *x = act8_row(P.x, row) + at, *r = act8_row(P.residual, row) + at;
        if (AHEAD) {
            ask(coming, ring + into);
            coming += stride;
            into = into + stage == rings ? 0 : into + stage;
            asm volatile("cp.async.wait_group %0;" ::"n"(kNormStages - 1) : "memory");
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            a[k] = {};
            b[k] = {};
            if (AHEAD) {
#pragma unroll
                for (int i = 0; i < kVecs; ++i) {
                    if (real && cols[k]) a[k].w[i] = lds16(ring + from + (k * kVecs + i) * piece);
                    if (real && cols[k] && P.residual.data) b[k].w[i] = lds16(ring + from + ((NV + k) * kVecs + i) * piece);
                }
            } else if (real && cols[k]) {
                get8<FULL>(P.x, x + k * step, nullptr, cols[k], a[k]);
                if (P.residual.data) get8<FULL>(P.residual, r + k * step, nullptr, cols[k], b[k]);
            }
        }
        if (AHEAD) from = from + stage == rings ? 0 : from + stage;
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
                if (!FULL || (real && cols[k])) put8<FULL, 32, T>(P.sum, to + k * step, real ? cols[k] : 0, s[k]);
        }
        if (P.sum8.data) act8_put_row<FULL, NV>(P.sum8, row, t, P.per_row, P.cols, real, s);
        squares = act8_row_sum(squares, slot, P.per_row, part, turn);
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
                if (!FULL || (real && cols[k])) put8<FULL, 32, T>(P.y, to + k * step, real ? cols[k] : 0, s[k]);
        }
        if (P.y8.data) act8_put_row<FULL, NV>(P.y8, row, t, P.per_row, P.cols, real, s);
    }
}

// (Two vectors of 32 bits: two CTAs of 512 have to fit, or the compiler takes 83 registers: 8192 x 4096 to 32 bits 63 -> 49 us,
// 4096 x 5120 61 -> 39.)
template <typename T, int NV>
__global__ void __launch_bounds__(512, NV == 2 && sizeof(T) == 4 ? 2 : 0) act8_norm_kernel(const __grid_constant__ Act8Norm P) {
    __shared__ float part[64];
    griddep_launch();
    griddep_wait();
    if (P.full) act8_norm_rows<T, NV, true, false>(P, part, nullptr);
    else act8_norm_rows<T, NV, false, false>(P, part, nullptr);
}
template <typename T, int NV>
__global__ void __launch_bounds__(512, NV == 4 ? 1 : 2) act8_norm_ahead_kernel(const __grid_constant__ Act8Norm P) {
    extern __shared__ __align__(16) unsigned char raw[];
    __shared__ float part[64];
    griddep_launch();
    griddep_wait();
    act8_norm_rows<T, NV, true, true>(P, part, raw);
}

// Its gradient.  With n = s rstd and g = d_out w:  d_x = rstd (g - n mean(g n)) + d_sum, and the weight's
// gradient is the sum over the rows of d_out n: each thread adds its columns' in registers over the
// rows that it has, a CTA its rows' at a time, and a second launch the CTAs' sums, all in a fixed order.  Bound by memory up to 8192
// columns (8192 x 4096 bf16 from 8 bits 42.3 us, 5.6 TB/s, without the weight's 37.7; 32 bits 71, 6.1); beyond, 32 entries a
// thread pass its 128 registers (844 to 1220 bytes in local memory; 2048 x 12288 74 us, 2.8).
struct Act8NormGrad {
    Act8Mat s, d_out, d_sum, d_x;
    const void* weight;
    const float* rstd;
    float* sums;                         // [grid][pitch], or NULL
    int weight_dtype;
    int full;                            // as Act8Norm's, and there is room for a row ahead
    uint32_t rows, cols, per_row, pitch;
    float inv_cols;
};

// What a thread reads of a row.  FULL: the next row's part is on its way to shared memory meanwhile, in places of the
// thread's own, so that nobody waits for anybody (registers have no room for it: 16 warps an SM then have
// their one row each on the way, 59 us for 8192 x 4096 against 42).
template <typename S, typename T, int NV>
struct NormRead {
    Raw8<S> a[NV];
    Raw8<T> b[NV], c[NV];
    float rstd;
    static constexpr uint32_t kBytes = NV * (8 * sizeof(S) + 2 * 8 * sizeof(T));   // a thread
    // 16 bytes (8 for a vector in 8 bits) of all threads lie together
    template <typename F>
    __device__ __forceinline__ static void places(uint32_t base, F f) {
        const uint32_t threads = blockDim.x, tid = threadIdx.x;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
                f(0, k, i, base + tid * 16);
                f(1, k, i, base + threads * 16 + tid * 16);
                base += threads * 32;
            }
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < (sizeof(S) == 1 ? 1 : (int)sizeof(S) / 2); ++i) {
                f(2, k, i, base + tid * (sizeof(S) == 1 ? 8u : 16u));
                base += threads * (sizeof(S) == 1 ? 8u : 16u);
            }
    }
};

template <typename S, typename T, int NV, bool FULL>
__device__ __forceinline__ void act8_norm_grad_rows(const Act8NormGrad& P, float* part, unsigned char* raw) {
    using Read = NormRead<S, T, NV>;
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
    const uint32_t ring = smem_u32(raw), stage = blockDim.x * Read::kBytes;
    // scale byte of a vector in 8 bits
    auto scale_of = [&](uint32_t row, int k) { return act8_row_scales(P.s, row) + act8_block_at((k * P.per_row + t) >> 4); };
    auto ask = [&](uint32_t row, uint32_t from) {                    // FULL
        const unsigned char* s = act8_row(P.s, row) + 8 * t * sizeof(S);
        const unsigned char *d = act8_row(P.d_out, row) + at, *e = act8_row(P.d_sum, row) + at;
        Read::places(from, [&](int m, int k, int i, uint32_t to) {
            if (!cols[k]) return;
            if (m == 2) copy_ahead<sizeof(S)>(to, s + k * P.per_row * 8 * sizeof(S) + 16 * i);
            else if (m == 0) copy_ahead<sizeof(T)>(to, d + k * step + 16 * i);
            else if (P.d_sum.data) copy_ahead<sizeof(T)>(to, e + k * step + 16 * i);
        });
    };
    const uint64_t stride = (uint64_t)gridDim.x * slots;
    uint32_t turn = 0;
    float next_rstd = 0.f;
    uint32_t next_scale[NV];
    if (FULL) {
        const uint64_t row = (uint64_t)blockIdx.x * slots + slot;
        if (row < P.rows) {
            ask((uint32_t)row, ring);
            next_rstd = P.rstd[row];
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (sizeof(S) == 1 && cols[k]) next_scale[k] = *scale_of((uint32_t)row, k);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    for (uint64_t first = (uint64_t)blockIdx.x * slots; first < P.rows; first += stride, ++turn) {
        const uint32_t row = (uint32_t)first + slot;
        const bool real = row < P.rows;
        Read in;
        if (FULL) {
            in.rstd = next_rstd;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                in.a[k] = {};
                in.b[k] = {};
                in.c[k] = {};
                if constexpr (sizeof(S) == 1) in.a[k].byte = real && cols[k] ? next_scale[k] : 127u;
            }
            const uint64_t ahead = first + stride + slot;
            if (ahead < P.rows) {
                ask((uint32_t)ahead, ring + ((turn + 1) & 1u) * stage);
                next_rstd = P.rstd[ahead];
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if (sizeof(S) == 1 && cols[k]) next_scale[k] = *scale_of((uint32_t)ahead, k);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            if (real)
                Read::places(ring + (turn & 1u) * stage, [&](int m, int k, int i, uint32_t from) {
                    if (!cols[k] || (m == 1 && !P.d_sum.data)) return;
                    if (m == 0) in.b[k].w[i] = lds16(from);
                    else if (m == 1) in.c[k].w[i] = lds16(from);
                    else if constexpr (sizeof(S) == 1) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(in.a[k].w.x), "=r"(in.a[k].w.y) : "r"(from));
                    else in.a[k].w[i] = lds16(from);
                });
        } else {
            in.rstd = real ? P.rstd[row] : 0.f;
            const unsigned char* s = act8_row(P.s, row) + 8 * t * sizeof(S);
            const unsigned char *d = act8_row(P.d_out, row) + at, *e = act8_row(P.d_sum, row) + at;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                in.a[k] = {};
                in.b[k] = {};
                in.c[k] = {};
                if (real && cols[k]) {
                    get8<false>(P.s, s + k * P.per_row * 8 * sizeof(S), sizeof(S) == 1 ? scale_of(row, k) : nullptr, cols[k], in.a[k]);
                    get8<false>(P.d_out, d + k * step, nullptr, cols[k], in.b[k]);
                    if (P.d_sum.data) get8<false>(P.d_sum, e + k * step, nullptr, cols[k], in.c[k]);
                }
            }
        }
        const float rstd = real ? in.rstd : 0.f;
        float normed[NV][8], g[NV][8], dot = 0.f;
        const uint64_t by = pack2(rstd, rstd);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            widen8(in.a[k], P.s.dtype, normed[k]);
            widen8(in.b[k], 0, g[k]);
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
        const float mean = __fmul_rn(act8_row_sum(dot, slot, P.per_row, part, turn), P.inv_cols);
        if (!P.d_x.data) continue;
        unsigned char* to = act8_row(P.d_x, row) + at;
        const uint64_t less = pack2(-mean, -mean);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (FULL && (!real || !cols[k])) continue;
            float x[8];
            widen8(in.c[k], 0, x);
#pragma unroll
            for (int i = 0; i < 8; i += 2)
                unpack2(fma2(by, fma2(pack2(normed[k][i], normed[k][i + 1]), less, pack2(g[k][i], g[k][i + 1])), pack2(x[i], x[i + 1])),
                        x[i], x[i + 1]);
            put8<FULL, 32, T>(P.d_x, to + k * step, real ? cols[k] : 0, x);
        }
    }
    if (!P.sums) return;
    float* to = P.sums + (uint64_t)blockIdx.x * P.pitch;
    if (slots == 1) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const uint32_t col = (k * P.per_row + t) * 8;
            if (!cols[k]) continue;
            *reinterpret_cast<uint4*>(to + col) = Elem<float>::narrow(dw[k]);
            *reinterpret_cast<uint4*>(to + col + 4) = Elem<float>::narrow(dw[k] + 4);
        }
        return;
    }
    // the rows at a time added up in shared memory
    if (FULL) {
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
    }
    float* all = reinterpret_cast<float*>(raw);
    const uint32_t width = P.per_row * NV * 8;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        uint4* mine = reinterpret_cast<uint4*>(all + slot * width + (k * P.per_row + t) * 8);
        mine[0] = Elem<float>::narrow(dw[k]);
        mine[1] = Elem<float>::narrow(dw[k] + 4);
    }
    __syncthreads();
    for (uint32_t col = threadIdx.x * 4; col < P.pitch; col += blockDim.x * 4) {
        float v[4], x[4];
        Elem<float>::widen(*reinterpret_cast<const uint4*>(all + col), v);
        for (uint32_t s = 1; s < slots; ++s) {
            Elem<float>::widen(*reinterpret_cast<const uint4*>(all + s * width + col), x);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __fadd_rn(v[i], x[i]);
        }
        *reinterpret_cast<uint4*>(to + col) = Elem<float>::narrow(v);
    }
}

template <typename S, typename T, int NV>
__global__ void __launch_bounds__(512) act8_norm_grad_kernel(const __grid_constant__ Act8NormGrad P) {
    extern __shared__ __align__(16) unsigned char raw[];
    __shared__ float part[64];
    griddep_launch();
    griddep_wait();
    if (P.full) act8_norm_grad_rows<S, T, NV, true>(P, part, raw);
    else act8_norm_grad_rows<S, T, NV, false>(P, part, raw);
}

// Columns of `count` vectors added: 32 columns a CTA, 32 threads a column.
__global__ void __launch_bounds__(1024) act8_add_kernel(const float* sums, uint32_t count, uint32_t pitch, uint32_t cols, float* out) {
    __shared__ float part[32][33];
    const uint32_t col = blockIdx.x * 32u + (threadIdx.x & 31u), lane = threadIdx.x & 31u, row = threadIdx.x >> 5;
    griddep_launch();
    griddep_wait();
    float v = 0.f;
    if (col < cols)
        for (uint32_t i = row; i < count; i += 32 * 8) {
            float x[8];
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) x[j] = i + 32 * j < count ? sums[(uint64_t)(i + 32 * j) * pitch + col] : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) v = __fadd_rn(v, x[j]);
        }
    part[row][lane] = v;
    __syncthreads();
    if (row || col >= cols) return;
#pragma unroll
    for (int i = 1; i < 32; ++i) v = __fadd_rn(v, part[i][lane]);
    out[col] = v;
}

}  // namespace ecq
