// Products of matrices in 8 bits with a power of two for each 128 entries of a row: D = A B^T (+ C).
#pragma once

#include <cstdint>

#include <cuda.h>

#include "ecq_act8.cuh"
#include "ecq_tensor.cuh"

namespace ecq {

// D_ij = sum over blocks of 128 along K of 2^(ea_i + eb_j) sum_k qa_ik qb_jk.  The tensor cores take the
// scales themselves (block-scaled products): each 32 entries along K of a row come with a byte, which
// here is the same for four such steps.  Sums are in 32 bits in tensor memory from the first step to
// the last (of a CTA that has a part of K: of its part).  The tensor cores cut off what an addition of 32 products shifts
// out, so that sums lose towards zero with their length: against 64 bits 5e-8 to 1.4e-7 of the result with 512 to 2048 terms, 1.2e-7 to
// 5e-7 with 8192, 2e-7 to 9e-7 with 16384, 9e-7 to 5e-6 with 65536 (fp32 on the other units: 3e-8 to 7e-7).  Results of 16 or 8 bits
// show none of it.
//
// Operands go to shared memory as they lie in memory, 128 bytes of 128 rows at a time, in the
// 128-byte swizzle; scale bytes in their groups of 512, from where tcgen05.cp takes them to tensor
// memory for each four blocks.

struct Product8 {
    CUtensorMap left, right, left_scales, right_scales, result;
    const unsigned char* add;            // C, or NULL
    uint64_t add_stride;                 // bytes
    Act8Mat out;
    uint32_t* status;                    // or NULL
    uint32_t rows, cols;                 // of the result
    uint32_t steps;                      // blocks along K
    uint32_t tail;                       // products of 32 in the last one
    uint32_t across, tiles;              // tiles along the right operand's rows, and in all
    uint32_t left_groups, right_groups;  // of scales, along K
    uint32_t formats;                    // of the operands, as bits of the instruction descriptor
    uint32_t wait_limit;
    int add_dtype, add_wide;             // wide: rows begin on 16-byte boundaries
    int add_quad, out_quad;              // on multiples of four entries
    int in_place;                        // C is D, in 32 bits
};

constexpr uint32_t kProdRow = 128;                                    // bytes along K of a step
constexpr uint32_t kProdBox = 128 * kProdRow;                         // 128 rows of them

__device__ __forceinline__ uint64_t umma_desc_swizzled(uint32_t addr) {   // groups of eight rows of 128 bytes
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

template <int CG>
__device__ __forceinline__ void umma_mx8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool add) {
    if (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
                     "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((uint32_t)add)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
                     "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((uint32_t)add)
                     : "memory");
}

// 512 bytes of scales to 32 lanes and four columns, for each quarter of tensor memory.
template <int CG>
__device__ __forceinline__ void umma_scales(uint32_t to, uint32_t from) {
    const uint64_t desc = umma_desc(from, 128, 128);
    if (CG == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(desc) : "memory");
}

template <int CG>
__device__ __forceinline__ void prod_load(uint32_t dst, const void* map, uint32_t x, uint32_t y, uint32_t bar) {
    if (CG == 1) tma_load_2d(dst, map, (int)x, (int)y, bar);
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
                     " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"((int)x), "r"((int)y), "r"(bar)
                     : "memory");
}

__device__ __forceinline__ void prefetch_map(const void* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// Adds a box of shared memory to 32-bit memory (subnormal results are zeros there).
__device__ __forceinline__ void tma_add_2d(const void* tmap, int x, int y, uint32_t src) {
    asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(tmap), "r"(x), "r"(y),
                 "r"(src)
                 : "memory");
}

// Stores to a CTA of the cluster that count their bytes on a barrier of it.
__device__ __forceinline__ void send4(uint32_t to, float v, uint32_t bar) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(to), "r"(__float_as_uint(v)), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void send16(uint32_t to, const float* v, uint32_t bar) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1,%2,%3,%4}, [%5];" ::"r"(to), "f"(v[0]), "f"(v[1]),
                 "f"(v[2]), "f"(v[3]), "r"(bar)
                 : "memory");
}

// Arrive on the first CTA's barrier where no memory is handed over (tensor memory that has been read): a release at cluster
// scope takes 1400 clocks (8192 x 4096 x 1024: 35.7 us against 30.2).
__device__ __forceinline__ void leader_arrive_relaxed(uint32_t leader_bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(leader_bar) : "memory");
}

// Arrive on a barrier of each of `ctas` when every product issued so far has completed.
__device__ __forceinline__ void umma_commit_to(uint32_t bar, uint16_t ctas) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(ctas)
                 : "memory");
}

// Four columns of C, as they lie in memory (16-bit ones in x and y), and widened.
__device__ __forceinline__ uint4 prod_fetch4(const Product8& P, uint32_t row, uint32_t col, uint32_t n) {
    const unsigned char* p = P.add + row * P.add_stride;
    uint32_t w[4] = {0, 0, 0, 0};
    if (P.add_dtype == 0) {
        const uint32_t* f = reinterpret_cast<const uint32_t*>(p) + col;
        if (n == 4 && P.add_quad) return *reinterpret_cast<const uint4*>(f);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (i < n) w[i] = f[i];
    } else {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(p) + col;
        if (n == 4 && P.add_quad) {
            const uint2 u = *reinterpret_cast<const uint2*>(h);
            return make_uint4(u.x, u.y, 0, 0);
        }
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (i < n) w[i >> 1] |= (uint32_t)h[i] << (16 * (i & 1));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void prod_widen4(int dtype, const uint4& w, float* c) {
    float x[8];
    if (dtype == 0) Elem<float>::widen(w, x);
    else if (dtype == 1) Elem<__nv_bfloat16>::widen(make_uint4(w.x, w.y, 0, 0), x);
    else Elem<__half>::widen(make_uint4(w.x, w.y, 0, 0), x);
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = x[i];
}
__device__ __forceinline__ void prod_get4(const Product8& P, uint32_t row, uint32_t col, uint32_t n, float* c) {
    prod_widen4(P.add_dtype, prod_fetch4(P, row, col, n), c);
}

// Four columns of a plain result.
__device__ __forceinline__ void prod_put4(const Product8& P, uint32_t row, uint32_t col, uint32_t n, const float* y) {
    unsigned char* p = P.out.data + row * P.out.stride;
    if (P.out.dtype == 0) {
        float* f = reinterpret_cast<float*>(p) + col;
        if (n == 4 && P.out_quad) {
            *reinterpret_cast<uint4*>(f) = Elem<float>::narrow(y);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (i < n) f[i] = y[i];
        }
        return;
    }
    uint16_t* h = reinterpret_cast<uint16_t*>(p) + col;
    const uint2 w = P.out.dtype == 1 ? make_uint2(Elem<__nv_bfloat16>::pair(y[0], y[1]), Elem<__nv_bfloat16>::pair(y[2], y[3]))
                                     : make_uint2(Elem<__half>::pair(y[0], y[1]), Elem<__half>::pair(y[2], y[3]));
    if (n == 4 && P.out_quad) {
        *reinterpret_cast<uint2*>(h) = w;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (i < n) h[i] = (uint16_t)((i < 2 ? w.x : w.y) >> (16 * (i & 1)));
    }
}

// One column.
template <typename Args>
__device__ __forceinline__ float prod_get1(const Args& P, uint32_t row, uint32_t col) {
    const unsigned char* p = P.add + row * P.add_stride;
    return P.add_dtype == 0 ? reinterpret_cast<const float*>(p)[col]
         : P.add_dtype == 1 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[col])
                            : __half2float(reinterpret_cast<const __half*>(p)[col]);
}
template <typename Args>
__device__ __forceinline__ void prod_put1(const Args& P, uint32_t row, uint32_t col, float y) {
    unsigned char* p = P.out.data + row * P.out.stride;
    if (P.out.dtype == 0) reinterpret_cast<float*>(p)[col] = y;
    else if (P.out.dtype == 1) reinterpret_cast<__nv_bfloat16*>(p)[col] = __float2bfloat16_rn(y);
    else reinterpret_cast<__half*>(p)[col] = __float2half_rn(y);
}
__device__ __forceinline__ float lds1(uint32_t addr) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr));
    return v;
}

// Sixteen columns of a row, which begin on a multiple of 16.
__device__ __forceinline__ void prod_get16(const Product8& P, uint32_t row, uint32_t col, float* c) {
    const uint32_t n = col >= P.cols ? 0 : min(16u, P.cols - col);
    if (P.add_dtype != 0 && n == 16 && P.add_wide) {
        const uint4* h = reinterpret_cast<const uint4*>(P.add + row * P.add_stride + 2ull * col);
        const uint4 a = h[0], b = h[1];
        if (P.add_dtype == 1) {
            Elem<__nv_bfloat16>::widen(a, c);
            Elem<__nv_bfloat16>::widen(b, c + 8);
        } else {
            Elem<__half>::widen(a, c);
            Elem<__half>::widen(b, c + 8);
        }
        return;
    }
#pragma unroll
    for (uint32_t i = 0; i < 16; i += 4) prod_get4(P, row, col + i, n > i ? min(4u, n - i) : 0, c + i);
}
__device__ __forceinline__ void prod_put16(const Product8& P, uint32_t row, uint32_t col, const float* y) {
    const uint32_t n = col >= P.cols ? 0 : min(16u, P.cols - col);
    if (P.out.dtype != 0 && n == 16 && P.out.wide) {
        uint4* h = reinterpret_cast<uint4*>(P.out.data + row * P.out.stride + 2ull * col);
        h[0] = P.out.dtype == 1 ? Elem<__nv_bfloat16>::narrow(y) : Elem<__half>::narrow(y);
        h[1] = P.out.dtype == 1 ? Elem<__nv_bfloat16>::narrow(y + 8) : Elem<__half>::narrow(y + 8);
        return;
    }
#pragma unroll
    for (uint32_t i = 0; i < 16; i += 4)
        if (n > i) prod_put4(P, row, col + i, min(4u, n - i), y + i);
}

__device__ __forceinline__ uint32_t inside4(uint32_t col, uint32_t cols) { return col >= cols ? 0u : min(4u, cols - col); }

// ---- one row of A ----------------------------------------------------------------------------------------
//
// One token and a matrix that is read in no time (1 x 4096 x 1024: 2.9 us, of which a launch is 2; through the tensor cores 4.4).
// A warp has four rows of B and steps of 512 along K, 16 bytes a lane; the lane's part of A is decoded once for the four.  Products of two 8-bit entries and
// their sums are taken unscaled in 32 bits (exact but for the sums' rounding), and each lane's 16 are scaled
// together.  `split` warps of a CTA share the steps of the same rows, so that short matrices fill the GPU too.  Decoding
// bounds it where there is more to read (1 x 8192 x 8192: 28 us, through the tensor cores 16).
struct Product8Few {
    Act8Mat a, b;
    Act8Mat out;
    const unsigned char* add;
    uint64_t add_stride;
    uint32_t cols, k, split;             // split: 1, 2, 4 or 8
    int add_dtype;
};

// Sixteen entries (zeros behind the last column).
__device__ __forceinline__ uint4 few_load(const Act8Mat& m, uint32_t row, uint32_t col, uint32_t k) {
    const unsigned char* p = m.data + row * m.stride + col;
    if (col + 16 <= k) return *reinterpret_cast<const uint4*>(p);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (uint32_t i = 0; i < 16; ++i)
        if (col + i < k) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// As pairs, unscaled.
__device__ __forceinline__ void few_decode(const uint4& q, int dtype, uint64_t (&x)[8]) {
    float y[16];
    act8_decode8(make_uint2(q.x, q.y), dtype, y);
    act8_decode8(make_uint2(q.z, q.w), dtype, y + 8);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = pack2(y[2 * i], y[2 * i + 1]);
}
__device__ __forceinline__ uint32_t few_scale(const Act8Mat& m, uint32_t row, uint32_t col, uint32_t k) {
    return col < k ? m.scales[act8_scale_at(row, col >> 7, m.groups)] : 127u;
}

constexpr uint32_t kFewThreads = 256, kFewRows = 4;

__global__ void __launch_bounds__(kFewThreads) act8_product_few_kernel(const __grid_constant__ Product8Few P) {
    __shared__ float part[kFewThreads / 32][kFewRows];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, slice = warp % P.split;
    const uint32_t row0 = (blockIdx.x * (kFewThreads / 32 / P.split) + warp / P.split) * kFewRows;   // of B
    griddep_launch();
    griddep_wait();
    float sum[kFewRows];
#pragma unroll
    for (uint32_t r = 0; r < kFewRows; ++r) sum[r] = 0.f;
    if (row0 < P.cols) {
        uint4 next[kFewRows];
        uint32_t scale[kFewRows];
        auto fetch = [&](uint32_t col) {
#pragma unroll
            for (uint32_t r = 0; r < kFewRows; ++r) {
                const uint32_t row = min(row0 + r, P.cols - 1);      // beyond the last: not written
                next[r] = few_load(P.b, row, col, P.k);
                scale[r] = few_scale(P.b, row, col, P.k);
            }
        };
        const uint32_t stride = P.split * 512u;
        if (slice * 512u < P.k) fetch(slice * 512u + lane * 16u);
        for (uint32_t at = slice * 512u; at < P.k; at += stride) {
            const uint32_t col = at + lane * 16u;
            uint64_t x[8];
            few_decode(few_load(P.a, 0, col, P.k), P.a.dtype, x);
            const uint32_t xs = few_scale(P.a, 0, col, P.k);
            uint4 now[kFewRows];
            uint32_t ws[kFewRows];
#pragma unroll
            for (uint32_t r = 0; r < kFewRows; ++r) { now[r] = next[r]; ws[r] = scale[r]; }
            if (at + stride < P.k) fetch(col + stride);
#pragma unroll
            for (uint32_t r = 0; r < kFewRows; ++r) {
                uint64_t w[8];
                few_decode(now[r], P.b.dtype, w);
                uint64_t d0 = mul2(w[0], x[0]), d1 = mul2(w[1], x[1]);
#pragma unroll
                for (int i = 2; i < 8; i += 2) {
                    d0 = fma2(w[i], x[i], d0);
                    d1 = fma2(w[i + 1], x[i + 1], d1);
                }
                float a, b;
                unpack2(add2(d0, d1), a, b);
                // 2^(ea + eb) as two factors: one of them alone may pass the range of fp32
                const uint32_t e = ws[r] + xs, h = e >> 1;
                const bool nan = ws[r] == 255u || xs == 255u;
                const float y = __fmul_rn(__fadd_rn(a, b), act8_up(nan ? 255u : h));
                sum[r] = __fmaf_rn(y, act8_up(e - h), sum[r]);
            }
        }
    }
#pragma unroll
    for (uint32_t r = 0; r < kFewRows; ++r) {
        float v = sum[r];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v = __fadd_rn(v, __shfl_xor_sync(~0u, v, o));
        if (lane == 0) part[warp][r] = v;
    }
    if (P.split > 1) __syncthreads();
    else __syncwarp();
    if (slice || lane >= kFewRows) return;
    float v = part[warp][lane];
    for (uint32_t s = 1; s < P.split; ++s) v = __fadd_rn(v, part[warp + s][lane]);
    const uint32_t col = row0 + lane;
    if (col >= P.cols) return;
    if (P.add) v = __fadd_rn(v, prod_get1(P, 0, col));
    prod_put1(P, 0, col, v);
}

// ---- a tile, K over a cluster ------------------------------------------------------------------------
//
// For products that have few tiles: tiles of 128 x 128 by one CTA or 256 x 128 by a pair (CG = 2: 24 KB for what
// two CTAs alone need 32 each), K shared out over the CTAs (pairs) of a cluster.  Each of them finishes its share of the
// tile: the others send it theirs, by stores that count bytes on a barrier of its own, to a place that no
// load uses, and it adds them in a fixed order.  (Both ways through the loads' ring, with a barrier of the cluster
// before and behind: 1.2 us more at 1024 x 1024 x 8192.)  SWAP: the left operand is B and the right one A (a few tokens), the tile is D's
// transposed; so a matrix of weights fills the 128 rows of an instruction.

template <int CG, int TN, bool SWAP>
struct ProdPart {
    static constexpr uint32_t kRight = TN / CG * kProdRow;
    static constexpr uint32_t kStage = kProdBox + kRight, kScales = 1024;
    static constexpr uint32_t kMostParts = CG == 2 ? 4 : 8;
    // what the others send: columns of 128 rows, or rows (tokens) of 128 columns (and this CTA's own)
    static constexpr uint32_t kSums = SWAP ? TN * 512u : 128u * TN * 4u / kMostParts * (kMostParts - 1);
    static constexpr uint32_t kFit = (226u * 1024u - kSums) / (kStage + kScales), kStages = kFit < 7 ? kFit : 7;
    static constexpr uint32_t kSmem = kStages * (kStage + kScales) + kSums + 1024;
    static constexpr uint32_t kScaleCols = TN < 32 ? 32 : TN;         // first column of scales in tensor memory
    static constexpr uint32_t kTmem = TN <= 64 ? 128 : 256;
    static constexpr uint32_t kThreads = 12 * 32;
    static_assert(CG == 1 || (TN == 128 && !SWAP), "");
};

template <int CG, int TN, bool SWAP>
__global__ void __launch_bounds__(ProdPart<CG, TN, SWAP>::kThreads, 1) act8_product_part_kernel(const __grid_constant__ Product8 P) {
    using S = ProdPart<CG, TN, SWAP>;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::kStages + 2];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t stop;
    __shared__ volatile RingEnd end;
    const uint32_t tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31;
    const uint32_t ring = (smem_u32(raw) + 1023u) & ~1023u, scales = ring + S::kStages * S::kStage, sums = scales + S::kStages * S::kScales;
    const uint32_t full = smem_u32(bars), empty = full + 8 * S::kStages, done = empty + 8 * S::kStages, come = done + 8;
    uint32_t ctas;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    const uint32_t cta = cta_rank(), rank = CG == 2 ? cta & 1u : 0, part = cta / CG, parts = ctas / CG, first = cta - rank;
    const uint32_t tile = blockIdx.x / ctas;
    const uint32_t left0 = tile / P.across * (128u * CG) + rank * 128u, right0 = tile % P.across * (uint32_t)TN;
    const uint32_t k0 = (uint32_t)((uint64_t)part * P.steps / parts), k1 = (uint32_t)((uint64_t)(part + 1) * P.steps / parts);
    const uint32_t own = TN / parts;                                  // columns that a CTA finishes (16 at least), or rows with SWAP
    const uint32_t own_row0 = right0 + part * own, own_rows = own_row0 < P.rows ? min(own, P.rows - own_row0) : 0;   // SWAP
    if (tid == 0) {
        for (uint32_t s = 0; s < S::kStages; ++s) { mbar_init(full + 8 * s, 2); mbar_init(empty + 8 * s, 1); }
        mbar_init(done, 1);
        mbar_init(come, 1);
        stop = 0;
        end.halted = 0;
        fence_mbar_init();
        mbar_arrive_expect_tx(come, (parts - 1) * (SWAP ? own_rows : own) * 512u);
    }
    if ((warp == 8 || warp == 10) && elect_one()) {
        prefetch_map(warp == 8 ? &P.left : &P.right);
        prefetch_map(warp == 8 ? &P.left_scales : &P.right_scales);
    }
    if (warp == 9) tmem_alloc<CG>(smem_u32(&tmem_slot), S::kTmem);
    tcgen05_before_sync();
    __syncthreads();
    cluster_sync_relaxed();                                           // the others' barriers are there
    tcgen05_after_sync();
    const uint32_t tmem = tmem_slot;
    griddep_launch();
    griddep_wait();

    if (warp == 8 || warp == 10) {
        // ---- loads: a warp for each operand; in a pair bytes are counted on the first CTA's barriers
        if (elect_one()) {
            const bool left = warp == 8;
            const void* map = left ? &P.left : &P.right;
            const void* smap = left ? &P.left_scales : &P.right_scales;
            const uint32_t at = left ? 0 : kProdBox, bytes = left ? kProdBox : S::kRight;
            const uint32_t row = left ? left0 : right0 + rank * (TN / CG), groups = left ? P.left_groups : P.right_groups;
            const uint32_t group0 = ((left ? left0 : right0) >> 7) * groups, sat = scales + (left ? 0 : 512);
            uint32_t it = 0;
            for (uint32_t k = k0; k < k1; ++k, ++it) {
                const uint32_t s = it % S::kStages, bar = CG == 1 ? full + 8 * s : peer_addr(full + 8 * s, first);
                if (!wait_or_stop(empty + 8 * s, ((it / S::kStages) & 1) ^ 1, P.wait_limit, &stop)) break;
                const bool with = k == k0 || (k & 3) == 0;
                if (rank == 0) mbar_arrive_expect_tx(full + 8 * s, CG * (bytes + (with ? 512u : 0u)));
                prod_load<CG>(ring + s * S::kStage + at, map, k * kProdRow, row, bar);
                if (with) prod_load<CG>(sat + s * S::kScales, smap, 0, group0 + (k >> 2), bar);
            }
            end.asked[left ? 0 : 1] = it;
            // none of them is in flight when this CTA leaves
            for (uint32_t b = 0; b < S::kStages && b < it; ++b) {
                const uint32_t last = it - 1 - b;
                if (!wait_or_stop(empty + 8 * (last % S::kStages), (last / S::kStages) & 1, P.wait_limit, &stop)) break;
            }
        }
        __syncwarp();
    } else if (warp == 9) {
        // ---- products
        if (rank == 0 && elect_one()) {
            const uint32_t idesc = P.formats | (1u << 23) | ((uint32_t)(TN / 8) << 17) | ((uint32_t)(CG * 128 / 16) << 24);
            const uint16_t both = (uint16_t)(3u << cta);
            // the right operand's scales begin at its row in their group of 128
            const uint32_t sb_at = 4 + ((right0 & 127u) >> 5);
            uint32_t it = 0, slot = 0;
            bool ok = true;
            for (uint32_t k = k0; k < k1; ++k, ++it) {
                const uint32_t s = it % S::kStages;
                if (!wait_or_stop(full + 8 * s, (it / S::kStages) & 1, P.wait_limit, &stop)) { ok = false; break; }
                tcgen05_after_sync();
                if (k == k0 || (k & 3) == 0) {
                    // one of three places in turn: what used it last is two whole groups behind, and over
                    const uint32_t base = tmem + S::kScaleCols;
                    slot = it == 0 || slot == base + 16 ? base : slot + 8;
                    umma_scales<CG>(slot, scales + s * S::kScales);
                    umma_scales<CG>(slot + 4, scales + s * S::kScales + 512);
                }
                const uint32_t id = idesc | (k & 3) << 29 | (k & 3) << 4, steps = k + 1 == P.steps ? P.tail : 4;
                const uint64_t a = umma_desc_swizzled(ring + s * S::kStage), b = umma_desc_swizzled(ring + s * S::kStage + kProdBox);
                for (uint32_t q = 0; q < steps; ++q) umma_mx8<CG>(tmem, a + 2 * q, b + 2 * q, id, slot, slot + sb_at, it > 0 || q > 0);
                if (CG == 1) umma_commit<1>(empty + 8 * s);
                else umma_commit_to(empty + 8 * s, both);
            }
            // a sum of fewer products is nobody's result: those who wait for it give up too
            if (ok) {
                if (CG == 1) umma_commit<1>(done);
                else umma_commit_to(done, both);
            }
            end.multiplied = it;
            end.committed = ok;
        }
        __syncwarp();
    }
    // ---- results, by eight warps: 32 rows of the tile and every second 16 columns of it
    const uint32_t quad = warp & 3, half = warp >> 2, from = tmem + ((quad * 32u) << 16);
    if (warp < 8) {
        const bool good = __all_sync(~0u, wait_or_stop(done, 0, P.wait_limit, &stop));
        tcgen05_after_sync();
        auto fetch = [&](uint32_t c, float* y) {
            tmem_load16(from + c, y);
            if (!good)
#pragma unroll
                for (int i = 0; i < 16; ++i) y[i] = __uint_as_float(0x7FC00000u);
        };
        if (SWAP) {
            // rows of the result (tokens) are shared out, a lane has a column
            for (uint32_t c = half * 16u; c < (uint32_t)TN; c += 32) {
                float y[16];
                fetch(c, y);
#pragma unroll
                for (uint32_t i = 0; i < 16; ++i) {
                    const uint32_t row = c + i, to = row / own, local = row - to * own;
                    if (right0 + row >= P.rows) break;
                    const uint32_t at = sums + (part * own + local) * 512u + 4 * (quad * 32u + lane);
                    if (to == part) asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(y[i]) : "memory");
                    else send4(peer_addr(at, to), y[i], peer_addr(come, to));
                }
            }
        } else {
            // 16 bytes of 32 rows lie together, then the next four columns
            for (uint32_t c = half * 16u; c < (uint32_t)TN; c += 32) {
                const uint32_t to = c / own, at = c - to * own;
                if (to == part) continue;
                float y[16];
                fetch(c, y);
                const uint32_t from_part = part > to ? part - 1 : part;   // places of the others, without its own
                const uint32_t base = peer_addr(sums + ((from_part * 4 + quad) * own + at) * 128u + lane * 16u, to * CG + rank);
                const uint32_t bar = peer_addr(come, to * CG + rank);
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) send16(base + i * 512u, y + 4 * i, bar);
            }
        }
        if (SWAP) named_bar_sync(1, 256);                             // this CTA's own sums
        const bool all = __all_sync(~0u, parts == 1 || wait_pair_or_stop(come, 0, P.wait_limit, &stop)) && good;
        if (!SWAP) {
            const bool straight = P.out.wide && (!P.add || P.add_wide);
            const uint32_t row = left0 + quad * 32u + lane;
            for (uint32_t c = half * 16u; c < own; c += 32) {
                const uint32_t col = right0 + part * own + c;
                float y[16], add[16];
                if (straight && P.add && row < P.rows) prod_get16(P, row, col, add);
                __syncwarp();
                fetch(part * own + c, y);
                for (uint32_t p = 0; p + 1 < parts; ++p) {
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        float x[4];
                        Elem<float>::widen(lds16(sums + ((p * 4 + quad) * own + c + 4 * i) * 128u + lane * 16u), x);
#pragma unroll
                        for (int j = 0; j < 4; ++j) y[4 * i + j] = __fadd_rn(y[4 * i + j], x[j]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (straight && P.add) y[i] = __fadd_rn(y[i], add[i]);
                    if (!all) y[i] = __uint_as_float(0x7FC00000u);
                }
                if (straight || !all) {                              // (not turned after a wait that ran out: loads may land there)
                    if (row < P.rows) prod_put16(P, row, col, y);
                    __syncwarp();
                    continue;
                }
                // rows that begin anywhere: turned, so that 16 lanes write a row's columns.  (The loads' ring is free.)
                const uint32_t turned = ring + warp * 2048u;
                __syncwarp();
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) sts16(turned + lane * 64u + ((i ^ ((lane >> 1) & 3u)) << 4), Elem<float>::narrow(y + 4 * i));
                __syncwarp();
                const uint32_t x = lane & 15u, row0 = left0 + quad * 32u;
                if (col + x < P.cols)
                    for (uint32_t r0 = lane >> 4; r0 < 32; r0 += 16) {
                        float add8[8];                               // all before the first is written: D may be C
#pragma unroll
                        for (uint32_t i = 0; i < 8; ++i)
                            add8[i] = P.add && row0 + r0 + 2 * i < P.rows ? prod_get1(P, row0 + r0 + 2 * i, col + x) : 0.f;
#pragma unroll
                        for (uint32_t i = 0; i < 8; ++i) {
                            const uint32_t r = r0 + 2 * i;
                            const float v = lds1(turned + r * 64u + (((x >> 2) ^ ((r >> 1) & 3u)) << 4) + 4 * (x & 3));
                            if (row0 + r < P.rows) prod_put1(P, row0 + r, col + x, P.add ? __fadd_rn(v, add8[i]) : v);
                        }
                    }
                __syncwarp();
            }
        } else {
            const uint32_t col = left0 + 4 * lane, n = inside4(col, P.cols);
            for (uint32_t local = warp; local < own_rows; local += 8) {
                const uint32_t row = own_row0 + local;
                float y[4] = {0.f, 0.f, 0.f, 0.f}, c[4];
                if (P.add) prod_get4(P, row, col, n, c);
                for (uint32_t p = 0; p < parts; ++p) {
                    float x[4];
                    Elem<float>::widen(lds16(sums + (p * own + local) * 512u + lane * 16u), x);
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = __fadd_rn(y[i], x[i]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (P.add) y[i] = __fadd_rn(y[i], c[i]);
                    if (!all) y[i] = __uint_as_float(0x7FC00000u);
                }
                if (P.out.dtype < 3) {
                    if (n) prod_put4(P, row, col, n, y);
                    continue;
                }
                uint32_t top = 0;
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)
                    if (i < n) top = max(top, __float_as_uint(y[i]) & 0x7FFFFFFFu);
                top = __reduce_max_sync(~0u, top);
                const uint32_t byte = act8_byte(top, P.out.dtype);
                uint32_t w;
                act8_code<4>(y, act8_down(byte), P.out.dtype, &w);
                unsigned char* to = P.out.data + row * P.out.stride + col;
                if (n == 4) {
                    *reinterpret_cast<uint32_t*>(to) = w;
                } else {
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i)
                        if (i < n) to[i] = (unsigned char)(w >> (8 * i));
                }
                if (lane == 0) P.out.scales[act8_scale_at(row, left0 >> 7, P.out.groups)] = (uint8_t)byte;
            }
        }
        tcgen05_before_sync();
    }
    __syncthreads();                                                  // tensor memory is read
    if (__builtin_expect(ring_end<false>(end, stop, ctas), 0)) {      // nobody sends any more
        const RingLoads loads = {S::kStages, CG, {kProdBox, S::kRight}, {512, 512}, k0, k1 - k0, {}};
        ring_settle<CG, 1>(end, loads, full, [&] { if (parts > 1) mbar_wait(come, 0); });   // and the sums that others sent
        if (tid == 0 && stop && P.status) atomicOr(P.status, kStatusTimeout);
    }
    tcgen05_after_sync();
    if (warp == 9) tmem_free<CG>(tmem, S::kTmem);
}

// ---- tiles of 256 x 256 by pairs of CTAs ------------------------------------------------------------
//
// A pair stays on the GPU and takes every n-th tile.  Each CTA stages its 128 rows of the left operand and
// half of the right one's: 32 KB for 512 clocks of the tensor cores.  Two accumulators of 256 columns and
// the scales do not fit the 512 of tensor memory, so the accumulators share 64: these are read first,
// and the next tile's products begin when they are.
struct ProdPair {
    static constexpr uint32_t kStage = 2 * kProdBox, kScales = 1536;
    static constexpr uint32_t kStages = 6;
    static constexpr uint32_t kEpiWarps = 8, kEpi = 2048;
    static constexpr uint32_t kThreads = 12 * 32;
    static constexpr uint32_t kSmem = kStages * (kStage + kScales) + kEpiWarps * kEpi + 1024;
    static constexpr uint32_t kSecond = 192, kScaleCols = 448, kSlots = 5, kSlotCols = 12;
    static constexpr uint32_t kTmem = 512;
};

// 16-byte piece c of row r in a warp's 2 KB of results, 32 rows of 64 bytes: where the 64-byte swizzle has it, and neither
// eight lanes with a row each nor eight with two whole rows meet in a bank.
__device__ __forceinline__ uint32_t prod_place(uint32_t own, uint32_t r, uint32_t c) { return own + r * 64u + ((c ^ ((r >> 1) & 3u)) << 4); }

// These at the last columns of rows that do not end on a 16-byte boundary, a lane a row.  (Not inline: it would be at every
// store, and cost 2 us in a product of 4096 x 4096 x 128.)
__device__ __noinline__ void prod_edge(const Product8& P, uint32_t own, uint32_t row, uint32_t col, uint32_t es) {
    const uint32_t lane = threadIdx.x & 31u;
    __syncwarp();
    if (row + lane < P.rows && col < P.cols) {
        unsigned char* to = P.out.data + (row + lane) * P.out.stride + (uint64_t)col * es;
        const uint32_t left = min(64u, (P.cols - col) * es);           // bytes
        if (P.in_place) {
            for (uint32_t i = 0; i < left; i += 4) {
                float* f = reinterpret_cast<float*>(to + i);
                *f = __fadd_rn(*f, lds1(prod_place(own, lane, i >> 4) + (i & 15u)));
            }
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 64; i += 16) {
                const uint4 w = lds16(prod_place(own, lane, i >> 4));
                if (i + 16 <= left) {
                    *reinterpret_cast<uint4*>(to + i) = w;
                    continue;
                }
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (uint32_t j = 0; j < 16; ++j) {
                    if (i + j >= left || j % es) continue;
                    const uint32_t v = u[j >> 2] >> (8 * (j & 3));
                    if (es == 4) *reinterpret_cast<uint32_t*>(to + i + j) = v;
                    else if (es == 2) *reinterpret_cast<uint16_t*>(to + i + j) = (uint16_t)v;
                    else to[i + j] = (unsigned char)v;
                }
            }
        }
    }
    __syncwarp();
}

// Results of tiles `begin`, `begin` + `step`, ..., by eight warps: each has 32 rows of its CTA's 128 and half of the columns.
__device__ __forceinline__ void prod_pair_results(const Product8& P, uint32_t tmem, uint32_t own, uint32_t acc_full, uint32_t shared_free,
                                                  uint32_t rank, uint32_t begin, uint32_t end, uint32_t step, volatile uint32_t* stop) {
    using S = ProdPair;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = warp & 3, half = warp >> 2, limit = P.wait_limit;
    // results go out through the warp's 2 KB of shared memory
    auto place = [&](uint32_t r, uint32_t c) { return prod_place(own, r, c); };
    // To the result (or added to it), which clips them, to 16 bytes: where its rows end between two such pieces, those that
    // end go out one by one.  And, before they are written again, whether they have been read.
    const uint32_t es = P.out.dtype == 0 ? 4 : P.out.dtype < 3 ? 2 : 1;
    const bool ragged = P.cols * es % 16 != 0;
    auto send = [&](uint32_t row, uint32_t col) {
        if (ragged && col + 64 / es > P.cols) {
            prod_edge(P, own, row, col, es);
            return;
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            if (P.in_place) tma_add_2d(&P.result, (int)col, (int)row, own);
            else tma_store_2d(&P.result, (int)col, (int)row, own);
            bulk_commit();
        }
    };
    auto sent = [&] {
        if (lane == 0) bulk_wait_read0();
        __syncwarp();
    };
    // what is added to 16 columns of a tile: four of four rows a lane
    const uint32_t piece = lane & 3u;
    auto ahead = [&](uint32_t row0, uint32_t col, uint4 (&to)[4]) {
        const uint32_t m = inside4(col + 4 * piece, P.cols), row = row0 + (lane >> 2);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) to[i] = prod_fetch4(P, row + 8 * i, col + 4 * piece, row + 8 * i < P.rows ? m : 0);
    };
    // A warp whose wait ran out waits for no other tile, whose barrier's phase could pass for an older one's, and says of none
    // any more that it has been read, as that would be taken for another warp's word.
    bool good = true;
    uint32_t n = 0;
    for (uint32_t tile = begin; tile < end; tile += step, ++n) {
        const uint32_t row0 = tile / P.across * 256u + rank * 128u + quad * 32u, col0 = tile % P.across * 256u + half * 128u;
        const bool out = row0 < P.rows && col0 < P.cols;
        if (P.add && !P.in_place && out && row0 + lane < P.rows) {   // C's lines of this warp, while the products run
            const uint32_t es = P.add_dtype ? 2 : 4;
            for (uint32_t at = 0; at < min(128u, P.cols - col0) * es; at += 128)
                asm volatile("prefetch.global.L2 [%0];" ::"l"(P.add + (row0 + lane) * P.add_stride + (uint64_t)col0 * es + at));
        }
        // Columns 192 .. 255 of tensor memory are the next tile's too: the second half's upper 64 in
        // even tiles, the first half's lower 64 in odd ones.  Columns are taken from there on.
        const bool shares = half != (n & 1);
        const uint32_t start = shares && half == 1 ? 64 : 0;
        // where all rows begin on 16-byte boundaries a lane reads what is added to its row, 32 columns ahead
        uint4 more[8];
        auto ask = [&](uint32_t c) {
            const uint32_t col = col0 + c, left = row0 + lane < P.rows && col < P.cols ? min(32u, P.cols - col) : 0;
            const unsigned char* p = P.add + (row0 + lane) * P.add_stride;
            if (left == 32) {
                const uint4* v = reinterpret_cast<const uint4*>(p + (uint64_t)col * (P.add_dtype ? 2 : 4));
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) more[i] = v[i];
                if (P.add_dtype == 0)
#pragma unroll
                    for (uint32_t i = 4; i < 8; ++i) more[i] = v[i];
                return;
            }
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) {                    // the last columns of a row
                uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) {
                    if (P.add_dtype == 0 && j < 4 && 4 * i + j < left) w[j] = reinterpret_cast<const uint32_t*>(p)[col + 4 * i + j];
                    if (P.add_dtype != 0 && i < 4 && 8 * i + j < left)
                        w[j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[col + 8 * i + j] << (16 * (j & 1));
                }
                more[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        };
        auto added = [&](float* y) {
            if (P.add_dtype == 0) {
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) {
                    float x[4];
                    Elem<float>::widen(more[i], x);
#pragma unroll
                    for (int j = 0; j < 4; ++j) y[4 * i + j] = __fadd_rn(y[4 * i + j], x[j]);
                }
                return;
            }
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                float x[8];
                if (P.add_dtype == 1) Elem<__nv_bfloat16>::widen(more[i], x);
                else Elem<__half>::widen(more[i], x);
#pragma unroll
                for (int j = 0; j < 8; ++j) y[8 * i + j] = __fadd_rn(y[8 * i + j], x[j]);
            }
        };
        const bool reads = P.add && !P.in_place && P.add_wide && P.out.wide && out;
        if (reads) ask(start);
        good = good && __all_sync(~0u, wait_or_stop(acc_full + 8 * (n & 1), (n >> 1) & 1, limit, stop));
        tcgen05_after_sync();
        const uint32_t from = tmem + ((quad * 32u) << 16) + (n & 1) * S::kSecond + half * 128u;
        // nobody waits for the last tile's: the first CTA could be gone when the word comes
        const bool tells = good && tile + step < end;
        auto release = [&] {
            tcgen05_before_sync();
            __syncwarp();
            if (lane == 0 && tells) leader_arrive_relaxed(leader_addr(shared_free));
        };
        if (!shares) release();
        if (!out) {
            if (shares) release();
            continue;
        }
        auto fetch32 = [&](uint32_t c, float* y) {
            tmem_load32(from + c, y);
            if (!good)
#pragma unroll
                for (int i = 0; i < 32; ++i) y[i] = __uint_as_float(0x7FC00000u);
        };
        auto fetch16 = [&](uint32_t c, float* y) {
            tmem_load16(from + c, y);
            if (!good)
#pragma unroll
                for (int i = 0; i < 16; ++i) y[i] = __uint_as_float(0x7FC00000u);
        };
        if (P.out.dtype >= 3) {
            // the largest magnitude of this lane's 128 columns first, then the entries; those that the next tile waits for
            // stay in registers meanwhile
            const uint32_t row = row0 + lane, dtype = P.out.dtype, nc = min(128u, P.cols - col0), other = start ^ 64u;
            uint32_t top = 0;
            auto largest = [&](uint32_t c, const float* y) {
#pragma unroll
                for (uint32_t i = 0; i < 32; ++i)
                    if (c + i < nc) top = max(top, __float_as_uint(y[i]) & 0x7FFFFFFFu);
            };
            float y[64];
            fetch32(start, y);
            fetch32(start + 32, y + 32);
            if (shares) release();
            largest(start, y);
            largest(start + 32, y + 32);
#pragma unroll 1
            for (uint32_t c = other; c < other + 64; c += 32) {
                float z[32];
                fetch32(c, z);
                largest(c, z);
            }
            const uint32_t byte = act8_byte(top, dtype);
            const float by = act8_down(byte);
#pragma unroll 1
            for (uint32_t c = start;; c = other) {
                sent();
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                    uint32_t w[4];
                    act8_code<16>(y + 16 * i, by, dtype, w);
                    sts16(place(lane, i), make_uint4(w[0], w[1], w[2], w[3]));
                }
                send(row0, col0 + c);
                if (c == other) break;
                fetch32(other, y);
                fetch32(other + 32, y + 32);
            }
            if (row < P.rows) P.out.scales[act8_scale_at(row, col0 >> 7, P.out.groups)] = (uint8_t)byte;
            continue;
        }
        if (P.out.wide && (!P.add || P.in_place || reads)) {
            // 64 columns to registers, and their place in tensor memory is free for the next tile
#pragma unroll 1
            for (uint32_t at = 0; at < 128; at += 64) {
                const uint32_t c = (at + start) & 127u;
                float y[64];
                fetch32(c, y);
                fetch32(c + 32, y + 32);
                if (at == 0 && shares) release();
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h) {
                    if (reads) {
                        added(y + 32 * h);
                        if (h == 0) ask(c + 32);
                        else if (at == 0) ask((c + 64) & 127u);
                    }
                    if (P.out.dtype == 0) {
#pragma unroll
                        for (uint32_t u = 0; u < 2; ++u) {
                            sent();
#pragma unroll
                            for (uint32_t i = 0; i < 4; ++i) sts16(place(lane, i), Elem<float>::narrow(y + 32 * h + 16 * u + 4 * i));
                            send(row0, col0 + c + 32 * h + 16 * u);
                        }
                    } else {
                        sent();
#pragma unroll
                        for (uint32_t i = 0; i < 4; ++i)
                            sts16(place(lane, i), P.out.dtype == 1 ? Elem<__nv_bfloat16>::narrow(y + 32 * h + 8 * i) : Elem<__half>::narrow(y + 32 * h + 8 * i));
                        send(row0, col0 + c + 32 * h);
                    }
                }
            }
            continue;
        }
        sent();
        if (!P.out_quad && !P.add) {
            // Rows that begin anywhere, in words of four bytes, 16 to a row and two rows at a time; a row of 16-bit
            // entries that begins between two words takes its words from both halves' neighbours, and its
            // first and last entry go out alone.  Word i of row r lies at i ^ (r / 2), so that neither 32
            // rows' same words nor two whole rows meet in a bank.
            const bool four = P.out.dtype == 0;
            const uint32_t rows = min(32u, P.rows - row0), x = lane & 15u, second = lane >> 4;
            const uint32_t step = four ? 16 : 32;                 // columns
#pragma unroll 1
            for (uint32_t at = 0; at < 128; at += step) {
                const uint32_t c = (at + start) & 127u, left = col0 + c < P.cols ? min(step, P.cols - col0 - c) : 0;
                unsigned char* first = P.out.data + row0 * P.out.stride + (uint64_t)(col0 + c) * (four ? 4 : 2);
                uint32_t w[16];
                if (four) {
                    fetch16(c, reinterpret_cast<float*>(w));
                } else {
                    float y[32];
                    fetch32(c, y);
#pragma unroll
                    for (uint32_t i = 0; i < 16; ++i)
                        w[i] = P.out.dtype == 1 ? Elem<__nv_bfloat16>::pair(y[2 * i], y[2 * i + 1]) : Elem<__half>::pair(y[2 * i], y[2 * i + 1]);
                }
                if (at + step == 64 && shares) release();
                __syncwarp();                                     // what was here has been read
                if (!left) continue;
#pragma unroll
                for (uint32_t i = 0; i < 16; ++i)
                    asm volatile("st.shared.u32 [%0], %1;" ::"r"(own + lane * 64u + ((i ^ (lane >> 1)) << 2)), "r"(w[i]) : "memory");
                if (!four) {
                    uint16_t* mine = reinterpret_cast<uint16_t*>(first + lane * P.out.stride);
                    if (lane < rows && (reinterpret_cast<uintptr_t>(mine) & 2u)) {
                        mine[0] = (uint16_t)w[0];
                        if (left == 32) mine[31] = (uint16_t)(w[15] >> 16);
                    }
                }
                __syncwarp();
                // this lane's word of rows `second`, `second` + 2, ...; rows alike in parity by the stride's
                unsigned char* to = first + second * P.out.stride + 4 * x;
#pragma unroll
                for (uint32_t k = 0; k < 16; ++k, to += 2 * P.out.stride) {
                    const uint32_t line = own + k * 128u + second * 64u;
                    uint32_t v, next = 0;
                    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(line + ((x ^ k) << 2)));
                    if (four) {
                        if (2 * k + second < rows && x < left) *reinterpret_cast<uint32_t*>(to) = v;
                        continue;
                    }
                    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(next) : "r"(line + (((x + 1) & 15u) ^ k) * 4u));
                    const uint32_t odd = (uint32_t)(reinterpret_cast<uintptr_t>(to) >> 1) & 1u, e = 2 * x + odd;   // first entry
                    v = __funnelshift_r(v, next, 16 * odd);
                    if (2 * k + second >= rows) continue;
                    if (e + 1 < left) *reinterpret_cast<uint32_t*>(to + 2 * odd) = v;
                    else if (e < left && !(odd && left == 32)) *reinterpret_cast<uint16_t*>(to + 2 * odd) = (uint16_t)v;
                }
            }
            continue;
        }
        if (!P.out_quad || (P.add && !P.add_quad)) {
            // rows that begin anywhere: a lane a column, two rows at a time
            const uint32_t rows = min(32u, P.rows - row0), x = lane & 15u;
            const bool four = P.out.dtype == 0, bf16 = P.out.dtype == 1;
#pragma unroll 1
            for (uint32_t at = 0; at < 128; at += 16) {
                const uint32_t c = (at + start) & 127u, col = col0 + c + x;
                float y[16];
                fetch16(c, y);
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) sts16(place(lane, i), Elem<float>::narrow(y + 4 * i));
                if (at == 48 && shares) release();
                __syncwarp();
                unsigned char* to = P.out.data + (row0 + (lane >> 4)) * P.out.stride + (uint64_t)col * (four ? 4 : 2);
                if (col < P.cols)
#pragma unroll 1
                    for (uint32_t r0 = lane >> 4; r0 < rows; r0 += 16) {
                        float add[8];                            // all before the first is written: D may be C
                        if (P.add)
#pragma unroll
                            for (uint32_t i = 0; i < 8; ++i) add[i] = r0 + 2 * i < rows ? prod_get1(P, row0 + r0 + 2 * i, col) : 0.f;
#pragma unroll
                        for (uint32_t i = 0; i < 8; ++i, to += 2 * P.out.stride) {
                            const uint32_t r = r0 + 2 * i;
                            float v = lds1(place(r, x >> 2) + 4 * (x & 3u));
                            if (P.add) v = __fadd_rn(v, add[i]);
                            if (r >= rows) continue;
                            if (four) *reinterpret_cast<float*>(to) = v;
                            else *reinterpret_cast<uint16_t*>(to) = bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
                        }
                    }
                __syncwarp();
            }
            continue;
        }
        // what is added is asked for 16 columns ahead
        uint4 next[4];
        if (P.add) ahead(row0, col0 + start, next);
#pragma unroll 1
        for (uint32_t at = 0; at < 128; at += 16) {
            const uint32_t c = (at + start) & 127u, col = col0 + c + 4 * piece, m = inside4(col, P.cols);
            float y[16];
            fetch16(c, y);
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) sts16(place(lane, i), Elem<float>::narrow(y + 4 * i));
            if (at == 48 && shares) release();
            __syncwarp();
            uint4 now[4];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) now[i] = next[i];
            if (P.add && at < 112) ahead(row0, col0 + ((c + 16) & 127u), next);
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                const uint32_t r = 8 * i + (lane >> 2);
                float x[4], add[4];
                Elem<float>::widen(lds16(place(r, piece)), x);
                if (row0 + r >= P.rows || !m) continue;
                if (P.add) {
                    prod_widen4(P.add_dtype, now[i], add);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = __fadd_rn(x[j], add[j]);
                }
                prod_put4(P, row0 + r, col, m, x);
            }
            __syncwarp();
        }
    }
    if (lane == 0) bulk_wait_all();
}

__global__ void __launch_bounds__(ProdPair::kThreads, 1) act8_product_pair_kernel(const __grid_constant__ Product8 P) {
    using S = ProdPair;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::kStages + 3];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t stop;
    __shared__ volatile RingEnd end;
    const uint32_t tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31;
    const uint32_t ring = (smem_u32(raw) + 1023u) & ~1023u, epi = ring + S::kStages * S::kStage, scales = epi + S::kEpiWarps * S::kEpi;
    const uint32_t full = smem_u32(bars), empty = full + 8 * S::kStages, acc_full = empty + 8 * S::kStages, shared_free = acc_full + 16;
    const uint32_t rank = cta_rank(), limit = P.wait_limit, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    if (tid == 0) {
        for (uint32_t s = 0; s < S::kStages; ++s) { mbar_init(full + 8 * s, 2); mbar_init(empty + 8 * s, 1); }
        mbar_init(acc_full, 1);
        mbar_init(acc_full + 8, 1);
        mbar_init(shared_free, 2 * S::kEpiWarps);
        stop = 0;
        end.halted = 0;
        fence_mbar_init();
    }
    if ((warp == 8 || warp == 10) && elect_one()) {
        prefetch_map(warp == 8 ? &P.left : &P.right);
        prefetch_map(warp == 8 ? &P.left_scales : &P.right_scales);
    }
    if (warp == 9) tmem_alloc<2>(smem_u32(&tmem_slot), S::kTmem);
    tcgen05_before_sync();
    __syncthreads();
    cluster_sync_relaxed();
    tcgen05_after_sync();
    const uint32_t tmem = tmem_slot;
    griddep_launch();
    griddep_wait();

    if (warp == 8 || warp == 10) {
        // ---- loads: a warp for each operand, in both CTAs; bytes are counted on the first CTA's barriers
        if (elect_one()) {
            const bool left = warp == 8;
            const void* map = left ? &P.left : &P.right;
            const void* smap = left ? &P.left_scales : &P.right_scales;
            const uint32_t at = left ? 0 : kProdBox, groups = left ? P.left_groups : P.right_groups;
            uint32_t it = 0;
            bool ok = true;
            for (uint32_t tile = pair; ok && tile < P.tiles; tile += pairs) {
                const uint32_t row = (left ? tile / P.across : tile % P.across) * 256u + rank * 128u;
                // the second half of the last tile's right rows may be beyond the scales: any will do
                const uint32_t group0 = (row >> 7) * groups, both0 = (tile % P.across) * 2u * groups;
                for (uint32_t k = 0; k < P.steps; ++k, ++it) {
                    const uint32_t s = it % S::kStages;
                    if (!wait_or_stop(empty + 8 * s, ((it / S::kStages) & 1) ^ 1, limit, &stop)) { ok = false; break; }
                    const bool with = (k & 3) == 0;
                    const uint32_t bar = leader_addr(full + 8 * s), sat = scales + s * S::kScales;
                    if (rank == 0) mbar_arrive_expect_tx(full + 8 * s, 2 * (kProdBox + (with ? left ? 512u : 1024u : 0u)));
                    prod_load<2>(ring + s * S::kStage + at, map, k * kProdRow, row, bar);
                    if (with) {
                        if (left) {
                            prod_load<2>(sat, smap, 0, group0 + (k >> 2), bar);
                        } else {
                            prod_load<2>(sat + 512, smap, 0, both0 + (k >> 2), bar);
                            prod_load<2>(sat + 1024, smap, 0, both0 + groups + (k >> 2), bar);
                        }
                    }
                }
            }
            end.asked[left ? 0 : 1] = it;
            // nothing of this CTA's is in flight when it leaves
            for (uint32_t b = 0; b < S::kStages && b < it; ++b) {
                const uint32_t last = it - 1 - b;
                if (!wait_or_stop(empty + 8 * (last % S::kStages), (last / S::kStages) & 1, limit, &stop)) break;
            }
        }
    } else if (warp == 9) {
        // ---- products, by the first CTA
        if (rank == 0 && elect_one()) {
            const uint32_t idesc = P.formats | (1u << 23) | ((256u / 8) << 17) | ((256u / 16) << 24);
            uint32_t it = 0, n = 0, group = 0, sc = 0;
            bool ok = true;
            for (uint32_t tile = pair; tile < P.tiles; tile += pairs, ++n) {
                if (n && !wait_pair_or_stop(shared_free, (n - 1) & 1, limit, &stop)) break;
                tcgen05_after_sync();
                const uint32_t d = tmem + (n & 1) * S::kSecond;
                for (uint32_t k = 0; k < P.steps; ++k, ++it) {
                    const uint32_t s = it % S::kStages;
                    if (!wait_or_stop(full + 8 * s, (it / S::kStages) & 1, limit, &stop)) { ok = false; break; }
                    tcgen05_after_sync();
                    if ((k & 3) == 0) {
                        // places in turn, whose last use is over: in a tile 16 steps are between, and a tile begins when the
                        // one before it is over
                        sc = tmem + S::kScaleCols + group * S::kSlotCols;
                        group = group + 1 == S::kSlots ? 0 : group + 1;
                        umma_scales<2>(sc, scales + s * S::kScales);
                        umma_scales<2>(sc + 4, scales + s * S::kScales + 512);
                        umma_scales<2>(sc + 8, scales + s * S::kScales + 1024);
                    }
                    const uint32_t id = idesc | (k & 3) << 29 | (k & 3) << 4, steps = k + 1 == P.steps ? P.tail : 4;
                    const uint64_t a = umma_desc_swizzled(ring + s * S::kStage), b = umma_desc_swizzled(ring + s * S::kStage + kProdBox);
                    for (uint32_t q = 0; q < steps; ++q) umma_mx8<2>(d, a + 2 * q, b + 2 * q, id, sc, sc + 4, k > 0 || q > 0);
                    umma_commit<2>(empty + 8 * s);
                }
                if (!ok) break;
                umma_commit<2>(acc_full + 8 * (n & 1));
            }
            end.multiplied = it;
            end.committed = n;
        }
    } else if (warp < S::kEpiWarps) {
        prod_pair_results(P, tmem, epi + warp * S::kEpi, acc_full, shared_free, rank, pair, P.tiles, pairs, &stop);
    }
    __syncwarp();
    tcgen05_before_sync();
    __syncthreads();
    if (__builtin_expect(ring_end<false>(end, stop, 2), 0)) {
        const RingLoads loads = {S::kStages, 2, {kProdBox, kProdBox}, {512, 1024}, 0, P.steps, {}};
        ring_settle<2, 2>(end, loads, full, [] {});
        if (tid == 0 && stop && P.status) atomicOr(P.status, kStatusTimeout);
    }
    tcgen05_after_sync();
    if (warp == 9) tmem_free<2>(tmem, S::kTmem);
}

}  // namespace ecq
