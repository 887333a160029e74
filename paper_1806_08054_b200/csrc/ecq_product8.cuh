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
// the last; against 64 bits, 5e-8 to 4e-7 of the result (1024 terms).
//
// Operands go to shared memory as they lie in memory, 128 bytes of 128 rows at a time, in the
// 128-byte swizzle; scale bytes in their groups of 512, from where tcgen05.cp takes them to tensor
// memory for each four blocks.

struct Product8 {
    CUtensorMap left, right, left_scales, right_scales;
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
    int add_dtype, add_wide;
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

// Four columns of C.
__device__ __forceinline__ void prod_add4(const Product8& P, uint32_t row, uint32_t col, uint32_t n, float* y) {
    const unsigned char* p = P.add + row * P.add_stride;
    float c[4] = {0.f, 0.f, 0.f, 0.f};
    if (P.add_dtype == 0) {
        const float* f = reinterpret_cast<const float*>(p) + col;
        if (n == 4 && P.add_wide) {
            Elem<float>::widen(*reinterpret_cast<const uint4*>(f), c);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (i < n) c[i] = f[i];
        }
    } else {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(p) + col;
        uint32_t w[2] = {0, 0};
        if (n == 4 && P.add_wide) {
            const uint2 u = *reinterpret_cast<const uint2*>(h);
            w[0] = u.x; w[1] = u.y;
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (i < n) w[i >> 1] |= (uint32_t)h[i] << (16 * (i & 1));
        }
        float x[8];
        if (P.add_dtype == 1) Elem<__nv_bfloat16>::widen(make_uint4(w[0], w[1], 0, 0), x);
        else Elem<__half>::widen(make_uint4(w[0], w[1], 0, 0), x);
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = x[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __fadd_rn(y[i], c[i]);
}

// Four columns of a plain result.
__device__ __forceinline__ void prod_put4(const Product8& P, uint32_t row, uint32_t col, uint32_t n, const float* y) {
    unsigned char* p = P.out.data + row * P.out.stride;
    if (P.out.dtype == 0) {
        float* f = reinterpret_cast<float*>(p) + col;
        if (n == 4 && P.out.wide) {
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
    if (n == 4 && P.out.wide) {
        *reinterpret_cast<uint2*>(h) = w;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (i < n) h[i] = (uint16_t)((i < 2 ? w.x : w.y) >> (16 * (i & 1)));
    }
}

__device__ __forceinline__ uint32_t inside4(uint32_t col, uint32_t cols) { return col >= cols ? 0u : min(4u, cols - col); }

// ---- tiles of 128 x TN, K over a cluster ------------------------------------------------------------
//
// For products that have few tiles: a cluster's CTAs have a part of K each.  Their sums meet through
// shared memory: each CTA finishes its share of the tile's rows, to which all others have sent theirs, and
// adds them in the CTAs' order.  SWAP: the left operand is B and the right one A (a few tokens), the tile
// is D's transposed; so a matrix of weights fills the 128 rows of an instruction.

template <int TN, bool SWAP>
struct ProdPart {
    static constexpr uint32_t kRight = TN * kProdRow;
    static constexpr uint32_t kStage = kProdBox + kRight;
    static constexpr uint32_t kStages = 6;
    static constexpr uint32_t kOutRows = SWAP ? TN : 128;             // of a tile, 128 columns each
    static constexpr uint32_t kRing = kStages * kStage;
    static constexpr uint32_t kSmem = (kRing > kOutRows * 512u ? kRing : kOutRows * 512u) + kStages * 1024u + 1024u;
    static constexpr uint32_t kScaleCols = TN < 32 ? 32 : TN;         // first column of scales in tensor memory
    static constexpr uint32_t kTmem = TN <= 32 ? 128 : TN <= 64 ? 128 : 256;
    static constexpr uint32_t kThreads = 12 * 32;
};

template <int TN, bool SWAP>
__global__ void __launch_bounds__(ProdPart<TN, SWAP>::kThreads, 1) act8_product_part_kernel(const __grid_constant__ Product8 P) {
    using S = ProdPart<TN, SWAP>;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::kStages + 1];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t stop;
    const uint32_t tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31;
    const uint32_t ring = (smem_u32(raw) + 1023u) & ~1023u, scales = ring + (S::kSmem - 1024u - S::kStages * 1024u);
    const uint32_t full = smem_u32(bars), empty = full + 8 * S::kStages, done = empty + 8 * S::kStages;
    uint32_t parts;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
    const uint32_t cta = cta_rank(), tile = blockIdx.x / parts;
    const uint32_t left0 = tile / P.across * 128u, right0 = tile % P.across * (uint32_t)TN;
    const uint32_t k0 = (uint32_t)((uint64_t)cta * P.steps / parts), k1 = (uint32_t)((uint64_t)(cta + 1) * P.steps / parts);
    if (tid == 0) {
        for (uint32_t s = 0; s < S::kStages; ++s) { mbar_init(full + 8 * s, 2); mbar_init(empty + 8 * s, 1); }
        mbar_init(done, 1);
        stop = 0;
        fence_mbar_init();
    }
    if (warp == 9) tmem_alloc<1>(smem_u32(&tmem_slot), S::kTmem);
    tcgen05_before_sync();
    __syncthreads();
    tcgen05_after_sync();
    const uint32_t tmem = tmem_slot;
    griddep_launch();
    griddep_wait();

    if (warp == 8 || warp == 10) {
        // ---- loads: a warp for each operand
        if (elect_one()) {
            const bool left = warp == 8;
            const void* map = left ? &P.left : &P.right;
            const void* smap = left ? &P.left_scales : &P.right_scales;
            const uint32_t at = left ? 0 : kProdBox, bytes = left ? kProdBox : S::kRight, row = left ? left0 : right0;
            const uint32_t group0 = (row >> 7) * (left ? P.left_groups : P.right_groups), sat = scales + (left ? 0 : 512);
            uint32_t it = 0;
            for (uint32_t k = k0; k < k1; ++k, ++it) {
                const uint32_t s = it % S::kStages;
                if (!wait_or_stop(empty + 8 * s, ((it / S::kStages) & 1) ^ 1, P.wait_limit, &stop)) break;
                const bool with = k == k0 || (k & 3) == 0;
                mbar_arrive_expect_tx(full + 8 * s, bytes + (with ? 512u : 0u));
                prod_load<1>(ring + s * S::kStage + at, map, k * kProdRow, row, full + 8 * s);
                if (with) prod_load<1>(sat + s * 1024u, smap, 0, group0 + (k >> 2), full + 8 * s);
            }
            // none of them is in flight when this CTA leaves
            for (uint32_t b = 0; b < S::kStages && b < it; ++b) {
                const uint32_t last = it - 1 - b, most = stop ? 1u << 12 : kWaitLimit;
                for (uint32_t n = 0; n < most; ++n)
                    if (mbar_try_wait(empty + 8 * (last % S::kStages), (last / S::kStages) & 1)) break;
            }
        }
        __syncwarp();
    } else if (warp == 9) {
        // ---- products
        if (elect_one()) {
            const uint32_t idesc = P.formats | (1u << 23) | ((uint32_t)(TN / 8) << 17) | ((128u / 16) << 24);
            uint32_t it = 0, slot = 0;
            // the right operand's scales begin at its row in their group of 128
            const uint32_t sb_at = S::kScaleCols + 4 + ((right0 & 127u) >> 5);
            for (uint32_t k = k0; k < k1; ++k, ++it) {
                const uint32_t s = it % S::kStages;
                if (!wait_or_stop(full + 8 * s, (it / S::kStages) & 1, P.wait_limit, &stop)) break;
                tcgen05_after_sync();
                if (k == k0 || (k & 3) == 0) {
                    // one of three places in turn: what used it last is two groups behind
                    slot = it == 0 ? 0 : slot == 16 ? 0 : slot + 8;
                    umma_scales<1>(tmem + S::kScaleCols + slot, scales + s * 1024u);
                    umma_scales<1>(tmem + S::kScaleCols + slot + 4, scales + s * 1024u + 512u);
                }
                const uint32_t id = idesc | (k & 3) << 29 | (k & 3) << 4, steps = k + 1 == P.steps ? P.tail : 4;
                const uint64_t a = umma_desc_swizzled(ring + s * S::kStage), b = umma_desc_swizzled(ring + s * S::kStage + kProdBox);
                for (uint32_t q = 0; q < steps; ++q)
                    umma_mx8<1>(tmem, a + 2 * q, b + 2 * q, id, tmem + S::kScaleCols + slot, tmem + sb_at + slot, it > 0 || q > 0);
                umma_commit<1>(empty + 8 * s);
            }
            umma_commit<1>(done);
        }
        __syncwarp();
    }
    // every product of this CTA is done, and with them its loads: the ring has room for sums
    const bool mine = wait_or_stop(done, 0, P.wait_limit, &stop);
    __syncwarp();
    tcgen05_after_sync();
    pair_sync();
    const uint32_t share = S::kOutRows / parts, quad = warp & 3, half = warp >> 2;
    if (warp < 8) {
        // this warp's 32 rows of the tile and half of its columns, to the CTAs that finish them
        const uint32_t from = tmem + ((quad * 32u) << 16);
        constexpr uint32_t kCols = TN / 2 < 16 ? 16 : TN / 2;
        const bool good = mine && !stop;
        if (half * kCols < (uint32_t)TN) {
#pragma unroll
            for (uint32_t b = 0; b < kCols; b += 16) {
                float y[16];
                tmem_load16(from + half * kCols + b, y);
                if (!good)
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] = __uint_as_float(0x7FC00000u);
                if (SWAP) {
                    const uint32_t c = quad * 32u + lane;
#pragma unroll
                    for (uint32_t i = 0; i < 16; ++i) {
                        const uint32_t row = half * kCols + b + i, to = row / share, local = row - to * share;
                        const uint32_t at = ring + (cta * share + local) * 512u + (((c >> 2) ^ (local & 7u)) << 4) + 4 * (c & 3);
                        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(peer_addr(at, to)), "f"(y[i]) : "memory");
                    }
                } else {
                    const uint32_t row = quad * 32u + lane, to = row / share, local = row - to * share;
                    const uint32_t base = peer_addr(ring + (cta * share + local) * 512u, to);
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        const uint32_t piece = (half * kCols + b) / 4 + i;
                        asm volatile("st.shared::cluster.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(base + ((piece ^ (local & 7u)) << 4)),
                                     "f"(y[4 * i]), "f"(y[4 * i + 1]), "f"(y[4 * i + 2]), "f"(y[4 * i + 3]) : "memory");
                    }
                }
            }
        }
    }
    tcgen05_before_sync();
    pair_sync();
    if (warp == 9) tmem_free<1>(tmem, S::kTmem);
    if (warp < 8) {
        const uint32_t row0 = (SWAP ? right0 : left0) + cta * share, col0 = SWAP ? left0 : right0, col = col0 + 4 * lane;
        const uint32_t n = inside4(col, P.cols);
        for (uint32_t local = warp; local < share && row0 + local < P.rows; local += 8) {
            const uint32_t row = row0 + local;
            float y[4] = {0.f, 0.f, 0.f, 0.f};
            for (uint32_t p = 0; p < parts; ++p) {
                float x[4];
                Elem<float>::widen(lds16(ring + (p * share + local) * 512u + ((lane ^ (local & 7u)) << 4)), x);
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = __fadd_rn(y[i], x[i]);
            }
            if (P.add && n) prod_add4(P, row, col, n, y);
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
            if (lane == 0) P.out.scales[act8_scale_at(row, col0 >> 7, P.out.groups)] = (uint8_t)byte;
        }
    }
    if (tid == 0 && stop && P.status) atomicOr(P.status, kStatusTimeout);
}

// ---- tiles of 256 x 256 by pairs of CTAs ------------------------------------------------------------
//
// A pair stays on the GPU and takes every n-th tile.  Each CTA stages its 128 rows of the left operand and
// half of the right one's: 32 KB for 512 clocks of the tensor cores.  Two accumulators of 256 columns and
// the scales do not fit the 512 of tensor memory, so the accumulators share 64: these are read first,
// and the next tile's products begin when they are.
struct ProdPair {
    static constexpr uint32_t kStage = 2 * kProdBox, kScales = 1536;
    static constexpr uint32_t kStages = 5;
    static constexpr uint32_t kEpiWarps = 8, kEpi = 4096;
    static constexpr uint32_t kThreads = 12 * 32;
    static constexpr uint32_t kSmem = kStages * (kStage + kScales) + kEpiWarps * kEpi + 1024;
    static constexpr uint32_t kSecond = 192, kScaleCols = 448, kSlots = 5, kSlotCols = 12;
    static constexpr uint32_t kTmem = 512;
};

__global__ void __launch_bounds__(ProdPair::kThreads, 1) act8_product_pair_kernel(const __grid_constant__ Product8 P) {
    using S = ProdPair;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::kStages + 3];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t stop;
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
        fence_mbar_init();
    }
    if (warp == 9) tmem_alloc<2>(smem_u32(&tmem_slot), S::kTmem);
    tcgen05_before_sync();
    __syncthreads();
    pair_sync();
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
            // nothing of this CTA's is in flight when it leaves
            for (uint32_t b = 0; b < S::kStages && b < it; ++b) {
                const uint32_t last = it - 1 - b, most = stop ? 1u << 12 : kWaitLimit;
                for (uint32_t n = 0; n < most; ++n)
                    if (mbar_try_wait(empty + 8 * (last % S::kStages), (last / S::kStages) & 1)) break;
            }
        }
    } else if (warp == 9) {
        // ---- products, by the first CTA
        if (rank == 0 && elect_one()) {
            const uint32_t idesc = P.formats | (1u << 23) | ((256u / 8) << 17) | ((256u / 16) << 24);
            uint32_t it = 0, n = 0, group = 0, sc = 0;
            bool ok = true;
            for (uint32_t tile = pair; ok && tile < P.tiles; tile += pairs, ++n) {
                if (n && !wait_pair_or_stop(shared_free, (n - 1) & 1, limit, &stop)) break;
                tcgen05_after_sync();
                const uint32_t d = tmem + (n & 1) * S::kSecond;
                for (uint32_t k = 0; k < P.steps; ++k, ++it) {
                    const uint32_t s = it % S::kStages;
                    if (!wait_or_stop(full + 8 * s, (it / S::kStages) & 1, limit, &stop)) { ok = false; break; }
                    tcgen05_after_sync();
                    if ((k & 3) == 0) {
                        // five places in turn: their last use is five steps behind, and over
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
                if (ok) umma_commit<2>(acc_full + 8 * (n & 1));
            }
        }
    } else if (warp < S::kEpiWarps) {
        // ---- results: a warp has 32 rows and half of the columns
        const uint32_t quad = warp & 3, half = warp >> 2, own = epi + warp * S::kEpi;
        uint32_t n = 0;
        for (uint32_t tile = pair; tile < P.tiles; tile += pairs, ++n) {
            const bool good = __all_sync(~0u, wait_or_stop(acc_full + 8 * (n & 1), (n >> 1) & 1, limit, &stop));
            tcgen05_after_sync();
            const uint32_t row0 = tile / P.across * 256u + rank * 128u + quad * 32u, col0 = tile % P.across * 256u + half * 128u;
            const uint32_t from = tmem + ((quad * 32u) << 16) + (n & 1) * S::kSecond + half * 128u;
            // Columns 192 .. 255 of tensor memory are the next tile's too: the second half's upper 64 in
            // even tiles, the first half's lower 64 in odd ones.  Blocks of 32 columns begin there.
            const bool shares = half != (n & 1), high = shares && half == 1;
            auto release = [&] {
                tcgen05_before_sync();
                __syncwarp();
                if (lane == 0) leader_arrive(leader_addr(shared_free));
            };
            if (!shares) release();
            const bool out = row0 < P.rows && col0 < P.cols;
            if (!out) {
                if (shares) release();
                continue;
            }
            auto fetch = [&](uint32_t b, float* y) {
                tmem_load32(from + 32 * b, y);
                if (!good)
#pragma unroll
                    for (int i = 0; i < 32; ++i) y[i] = __uint_as_float(0x7FC00000u);
            };
            if (P.out.dtype >= 3) {
                // the largest magnitude of this lane's 128 columns first, then the entries
                const uint32_t row = row0 + lane, dtype = P.out.dtype;
                uint32_t top = 0;
                const uint32_t nc = min(128u, P.cols - col0);
#pragma unroll 1
                for (uint32_t b = 0; b < 4; ++b) {
                    float y[32];
                    fetch(b, y);
#pragma unroll
                    for (uint32_t i = 0; i < 32; ++i)
                        if (32 * b + i < nc) top = max(top, __float_as_uint(y[i]) & 0x7FFFFFFFu);
                }
                const uint32_t byte = act8_byte(top, dtype);
                const float by = act8_down(byte);
#pragma unroll 1
                for (uint32_t b = 0; b < 4; ++b) {
                    float y[32];
                    fetch(b, y);
#pragma unroll
                    for (uint32_t c = 0; c < 2; ++c) {
                        uint32_t w[4];
                        act8_code<16>(y + 16 * c, by, dtype, w);
                        sts16(own + lane * 128u + (((2 * b + c) ^ (lane & 7u)) << 4), make_uint4(w[0], w[1], w[2], w[3]));
                    }
                }
                if (shares) release();
                __syncwarp();
                if (row < P.rows) P.out.scales[act8_scale_at(row, col0 >> 7, P.out.groups)] = (uint8_t)byte;
                const uint32_t piece = lane & 7u, left = col0 + 16 * piece < P.cols ? P.cols - col0 - 16 * piece : 0;
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) {
                    const uint32_t r = 4 * i + (lane >> 3);
                    const uint4 w = lds16(own + r * 128u + ((piece ^ (r & 7u)) << 4));
                    if (row0 + r >= P.rows) continue;
                    unsigned char* to = P.out.data + (row0 + r) * P.out.stride + col0 + 16 * piece;
                    if (left >= 16) {
                        *reinterpret_cast<uint4*>(to) = w;
                    } else {
                        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (uint32_t j = 0; j < 16; ++j)
                            if (j < left) to[j] = (unsigned char)(u[j >> 2] >> (8 * (j & 3)));
                    }
                }
                __syncwarp();
                continue;
            }
            if (P.out.dtype != 0 && !P.add && P.out.wide && col0 + 128 <= P.cols) {
                // 16 bits, whole rows of 64 columns: 128 bytes a row
#pragma unroll 1
                for (uint32_t c = 0; c < 2; ++c) {
                    const uint32_t b = 2 * (c ^ (high ? 1u : 0u));
#pragma unroll
                    for (uint32_t h = 0; h < 2; ++h) {
                        float y[32];
                        fetch(b + h, y);
#pragma unroll
                        for (uint32_t i = 0; i < 4; ++i)
                            sts16(own + lane * 128u + (((4 * h + i) ^ (lane & 7u)) << 4),
                                  P.out.dtype == 1 ? Elem<__nv_bfloat16>::narrow(y + 8 * i) : Elem<__half>::narrow(y + 8 * i));
                    }
                    if (c == 0 && shares) release();
                    __syncwarp();
                    const uint32_t piece = lane & 7u;
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) {
                        const uint32_t r = 4 * i + (lane >> 3);
                        const uint4 w = lds16(own + r * 128u + ((piece ^ (r & 7u)) << 4));
                        if (row0 + r < P.rows)
                            *reinterpret_cast<uint4*>(P.out.data + (row0 + r) * P.out.stride + (col0 + 32 * b + 8 * piece) * 2ull) = w;
                    }
                    __syncwarp();
                }
                continue;
            }
#pragma unroll 1
            for (uint32_t c = 0; c < 4; ++c) {
                const uint32_t b = high ? c ^ 2u : c;
                float y[32];
                fetch(b, y);
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) sts16(own + lane * 128u + ((i ^ (lane & 7u)) << 4), Elem<float>::narrow(y + 4 * i));
                if (c == 1 && shares) release();
                __syncwarp();
                const uint32_t piece = lane & 7u, col = col0 + 32 * b + 4 * piece, m = inside4(col, P.cols);
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) {
                    const uint32_t r = 4 * i + (lane >> 3);
                    float x[4];
                    Elem<float>::widen(lds16(own + r * 128u + ((piece ^ (r & 7u)) << 4)), x);
                    if (row0 + r >= P.rows || !m) continue;
                    if (P.add) prod_add4(P, row0 + r, col, m, x);
                    prod_put4(P, row0 + r, col, m, x);
                }
                __syncwarp();
            }
        }
    }
    __syncwarp();
    tcgen05_before_sync();
    __syncthreads();
    pair_sync();
    tcgen05_after_sync();
    // after a wait that ran out, loads and arrivals for this CTA may still be on their way
    if (stop)
        for (const long long since = clock64(); clock64() - since < 20000;) {}
    if (tid == 0 && stop && P.status) atomicOr(P.status, kStatusTimeout);
    if (warp == 9) tmem_free<2>(tmem, S::kTmem);
}

}  // namespace ecq
