// Newton-Schulz orthogonalisation of the matrices of a flat vector, with the momentum in front of
// it and the weight update behind it.
#pragma once

#include <cstdint>

#include <cuda.h>

#include "ecq_common.cuh"
#include "ecq_elem.cuh"

namespace ecq {

// The iteration, for a matrix taken with m <= n (a tall one is transposed on the way in and out):
//     X_0 = U / |U|_F,   X <- a X + (b G + c G^2) X,   G = X X^T
// Three products a step: G and G^2 are symmetric, so only tiles that touch the lower triangle are
// computed and written twice; the third is full.
//
// Merged steps.  For wide matrices the first steps need not touch X one by one: with B = b G + c G^2,
//     X' = (alpha I + R) X,  G' = (a I + B) G (a I + B)
// every matrix being a polynomial in the first G, all of them commute and all products are
// symmetric.  A further step costs, instead of G and a product with X (3 m^2 n), the products
//     S = a G + B G,  G' = a S + B S,  R' = a R + alpha B + B R,  alpha' = a alpha
// (3 m^3) and none of X's memory traffic.  Rounding errors of G' grow by a^2 a step relative to
// small eigenvalues, so this is done for the first three steps at most, in which singular values
// are brought up to order 1, with G and S as pairs: no difference in the result's error was
// measured against single steps.  (All five merged: up to 0.5.)
//
// Numbers.  The products run on the tensor cores with fp16 operands and fp32 accumulators.  What
// keeps the result accurate is that X itself is not rounded to 11 bits: it is a pair hi + lo of fp16
// (22 bits) of which the products take hi, and the linear term a X both.  A rounding error of X in the
// directions of small singular values would be multiplied by a (3.44) in every step.  Against 64
// bits, relative error of the result for spectra from flat to 1/i^1.5: bf16 throughout 1e-2 to
// 9e-2, fp16 throughout 1e-3 to 1e-2, with the pair 3e-4 to 1.7e-3.  The last two steps have
// nothing left to amplify, and X has no low half there (no difference measured).
// In the last two steps, where most singular values are near 1, G is replaced by D = G - I
// (exactly the same polynomial: b G + c G^2 = (b + c) I + (b + 2c) D + c D^2), so that the
// rounding of G's diagonal does not cancel against a X: 5e-4 to 1.1e-3.  (Not with coefficients whose
// iterates stay far below 1, for which it would.)
// With SPLIT, operands are pairs hi + lo of fp16 (22 bits), of which three products are taken
// (hi hi, hi lo, lo hi), and the result's error is that of fp32 arithmetic.
//
// X, G and the polynomial are stored scaled by powers of two, so that fp16's narrow range holds
// entries as small as 1 / (m n)^0.5 and their low halves.

constexpr float kMuonScaleX = 4096.f;
constexpr float kMuonScaleG = 256.f;

struct MuonMat {
    uint64_t offset, stride;             // in the caller's flat vectors, entries
    uint32_t rows, cols, m, n;
    uint32_t x_tile, m_tile;             // first tile in each X and m x m buffer of the workspace
    uint32_t pad, down;                  // m rounded up to 64; tiles below each other, of 128 rows
    uint32_t part0, parts;               // its partial sums of squares
    uint32_t tall;
    float scale;
};

// What the passes over the caller's vectors take.
struct MuonIn {
    const void* grad;
    float* momentum;                     // NULL: the matrices themselves are orthogonalised
    float mu;
    int nesterov;
};

struct MuonOut {
    float* params;                       // NULL, or params <- keep * params - rate * scale * O
    void* update;                        // NULL, or update = scale * O
    float keep, rate;
    int scaled;                          // 0: the update is O itself
};


// The workspace is an array of tiles of 128 rows and 64 columns of fp16, 16 KB each, those of a
// matrix's first 64 columns below each other first.  In a tile 16-byte pieces of 128 rows follow
// each other, then the next pieces: the image that a tensor-core operand without swizzle has in
// shared memory, with K along a row or along the rows alike.  Loads are plain boxes, and the 32
// threads that have a row of an accumulator each read and write 512 contiguous bytes at a time:
// results do not pass through shared memory, whose bandwidth the operands use up, and an SM's
// stores, which leave it at 32 bytes a clock, are whole lines.  (Row-major operands, turned in shared
// memory, with fp32 copies beside them for what is added: 2 bytes an entry more to store; rows of
// 128 swizzled bytes, a row per thread: 32 lines an instruction, and slower still.)  Up to the next
// multiple of 64, entries beyond a matrix's rows and columns are zeros.
constexpr int kMuonSquare = 5;           // m x m buffers: G, B, another B, S, R
struct MuonWork {
    unsigned char* base;
    uint32_t x[2][2], m[kMuonSquare][2]; // first tile of each buffer; copies of X; hi, lo
};
constexpr uint32_t kMuonTileBytes = 16384, kMuonPiece = 2048;

__device__ __forceinline__ unsigned char* muon_tile(const MuonWork& ws, uint32_t tile) { return ws.base + (uint64_t)tile * kMuonTileBytes; }

__device__ __forceinline__ float muon_direction(const MuonIn& in, float g, float m_new) {
    return in.nesterov ? __fmaf_rn(in.mu, m_new, g) : m_new;
}

// ---- sum of squares, X_0 and the new momentum --------------------------------------------------
//
// Two passes over the gradient and the momentum: the first adds the squares of U, the second reads
// both again and writes the new momentum and X_0 (8 + 8 + 8 bytes an entry), so that a matrix that
// holds a NaN or Inf is found before anything of it is changed.  Squares are added in 64 bits: no
// fp32 value overflows or vanishes.  Where the tasks of both fit the GPU at once they are one
// launch: they are handed out in order, sums first, and the second pass waits for its matrix's
// factor.  (One launch for large vectors too, with the second pass close behind the first so that it
// finds its entries in the L2 cache, was tried: 132 us against 103 for 25 M entries.)

constexpr int kMuonPrepThreads = 256;
constexpr uint32_t kMuonSpan = 8192;

struct MuonSpan { uint64_t start, stride; uint32_t mat, rows, len; };   // rows of len entries
struct MuonTile { uint32_t mat; uint16_t i, j; };                       // of 64 x 64

struct MuonPrepare {
    const MuonSpan* spans;
    const MuonTile* tiles;
    const MuonMat* mats;
    MuonIn in;
    MuonWork ws;
    double* partial;                     // a sum per span
    uint32_t* added;                     // per matrix: spans added up since the call began
    unsigned long long* factor;          // per matrix: the factor of U, as two of fp32, 0 until it is known
    uint32_t* next;                      // the next task that nobody has taken
    uint32_t* sound;
    unsigned long long *done, *tile;     // of the products that follow
    uint32_t* status;
    uint32_t n_spans, wait_limit;
    int what;                            // 0 spans, 1 tiles, 2 both, handed out by `next`
};

template <typename T, bool MOM>
__device__ __forceinline__ void muon_add_squares(const MuonPrepare& P, uint32_t index, double* part) {
    constexpr uint32_t E = Elem<T>::kPer16;
    const MuonSpan sp = P.spans[index];
    const MuonIn& in = P.in;
    const uint32_t tid = threadIdx.x;
    double sum = 0.0;
    auto direction = [&](float g, float m) { return MOM ? muon_direction(in, g, __fmaf_rn(in.mu, m, g)) : g; };
    for (uint32_t r = 0; r < sp.rows; ++r) {
        const T* g = reinterpret_cast<const T*>(in.grad) + sp.start + r * sp.stride;
        const float* mo = MOM ? in.momentum + sp.start + r * sp.stride : nullptr;
        const uint32_t odd = (uint32_t)((16u - (reinterpret_cast<uintptr_t>(g) & 15u)) & 15u) / (uint32_t)sizeof(T);
        const uint32_t head = odd < sp.len ? odd : sp.len;
        const uint32_t nv = (sp.len - head) / E;
#pragma unroll 4
        for (uint32_t v = tid; v < nv; v += kMuonPrepThreads) {
            float x[E];
            Elem<T>::widen(*(reinterpret_cast<const uint4*>(g + head) + v), x);
            if (MOM) {                                               // fp32 beside fp32: the same alignment
                float y[4];
                Elem<float>::widen(*(reinterpret_cast<const uint4*>(mo + head) + v), y);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = direction(x[i], y[i]);
            }
#pragma unroll
            for (uint32_t i = 0; i < E; ++i) sum = fma((double)x[i], (double)x[i], sum);
        }
        const uint32_t edge = tid < head ? tid : head + nv * E + (tid - head);
        if (edge < sp.len && (tid < head || edge >= head + nv * E) && tid < head + E) {
            const float x = direction(Elem<T>::load(g + edge), MOM ? mo[edge] : 0.f);
            sum = fma((double)x, (double)x, sum);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if ((tid & 31) == 0) part[tid >> 5] = sum;
    __syncthreads();
    if (tid >= 32) return;
    uint32_t before = 0;
    if (tid == 0) {
        for (int w = 1; w < kMuonPrepThreads / 32; ++w) sum += part[w];
        __stcg(P.partial + index, sum);
        asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(before) : "l"(P.added + sp.mat) : "memory");
    }
    // whoever adds a matrix's last span has its norm
    const MuonMat& mat = P.mats[sp.mat];
    if (__shfl_sync(~0u, before, 0) + 1 != mat.parts) return;
    sum = 0.0;
    for (uint32_t i = tid; i < mat.parts; i += 32) sum += __ldcg(P.partial + mat.part0 + i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (tid == 0) {
        const bool ok = sum < INFINITY;                              // false for NaN
        // S / |U| as two factors: one of them alone may pass the range of fp32
        int e = 0;
        const double inv = ok && sum > 0.0 ? frexp((double)kMuonScaleX / sqrt(sum), &e) : 0.0;
        const float f0 = (float)ldexp(inv, e / 2), f1 = ok ? (float)ldexp(1.0, e - e / 2) : NAN;
        P.sound[sp.mat] = ok ? 1u : 0u;
        if (!ok) atomicOr(P.status, kStatusNonFinite);
        P.done[sp.mat] = 0;                                          // for the products that follow
        if (sp.mat == 0) *P.tile = 0;
        asm volatile("st.release.gpu.global.u64 [%0], %1;"
                     ::"l"(P.factor + sp.mat), "l"((unsigned long long)__float_as_uint(f0) | ((unsigned long long)__float_as_uint(f1) << 32))
                     : "memory");
    }
}

__device__ __forceinline__ void muon_split(float v, __half& hi, __half& lo) {
    hi = __float2half_rn(v);
    lo = __float2half_rn(__fsub_rn(v, __half2float(hi)));
}

// A tile of a matrix.  sound[mat] gets 1 where the matrix is sound and 0 where it
// holds a NaN or Inf: then X_0 = 0 and its momentum (and later its weights) stay as they are.
template <typename T, bool MOM>
__device__ __forceinline__ void muon_make_x(const MuonPrepare& P, uint32_t index, float (*stage)[65], float* factor) {
    const MuonTile tile = P.tiles[index];
    const MuonMat mat = P.mats[tile.mat];
    const MuonIn& in = P.in;
    const uint32_t tid = threadIdx.x;
    if (tid == 0) {
        unsigned long long f = 0;
        for (uint32_t it = 0; it < P.wait_limit && !f; ++it)
            asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(f) : "l"(P.factor + tile.mat) : "memory");
        if (!f) {                                                    // a matrix left alone, as if it held a NaN
            atomicOr(P.status, kStatusTimeout);
            P.sound[tile.mat] = 0;
            f = 0x7FC00000ull << 32;
        }
        factor[0] = __uint_as_float((uint32_t)f);
        factor[1] = __uint_as_float((uint32_t)(f >> 32));
    }
    __syncthreads();
    const float f0 = factor[0], f1 = factor[1];
    const bool ok = f1 == f1;
    const uint32_t tx = tid & 15, ty = tid >> 4;
    const uint32_t c0 = tile.j * 64u + tx * 4;
    float x[4][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t r = tile.i * 64u + ty + 16 * k;
        const uint64_t at = mat.offset + (uint64_t)r * mat.stride + c0;
        const T* g = reinterpret_cast<const T*>(in.grad) + at;
        float* mo = MOM ? in.momentum + at : nullptr;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[k][i] = 0.f;
        if (r < mat.rows && c0 < mat.cols && ok) {
            const bool whole = c0 + 4 <= mat.cols;
            if (whole && (reinterpret_cast<uintptr_t>(g) & (4 * sizeof(T) - 1)) == 0) {
                if (sizeof(T) == 4) {
                    Elem<float>::widen(*reinterpret_cast<const uint4*>(g), x[k]);
                } else {
                    const uint2 w = *reinterpret_cast<const uint2*>(g);
                    float y[Elem<T>::kPer16];
                    Elem<T>::widen(make_uint4(w.x, w.y, 0, 0), y);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[k][i] = y[i];
                }
                if (MOM) {
                    float m[4];
                    Elem<float>::widen(*reinterpret_cast<const uint4*>(mo), m);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        m[i] = __fmaf_rn(in.mu, m[i], x[k][i]);
                        x[k][i] = muon_direction(in, x[k][i], m[i]);
                    }
                    *reinterpret_cast<uint4*>(mo) = Elem<float>::narrow(m);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (c0 + i < mat.cols) {
                        x[k][i] = Elem<T>::load(g + i);
                        if (MOM) {
                            const float m = __fmaf_rn(in.mu, mo[i], x[k][i]);
                            x[k][i] = muon_direction(in, x[k][i], m);
                            mo[i] = m;
                        }
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x[k][i] = ok ? __fmul_rn(__fmul_rn(x[k][i], f0), f1) : 0.f;
    }
    if (mat.tall) {                                                  // X is the transpose
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) stage[ty + 16 * k][tx * 4 + i] = x[k][i];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[k][i] = stage[tx * 4 + i][ty + 16 * k];
    }
    const uint32_t xr0 = (mat.tall ? tile.j : tile.i) * 64u, xc = (mat.tall ? tile.i : tile.j) * 64u + tx * 4;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t xr = xr0 + ty + 16 * k;
        __half hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) muon_split(x[k][i], hi[i], lo[i]);
        const uint32_t at_tile = mat.x_tile + (xc >> 6) * mat.down + (xr >> 7);
        const uint32_t at = (tx >> 1) * kMuonPiece + (xr & 127) * 16 + (tx & 1) * 8;
        *reinterpret_cast<uint2*>(muon_tile(P.ws, P.ws.x[0][0] + at_tile) + at) = *reinterpret_cast<uint2*>(hi);
        *reinterpret_cast<uint2*>(muon_tile(P.ws, P.ws.x[0][1] + at_tile) + at) = *reinterpret_cast<uint2*>(lo);
    }
}

template <typename T, bool MOM>
__global__ void __launch_bounds__(kMuonPrepThreads, 5) muon_prepare_kernel(const __grid_constant__ MuonPrepare P) {
    __shared__ float stage[64][65];
    __shared__ double part[kMuonPrepThreads / 32];
    __shared__ float factor[2];
    __shared__ uint32_t slot;
    griddep_launch();
    griddep_wait();
    uint32_t n = blockIdx.x;
    if (P.what == 2) {
        if (threadIdx.x == 0) slot = atomicAdd(P.next, 1u);
        __syncthreads();
        n = slot;
    }
    if (P.what == 0 || (P.what == 2 && n < P.n_spans)) muon_add_squares<T, MOM>(P, n, part);
    // last tiles first: their entries are still in the L2 cache, and the products begin with the first
    // (two lm layers, 201 MB: 613 -> 606 us)
    else muon_make_x<T, MOM>(P, P.what == 2 ? n - P.n_spans : gridDim.x - 1 - n, stage, factor);
}

// ---- tensor-core products --------------------------------------------------------------------

// Shared-memory descriptor of an operand without swizzle: units of eight rows of 16 bytes, 128 bytes
// each.  `lead` is the byte distance from a unit to the next one along K, `step` to the next one
// along M or N.
__device__ __forceinline__ uint64_t umma_desc(uint32_t addr, uint32_t lead, uint32_t step) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(step >> 4) << 32) | (1ull << 46);
}

template <int CG>
__device__ __forceinline__ void umma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    if (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                     "r"(idesc), "r"((uint32_t)add)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                     "r"(idesc), "r"((uint32_t)add)
                     : "memory");
}

// Arrive on a barrier (of both CTAs of a pair) when every product issued so far has completed.
template <int CG>
__device__ __forceinline__ void umma_commit(uint32_t bar) {
    if (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)3)
                     : "memory");
}

template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t cols) {
    if (CG == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
}
template <int CG>
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t cols) {
    if (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols));
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols));
}

__device__ __forceinline__ void tmem_load32(uint32_t addr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,"
        "%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_load16(uint32_t addr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tcgen05_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tcgen05_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

__device__ __forceinline__ uint32_t cta_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void pair_sync() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// The same shared-memory location in another CTA of the cluster; in its first.
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t cta) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(cta));
    return a;
}
__device__ __forceinline__ uint32_t leader_addr(uint32_t addr) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(addr));
    return a;
}
__device__ __forceinline__ void leader_arrive(uint32_t leader_bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(leader_bar) : "memory");
}

// Eight pieces of a tile's 128 or 64 rows (from the unit-th eight on) into this CTA's shared memory; in a pair the bytes are counted on the first
// CTA's barrier.
template <int CG>
__device__ __forceinline__ void muon_load(uint32_t dst, const void* map, uint32_t unit, uint32_t piece, uint32_t bar) {
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
                     " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(0), "r"(unit), "r"(piece), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
                     " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(0), "r"(unit), "r"(piece), "r"(bar)
                     : "memory");
}

enum { kMuonGram = 0, kMuonSym = 1, kMuonApply = 2 };                // X X^T, m x m, m x m times X

// One product of the iteration: out = lin * in + lin2 * in2 + acc * left right, less `shift` on the
// diagonal.  Buffers are copies of X or m x m ones by the kind.  Low halves of in are read and of out
// written with the flags (with SPLIT always, and then of in2, too).
enum { kMuonReadLow = 1, kMuonWriteLow = 2, kMuonLast = 4 };
struct MuonProduct {
    float lin, lin2, acc, shift;
    uint8_t kind, left, right, out;
    uint8_t in, in2, flags;              // 255: none
    uint8_t after;                       // products before it that have to be finished
};

// One tile of the whole computation; the list of them is in the order in which they are handed out.
struct MuonTask {
    uint32_t mat;
    uint16_t i, j;
    uint16_t product, mirror;
    uint32_t need;                       // tiles of the matrix that have to be finished before
};

struct MuonIterate {
    CUtensorMap rows128, rows64;         // the workspace, in boxes of 128 or 64 rows of a tile
    const MuonMat* mats;
    const MuonTask* tasks;
    const MuonProduct* products;
    const uint32_t* sound;
    MuonWork ws;
    unsigned long long* done;            // per matrix: parts of tiles finished since the call began
    unsigned long long* next;            // the next tile that nobody has taken
    uint32_t *added, *prepare_next;      // set to zero for the next call, and factor
    unsigned long long* factor;
    uint32_t* status;
    MuonOut out;
    int out_dtype;
    uint32_t n_tasks, n_mats;
    uint32_t wait_limit;
};

constexpr uint32_t kMuonBox = 8192;                                   // 64 x 64 fp16
constexpr uint32_t kMuonBlock = 2048;                                 // 32 x 32 fp16
constexpr uint32_t kMuonQueue = 2;
constexpr uint32_t kMuonShare = 128 * 32 * 4;                         // partial sums from one CTA to another
constexpr uint32_t kMuonChunk = 4;                                    // 64-wide steps along K per partial sum (SPLIT)

// CG CTAs work on one tile of CG * 128 rows and TN columns; each stages its 128 rows of the left
// operand and TN / CG rows of the right one, 64 along K at a time, both halves of each with SPLIT.
//
// With KS two CTAs have half of a tile's K each, for matrices with few tiles and long products: an SM
// takes 48 bytes a clock from L2, 2.1 us for 8 steps of 24 KB.  Each finishes 32 columns of the tile,
// with the other's partial sums added that come through its shared memory; that takes about 0.9 us a
// product.  (Four CTAs a tile were never faster: 2497 x 85 with 22 bits took 186 us with one, 147 with
// two and 154 with four, 1000 x 2048 301, 264 and 460.)
template <int CG, int TN, bool SPLIT, bool KS = false>
struct MuonShape {
    static constexpr uint32_t kHalves = SPLIT ? 2 : 1;
    static constexpr uint32_t kBoxesA = 2, kBoxesB = TN / CG / 64;
    static constexpr uint32_t kBytesA = kBoxesA * kMuonBox, kBytesB = kBoxesB * kMuonBox;
    static constexpr uint32_t kStageBytes = kHalves * (kBytesA + kBytesB);
    static constexpr uint32_t kEpiWarps = 8;
    static constexpr uint32_t kCols = TN / (kEpiWarps / 4);           // columns of an epilogue warp
    static constexpr uint32_t kThreads = (kEpiWarps + 4) * 32;        // + two for loads, products, signals
    static constexpr uint32_t kFinish = KS ? 4 : kEpiWarps;           // of them, warps that finish results
    static constexpr uint32_t kEpiBytes = kFinish * 2 * kMuonBlock;
    static constexpr uint32_t kShareBytes = KS ? kMuonShare : 0;
    static constexpr uint32_t kStagesFit = (230u * 1024u - 2048u - kEpiBytes - kShareBytes) / kStageBytes;
    static constexpr uint32_t kStages = kStagesFit < 6 ? kStagesFit : 6;
    static constexpr uint32_t kSmem = kStages * kStageBytes + kEpiBytes + kShareBytes + 1024;   // + alignment
    static constexpr uint32_t kAccCols = SPLIT ? 2 * TN : TN;         // hi hi, and the two small products
    static constexpr uint32_t kTmemCols = 2 * kAccCols;
    // counts per tile on MuonIterate::done
    static constexpr uint32_t kParts = KS ? 2 : CG;
    static_assert(!KS || (CG == 1 && TN == 64), "");
};

// Waits that give up: the limit is per wait, and one that ran out ends all others soon.
__device__ __forceinline__ bool muon_wait(uint32_t bar, uint32_t parity, uint32_t limit, volatile uint32_t* stop) {
    for (uint32_t it = 0; it < limit; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if (*stop) return false;
    }
    *stop = 1;
    return false;
}
// The same where the other CTA of a pair arrives and its writes are read.
__device__ __forceinline__ bool muon_wait_pair(uint32_t bar, uint32_t parity, uint32_t limit, volatile uint32_t* stop) {
    for (uint32_t it = 0; it < limit; ++it) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\t"
                     "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                     "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
        if (*stop) return false;
    }
    *stop = 1;
    return false;
}
// Until `need` parts of a matrix's tiles are finished; then their results may be loaded.
__device__ __forceinline__ bool muon_wait_done(const unsigned long long* done, unsigned long long need, uint32_t limit,
                                               volatile uint32_t* stop, uint32_t pause) {
    for (uint32_t it = 0; it < limit; ++it) {
        unsigned long long v;
        asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(done) : "memory");
        if (v >= need) {
            asm volatile("fence.proxy.async;" ::: "memory");
            return true;
        }
        if (*stop) return false;
        if (pause) __nanosleep(pause);
    }
    *stop = 1;
    return false;
}

// Place of the 16 bytes with columns 8 c .. 8 c + 7 of row r in a block of 64-byte rows: neither
// eight lanes with a row each nor eight with two whole rows meet in a bank.
__device__ __forceinline__ uint32_t muon_swizzle(uint32_t r, uint32_t c) { return r * 64u + ((c ^ ((r >> 1) & 3u)) << 4); }

__device__ __forceinline__ uint4 lds16(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ void sts16(uint32_t addr, uint4 v) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// A row's 32 columns of a block: four pieces.  (Reads of what other SMs have written come behind an
// acquire.)
__device__ __forceinline__ void muon_get(const unsigned char* p, uint4 (&v)[4]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = __ldcg(reinterpret_cast<const uint4*>(p + c * kMuonPiece));
}
__device__ __forceinline__ void muon_put(unsigned char* p, const uint4 (&v)[4]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) __stcg(reinterpret_cast<uint4*>(p + c * kMuonPiece), v[c]);
}

// A block of 32 x 32 finished entries, row or0 and column oc0 of the caller's matrix, from shared
// memory (rows of 64 or 128 bytes) to the update and the weights.
__device__ __forceinline__ void muon_out_narrow(const MuonIterate& P, const MuonMat& mat, uint32_t block, uint32_t or0, uint32_t oc0) {
    const uint32_t lane = threadIdx.x & 31, cr = lane >> 2, cc = lane & 3, oc = oc0 + 8 * cc;
    if (oc >= mat.cols) return;
    uint16_t* to = reinterpret_cast<uint16_t*>(P.out.update) + mat.offset + (uint64_t)(or0 + cr) * mat.stride + oc;
    const uint64_t down = 8 * mat.stride;
    if (((mat.offset | mat.stride) & 7) == 0 && oc + 8 <= mat.cols) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i, to += down)
            if (or0 + cr + 8 * i < mat.rows) *reinterpret_cast<uint4*>(to) = lds16(block + muon_swizzle(cr, cc) + 512 * i);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i, to += down) {
            if (or0 + cr + 8 * i >= mat.rows) break;
            const uint4 v = lds16(block + muon_swizzle(cr, cc) + 512 * i);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (oc + k < mat.cols) to[k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
        }
    }
}

// Weights are read before any is written: a block waits for memory once.
__device__ __forceinline__ void muon_out_wide(const MuonIterate& P, const MuonMat& mat, uint32_t block, uint32_t or0, uint32_t oc0,
                                           bool sound) {
    const uint32_t lane = threadIdx.x & 31;
    const float rate = -__fmul_rn(P.out.rate, mat.scale), up = P.out.scaled ? mat.scale : 1.f, keep = P.out.keep;
    float* params = sound ? P.out.params : nullptr;
    void* update = P.out.update;
    if (((mat.offset | mat.stride) & 3) == 0 && oc0 + 32 <= mat.cols && P.out_dtype == 0) {
        const uint32_t fr = lane >> 3, fc = lane & 7;                  // eight lanes with 16 bytes each to a row
        const uint64_t to = mat.offset + (uint64_t)(or0 + fr) * mat.stride + oc0 + 4 * fc, down = 4 * mat.stride;
        uint4 p[8];
        if (params) {
            const float* from = params + to;
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i, from += down)
                if (or0 + fr + 4 * i < mat.rows) p[i] = *reinterpret_cast<const uint4*>(from);
        }
        float* out = reinterpret_cast<float*>(update) + to;
        float* par = params + to;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i, out += down, par += down) {
            const uint32_t rr = i * 4 + fr;
            if (or0 + rr >= mat.rows) break;
            float o[4], w[4];
            Elem<float>::widen(lds16(block + rr * 128 + ((fc ^ (rr & 7)) << 4)), o);
            if (params) {
                Elem<float>::widen(p[i], w);
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = __fmaf_rn(rate, o[k], __fmul_rn(keep, w[k]));
                *reinterpret_cast<uint4*>(par) = Elem<float>::narrow(w);
            }
            if (update) {
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = __fmul_rn(up, o[k]);
                *reinterpret_cast<uint4*>(out) = Elem<float>::narrow(w);
            }
        }
        return;
    }
    if (oc0 + lane >= mat.cols) return;                                // any alignment: the lanes along a row
    uint64_t to = mat.offset + (uint64_t)or0 * mat.stride + oc0 + lane;
    for (uint32_t half = 0; half < 32; half += 16) {
        float p[16];
        if (params) {
            const float* from = params + to;
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i, from += mat.stride)
                if (or0 + half + i < mat.rows) p[i] = *from;
        }
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i, to += mat.stride) {
            const uint32_t rr = half + i;
            if (or0 + rr >= mat.rows) return;
            float o;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(o) : "r"(block + rr * 128 + (((lane >> 2) ^ (rr & 7)) << 4) + 4 * (lane & 3)));
            if (params) params[to] = __fmaf_rn(rate, o, __fmul_rn(keep, p[i]));
            if (update) {
                const float u = __fmul_rn(up, o);
                if (P.out_dtype == 0) reinterpret_cast<float*>(update)[to] = u;
                else if (P.out_dtype == 1) reinterpret_cast<__nv_bfloat16*>(update)[to] = __float2bfloat16_rn(u);
                else reinterpret_cast<__half*>(update)[to] = __float2half_rn(u);
            }
        }
    }
}

// One lane of a converged warp, in a form from which the compiler can tell that it is one: TMA and
// tcgen05 instructions take their operands from uniform registers, and behind a plain comparison of
// the lane's number each of them costs about 0.1 us to issue.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

// Every step of every matrix in one launch.  Tiles are taken from a counter in a fixed order; each
// waits until the tiles that its operands come from are finished.  Those are earlier in the order,
// so they have been taken by CTAs that are running: some tile can always go on, whatever number
// of CTAs the GPU has room for.
//
// What bounds it.  Large matrices (two layers of 1024 x 1024 to 1024 x 4096, 460 us of the call's 548): operands
// and results through L2, 9.8 TB/s, with the tensor pipe busy 40 % of the time; 24 such layers (5.9 ms
// undisturbed, 6.5 among others, 2.36 at the tensor cores' rate) meet the power cap besides.  Few tiles (1024 x
// 1024, 137 us): 15 products one after the other, 9 us each: 0.7 for the first load, 4.2 for 16 steps of
// 24 KB at the 48 bytes a clock that an SM takes from L2 (the products alone: 1.6), 1.5 for the results, 1 to
// make them visible, 0.5 to see that.  Smallest (96 x 160, 63 us): the same with 0.5 for the products.
template <int CG, int TN, bool SPLIT, bool KS>
__global__ void __launch_bounds__(MuonShape<CG, TN, SPLIT, KS>::kThreads, 1) muon_iterate_kernel(const __grid_constant__ MuonIterate P) {
    using S = MuonShape<CG, TN, SPLIT, KS>;
    constexpr bool kJoint = CG == 2 || KS;                            // two CTAs work together
    constexpr uint32_t ctas = kJoint ? 2 : 1;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::kStages + 6 + 4 * kMuonQueue + (KS ? 8 : 0)];
    __shared__ uint32_t tmem_slot, queue[kMuonQueue], passed[kMuonQueue];
    __shared__ volatile uint32_t stop;
    const uint32_t tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31;
    const uint32_t ring = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t full = smem_u32(bars), empty = full + 8 * S::kStages;
    const uint32_t acc_full = empty + 8 * S::kStages, acc_empty = acc_full + 16;
    const uint32_t q_full = acc_empty + 16, q_empty = q_full + 8 * kMuonQueue;
    const uint32_t pass_full = q_empty + 8 * kMuonQueue, pass_empty = pass_full + 8 * kMuonQueue, stored = pass_empty + 8 * kMuonQueue;
    // the other's partial sums, by warp: come, and read
    const uint32_t share_full = stored + 16, share_empty = share_full + 32;
    const uint32_t cta = kJoint ? cta_rank() : 0, rank = KS ? 0 : cta;   // rank: which rows of the tile
    const uint32_t limit = P.wait_limit;
    // this CTA's steps along K
    auto steps_from = [&](uint32_t kb) { return KS ? min(cta * ((kb + ctas - 1) / ctas), kb) : 0; };
    auto steps_to = [&](uint32_t kb) { return KS ? min((cta + 1) * ((kb + ctas - 1) / ctas), kb) : kb; };

    if (tid == 0) {
        for (uint32_t s = 0; s < S::kStages; ++s) { mbar_init(full + 8 * s, 2); mbar_init(empty + 8 * s, 1); }
        for (uint32_t b = 0; b < 2; ++b) { mbar_init(acc_full + 8 * b, 1); mbar_init(acc_empty + 8 * b, CG * S::kEpiWarps); }
        for (uint32_t q = 0; q < kMuonQueue; ++q) {
            mbar_init(q_full + 8 * q, 1);
            mbar_init(q_empty + 8 * q, S::kEpiWarps + 2 + (rank == 0 ? 1 : 0));   // results, right operands, signals, products
            mbar_init(pass_full + 8 * q, 1);
            mbar_init(pass_empty + 8 * q, 1);
        }
        mbar_init(stored, S::kFinish);
        mbar_init(stored + 8, S::kFinish);
        if (KS)
            for (uint32_t i = 0; i < 8; ++i) mbar_init(share_full + 8 * i, 1);
        stop = 0;
        fence_mbar_init();
    }
    if (warp == S::kEpiWarps + 1) tmem_alloc<CG>(smem_u32(&tmem_slot), S::kTmemCols);
    tcgen05_before_sync();
    __syncthreads();
    if (kJoint) pair_sync();
    tcgen05_after_sync();
    const uint32_t tmem = tmem_slot;
    griddep_wait();
    if (blockIdx.x == 0) {
        for (uint32_t i = tid; i < P.n_mats; i += S::kThreads) { P.added[i] = 0; P.factor[i] = 0; }
        if (tid == 0) *P.prepare_next = 0;
    }

    // Numbers of tiles go from the thread that loads left operands to the other roles of its CTA through
    // `queue`; those of a second CTA are passed to that thread of it first.  So what crosses CTAs is
    // released by threads that have written no results: a release to the other CTA would wait for
    // those on their way to memory (all roles arriving at the first CTA: two lm layers 550 -> 561 us, 48 of 512 x
    // 512 324 -> 340; this way 553 and 318).
    //
    // n-th tile of this CTA (or pair); false when a wait ran out
    auto take = [&](uint32_t n, uint32_t& t) {
        const uint32_t q = n % kMuonQueue;
        if (!muon_wait(q_full + 8 * q, (n / kMuonQueue) & 1, limit, &stop)) return false;
        t = *reinterpret_cast<volatile uint32_t*>(&queue[q]);
        return true;
    };
    auto taken = [&](uint32_t n) { mbar_arrive(q_empty + 8 * (n % kMuonQueue)); };
    auto give = [&](uint32_t n, uint32_t t) {
        const uint32_t q = n % kMuonQueue;
        if (!muon_wait(q_empty + 8 * q, ((n / kMuonQueue) & 1) ^ 1, limit, &stop)) return false;
        *reinterpret_cast<volatile uint32_t*>(&queue[q]) = t;
        mbar_arrive(q_full + 8 * q);
        return true;
    };
    auto pass = [&](uint32_t n, uint32_t t) {                          // by the first CTA
        const uint32_t q = n % kMuonQueue;
        if (!muon_wait_pair(pass_empty + 8 * q, ((n / kMuonQueue) & 1) ^ 1, limit, &stop)) return false;
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(peer_addr(smem_u32(&passed[q]), 1)), "r"(t) : "memory");
        leader_arrive(peer_addr(pass_full + 8 * q, 1));
        return true;
    };
    auto receive = [&](uint32_t n, uint32_t& t) {                      // by the second
        const uint32_t q = n % kMuonQueue;
        if (!muon_wait_pair(pass_full + 8 * q, (n / kMuonQueue) & 1, limit, &stop)) return false;
        t = *reinterpret_cast<volatile uint32_t*>(&passed[q]);
        leader_arrive(leader_addr(pass_empty + 8 * q));
        return true;
    };

    if (warp == S::kEpiWarps || warp == S::kEpiWarps + 3) {
        // ---- loads -------------------------------------------------------------------------------
        // One warp for the left operands, one for the right: a thread issues a TMA load in about 200
        // clocks, and 32 KB in two boxes by one take 756 clocks, by two 580 (in three 789 and 616).
        // Each load thread of each CTA has part in every stage: one that had none could fall two
        // rounds of the ring behind, where the barriers' parities are the same again.
        if (elect_one()) {
            const bool first = warp == S::kEpiWarps, giver = first && cta == 0;
            uint32_t it = 0, t = 0;
            bool ok = true;
            const uint32_t total = P.n_tasks;
            // a tile is claimed when the loads of the one before it are issued: one that waits for
            // its operands then holds up no tile that another CTA could have had
            unsigned long long claim = giver ? atomicAdd(P.next, 1ull) : 0;
            for (uint32_t n = 0; ok; ++n) {
                if (giver) {
                    t = (uint32_t)min(claim, (unsigned long long)total);
                    if ((kJoint && !pass(n, t)) || !give(n, t)) break;
                } else if (first) {
                    if (!receive(n, t) || !give(n, t)) break;
                } else {
                    if (!take(n, t)) break;
                    taken(n);
                }
                if (t >= total) break;
                const MuonTask task = P.tasks[t];
                const MuonProduct& pr = P.products[task.product];
                const int kind = pr.kind;
                const MuonMat& mat = P.mats[task.mat];
                const uint32_t kb = ((kind == kMuonGram ? mat.n : mat.m) + 63) / 64, down = mat.down;
                const uint32_t row = task.i * (CG * 128u) + rank * 128u;
                const uint32_t col = task.j * (uint32_t)TN + rank * (TN / CG);
                const bool along_n = kind == kMuonApply;
                uint32_t from[2];                                      // tiles
#pragma unroll
                for (uint32_t h = 0; h < S::kHalves; ++h) {
                    if (first)
                        from[h] = (kind == kMuonGram ? P.ws.x[pr.left][h] + mat.x_tile : P.ws.m[pr.left][h] + mat.m_tile) + row / 128;
                    else
                        from[h] = (kind == kMuonSym ? P.ws.m[pr.right][h] + mat.m_tile : P.ws.x[pr.right][h] + mat.x_tile) +
                                  (along_n ? col / 64 * down : col / 128);
                }
                if (!muon_wait_done(P.done + task.mat, (unsigned long long)S::kParts * task.need, limit, &stop, 0)) break;
                const uint32_t k1 = steps_to(kb);
                for (uint32_t k = steps_from(kb); k < k1; ++k, ++it) {
                    const uint32_t s = it % S::kStages, ph = (it / S::kStages) & 1;
                    if (!muon_wait(empty + 8 * s, ph ^ 1, limit, &stop)) { ok = false; break; }
                    const uint32_t bar = CG == 1 ? full + 8 * s : leader_addr(full + 8 * s);
                    const uint32_t da = ring + s * S::kStageBytes, db = da + S::kHalves * S::kBytesA;
                    if (first) {
                        if (rank == 0) mbar_arrive_expect_tx(full + 8 * s, CG * S::kHalves * S::kBytesA);
#pragma unroll
                        for (uint32_t h = 0; h < S::kHalves; ++h)
                            muon_load<CG>(da + h * S::kBytesA, &P.rows128, 0, 8 * (from[h] + k * down), bar);
                        if (giver && k + 1 == k1) claim = atomicAdd(P.next, 1ull);
                    } else {
                        if (rank == 0) mbar_arrive_expect_tx(full + 8 * s, CG * S::kHalves * S::kBytesB);
#pragma unroll
                        for (uint32_t h = 0; h < S::kHalves; ++h) {
                            if (along_n) {                             // 64 columns a box, their rows along K
#pragma unroll
                                for (uint32_t b = 0; b < S::kBoxesB; ++b)
                                    muon_load<CG>(db + h * S::kBytesB + b * kMuonBox, &P.rows64, (k & 1) * 8,
                                                  8 * (from[h] + b * down + k / 2), bar);
                            } else if (S::kBoxesB == 2) {
                                muon_load<CG>(db + h * S::kBytesB, &P.rows128, 0, 8 * (from[h] + k * down), bar);
                            } else {
                                muon_load<CG>(db + h * S::kBytesB, &P.rows64, (col & 64) / 8, 8 * (from[h] + k * down), bar);
                            }
                        }
                    }
                }
            }
            // nothing of this CTA's is in flight when it leaves: every stage's last load was consumed
            // (or, where a wait ran out and nobody consumes them any more, has had time to land)
            for (uint32_t b = 0; b < S::kStages && b < it; ++b) {
                const uint32_t last = it - 1 - b, most = stop ? 1u << 12 : kWaitLimit;
                for (uint32_t n = 0; n < most; ++n)
                    if (mbar_try_wait(empty + 8 * (last % S::kStages), (last / S::kStages) & 1)) break;
            }
        }
    } else if (warp == S::kEpiWarps + 1) {
        // ---- products ----------------------------------------------------------------------------
        if (rank == 0 && elect_one()) {
            uint32_t it = 0, acc = 0, t;
            bool ok = true;
            for (uint32_t n = 0; ok && take(n, t); ++n) {
                taken(n);
                if (t >= P.n_tasks) break;
                const MuonTask task = P.tasks[t];
                const MuonProduct& pr = P.products[task.product];
                const int kind = pr.kind;
                const MuonMat& mat = P.mats[task.mat];
                const uint32_t kb = ((kind == kMuonGram ? mat.n : mat.m) + 63) / 64;
                const bool along_n = kind == kMuonApply;               // right operand's rows run along K
                // fp32 accumulators, fp16 operands
                const uint32_t idesc = (1u << 4) | ((uint32_t)(TN / 8) << 17) | ((uint32_t)(CG * 128 / 16) << 24) |
                                       (along_n ? 1u << 16 : 0u);
                // bytes from a unit to the next along K and along M or N, and from 16 along K to the next
                constexpr uint32_t a_lead = kMuonPiece, b_rows = S::kBoxesB * 1024;
                const uint32_t b_lead = along_n ? 128 : b_rows, b_step = along_n ? 1024 : 128;
                const uint32_t b_k16 = along_n ? 256 : 2 * b_rows;
                uint32_t in_chunk = 0, d = 0;
                const uint32_t k0 = steps_from(kb), k1 = steps_to(kb);
                for (uint32_t k = k0; k < k1; ++k, ++it) {
                    if (in_chunk == 0) {
                        ok = CG == 1 ? muon_wait(acc_empty + 8 * (acc & 1), ((acc >> 1) & 1) ^ 1, limit, &stop)
                                     : muon_wait_pair(acc_empty + 8 * (acc & 1), ((acc >> 1) & 1) ^ 1, limit, &stop);
                        if (!ok) break;
                        d = tmem + (acc & 1) * S::kAccCols;
                    }
                    const uint32_t s = it % S::kStages, ph = (it / S::kStages) & 1;
                    if (!muon_wait(full + 8 * s, ph, limit, &stop)) { ok = false; break; }
                    tcgen05_after_sync();
                    const uint32_t a0 = ring + s * S::kStageBytes, b0 = a0 + S::kHalves * S::kBytesA;
                    const uint64_t da = umma_desc(a0, a_lead, 128), db = umma_desc(b0, b_lead, b_step);
                    const uint64_t dal = umma_desc(a0 + S::kBytesA, a_lead, 128), dbl = umma_desc(b0 + S::kBytesB, b_lead, b_step);
#pragma unroll
                    for (uint32_t q = 0; q < 4; ++q) {
                        const bool add = in_chunk > 0 || q > 0;
                        const uint64_t qa = (2 * a_lead * q) >> 4, qb = (b_k16 * q) >> 4;
                        umma_f16<CG>(d, da + qa, db + qb, idesc, add);
                        if (SPLIT) {
                            umma_f16<CG>(d + TN, da + qa, dbl + qb, idesc, add);
                            umma_f16<CG>(d + TN, dal + qa, db + qb, idesc, true);
                        }
                    }
                    umma_commit<CG>(empty + 8 * s);
                    if (++in_chunk == (SPLIT ? kMuonChunk : k1 - k0) || k + 1 == k1) {
                        umma_commit<CG>(acc_full + 8 * (acc & 1));
                        in_chunk = 0;
                        ++acc;
                    }
                }
            }
        }
    } else if (warp == S::kEpiWarps + 2) {
        // ---- signals -----------------------------------------------------------------------------
        // Making a tile's results visible to the other SMs takes a microsecond; the warps that wrote
        // them have the next tile to do meanwhile.  The release covers their writes, which came
        // before their arrivals here; whoever acquires the count puts the fence between it and TMA.
        if (lane == 0) {
            uint32_t t;
            for (uint32_t n = 0; take(n, t); ++n) {
                taken(n);
                if (t >= P.n_tasks) break;
                const uint32_t mat = P.tasks[t].mat;
                if (!muon_wait(stored + 8 * (n & 1), (n >> 1) & 1, limit, &stop)) break;
                asm volatile("red.release.gpu.global.add.u64 [%0], %1;" ::"l"(P.done + mat), "l"(1ull) : "memory");
            }
        }
    } else {
        // ---- results -----------------------------------------------------------------------------
        // Every warp has 32 rows and kCols columns of a tile, taken in blocks of 32 x 32.  What a
        // block's results are added to is read ahead into registers.
        const uint32_t quad = warp & 3, half = KS ? (warp >> 2) ^ cta : warp >> 2, c0 = half * S::kCols;
        const bool finish = !KS || warp < 4;
        const uint32_t block = ring + S::kStages * S::kStageBytes + (finish ? warp : 0) * 2 * kMuonBlock;
        // the other CTA's sums for this warp's rows: 16 bytes of 32 rows, then the next
        const uint32_t share = ring + S::kStages * S::kStageBytes + S::kEpiBytes + quad * (kMuonShare / 4) + lane * 16;
        const uint32_t lane_addr = tmem + ((quad * 32u) << 16);
        constexpr uint32_t kBlocks = S::kCols / 32;
        const uint32_t own = block + lane * 64, flip = (lane >> 1) & 3;   // this lane's row in shared memory: piece c at own + ((c ^ flip) << 4)
        uint32_t acc = 0, t;
        bool ok = true;
        for (uint32_t n = 0; ok && __all_sync(~0u, take(n, t)); ++n) {
            __syncwarp();
            if (lane == 0) taken(n);
            if (t >= P.n_tasks) break;
            const MuonTask task = P.tasks[t];
            const MuonProduct& pr = P.products[task.product];
            const MuonMat& mat = P.mats[task.mat];
            const bool apply = pr.kind == kMuonApply, gram = pr.kind == kMuonGram;
            const uint32_t flags = pr.flags;
            const bool last = (flags & kMuonLast) != 0, mirror = task.mirror != 0;
            const bool read_low = SPLIT || (flags & kMuonReadLow), write_low = SPLIT || (flags & kMuonWriteLow);
            const uint32_t m = mat.m, pad = mat.pad, width = ((apply ? mat.n : m) + 63) / 64 * 64;
            const uint32_t row0 = task.i * (CG * 128u) + rank * 128u + quad * 32u;
            const uint32_t col0 = task.j * (uint32_t)TN + c0;
            const uint32_t r = row0 + lane;
            const float lin = pr.lin, mul = pr.acc, shift = pr.shift;
            // this lane's first piece of the warp's first block, in any buffer
            const uint32_t tile = (apply ? mat.x_tile : mat.m_tile) + (col0 >> 6) * mat.down + (row0 >> 7);
            const uint32_t piece = (col0 & 32) * (kMuonPiece / 8) + (r & 127) * 16;
            const uint64_t right = (uint64_t)mat.down * kMuonTileBytes;   // to the next 64 columns
            auto place = [&](uint32_t buffer, uint32_t b) {
                return muon_tile(P.ws, buffer + tile) + piece + (b >> 1) * right + (b & 1) * (4 * kMuonPiece);
            };
            const uint32_t (*const buffers)[2] = apply ? P.ws.x : P.ws.m;
            const uint32_t in_at = gram ? 0 : apply ? pr.right : pr.in;
            // blocks inside the matrix; 0 for a warp whose rows are all below it
            const uint32_t blocks = row0 >= pad || col0 >= width ? 0 : min(kBlocks, (width - col0) / 32);

            uint4 in[4], low[4];
            auto fetch = [&](uint32_t b) {
                if (gram || b >= blocks) return;
                muon_get(place(buffers[in_at][0], b), in);
                if (read_low) muon_get(place(buffers[in_at][1], b), low);
            };
            if (!gram && blocks && finish) {
                int go = 1;
                if (lane == 0)
                    go = muon_wait_done(P.done + task.mat, (unsigned long long)S::kParts * task.need, limit, &stop, 100);
                go = __shfl_sync(~0u, go, 0);
                __syncwarp();                                          // the shuffle alone orders no memory for the other lanes
                if (!go) break;
            }
            if ((!SPLIT || S::kCols == 32) && finish) fetch(0);
            uint32_t steps = 1;                                        // along K; without SPLIT, whether there is one
            if (KS || SPLIT) {
                const uint32_t kb = ((gram ? mat.n : m) + 63) / 64;
                steps = steps_to(kb) - steps_from(kb);
            }

            float sum[SPLIT ? S::kCols : 1];
            if (SPLIT) {
#pragma unroll
                for (uint32_t i = 0; i < S::kCols; ++i) sum[SPLIT ? i : 0] = 0.f;
                for (uint32_t chunk = 0; chunk < (steps + kMuonChunk - 1) / kMuonChunk; ++chunk, ++acc) {
                    ok = __all_sync(~0u, muon_wait(acc_full + 8 * (acc & 1), (acc >> 1) & 1, limit, &stop));
                    if (!ok) break;
                    tcgen05_after_sync();
#pragma unroll
                    for (uint32_t h = 0; h < S::kCols / 16; ++h) {
                        float v[16], w[16];
                        tmem_load16(lane_addr + (acc & 1) * S::kAccCols + c0 + 16 * h, v);
                        tmem_load16(lane_addr + (acc & 1) * S::kAccCols + TN + c0 + 16 * h, w);
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            sum[SPLIT ? 16 * h + i : 0] = __fadd_rn(sum[SPLIT ? 16 * h + i : 0], __fadd_rn(v[i], w[i]));
                    }
                    tcgen05_before_sync();
                    __syncwarp();
                    if (lane == 0) {
                        if (CG == 1) mbar_arrive(acc_empty + 8 * (acc & 1));
                        else leader_arrive(leader_addr(acc_empty + 8 * (acc & 1)));
                    }
                }
            } else if (steps) {
                ok = __all_sync(~0u, muon_wait(acc_full + 8 * (acc & 1), (acc >> 1) & 1, limit, &stop));
                tcgen05_after_sync();
            }
            if (!ok) break;
            if (SPLIT && S::kCols != 32) fetch(0);                     // not before: the sums take the registers
            // this warp's block of the accumulators is read
            auto release = [&] {
                tcgen05_before_sync();
                __syncwarp();
                if (lane == 0) {
                    if (CG == 1) mbar_arrive(acc_empty + 8 * (acc & 1));
                    else leader_arrive(leader_addr(acc_empty + 8 * (acc & 1)));
                }
                ++acc;
            };
            if (!finish) {
                // to the CTA that finishes these columns; it has read the last tile's before
                float y[32];
                if (SPLIT) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) y[i] = sum[SPLIT ? i : 0];
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) y[i] = 0.f;
                    if (steps) {
                        tmem_load32(lane_addr + (acc & 1) * S::kAccCols + c0, y);
                        release();
                    }
                }
                ok = __all_sync(~0u, muon_wait_pair(share_empty + 8 * quad, (n & 1) ^ 1, limit, &stop));
                if (!ok) break;
                const uint32_t to = peer_addr(share, half);
                const uint32_t bar = peer_addr(share_full + 8 * quad, half);
                if (lane == 0)
                    asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(kMuonShare / 4) : "memory");
#pragma unroll
                for (uint32_t c = 0; c < 8; ++c)
                    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1,%2,%3,%4}, [%5];"
                                 ::"r"(to + c * 512), "f"(y[4 * c]), "f"(y[4 * c + 1]), "f"(y[4 * c + 2]), "f"(y[4 * c + 3]), "r"(bar) : "memory");
                continue;
            }

            if (KS) {
                ok = __all_sync(~0u, muon_wait_pair(share_full + 8 * quad, n & 1, limit, &stop));
                if (!ok) break;
            }


            // a finished block, 32 columns of this lane's row
            auto result = [&](uint32_t b, float* y) {
                const uint32_t col = col0 + 32 * b;
                if (SPLIT) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) y[i] = sum[SPLIT ? 32 * b + i : 0];
                } else if (!KS || steps) {
                    tmem_load32(lane_addr + (acc & 1) * S::kAccCols + c0 + 32 * b, y);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) y[i] = 0.f;
                }
                if (KS) {
#pragma unroll
                    for (uint32_t c = 0; c < 8; ++c) {
                        const uint4 w = lds16(share + c * 512);
                        y[4 * c] = __fadd_rn(y[4 * c], __uint_as_float(w.x));
                        y[4 * c + 1] = __fadd_rn(y[4 * c + 1], __uint_as_float(w.y));
                        y[4 * c + 2] = __fadd_rn(y[4 * c + 2], __uint_as_float(w.z));
                        y[4 * c + 3] = __fadd_rn(y[4 * c + 3], __uint_as_float(w.w));
                    }
                }
                // pairs of columns in one operation each
                const uint64_t mul2v = pack2(mul, mul);
                if (gram) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) unpack2(mul2(pack2(y[2 * i], y[2 * i + 1]), mul2v), y[2 * i], y[2 * i + 1]);
                    if (col < row0 + 32 && row0 < col + 32) {          // the block meets the diagonal
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (r == col + i && r < m) y[i] = __fsub_rn(y[i], shift);
                    }
                } else {
                    // y = mul * y + by * v, or y + by * v
                    auto add = [&](const uint4 (&v)[4], float by, bool first) {
                        const uint64_t by2 = pack2(by, by);
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            float x[8];
                            Elem<__half>::widen(v[c], x);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float &u = y[8 * c + 2 * i], &w = y[8 * c + 2 * i + 1];
                                uint64_t before = pack2(u, w);
                                if (first) before = mul2(before, mul2v);
                                unpack2(fma2(by2, pack2(x[2 * i], x[2 * i + 1]), before), u, w);
                            }
                        }
                    };
                    add(in, lin, true);
                    if (read_low) add(low, lin, false);
                    if (pr.in2 != 255) {
                        muon_get(place(P.ws.m[pr.in2][0], b), in);
                        if (SPLIT) muon_get(place(P.ws.m[pr.in2][1], b), low);
                        add(in, pr.lin2, false);
                        if (SPLIT) add(low, pr.lin2, false);
                    }
                    fetch(b + 1);
                }
            };
            auto keep_block = [&](uint32_t b) {
                const uint32_t col = col0 + 32 * b;
                float y[32];
                result(b, y);
                // the transposed block: row c of it has the 32 lanes' entries of column c
                auto turn = [&](const uint4 (&v)[4], uint32_t buffer) {
                    __syncwarp();
#pragma unroll
                    for (uint32_t c = 0; c < 4; ++c) {
                        const uint32_t w[4] = {v[c].x, v[c].y, v[c].z, v[c].w};
#pragma unroll
                        for (uint32_t i = 0; i < 8; ++i)
                            asm volatile("st.shared.b16 [%0], %1;"
                                         ::"r"(block + (8 * c + i) * 64 + (((lane >> 3) ^ ((i >> 1) & 3)) << 4) + 2 * (lane & 7)),
                                         "h"((uint16_t)(w[i >> 1] >> (16 * (i & 1)))) : "memory");
                    }
                    __syncwarp();
                    uint4 t[4];
#pragma unroll
                    for (uint32_t c = 0; c < 4; ++c) t[c] = lds16(own + ((c ^ flip) << 4));
                    if (col + lane < pad)
                        muon_put(muon_tile(P.ws, buffer + mat.m_tile + (row0 >> 6) * mat.down + (col >> 7)) +
                                     (row0 & 32) * (kMuonPiece / 8) + ((col & 127) + lane) * 16, t);
                };
                uint4 v[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] = Elem<__half>::narrow(y + 8 * c);
                if (r < pad) muon_put(place(buffers[pr.out][0], b), v);
                if (mirror) turn(v, P.ws.m[pr.out][0]);
                if (write_low) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float f[8];
                        Elem<__half>::widen(v[c], f);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            unpack2(sub2(pack2(y[8 * c + 2 * i], y[8 * c + 2 * i + 1]), pack2(f[2 * i], f[2 * i + 1])), f[2 * i], f[2 * i + 1]);
                        v[c] = Elem<__half>::narrow(f);
                    }
                    if (r < pad) muon_put(place(buffers[pr.out][1], b), v);
                    if (mirror) turn(v, P.ws.m[pr.out][1]);
                }
            };
            auto out_block = [&](uint32_t b) {
                const uint32_t col = col0 + 32 * b;
                float y[32];
                result(b, y);
                // to the caller's vectors: the block turned in shared memory to the caller's rows
                // (where X is the transpose, its columns)
                const bool narrow = !P.out.params && P.out_dtype != 0;
                __syncwarp();
                if (narrow) {
                    const float scale = P.out.scaled ? mat.scale : 1.f;
#pragma unroll
                    for (uint32_t c = 0; c < 4; ++c) {
                        uint32_t w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float u = __fmul_rn(scale, y[8 * c + 2 * i]), v = __fmul_rn(scale, y[8 * c + 2 * i + 1]);
                            w[i] = P.out_dtype == 1 ? Elem<__nv_bfloat16>::pair(u, v) : Elem<__half>::pair(u, v);
                        }
                        if (!mat.tall) {
                            sts16(own + ((c ^ flip) << 4), make_uint4(w[0], w[1], w[2], w[3]));
                        } else {
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                asm volatile("st.shared.b16 [%0], %1;"
                                             ::"r"(block + muon_swizzle(8 * c + i, lane >> 3) + 2 * (lane & 7)),
                                             "h"((uint16_t)(w[i >> 1] >> (16 * (i & 1)))) : "memory");
                        }
                    }
                } else {                                           // 16-byte pieces of a row exchanged by its number
#pragma unroll
                    for (uint32_t c = 0; c < 8; ++c) {
                        if (!mat.tall) {
                            sts16(block + lane * 128 + ((c ^ (lane & 7)) << 4), Elem<float>::narrow(y + 4 * c));
                        } else {
#pragma unroll
                            for (uint32_t i = 4 * c; i < 4 * c + 4; ++i)
                                asm volatile("st.shared.f32 [%0], %1;"
                                             ::"r"(block + i * 128 + (((lane >> 2) ^ (i & 7)) << 4) + 4 * (lane & 3)), "f"(y[i])
                                             : "memory");
                        }
                    }
                }
                __syncwarp();
                const uint32_t or0 = mat.tall ? col : row0, oc0 = mat.tall ? row0 : col;
                if (narrow) muon_out_narrow(P, mat, block, or0, oc0);
                else muon_out_wide(P, mat, block, or0, oc0, P.sound[task.mat] != 0);
                __syncwarp();
            };
            // sums in registers need fixed places; elsewhere a loop is kept, as unrolled code spills
            if constexpr (SPLIT) {
#pragma unroll
                for (uint32_t b = 0; b < kBlocks; ++b)
                    if (b < blocks) {                                  // the whole warp
                        if (!last) keep_block(b);
                        else out_block(b);
                    }
            } else if (!last) {
#pragma unroll 1
                for (uint32_t b = 0; b < blocks; ++b) keep_block(b);
            } else {
#pragma unroll 1
                for (uint32_t b = 0; b < blocks; ++b) out_block(b);
            }
            if (!SPLIT && steps) release();
            __syncwarp();
            // the signal warp does the rest; the barrier's last use, two tiles ago, is over first
            if (lane == 0 && muon_wait(stored + 8 * (n & 1), ((n >> 1) & 1) ^ 1, limit, &stop)) mbar_arrive(stored + 8 * (n & 1));
            // and the other may send the next tile's sums: last, as this release waits for the results
            // on their way to memory (before them: 1.2 us more a product)
            if (KS && lane == 0) leader_arrive(peer_addr(share_empty + 8 * quad, cta ^ 1));
        }
    }
    __syncwarp();
    tcgen05_before_sync();
    __syncthreads();
    if (kJoint) pair_sync();
    tcgen05_after_sync();
    // After a wait that ran out, partial sums and arrivals that this CTA did not wait for may still be on
    // their way to it from the other one, which has issued its last by now: 20,000 clocks to land.
    if (kJoint && stop)
        for (const long long from = clock64(); clock64() - from < 20000;) {}
    if (tid == 0 && stop) atomicOr(P.status, kStatusTimeout);
    if (warp == S::kEpiWarps + 1) tmem_free<CG>(tmem, S::kTmemCols);
}

}  // namespace ecq
