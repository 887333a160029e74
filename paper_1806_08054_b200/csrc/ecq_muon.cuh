// Newton-Schulz orthogonalisation of the matrices of a flat vector, with the momentum in front of
// it and the weight update behind it.
#pragma once

#include <cstdint>

#include "ecq_common.cuh"
#include "ecq_elem.cuh"

namespace ecq {

// The iteration, for a matrix taken with m <= n (a tall one is transposed on the way in and out):
//     X_0 = U / |U|_F,   X <- a X + (b G + c G^2) X,   G = X X^T
// Three products a step: G and G^2 are symmetric, so only tiles that touch the lower triangle are
// computed and written twice; the third is full.
//
// Numbers.  The products run on the tensor cores with fp16 operands and fp32 accumulators.  What
// keeps the result accurate is that X itself is never rounded to 11 bits: it is kept as a pair
// hi + lo of fp16 (22 bits), and the linear term a X takes both.  A rounding error of X in the
// directions of small singular values would be multiplied by a (3.44) in every step.  Against 64
// bits, relative error of the result for spectra from flat to 1/i^1.5: bf16 throughout 1e-2 to
// 9e-2, fp16 throughout 1e-3 to 1e-2, with the pair 3e-4 to 1.7e-3.
// In the last two steps, where most singular values are near 1, G is replaced by D = G - I
// (exactly the same polynomial: b G + c G^2 = (b + c) I + (b + 2c) D + c D^2), so that the
// rounding of G's diagonal does not cancel against a X: 5e-4 to 1.1e-3.
// With three products per product (hi hi + hi lo + lo hi) all operands have 22 bits and the
// result's error is that of fp32 arithmetic.
//
// X, G and the polynomial are stored scaled by powers of two, so that fp16's narrow range holds
// entries as small as 1 / (m n)^0.5 and their low halves.

constexpr float kMuonScaleX = 4096.f;
constexpr float kMuonScaleG = 256.f;

struct MuonMat {
    uint64_t offset, stride;             // in the caller's flat vectors, entries
    uint64_t x_at, g_at;                 // in the workspace, entries of fp16 (each of hi and lo)
    uint32_t rows, cols, m, n;
    uint32_t ld_x, ld_g;                 // padded to 64 entries
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

struct MuonSpan { uint64_t start, stride; uint32_t mat, rows, len; };   // rows of len entries
struct MuonTile { uint32_t mat; uint16_t i, j; };

struct MuonWork {
    __half *xh[2], *xl[2], *gh, *gl, *bh, *bl;
};

__device__ __forceinline__ float muon_direction(const MuonIn& in, float g, float m_new) {
    return in.nesterov ? __fmaf_rn(in.mu, m_new, g) : m_new;
}

// ---- sum of squares --------------------------------------------------------------------------
//
// First of two passes over the gradient and the momentum (8 bytes an entry; the second reads them
// again and writes the new momentum, so a matrix that holds a NaN or Inf is found before anything
// of it is changed).  Squares are added in 64 bits: no fp32 value overflows or vanishes.

constexpr int kMuonSpanThreads = 256;
constexpr uint32_t kMuonSpan = 32768;

template <typename T, bool MOM>
__global__ void __launch_bounds__(kMuonSpanThreads) muon_norm_kernel(const MuonSpan* spans, MuonIn in, double* partial) {
    constexpr uint32_t E = Elem<T>::kPer16;
    const MuonSpan sp = spans[blockIdx.x];
    const uint32_t tid = threadIdx.x;
    double sum = 0.0;
    auto direction = [&](float g, float m) { return MOM ? muon_direction(in, g, __fmaf_rn(in.mu, m, g)) : g; };
    for (uint32_t r = 0; r < sp.rows; ++r) {
        const T* g = reinterpret_cast<const T*>(in.grad) + sp.start + r * sp.stride;
        const float* mo = MOM ? in.momentum + sp.start + r * sp.stride : nullptr;
        const uint32_t odd = (uint32_t)((16u - (reinterpret_cast<uintptr_t>(g) & 15u)) & 15u) / (uint32_t)sizeof(T);
        const uint32_t head = odd < sp.len ? odd : sp.len;
        const uint32_t nv = (sp.len - head) / E;
        for (uint32_t v = tid; v < nv; v += kMuonSpanThreads) {
            float x[E];
            Elem<T>::widen(__ldg(reinterpret_cast<const uint4*>(g + head) + v), x);
            if (MOM) {                                               // fp32 beside fp32: the same alignment
                float y[4];
                Elem<float>::widen(__ldg(reinterpret_cast<const uint4*>(mo + head) + v), y);
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
    __shared__ double part[kMuonSpanThreads / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if ((tid & 31) == 0) part[tid >> 5] = sum;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kMuonSpanThreads / 32; ++w) sum += part[w];
        partial[blockIdx.x] = sum;
    }
}

// ---- X_0 and the new momentum ----------------------------------------------------------------

constexpr int kMuonPrepThreads = 256;

__device__ __forceinline__ void muon_split(float v, __half& hi, __half& lo) {
    hi = __float2half_rn(v);
    lo = __float2half_rn(__fsub_rn(v, __half2float(hi)));
}

// One 64 x 64 tile of a matrix.  norm[mat] gets 1 where the matrix is sound and 0 where it holds a
// NaN or Inf: then X_0 = 0 and its momentum (and later its weights) stay as they are.
template <typename T, bool MOM>
__global__ void __launch_bounds__(kMuonPrepThreads) muon_prepare_kernel(
    const MuonMat* mats, const MuonTile* tiles, const double* partial, MuonIn in, MuonWork ws, uint32_t* sound,
    uint32_t* status) {
    const MuonTile tile = tiles[blockIdx.x];
    const MuonMat mat = mats[tile.mat];
    const uint32_t tid = threadIdx.x;
    __shared__ float stage[64][65];
    __shared__ float factor[2];
    if (tid < 32) {
        double sum = 0.0;
        for (uint32_t i = tid; i < mat.parts; i += 32) sum += partial[mat.part0 + i];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        if (tid == 0) {
            const bool ok = sum < INFINITY;                          // false for NaN
            // S / |U| as two factors: one of them alone may pass the range of fp32
            int e = 0;
            const double inv = ok && sum > 0.0 ? frexp((double)kMuonScaleX / sqrt(sum), &e) : 0.0;
            factor[0] = (float)ldexp(inv, e / 2);
            factor[1] = (float)ldexp(1.0, e - e / 2);
            if (!ok) factor[1] = NAN;
            if (tile.i == 0 && tile.j == 0) {
                sound[tile.mat] = ok ? 1u : 0u;
                if (!ok) atomicOr(status, kStatusNonFinite);
            }
        }
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
        if (xr >= mat.m) continue;
        __half hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) muon_split(x[k][i], hi[i], lo[i]);
        const uint64_t to = mat.x_at + (uint64_t)xr * mat.ld_x + xc;  // xc + 4 <= ld_x: a tile is 64 wide
        *reinterpret_cast<uint2*>(ws.xh[0] + to) = *reinterpret_cast<uint2*>(hi);
        *reinterpret_cast<uint2*>(ws.xl[0] + to) = *reinterpret_cast<uint2*>(lo);
    }
}

// ---- tensor-core products --------------------------------------------------------------------

// Shared-memory matrix descriptor of a tile in 128-byte swizzled rows: `lead` and `step` are the
// byte distances between 64-wide column blocks (where the tile's rows are along K) and between
// groups of eight 128-byte rows.
__device__ __forceinline__ uint64_t umma_desc(uint32_t addr, uint32_t lead, uint32_t step) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(step >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
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
// The same shared-memory location in the pair's first CTA.
__device__ __forceinline__ uint32_t leader_addr(uint32_t addr) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(addr));
    return a;
}
__device__ __forceinline__ void leader_arrive(uint32_t leader_bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(leader_bar) : "memory");
}

// A 64 x 64 box of fp16 into this CTA's shared memory; in a pair the bytes are counted on the
// first CTA's barrier.
template <int CG>
__device__ __forceinline__ void muon_load(uint32_t dst, const void* map, uint32_t x, uint32_t y, uint32_t bar) {
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
                     " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
                     " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar)
                     : "memory");
}

enum { kMuonGram = 0, kMuonPoly = 1, kMuonApply = 2 };
enum { kMapX = 0, kMapG = 4, kMapB = 6, kMapsPerMat = 8 };           // X: hi, lo of each copy; G, B: hi, lo

struct MuonPhase {
    const MuonMat* mats;
    const unsigned char* maps;           // 8 tensor maps of 128 bytes per matrix
    const MuonTile* tiles;
    const uint32_t* sound;
    uint32_t* status;
    MuonWork ws;
    MuonOut out;
    uint32_t n_tiles;
    int kind;                            // kMuonGram, kMuonPoly, kMuonApply
    int src;                             // copy of X that is read
    int terms;                           // 1, or 3: hi hi, hi lo, lo hi
    int last;                            // kMuonApply of the last step: to the caller's vectors
    float lin, acc, shift;               // out = lin * in + acc * product - shift on the diagonal
    uint32_t wait_limit;
};

constexpr int kMuonEpiWarps = 8;
constexpr int kMuonThreads = (kMuonEpiWarps + 2) * 32;
constexpr uint32_t kMuonBox = 8192;                                   // 64 x 64 fp16

// CG CTAs work on one tile of CG * 128 rows and TN columns; each stages its 128 rows of the left
// operand and TN / CG rows of the right one, 64 along K at a time.
template <int CG, int TN>
struct MuonShape {
    static constexpr uint32_t kBoxesA = 2, kBoxesB = TN / CG / 64;
    static constexpr uint32_t kStageBytes = (kBoxesA + kBoxesB) * kMuonBox;
    static constexpr uint32_t kStages = 6;
    static constexpr uint32_t kBars = 2 * kStages + 4;
    static constexpr uint32_t kSmem = kStages * kStageBytes + 1024;   // + alignment
    static constexpr uint32_t kTmemCols = 2 * TN < 32 ? 32 : 2 * TN;
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

template <typename TO>
__device__ __forceinline__ void muon_write_last(const MuonPhase& P, const MuonMat& mat, uint64_t at, float o, bool sound) {
    if (P.out.update)
        Elem<TO>::store(reinterpret_cast<TO*>(P.out.update) + at, P.out.scaled ? __fmul_rn(mat.scale, o) : o);
    if (P.out.params && sound) {
        const float p = P.out.params[at];
        P.out.params[at] = __fmaf_rn(-__fmul_rn(P.out.rate, mat.scale), o, __fmul_rn(P.out.keep, p));
    }
}

template <int CG, int TN, typename TO>
__global__ void __launch_bounds__(kMuonThreads, 1) muon_product_kernel(const MuonPhase P) {
    using S = MuonShape<CG, TN>;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t bars[S::kBars];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t stop;
    __shared__ float turn[kMuonEpiWarps][32][33];
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t ring = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t full = bar0, empty = bar0 + 8 * S::kStages, acc_full = bar0 + 16 * S::kStages, acc_empty = acc_full + 16;
    const uint32_t rank = CG == 1 ? 0 : cta_rank();
    const uint32_t group = blockIdx.x / CG, groups = gridDim.x / CG;

    if (tid == 0) {
        for (uint32_t s = 0; s < S::kStages; ++s) { mbar_init(full + 8 * s, 1); mbar_init(empty + 8 * s, 1); }
        for (uint32_t b = 0; b < 2; ++b) { mbar_init(acc_full + 8 * b, 1); mbar_init(acc_empty + 8 * b, CG * kMuonEpiWarps); }
        stop = 0;
        fence_mbar_init();
    }
    if (warp == kMuonEpiWarps + 1) tmem_alloc<CG>(smem_u32(&tmem_slot), S::kTmemCols);
    tcgen05_before_sync();
    __syncthreads();
    if (CG == 2) pair_sync();
    tcgen05_after_sync();
    const uint32_t tmem = tmem_slot;

    if (warp == kMuonEpiWarps) {
        // ---- loads -------------------------------------------------------------------------------
        if (lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            for (uint32_t t = group; t < P.n_tiles && ok; t += groups) {
                const MuonTile tile = P.tiles[t];
                const unsigned char* map = P.maps + (uint64_t)tile.mat * kMapsPerMat * 128;
                const uint32_t m = P.mats[tile.mat].m, n = P.mats[tile.mat].n;
                const uint32_t K = P.kind == kMuonGram ? n : m;
                const uint32_t kb = (K + 63) / 64;
                const uint32_t row = tile.i * (CG * 128u) + rank * 128u;
                const uint32_t col = tile.j * (uint32_t)TN + rank * (TN / CG);
                const int left = P.kind == kMuonGram ? kMapX + 2 * P.src : P.kind == kMuonPoly ? kMapG : kMapB;
                const int right = P.kind == kMuonPoly ? kMapG : kMapX + 2 * P.src;
                for (int term = 0; term < P.terms && ok; ++term) {
                    const unsigned char* ma = map + (left + (term == 2 ? 1 : 0)) * 128;
                    const unsigned char* mb = map + (right + (term == 1 ? 1 : 0)) * 128;
                    for (uint32_t k = 0; k < kb; ++k, ++it) {
                        const uint32_t s = it % S::kStages, ph = (it / S::kStages) & 1;
                        if (!muon_wait(empty + 8 * s, ph ^ 1, P.wait_limit, &stop)) { ok = false; break; }
                        if (rank == 0) mbar_arrive_expect_tx(full + 8 * s, CG * S::kStageBytes);
                        const uint32_t bar = CG == 1 ? full + 8 * s : leader_addr(full + 8 * s);
                        const uint32_t dst = ring + s * S::kStageBytes;
                        for (uint32_t b = 0; b < S::kBoxesA; ++b)
                            muon_load<CG>(dst + b * kMuonBox, ma, k * 64, row + b * 64, bar);
                        for (uint32_t b = 0; b < S::kBoxesB; ++b) {
                            const uint32_t to = dst + (S::kBoxesA + b) * kMuonBox;
                            if (P.kind == kMuonApply) muon_load<CG>(to, mb, col + b * 64, k * 64, bar);
                            else muon_load<CG>(to, mb, k * 64, col + b * 64, bar);
                        }
                    }
                }
            }
            // nothing of this CTA's is in flight when it leaves: every stage's last load was consumed
            // (or, where a wait ran out and nobody consumes them any more, has had time to land)
            for (uint32_t b = 0; b < S::kStages && b < it; ++b) {
                const uint32_t last = it - 1 - b, limit = stop ? 1u << 12 : kWaitLimit;
                for (uint32_t n = 0; n < limit; ++n)
                    if (mbar_try_wait(empty + 8 * (last % S::kStages), (last / S::kStages) & 1)) break;
            }
        }
    } else if (warp == kMuonEpiWarps + 1) {
        // ---- products ----------------------------------------------------------------------------
        if (lane == 0 && rank == 0) {
            // fp32 accumulators; fp16 operands; right operand along N (bit 16) in kMuonApply
            const uint32_t idesc = (1u << 4) | ((uint32_t)(TN / 8) << 17) | ((uint32_t)(CG * 128 / 16) << 24) |
                                   (P.kind == kMuonApply ? 1u << 16 : 0u);
            const uint32_t b_lead = P.kind == kMuonApply ? kMuonBox : 16;
            const uint32_t b_k16 = P.kind == kMuonApply ? 2048u : 32u;   // bytes to the next 16 along K
            uint32_t it = 0, n = 0;
            bool ok = true;
            for (uint32_t t = group; t < P.n_tiles && ok; t += groups, ++n) {
                const MuonTile tile = P.tiles[t];
                const uint32_t K = P.kind == kMuonGram ? P.mats[tile.mat].n : P.mats[tile.mat].m;
                const uint32_t total = (K + 63) / 64 * P.terms;
                const uint32_t buf = n & 1;
                if (!muon_wait(acc_empty + 8 * buf, ((n >> 1) & 1) ^ 1, P.wait_limit, &stop)) break;
                tcgen05_after_sync();
                const uint32_t d = tmem + buf * TN;
                for (uint32_t k = 0; k < total; ++k, ++it) {
                    const uint32_t s = it % S::kStages, ph = (it / S::kStages) & 1;
                    if (!muon_wait(full + 8 * s, ph, P.wait_limit, &stop)) { ok = false; break; }
                    tcgen05_after_sync();
                    const uint32_t a0 = ring + s * S::kStageBytes, b0 = a0 + S::kBoxesA * kMuonBox;
#pragma unroll
                    for (uint32_t q = 0; q < 4; ++q)
                        umma_f16<CG>(d, umma_desc(a0 + 32 * q, 16, 1024), umma_desc(b0 + b_k16 * q, b_lead, 1024), idesc,
                                     k > 0 || q > 0);
                    umma_commit<CG>(empty + 8 * s);
                }
                if (ok) umma_commit<CG>(acc_full + 8 * buf);
            }
        }
    } else {
        // ---- results -----------------------------------------------------------------------------
        const uint32_t quad = warp & 3, half = warp >> 2;
        uint32_t n = 0;
        for (uint32_t t = group; t < P.n_tiles; t += groups, ++n) {
            const MuonTile tile = P.tiles[t];
            const MuonMat mat = P.mats[tile.mat];
            const uint32_t buf = n & 1;
            if (!__all_sync(~0u, muon_wait(acc_full + 8 * buf, (n >> 1) & 1, P.wait_limit, &stop))) break;
            tcgen05_after_sync();
            const uint32_t row0 = tile.i * (CG * 128u) + rank * 128u + quad * 32u;
            const uint32_t r = row0 + lane;
            const bool sound = P.last ? P.sound[tile.mat] != 0 : true;
            const bool mirror = P.kind != kMuonApply && tile.j * (uint32_t)TN / (CG * 128u) < tile.i;
            const uint32_t width = P.kind == kMuonApply ? mat.n : mat.m, ld = P.kind == kMuonApply ? mat.ld_x : mat.ld_g;
            for (uint32_t c = half * (TN / 2); c < (half + 1) * (uint32_t)(TN / 2); c += 32) {
                const uint32_t col = tile.j * (uint32_t)TN + c;
                if (row0 >= mat.m || col >= width) continue;          // the whole warp
                const bool in = r < mat.m;
                float v[32], x[32];
                const uint64_t at = (P.kind == kMuonApply ? mat.x_at : mat.g_at) + (uint64_t)r * ld + col;
                if (P.kind == kMuonGram || !in) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = 0.f;
                } else {
                    const __half* ph = (P.kind == kMuonApply ? P.ws.xh[P.src] : P.ws.gh) + at;
                    const __half* pl = (P.kind == kMuonApply ? P.ws.xl[P.src] : P.ws.gl) + at;
                    const bool low = P.kind == kMuonApply || P.terms == 3;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float h[8], l[8];
                        Elem<__half>::widen(*reinterpret_cast<const uint4*>(ph + 8 * i), h);
                        if (low) Elem<__half>::widen(*reinterpret_cast<const uint4*>(pl + 8 * i), l);
#pragma unroll
                        for (int j = 0; j < 8; ++j) x[8 * i + j] = low ? __fadd_rn(h[j], l[j]) : h[j];
                    }
                }
                tmem_load32(tmem + ((quad * 32u) << 16) + buf * TN + c, v);
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    v[i] = __fmaf_rn(P.lin, x[i], __fmul_rn(P.acc, v[i]));
                    if (P.kind == kMuonGram && r == col + i) v[i] = __fsub_rn(v[i], P.shift);
                }
                if (P.last) {
                    if (mat.tall) {
                        // the caller's rows run along the lanes
                        for (int i = 0; i < 32; ++i)
                            if (in && col + i < width)
                                muon_write_last<TO>(P, mat, mat.offset + (uint64_t)(col + i) * mat.stride + r, v[i], sound);
                    } else {
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 32; ++i) turn[warp][lane][i] = v[i];
                        __syncwarp();
                        for (uint32_t i = 0; i < 32; ++i)
                            if (row0 + i < mat.m && col + lane < width)
                                muon_write_last<TO>(P, mat, mat.offset + (uint64_t)(row0 + i) * mat.stride + col + lane,
                                                    turn[warp][i][lane], sound);
                    }
                    continue;
                }
                __half* oh = (P.kind == kMuonGram ? P.ws.gh : P.kind == kMuonPoly ? P.ws.bh : P.ws.xh[P.src ^ 1]);
                __half* ol = (P.kind == kMuonGram ? P.ws.gl : P.kind == kMuonPoly ? P.ws.bl : P.ws.xl[P.src ^ 1]);
                const bool low = P.kind == kMuonApply || P.terms == 3;
                if (in) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        __half hi[8], lo[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) muon_split(v[8 * i + j], hi[j], lo[j]);
                        *reinterpret_cast<uint4*>(oh + at + 8 * i) = *reinterpret_cast<uint4*>(hi);
                        if (low) *reinterpret_cast<uint4*>(ol + at + 8 * i) = *reinterpret_cast<uint4*>(lo);
                    }
                    if (mirror) {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (col + i < mat.m) {
                                __half hi, lo;
                                muon_split(v[i], hi, lo);
                                const uint64_t to = mat.g_at + (uint64_t)(col + i) * ld + r;
                                oh[to] = hi;
                                if (low) ol[to] = lo;
                            }
                    }
                }
            }
            tcgen05_before_sync();
            __syncwarp();
            if (lane == 0) {
                if (CG == 1) mbar_arrive(acc_empty + 8 * buf);
                else leader_arrive(leader_addr(acc_empty + 8 * buf));
            }
        }
    }
    __syncwarp();
    tcgen05_before_sync();
    __syncthreads();
    if (CG == 2) pair_sync();
    tcgen05_after_sync();
    if (tid == 0 && stop) atomicOr(P.status, kStatusTimeout);
    if (warp == kMuonEpiWarps + 1) tmem_free<CG>(tmem, S::kTmemCols);
}

}  // namespace ecq
