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
    uint32_t tiles_sym[4], tiles_full[4];  // tiles of its products, by tile shape
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
    unsigned long long* done, unsigned long long* next, uint32_t* status) {
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
                done[tile.mat] = 0;                                  // for the products that follow
                if (tile.mat == 0) *next = 0;
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
// Tensor maps of a matrix.  Loads of operands take 64 x 64 boxes, the epilogue reads and writes
// blocks of 32 rows and 64 columns, and the mirrored halves of symmetric products are written in
// blocks of 64 rows and 32 columns.  Each group: X (hi, lo of two copies), G (hi, lo), B (hi, lo).
enum { kMapX = 0, kMapG = 4, kMapB = 6, kMapOperand = 0, kMapBlock = 8, kMapMirror = 16, kMapsPerMat = 20 };

struct MuonStep { float poly_lin, poly_acc, apply_lin, apply_acc, shift; };

struct MuonIterate {
    const MuonMat* mats;
    const unsigned char* maps;           // kMapsPerMat tensor maps of 128 bytes per matrix
    const MuonTile *sym, *full;          // tiles of a symmetric product, of the product with X
    const MuonStep* steps;
    const uint32_t* sound;
    unsigned long long* done;            // per matrix: parts of tiles finished since the call began
    unsigned long long* next;            // the next tile that nobody has taken
    uint32_t* status;
    MuonOut out;
    int out_dtype;
    uint32_t n_sym, n_full, n_steps;
    uint32_t shape;                      // index of MuonMat::tiles_sym, tiles_full
    uint32_t wait_limit;
};

constexpr uint32_t kMuonBox = 8192;                                   // 64 x 64 fp16
constexpr uint32_t kMuonBlock = 4096;                                 // 32 x 64 fp16
constexpr uint32_t kMuonQueue = 2;
constexpr uint32_t kMuonChunk = 4;                                    // 64-wide steps along K per partial sum (SPLIT)

// CG CTAs work on one tile of CG * 128 rows and TN columns; each stages its 128 rows of the left
// operand and TN / CG rows of the right one, 64 along K at a time, both halves of each with SPLIT.
template <int CG, int TN, bool SPLIT>
struct MuonShape {
    static constexpr uint32_t kHalves = SPLIT ? 2 : 1;
    static constexpr uint32_t kBoxesA = 2, kBoxesB = TN / CG / 64;
    static constexpr uint32_t kBytesA = kBoxesA * kMuonBox, kBytesB = kBoxesB * kMuonBox;
    static constexpr uint32_t kStageBytes = kHalves * (kBytesA + kBytesB);
    static constexpr uint32_t kEpiWarps = TN >= 128 ? 8 : 4;
    static constexpr uint32_t kCols = TN / (kEpiWarps / 4);           // columns of an epilogue warp
    static constexpr uint32_t kThreads = (kEpiWarps + 3) * 32;        // + loads, products, tile queue
    static constexpr uint32_t kEpiBytes = kEpiWarps * 2 * kMuonBlock;
    static constexpr uint32_t kStagesFit = (230u * 1024u - 2048u - kEpiBytes) / kStageBytes;
    static constexpr uint32_t kStages = kStagesFit < 6 ? kStagesFit : 6;
    static constexpr uint32_t kSmem = kStages * kStageBytes + kEpiBytes + 1024;   // + alignment
    static constexpr uint32_t kAccCols = SPLIT ? 2 * TN : TN;         // hi hi, and the two small products
    static constexpr uint32_t kTmemCols = 2 * kAccCols;
    // arrivals per tile on MuonIterate::done, and on a queue slot
    static constexpr uint32_t kParts = CG * kEpiWarps, kReaders = CG * (kEpiWarps + 1) + 1;
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

// One tile of the whole computation, in the order in which they are handed out: for each step G
// of all matrices, then the polynomials, then the products with X.
struct MuonTask {
    MuonTile tile;
    uint32_t step;
    int kind;
    unsigned long long need;             // parts of the matrix's earlier tiles that it waits for
    bool end;
};

template <typename S>
__device__ __forceinline__ MuonTask muon_task(const MuonIterate& P, uint32_t t) {
    MuonTask k;
    const uint32_t per = 2 * P.n_sym + P.n_full;
    k.step = t / per;
    k.end = k.step >= P.n_steps;
    if (k.end) return k;
    const uint32_t r = t - k.step * per;
    k.kind = r < P.n_sym ? kMuonGram : r < 2 * P.n_sym ? kMuonPoly : kMuonApply;
    k.tile = k.kind == kMuonApply ? P.full[r - 2 * P.n_sym] : P.sym[k.kind == kMuonGram ? r : r - P.n_sym];
    const MuonMat& mat = P.mats[k.tile.mat];
    const unsigned long long sym = mat.tiles_sym[P.shape], full = mat.tiles_full[P.shape];
    k.need = S::kParts * (k.step * (2 * sym + full) + k.kind * sym);
    return k;
}

__device__ __forceinline__ void muon_write_last(const MuonIterate& P, const MuonMat& mat, uint64_t at, float o, bool sound) {
    if (P.out.update) {
        const float u = P.out.scaled ? __fmul_rn(mat.scale, o) : o;
        if (P.out_dtype == 0) reinterpret_cast<float*>(P.out.update)[at] = u;
        else if (P.out_dtype == 1) reinterpret_cast<__nv_bfloat16*>(P.out.update)[at] = __float2bfloat16_rn(u);
        else reinterpret_cast<__half*>(P.out.update)[at] = __float2half_rn(u);
    }
    if (P.out.params && sound) {
        const float p = P.out.params[at];
        P.out.params[at] = __fmaf_rn(-__fmul_rn(P.out.rate, mat.scale), o, __fmul_rn(P.out.keep, p));
    }
}

// Place of the 16 bytes with columns 8 c .. 8 c + 7 of row r in a block of 128-byte swizzled rows.
__device__ __forceinline__ uint32_t muon_swizzle(uint32_t r, uint32_t c) { return r * 128u + ((c ^ (r & 7u)) << 4); }

__device__ __forceinline__ uint4 lds16(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ void sts16(uint32_t addr, uint4 v) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// Every step of every matrix in one launch.  Tiles are taken from a counter in a fixed order; each
// waits until the tiles that its operands come from are finished.  Those are earlier in the order,
// so they have been taken by CTAs that are running: some tile can always go on, whatever number
// of CTAs the GPU has room for.
template <int CG, int TN, bool SPLIT>
__global__ void __launch_bounds__(MuonShape<CG, TN, SPLIT>::kThreads, 1) muon_iterate_kernel(const MuonIterate P) {
    using S = MuonShape<CG, TN, SPLIT>;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::kStages + 4 + 2 * kMuonQueue + S::kEpiWarps];
    __shared__ uint32_t tmem_slot, queue[kMuonQueue];
    __shared__ volatile uint32_t stop;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t ring = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t full = smem_u32(bars), empty = full + 8 * S::kStages;
    const uint32_t acc_full = empty + 8 * S::kStages, acc_empty = acc_full + 16;
    const uint32_t q_full = acc_empty + 16, q_empty = q_full + 8 * kMuonQueue, loaded = q_empty + 8 * kMuonQueue;
    const uint32_t rank = CG == 1 ? 0 : cta_rank();
    const uint32_t limit = P.wait_limit;

    if (tid == 0) {
        for (uint32_t s = 0; s < S::kStages; ++s) { mbar_init(full + 8 * s, 1); mbar_init(empty + 8 * s, 1); }
        for (uint32_t b = 0; b < 2; ++b) { mbar_init(acc_full + 8 * b, 1); mbar_init(acc_empty + 8 * b, S::kParts); }
        for (uint32_t q = 0; q < kMuonQueue; ++q) { mbar_init(q_full + 8 * q, 1); mbar_init(q_empty + 8 * q, S::kReaders); }
        for (uint32_t w = 0; w < S::kEpiWarps; ++w) mbar_init(loaded + 8 * w, 1);
        stop = 0;
        fence_mbar_init();
    }
    if (warp == S::kEpiWarps + 1) tmem_alloc<CG>(smem_u32(&tmem_slot), S::kTmemCols);
    tcgen05_before_sync();
    __syncthreads();
    if (CG == 2) pair_sync();
    tcgen05_after_sync();
    const uint32_t tmem = tmem_slot;

    // n-th tile of this CTA (or pair); false when there is none or a wait ran out
    auto take = [&](uint32_t n, uint32_t& t) {
        const uint32_t q = n % kMuonQueue;
        if (!(CG == 1 ? muon_wait(q_full + 8 * q, (n / kMuonQueue) & 1, limit, &stop)
                      : muon_wait_pair(q_full + 8 * q, (n / kMuonQueue) & 1, limit, &stop)))
            return false;
        t = *reinterpret_cast<volatile uint32_t*>(&queue[q]);
        return true;
    };
    auto taken = [&](uint32_t n) {
        const uint32_t bar = q_empty + 8 * (n % kMuonQueue);
        if (CG == 1) mbar_arrive(bar);
        else leader_arrive(leader_addr(bar));
    };

    if (warp == S::kEpiWarps) {
        // ---- loads -------------------------------------------------------------------------------
        if (lane == 0) {
            uint32_t it = 0, t;
            bool ok = true;
            for (uint32_t n = 0; ok && take(n, t); ++n) {
                taken(n);
                const MuonTask task = muon_task<S>(P, t);
                if (task.end) break;
                const unsigned char* map = P.maps + (uint64_t)task.tile.mat * kMapsPerMat * 128;
                const MuonMat& mat = P.mats[task.tile.mat];
                const uint32_t kb = ((task.kind == kMuonGram ? mat.n : mat.m) + 63) / 64;
                const uint32_t row = task.tile.i * (CG * 128u) + rank * 128u;
                const uint32_t col = task.tile.j * (uint32_t)TN + rank * (TN / CG);
                const int x = kMapX + 2 * (task.step & 1);
                const unsigned char* ma = map + (task.kind == kMuonGram ? x : task.kind == kMuonPoly ? kMapG : kMapB) * 128;
                const unsigned char* mb = map + (task.kind == kMuonPoly ? kMapG : x) * 128;
                if (!muon_wait_done(P.done + task.tile.mat, task.need, limit, &stop, 0)) break;
                for (uint32_t k = 0; k < kb; ++k, ++it) {
                    const uint32_t s = it % S::kStages, ph = (it / S::kStages) & 1;
                    if (!muon_wait(empty + 8 * s, ph ^ 1, limit, &stop)) { ok = false; break; }
                    if (rank == 0) mbar_arrive_expect_tx(full + 8 * s, CG * S::kStageBytes);
                    const uint32_t bar = CG == 1 ? full + 8 * s : leader_addr(full + 8 * s);
                    uint32_t dst = ring + s * S::kStageBytes;
#pragma unroll
                    for (uint32_t h = 0; h < S::kHalves; ++h)
#pragma unroll
                        for (uint32_t b = 0; b < S::kBoxesA; ++b, dst += kMuonBox)
                            muon_load<CG>(dst, ma + 128 * h, k * 64, row + b * 64, bar);
#pragma unroll
                    for (uint32_t h = 0; h < S::kHalves; ++h)
#pragma unroll
                        for (uint32_t b = 0; b < S::kBoxesB; ++b, dst += kMuonBox) {
                            if (task.kind == kMuonApply) muon_load<CG>(dst, mb + 128 * h, col + b * 64, k * 64, bar);
                            else muon_load<CG>(dst, mb + 128 * h, k * 64, col + b * 64, bar);
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
        if (lane == 0 && rank == 0) {
            uint32_t it = 0, acc = 0, t;
            bool ok = true;
            for (uint32_t n = 0; ok && take(n, t); ++n) {
                taken(n);
                const MuonTask task = muon_task<S>(P, t);
                if (task.end) break;
                const MuonMat& mat = P.mats[task.tile.mat];
                const uint32_t kb = ((task.kind == kMuonGram ? mat.n : mat.m) + 63) / 64;
                const bool along_n = task.kind == kMuonApply;          // right operand's rows run along K
                // fp32 accumulators, fp16 operands
                const uint32_t idesc = (1u << 4) | ((uint32_t)(TN / 8) << 17) | ((uint32_t)(CG * 128 / 16) << 24) |
                                       (along_n ? 1u << 16 : 0u);
                const uint32_t b_lead = along_n ? kMuonBox : 16;
                const uint32_t b_k16 = along_n ? 2048u : 32u;          // bytes to the next 16 along K
                uint32_t in_chunk = 0, d = 0;
                for (uint32_t k = 0; k < kb; ++k, ++it) {
                    if (in_chunk == 0) {
                        if (!muon_wait(acc_empty + 8 * (acc & 1), ((acc >> 1) & 1) ^ 1, limit, &stop)) { ok = false; break; }
                        d = tmem + (acc & 1) * S::kAccCols;
                    }
                    const uint32_t s = it % S::kStages, ph = (it / S::kStages) & 1;
                    if (!muon_wait(full + 8 * s, ph, limit, &stop)) { ok = false; break; }
                    tcgen05_after_sync();
                    const uint32_t a0 = ring + s * S::kStageBytes, b0 = a0 + S::kHalves * S::kBytesA;
                    const uint64_t da = umma_desc(a0, 16, 1024), db = umma_desc(b0, b_lead, 1024);
                    const uint64_t dal = umma_desc(a0 + S::kBytesA, 16, 1024), dbl = umma_desc(b0 + S::kBytesB, b_lead, 1024);
#pragma unroll
                    for (uint32_t q = 0; q < 4; ++q) {
                        const bool add = in_chunk > 0 || q > 0;
                        const uint64_t qa = (32 * q) >> 4, qb = (uint64_t)((b_k16 * q) >> 4);
                        umma_f16<CG>(d, da + qa, db + qb, idesc, add);
                        if (SPLIT) {
                            umma_f16<CG>(d + TN, da + qa, dbl + qb, idesc, add);
                            umma_f16<CG>(d + TN, dal + qa, db + qb, idesc, true);
                        }
                    }
                    umma_commit<CG>(empty + 8 * s);
                    if (++in_chunk == (SPLIT ? kMuonChunk : kb) || k + 1 == kb) {
                        umma_commit<CG>(acc_full + 8 * (acc & 1));
                        in_chunk = 0;
                        ++acc;
                    }
                }
            }
        }
    } else if (warp == S::kEpiWarps + 2) {
        // ---- tile queue --------------------------------------------------------------------------
        if (lane == 0 && rank == 0) {
            const uint32_t total = (2 * P.n_sym + P.n_full) * P.n_steps;
            uint32_t t = (uint32_t)min(atomicAdd(P.next, 1ull), (unsigned long long)total);
            for (uint32_t n = 0;; ++n) {
                const uint32_t q = n % kMuonQueue;
                if (!muon_wait(q_empty + 8 * q, ((n / kMuonQueue) & 1) ^ 1, limit, &stop)) break;
                *reinterpret_cast<volatile uint32_t*>(&queue[q]) = t;
                mbar_arrive(q_full + 8 * q);
                if (CG == 2) {
                    uint32_t v, b;
                    asm("mapa.shared::cluster.u32 %0, %1, 1;" : "=r"(v) : "r"(smem_u32(&queue[q])));
                    asm("mapa.shared::cluster.u32 %0, %1, 1;" : "=r"(b) : "r"(q_full + 8 * q));
                    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(v), "r"(t) : "memory");
                    leader_arrive(b);
                }
                if (t >= total) break;
                t = (uint32_t)min(atomicAdd(P.next, 1ull), (unsigned long long)total);
            }
        }
    } else {
        // ---- results -----------------------------------------------------------------------------
        // Every warp has 32 rows and kCols columns of a tile.  What its results are added to comes
        // in blocks of 32 x 64 by TMA, is replaced by the result in place, and leaves by TMA.
        const uint32_t quad = warp & 3, c0 = (warp >> 2) * S::kCols;
        const uint32_t block = ring + S::kStages * S::kStageBytes + warp * 2 * kMuonBlock;
        const uint32_t lane_addr = tmem + ((quad * 32u) << 16);
        uint32_t acc = 0, loads = 0, t;
        bool ok = true;
        for (uint32_t n = 0; ok && __all_sync(~0u, take(n, t)); ++n) {
            __syncwarp();
            if (lane == 0) taken(n);
            const MuonTask task = muon_task<S>(P, t);
            if (task.end) break;
            const MuonMat mat = P.mats[task.tile.mat];
            const MuonStep step = P.steps[task.step];
            const unsigned char* map = P.maps + (uint64_t)task.tile.mat * kMapsPerMat * 128;
            const bool apply = task.kind == kMuonApply, gram = task.kind == kMuonGram;
            const bool last = apply && task.step + 1 == P.n_steps;
            const int src = task.step & 1;
            const uint32_t row0 = task.tile.i * (CG * 128u) + rank * 128u + quad * 32u;
            const uint32_t col0 = task.tile.j * (uint32_t)TN + c0;
            const uint32_t r = row0 + lane;
            const uint32_t width = apply ? mat.n : mat.m;
            const bool rows_in = row0 < mat.m;
            const bool low = SPLIT || apply;                           // hi and lo, or hi alone
            const bool mirror = !apply && task.tile.j * (uint32_t)TN / (CG * 128u) < task.tile.i;
            const bool sound = last ? P.sound[task.tile.mat] != 0 : true;
            const unsigned char* in_map = map + (kMapBlock + (apply ? kMapX + 2 * src : kMapG)) * 128;
            const unsigned char* out_map = map + (kMapBlock + (gram ? kMapG : apply ? kMapX + 2 * (src ^ 1) : kMapB)) * 128;
            const unsigned char* mir_map = map + (kMapMirror + (gram ? 0 : 2)) * 128;
            const float lin = apply ? step.apply_lin : step.poly_lin;
            const float mul = gram ? kMuonScaleG / (kMuonScaleX * kMuonScaleX) : apply ? step.apply_acc : step.poly_acc;

            auto fetch = [&](uint32_t col) {                           // lane 0
                mbar_arrive_expect_tx(loaded + 8 * warp, (low ? 2 : 1) * kMuonBlock);
                tma_load_2d(block, in_map, (int)col, (int)row0, loaded + 8 * warp);
                if (low) tma_load_2d(block + kMuonBlock, in_map + 128, (int)col, (int)row0, loaded + 8 * warp);
            };
            const bool any = rows_in && col0 < width;
            if (!gram && any) {
                int go = 1;
                if (lane == 0) {
                    go = muon_wait_done(P.done + task.tile.mat, task.need, limit, &stop, 100);
                    if (go) fetch(col0);
                }
                if (!__shfl_sync(~0u, go, 0)) break;
            }

            float sum[SPLIT ? S::kCols : 1];
            if (SPLIT) {
#pragma unroll
                for (uint32_t i = 0; i < S::kCols; ++i) sum[i] = 0.f;
                const uint32_t kb = ((gram ? mat.n : mat.m) + 63) / 64;
                for (uint32_t chunk = 0; chunk < (kb + kMuonChunk - 1) / kMuonChunk; ++chunk, ++acc) {
                    ok = __all_sync(~0u, muon_wait(acc_full + 8 * (acc & 1), (acc >> 1) & 1, limit, &stop));
                    if (!ok) break;
                    tcgen05_after_sync();
#pragma unroll
                    for (uint32_t h = 0; h < S::kCols / 32; ++h) {
                        float v[32], w[32];
                        tmem_load32(lane_addr + (acc & 1) * S::kAccCols + c0 + 32 * h, v);
                        tmem_load32(lane_addr + (acc & 1) * S::kAccCols + TN + c0 + 32 * h, w);
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            sum[(SPLIT ? 32 * h : 0) + (SPLIT ? i : 0)] =
                                __fadd_rn(sum[(SPLIT ? 32 * h : 0) + (SPLIT ? i : 0)], __fadd_rn(v[i], w[i]));
                    }
                    tcgen05_before_sync();
                    __syncwarp();
                    if (lane == 0) {
                        if (CG == 1) mbar_arrive(acc_empty + 8 * (acc & 1));
                        else leader_arrive(leader_addr(acc_empty + 8 * (acc & 1)));
                    }
                }
            } else {
                ok = __all_sync(~0u, muon_wait(acc_full + 8 * (acc & 1), (acc >> 1) & 1, limit, &stop));
                tcgen05_after_sync();
            }
            if (!ok) break;

#pragma unroll
            for (uint32_t b = 0; b < S::kCols / 64; ++b) {
                const uint32_t col = col0 + 64 * b;
                if (!rows_in || col >= width) continue;                // the whole warp
                if (b > 0) {                                           // the buffer's last block has left
                    if (lane == 0) {
                        bulk_wait_read0();
                        if (!gram) fetch(col);
                    }
                    __syncwarp();
                }
                float y[64];
                if (SPLIT) {
#pragma unroll
                    for (int i = 0; i < 64; ++i) y[i] = sum[SPLIT ? 64 * b + i : 0];
                } else {
                    tmem_load32(lane_addr + (acc & 1) * S::kAccCols + c0 + 64 * b, y);
                    tmem_load32(lane_addr + (acc & 1) * S::kAccCols + c0 + 64 * b + 32, y + 32);
                }
#pragma unroll
                for (int i = 0; i < 64; ++i) y[i] = __fmul_rn(mul, y[i]);
                if (gram) {
#pragma unroll
                    for (int i = 0; i < 64; ++i)
                        if (r == col + i) y[i] = __fsub_rn(y[i], step.shift);
                } else {
                    ok = __all_sync(~0u, muon_wait(loaded + 8 * warp, loads & 1, limit, &stop));
                    ++loads;
                    if (!ok) break;
#pragma unroll
                    for (uint32_t c = 0; c < 8; ++c) {
                        float x[8], l[8];
                        Elem<__half>::widen(lds16(block + muon_swizzle(lane, c)), x);
                        if (low) {
                            Elem<__half>::widen(lds16(block + kMuonBlock + muon_swizzle(lane, c)), l);
#pragma unroll
                            for (int i = 0; i < 8; ++i) x[i] = __fadd_rn(x[i], l[i]);
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[8 * c + i] = __fmaf_rn(lin, x[i], y[8 * c + i]);
                    }
                }
                if (!last) {
#pragma unroll
                    for (uint32_t c = 0; c < 8; ++c) {
                        __half hi[8], lo[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) muon_split(y[8 * c + i], hi[i], lo[i]);
                        sts16(block + muon_swizzle(lane, c), *reinterpret_cast<uint4*>(hi));
                        if (low) sts16(block + kMuonBlock + muon_swizzle(lane, c), *reinterpret_cast<uint4*>(lo));
                    }
                    // mirrored: 64 rows of 32 entries, into the half that HALF leaves free
                    auto turn = [&](uint32_t to, bool high) {
#pragma unroll
                        for (int i = 0; i < 64; ++i) {
                            __half hi, lo;
                            muon_split(y[i], hi, lo);
                            asm volatile("st.shared.b16 [%0], %1;" ::"r"(to + i * 64 + 2 * lane),
                                         "h"(__half_as_ushort(high ? hi : lo)) : "memory");
                        }
                    };
                    if (!SPLIT && mirror) turn(block + kMuonBlock, true);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d(out_map, (int)col, (int)row0, block);
                        if (low) tma_store_2d(out_map + 128, (int)col, (int)row0, block + kMuonBlock);
                        if (!SPLIT && mirror) tma_store_2d(mir_map, (int)row0, (int)col, block + kMuonBlock);
                        bulk_commit();
                    }
                    if (SPLIT && mirror) {
                        if (lane == 0) bulk_wait_read0();
                        __syncwarp();
                        turn(block, true);
                        turn(block + kMuonBlock, false);
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            tma_store_2d(mir_map, (int)row0, (int)col, block);
                            tma_store_2d(mir_map + 128, (int)row0, (int)col, block + kMuonBlock);
                            bulk_commit();
                        }
                    }
                } else if (mat.tall) {                                 // the caller's rows run along the lanes
#pragma unroll
                    for (int i = 0; i < 64; ++i)
                        if (r < mat.m && col + i < width)
                            muon_write_last(P, mat, mat.offset + (uint64_t)(col + i) * mat.stride + r, y[i], sound);
                } else {                                               // turned in the buffer, rotated by the row
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 64; ++i)
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(block + lane * 256 + ((i + lane) & 63) * 4), "f"(y[i])
                                     : "memory");
                    __syncwarp();
                    for (uint32_t i = 0; i < 32 && row0 + i < mat.m; ++i)
#pragma unroll
                        for (uint32_t g = 0; g < 64; g += 32)
                            if (col + g + lane < width) {
                                float o;
                                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(o) : "r"(block + i * 256 + ((g + lane + i) & 63) * 4));
                                muon_write_last(P, mat, mat.offset + (uint64_t)(row0 + i) * mat.stride + col + g + lane, o, sound);
                            }
                    fence_proxy_async_smem();                          // the next block comes by TMA
                    __syncwarp();
                }
            }
            if (!ok) break;
            if (!SPLIT) {
                tcgen05_before_sync();
                __syncwarp();
                if (lane == 0) {
                    if (CG == 1) mbar_arrive(acc_empty + 8 * (acc & 1));
                    else leader_arrive(leader_addr(acc_empty + 8 * (acc & 1)));
                }
                ++acc;
            }
            if (lane == 0) {
                bulk_wait_all();                                       // written, not only read
                asm volatile("red.release.gpu.global.add.u64 [%0], %1;" ::"l"(P.done + task.tile.mat), "l"(1ull) : "memory");
            }
            __syncwarp();
        }
        if (lane == 0) {
            bulk_wait_all();
            if (stop)                                                  // a block may still be on its way
                for (uint32_t i = 0; i < 1u << 12 && !mbar_try_wait(loaded + 8 * warp, loads & 1); ++i) {}
        }
    }
    __syncwarp();
    tcgen05_before_sync();
    __syncthreads();
    if (CG == 2) pair_sync();
    tcgen05_after_sync();
    if (tid == 0 && stop) atomicOr(P.status, kStatusTimeout);
    if (warp == S::kEpiWarps + 1) tmem_free<CG>(tmem, S::kTmemCols);
}

}  // namespace ecq
