// C ABI of the Newton-Schulz orthogonaliser: plan, tables, launches.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <mutex>
#include <new>
#include <vector>

#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/ecq.h"
#include "ecq_host.h"
#include "ecq_muon.cuh"

using namespace ecq;

namespace {

struct Step { float a, b, c, shift; };

// Tile shapes of the product kernel: CTAs per tile and columns (rows are 128 a CTA).
struct Shape { uint32_t cg, tn; };
constexpr Shape kShapes[] = {{2, 256}, {2, 128}, {1, 128}, {1, 64}};
constexpr int kShapeCount = 4;

// With 11-bit operands a sum along K stays in one accumulator, whose rounding errors grow with its length:
// 64 rows, by columns, error of the result with 11 and with 22 bits (sums of 256 terms):
//     65536 1.2e-3 2.3e-6   262144 1.9e-3 2.2e-6   1048576 4.9e-3 2.2e-6   4194304 2.2e-2 2.2e-6
// Plans with longer matrices than this take 22 bits for all: at 262144 columns, 64 rows 5.6 -> 6.1 ms, 1024 rows
// 6.2 -> 11.6 ms.
constexpr uint32_t kHalfLongest = 262144;

uint64_t round64(uint64_t x) { return (x + 63) / 64 * 64; }

}  // namespace

struct ecq_muon {
    int device, sms;
    int precision;
    int tiles;                           // ECQ_MUON_TILES_*
    uint32_t wait_limit;
    std::vector<Step> steps;
    std::vector<MuonMat> mats;
    uint64_t x_tiles, m_tiles;           // tiles of one X buffer, of one m x m buffer
    // device tables, one allocation
    unsigned char* block;
    MuonMat* d_mats;
    MuonSpan* d_spans;
    MuonTile* d_prep;
    unsigned char* d_tasks[kShapeCount]; // products and tiles by tile shape, each an allocation, NULL until needed
    double* d_partial;
    unsigned long long *d_done, *d_next, *d_factor;
    uint32_t *d_added, *d_prep_next, *d_sound, *d_status, *h_status;
    CUtensorMap rows128, rows64;         // of the bound workspace
    uint32_t n_spans, n_prep, n_tasks[kShapeCount], tasks_at[kShapeCount];
    uint64_t n_full[kShapeCount];        // tiles of one product with X, over all matrices
    uint64_t n_sym;                      // tiles of 128 x 64 of one symmetric product
    uint64_t k_steps, chain;             // steps of 64 along K of every product, and products, over all matrices
    uint64_t padded[2];                  // entries of all X with rows in whole 128s, in whole 256s
    unsigned char* workspace;            // the caller's, NULL until bound
    uint64_t reset_bytes;                // from d_added on: what a call's first launches count in
    bool unfinished;                     // the last call could not launch all of its kernels
    bool long_sums;                      // a matrix has more than kHalfLongest columns
};

namespace {

// Map of `tiles` tiles as pieces of 16 times eight rows of 16 bytes, loaded in boxes of eight pieces
// of `units` times eight rows.
bool tensor_map(CUtensorMap* tm, void* base, uint64_t tiles, uint32_t units) {
    typedef CUresult (*Fn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                           const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                           CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static Fn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<Fn>(p);
    });
    if (!fn) return false;
    const cuuint64_t dims[3] = {64, 16, 8 * tiles}, strides[2] = {128, kMuonPiece};
    const cuuint32_t box[3] = {64, units, 8}, unit[3] = {1, 1, 1};
    return fn(tm, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, base, dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

uint64_t workspace_tiles(const ecq_muon* p) { return 4 * p->x_tiles + 2 * kMuonSquare * p->m_tiles; }

MuonWork work_of(const ecq_muon* p) {
    MuonWork w;
    uint32_t at = 0;
    w.base = p->workspace;
    for (auto& copy : w.x)
        for (uint32_t& half : copy) { half = at; at += (uint32_t)p->x_tiles; }
    for (auto& square : w.m)
        for (uint32_t& half : square) { half = at; at += (uint32_t)p->m_tiles; }
    return w;
}

// Singular values start in (0, 1]; the scaled fp16 copies hold iterates up to 8 and polynomials
// b s^2 + c s^4 up to 128.
bool steps_in_range(const std::vector<Step>& steps) {
    for (int i = 0; i <= 4096; ++i) {
        double s = i / 4096.0;
        for (const Step& k : steps) {
            const double g = s * s;
            if (!(std::fabs(k.b * g) + std::fabs(k.c * g * g) <= 128.0)) return false;
            s = std::fabs(s * (k.a + k.b * g + k.c * g * g));
            if (!(s <= 8.0)) return false;
        }
    }
    return true;
}

// The last two steps work with D = G - I where that keeps what is stored small: its polynomial
// (b + 2c) D + c D^2 is b G + c G^2 less (b + c) I, which is near zero for singular values near 1, and
// -(b + c) I for those near 0.  Iterates that stay far below 1 get the larger numbers from it: rounding
// errors that then cancel against a X, or numbers out of fp16's range.  So it is done where the
// polynomial reaches no more than twice what b G + c G^2 does (0.98 times with the default
// coefficients; 1 for coefficients that converge to 1), and 128.
void choose_shifts(std::vector<Step>& steps) {
    if (steps.size() <= 2) return;
    for (size_t k = steps.size() - 2; k < steps.size(); ++k) {
        double plain = 0.0, shifted = 0.0;
        for (int i = 0; i <= 4096; ++i) {
            double s = i / 4096.0;
            for (size_t j = 0; j < k; ++j) {
                const double g = s * s;
                s = std::fabs(s * (steps[j].a + steps[j].b * g + steps[j].c * g * g));
            }
            const double b = steps[k].b, c = steps[k].c, g = s * s, d = g - 1.0;
            plain = std::max(plain, std::fabs(b * g + c * g * g));
            shifted = std::max(shifted, std::fabs((b + 2 * c) * d + c * d * d));
        }
        steps[k].shift = shifted <= 2 * plain && shifted <= 128.0 ? 1.f : 0.f;
    }
}

// First steps of an iteration that may be merged: at most three, not among the last two, and only
// while the polynomials stay in the range of their fp16 copies (R up to 200; G, B, S as in single
// steps).
uint32_t mergeable(const std::vector<Step>& steps) {
    uint32_t k = steps.size() > 2 ? std::min<uint32_t>(3, (uint32_t)steps.size() - 2) : 1;
    for (; k > 1; --k) {
        bool ok = true;
        for (int i = 0; i <= 4096 && ok; ++i) {
            double g = (i / 4096.0) * (i / 4096.0), alpha = 1.0, whole = 1.0;
            for (uint32_t j = 0; j < k && ok; ++j) {
                const double p = steps[j].a + steps[j].b * g + steps[j].c * g * g;
                alpha *= steps[j].a;
                whole *= p;
                ok = std::fabs(whole - alpha) <= 200.0 && std::fabs(p * g) <= 128.0;
                g *= p * p;
            }
        }
        if (ok) return k;
    }
    return 1;
}

// Products of one matrix in their order.  m x m buffers: 0 G, 1 and 2 B, 3 S, 4 R; the last R of
// merged steps goes to S's place.
std::vector<MuonProduct> program(const std::vector<Step>& steps, uint32_t merge) {
    constexpr uint8_t none = 255;
    const float sx = kMuonScaleX, sg = kMuonScaleG;
    const int in_low = kMuonReadLow, out_low = kMuonWriteLow, both = in_low | out_low;
    const uint32_t n = (uint32_t)steps.size();
    std::vector<MuonProduct> out;
    auto put = [&](int kind, int left, int right, int to, int in, int in2, float lin, float lin2, float acc, float shift,
                   int flags) {
        out.push_back({lin, lin2, acc, shift, (uint8_t)kind, (uint8_t)left, (uint8_t)right, (uint8_t)to, (uint8_t)in,
                       (uint8_t)in2, (uint8_t)flags, (uint8_t)0});
        out.back().after = (uint8_t)(out.size() - 1);
    };
    uint32_t copy = 0;
    for (uint32_t k = 0; k < n;) {
        // X has a low half while small singular values are still to be amplified: an error made in
        // the last two steps is not
        const uint32_t end = k == 0 ? merge : k + 1;
        const float unscale = end == n ? 1.f / sx : 1.f;
        const int x_flags = (k + 2 < n ? in_low : 0) | (end == n ? kMuonLast : end + 2 < n ? out_low : 0);
        if (end == k + 1) {
            // b G + c G^2 with G = D + t I, of D as the operands have it: their rounding errors
            // cancel in part
            const Step& s = steps[k];
            const float t = s.shift;
            put(kMuonGram, copy, copy, 0, none, none, 0.f, 0.f, sg / (sx * sx), sg * t, 0);
            put(kMuonSym, 0, 0, 1, 0, none, s.b + 2 * s.c * t, 0.f, s.c / sg, 0.f, 0);
            put(kMuonApply, 1, copy, copy ^ 1, 0, none, (s.a + s.b * t + s.c * t * t) * unscale, 0.f, unscale / sg, 0.f, x_flags);
        } else {
            float alpha = steps[0].a;
            int r = 1, b = 1;                                          // the first R is the first B
            put(kMuonGram, copy, copy, 0, none, none, 0.f, 0.f, sg / (sx * sx), 0.f, out_low);
            put(kMuonSym, 0, 0, 1, 0, none, steps[0].b, 0.f, steps[0].c / sg, 0.f, in_low);
            for (uint32_t j = 1; j < end; ++j) {
                const Step &before = steps[j - 1], &s = steps[j];
                put(kMuonSym, b, 0, 3, 0, none, before.a, 0.f, 1.f / sg, 0.f, both);
                if (j == 2) {
                    // R of the step before last is formed beside S: it needs no more than B
                    put(kMuonSym, 2, 1, 4, 1, 2, steps[1].a, alpha, 1.f / sg, 0.f, 0);
                    out.back().after -= 1;
                    alpha *= steps[1].a;
                    r = 4;
                }
                put(kMuonSym, b, 3, 0, 3, none, before.a, 0.f, 1.f / sg, 0.f, both);
                b = j == 1 ? 2 : 1;
                put(kMuonSym, 0, 0, b, 0, none, s.b, 0.f, s.c / sg, 0.f, in_low);
            }
            const Step& s = steps[end - 1];
            put(kMuonSym, b, r, 3, r, b, s.a, alpha, 1.f / sg, 0.f, 0);
            alpha *= s.a;
            put(kMuonApply, 3, copy, copy ^ 1, 0, none, alpha * unscale, 0.f, unscale / sg, 0.f, x_flags);
        }
        copy ^= 1;
        k = end;
    }
    return out;
}

// Entries of the matrices that are worked on together.  Three such groups are under way at a time,
// each with 8 bytes an entry of X, of which about half is alive: they about fill the L2 cache.  Smaller
// groups leave SMs without a tile, larger ones make no difference.  In ms with groups of 3, 6, 12, 24 and
// 48 M entries, layers of (w, 4w), (4w, w) and four (w, w) to a bf16 update:
//     w 640, 20 layers   2.38 2.02 2.05 2.06 2.07     w 1024, 12   4.60 3.62 3.20 3.20 3.21
//     w 1280, 8          4.80 4.10 3.80 3.75 3.85     w 2048, 4    6.4  6.2  6.3  6.2  6.1
constexpr uint64_t kGroupEntries = 12ull << 20;
constexpr uint64_t kLanes = 3;

// Tiles of all products in the order in which they are handed out.  Matrices are taken in groups, and
// kLanes groups at a time go through their products one by one in turn: between a group's product
// and the next one, which waits for all of it, there is the other groups' work.
struct TaskList {
    const std::vector<MuonMat>& mats;
    Shape shape;
    std::vector<MuonProduct> products;   // the single-step program, then the merged one
    uint32_t count[2];                   // products of either
    std::vector<MuonTask> tasks;
    std::vector<uint64_t> sym, full;     // tiles per product, by matrix

    TaskList(const std::vector<MuonMat>& all, Shape s, const std::vector<Step>& steps)
        : mats(all), shape(s), sym(all.size()), full(all.size()) {
        products = program(steps, 1);
        const std::vector<MuonProduct> merged = program(steps, mergeable(steps));
        count[0] = (uint32_t)products.size();
        count[1] = (uint32_t)merged.size();
        products.insert(products.end(), merged.begin(), merged.end());
        for (size_t i = 0; i < mats.size(); ++i) {
            const uint32_t tm = shape.cg * 128, rb = (mats[i].m + tm - 1) / tm;
            for (uint32_t r = 0; r < rb; ++r) sym[i] += sym_columns(mats[i], r);
            full[i] = (uint64_t)rb * ((mats[i].n + shape.tn - 1) / shape.tn);
        }
    }
    // Merging three steps saves two products X X^T and two with X, 6 m^2 n, and costs 6 m^3; with
    // tiles that reach over the diagonal, 6.5 against 7.5.  Singular values near 1 lose a factor
    // alpha (41) in alpha X + R X: small matrices, whose singular values are all large in X_0,
    // take single steps (error of 96 x 160: 7e-4, merged 1.4e-3).
    bool merged(uint32_t i) const { return 5ull * mats[i].n >= 6ull * mats[i].m && mats[i].m >= 256; }
    uint64_t tiles(uint32_t i, const MuonProduct& p) const { return p.kind == kMuonApply ? full[i] : sym[i]; }
    uint64_t all_tiles(uint32_t i) const {
        uint64_t n = 0;
        const uint32_t from = merged(i) ? count[0] : 0;
        for (uint32_t k = 0; k < count[merged(i)]; ++k) n += tiles(i, products[from + k]);
        return n;
    }
    // tiles of row block r that touch the lower triangle
    uint32_t sym_columns(const MuonMat& mat, uint32_t r) const {
        return (std::min(mat.m, (r + 1) * shape.cg * 128) + shape.tn - 1) / shape.tn;
    }
    void add(uint32_t i, uint32_t at) {
        const MuonMat& mat = mats[i];
        const uint32_t from = merged(i) ? count[0] : 0;
        if (at >= count[merged(i)]) return;
        const MuonProduct& p = products[from + at];
        const uint32_t tm = shape.cg * 128, rb = (mat.m + tm - 1) / tm;
        uint64_t need = 0;
        for (uint32_t k = 0; k < p.after; ++k) need += tiles(i, products[from + k]);
        for (uint32_t r = 0; r < rb; ++r) {
            const uint32_t cb = p.kind == kMuonApply ? (mat.n + shape.tn - 1) / shape.tn : sym_columns(mat, r);
            for (uint32_t c = 0; c < cb; ++c)
                tasks.push_back({i, (uint16_t)r, (uint16_t)c, (uint16_t)(from + at),
                                 (uint16_t)(p.kind != kMuonApply && c * shape.tn / tm < r), (uint32_t)need});
        }
    }
    void measure(uint64_t& n_sym, uint64_t& k_steps, uint64_t& chain) const {
        n_sym = k_steps = chain = 0;
        for (uint32_t i = 0; i < mats.size(); ++i) {
            const uint32_t from = merged(i) ? count[0] : 0;
            n_sym += sym[i];
            chain += count[merged(i)];
            for (uint32_t k = 0; k < count[merged(i)]; ++k)
                k_steps += ((products[from + k].kind == kMuonGram ? mats[i].n : mats[i].m) + 63) / 64;
        }
    }
    void build() {
        std::vector<std::pair<uint32_t, uint32_t>> groups;
        uint64_t all = 0, held = 0;
        for (const MuonMat& mat : mats) all += (uint64_t)mat.m * mat.n;
        const uint64_t most = std::min<uint64_t>(kGroupEntries, (all + kLanes - 1) / kLanes);
        uint32_t from = 0;
        for (uint32_t i = 0; i < mats.size(); ++i) {
            held += (uint64_t)mats[i].m * mats[i].n;
            if (held >= most || i + 1 == mats.size()) {
                groups.push_back({from, i + 1});
                from = i + 1;
                held = 0;
            }
        }
        // lane l takes the groups l, l + kLanes, ...; in every turn each lane has one product, and lane
        // l starts l turns later
        const uint64_t length = std::max(count[0], count[1]);
        const uint64_t turns = (groups.size() + kLanes - 1) / kLanes * length + kLanes;
        for (uint64_t turn = 0; turn < turns; ++turn)
            for (uint64_t lane = 0; lane < kLanes && lane <= turn; ++lane) {
                const uint64_t at = turn - lane, g = at / length * kLanes + lane;
                if (g >= groups.size()) continue;
                for (uint32_t i = groups[g].first; i < groups[g].second; ++i) add(i, (uint32_t)(at % length));
            }
    }
};

template <int CG, int TN, bool SPLIT, bool KS>
cudaLaunchConfig_t iterate_config(cudaLaunchAttribute (&at)[2]) {
    constexpr uint32_t kCluster = KS ? 2 : CG;
    using S = MuonShape<CG, TN, SPLIT, KS>;
    cudaLaunchConfig_t cfg = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = kCluster;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.attrs = at;
    cfg.numAttrs = kCluster > 1 ? 2 : 1;
    return cfg;
}

// Clusters of the kernel that the plan's device holds at a time, with the kernel's attributes set; 0
// where one of the queries fails, which the next call asks again.
template <int CG, int TN, bool SPLIT, bool KS>
uint32_t iterate_clusters(const ecq_muon* p) {
    constexpr int kCluster = KS ? 2 : CG;
    static std::atomic<uint32_t> known[kMaxDevices];
    uint32_t have = known[p->device].load(std::memory_order_acquire);
    if (have) return have;
    auto kern = muon_iterate_kernel<CG, TN, SPLIT, KS>;
    cudaLaunchAttribute at[2] = {};
    cudaLaunchConfig_t cfg = iterate_config<CG, TN, SPLIT, KS>(at);
    cfg.gridDim = dim3(p->sms / kCluster * kCluster);
    int n = p->sms;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg.dynamicSmemBytes) != cudaSuccess ||
        (kCluster > 1 && cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess)) {
        cudaGetLastError();
        return 0;
    }
    have = (uint32_t)std::max(0, std::min(n, p->sms / kCluster));
    known[p->device].store(have, std::memory_order_release);
    return have;
}

template <int CG, int TN, bool SPLIT, bool KS>
int launch_iterate(const ecq_muon* p, const MuonIterate& it, uint64_t clusters, cudaStream_t st) {
    cudaLaunchAttribute at[2] = {};
    cudaLaunchConfig_t cfg = iterate_config<CG, TN, SPLIT, KS>(at);
    cfg.gridDim = dim3((uint32_t)clusters * (KS ? 2 : CG));
    cfg.stream = st;
    if (cudaLaunchKernelEx(&cfg, muon_iterate_kernel<CG, TN, SPLIT, KS>, it) != cudaSuccess) {
        cudaGetLastError();
        return ECQ_ERR_CUDA;
    }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return ECQ_OK;
}

struct IterateKernel {
    uint32_t (*clusters)(const ecq_muon*);
    int (*launch)(const ecq_muon*, const MuonIterate&, uint64_t, cudaStream_t);
};
template <int CG, int TN, bool SPLIT, bool KS = false>
IterateKernel iterate_kernel() { return {iterate_clusters<CG, TN, SPLIT, KS>, launch_iterate<CG, TN, SPLIT, KS>}; }

// The launches may be scheduled while what is ahead of them in the stream drains; they touch no
// global memory before it has completed.
template <typename T, bool MOM>
int launch_prepare(const ecq_muon* p, MuonPrepare pre, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.blockDim = dim3(kMuonPrepThreads);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const bool both = p->n_spans + p->n_prep <= 5u * (uint32_t)p->sms;
    for (pre.what = both ? 2 : 0; pre.what < 3; ++pre.what) {
        cfg.gridDim = dim3(both ? p->n_spans + p->n_prep : pre.what ? p->n_prep : p->n_spans);
        if (cudaLaunchKernelEx(&cfg, muon_prepare_kernel<T, MOM>, pre) != cudaSuccess) {
            cudaGetLastError();
            return ECQ_ERR_CUDA;
        }
        g_launches.fetch_add(1, std::memory_order_relaxed);
        if (pre.what == 1) break;
    }
    return ECQ_OK;
}

// Tiles of a call: the plan's choice, or the largest of which there are enough for every SM.  Pairs
// take 256 rows at a time, which has to fill.  In us with 256 x 256, 128 x 128 and 128 x 64, 11 bits, and
// with 256 x 128 and 128 x 64, 22 bits, by the rows that pairs compute for one of 128-row tiles:
//     2.00  48 of 128 x 512    160 116 102 | 195 131     1.14  6 of 896 x 1792    351 296 396 | 554 589
//     1.33  60 of 384 x 384    357 255 368 | 540 439     1.11  4 of 1152 x 2304   401 361 527 | 665 771
//     1.20  3 of 1537 x 611    288 214 188 | 311 266     1.09  4 of 1408 x 1408   372 380 603 | 730 929
//     1.20  30 of 640 x 640    419 366 603 | 816 798     1.00  2048 x 2048        327 306 478 | 505 787
// With 22 bits the crossing is the rule's; with 11 bits it lies lower, at 1.10 (the rule costs the 1.14 and
// 1.11 lines 50 and 40 us).  Too few tiles for the SMs: one 1024 x 1024 takes 222, 165 and 148 us, 263 and
// 194 with 22 bits; three of them 256, 196 and 216, and 308 and 335.
int choose_tiles(const ecq_muon* p, bool split) {
    if (p->tiles != ECQ_MUON_TILES_AUTO) return p->tiles;
    if (p->n_full[split ? 1 : 0] * 2 >= (uint64_t)p->sms && 100 * p->padded[1] <= 115 * p->padded[0]) return ECQ_MUON_TILES_256X256;
    if (!split && p->n_full[2] >= (uint64_t)p->sms) return ECQ_MUON_TILES_128X128;
    return ECQ_MUON_TILES_128X64;
}

// Whether two CTAs share the K of a tile of 128 x 64: where the symmetric products have no more tiles
// than there are pairs, and the products are long enough, counted in steps of 64 along K.  In us, one
// CTA a tile and two (22-bit operands: three times the work a step):
//     22 bits  96 x 160  (2.3 steps) 90 97     1024 x 1024 (16) 228 193   1000 x 2048 (20) 301 250
//              2497 x 85 (15) 186 136          1537 x 611 (13) 217 181, three of them (90 tiles) 264 284
//     11 bits  64 x 1024 (6) 82 94   512 x 2048 (12) 144 147   128 x 4096 (23) 150 120
//              1024 x 1024 (16, but 128 tiles in every third product) 148 155
bool share_along_k(const ecq_muon* p, bool split) {
    return p->n_sym * 2 <= (uint64_t)p->sms && (split || p->n_full[3] * 2 <= (uint64_t)p->sms) &&
           p->k_steps >= (split ? 5u : 16u) * p->chain;
}

// Index in kShapes of a tile choice.
int shape_of(int tiles, bool split) {
    if (split) return tiles == ECQ_MUON_TILES_256X256 ? 1 : 3;
    return tiles == ECQ_MUON_TILES_256X256 ? 0 : tiles == ECQ_MUON_TILES_128X128 ? 2 : 3;
}

IterateKernel choose_kernel(const ecq_muon* p, int shape, bool split) {
    const bool joint = shape == 3 && share_along_k(p, split);
    if (split) {
        if (shape == 1) return iterate_kernel<2, 128, true>();
        return joint ? iterate_kernel<1, 64, true, true>() : iterate_kernel<1, 64, true>();
    }
    if (shape == 0) return iterate_kernel<2, 256, false>();
    if (shape == 2) return iterate_kernel<1, 128, false>();
    return joint ? iterate_kernel<1, 64, false, true>() : iterate_kernel<1, 64, false>();
}

int iterate(ecq_muon* p, const MuonIn& in, int in_dtype, const MuonOut& out, int out_dtype, cudaStream_t st) {
    const MuonWork ws = work_of(p);
    const bool split = p->precision == ECQ_MUON_SPLIT || p->long_sums ||
                       (p->precision == ECQ_MUON_AUTO && (out.params || out_dtype != ECQ_BF16));
    const int shape = shape_of(choose_tiles(p, split), split);
    // what can fail does so before the momentum is touched
    const IterateKernel kernel = choose_kernel(p, shape, split);
    const uint32_t clusters = kernel.clusters(p);
    if (!clusters) return ECQ_ERR_CUDA;
    if (!p->d_tasks[shape]) return ECQ_ERR_ARG;

    // The first launches count in these, the last one sets them to zero again.  Where a call could not
    // launch all of its kernels, the next one does.
    if (p->unfinished && cudaMemsetAsync(p->d_added, 0, p->reset_bytes, st) != cudaSuccess) {
        cudaGetLastError();
        return ECQ_ERR_CUDA;
    }
    p->unfinished = true;
    const MuonPrepare pre = {p->d_spans, p->d_prep, p->d_mats, in, ws, p->d_partial, p->d_added, p->d_factor, p->d_prep_next,
                             p->d_sound, p->d_done, p->d_next, p->d_status, p->n_spans, p->wait_limit, 0};
    int rc = in.momentum              ? launch_prepare<float, true>(p, pre, st)
             : in_dtype == ECQ_F32    ? launch_prepare<float, false>(p, pre, st)
             : in_dtype == ECQ_BF16   ? launch_prepare<__nv_bfloat16, false>(p, pre, st)
                                      : launch_prepare<__half, false>(p, pre, st);
    if (rc != ECQ_OK) return rc;

    MuonIterate m = {};
    m.mats = p->d_mats;
    m.products = reinterpret_cast<const MuonProduct*>(p->d_tasks[shape]);
    m.tasks = reinterpret_cast<const MuonTask*>(p->d_tasks[shape] + p->tasks_at[shape]);
    m.n_tasks = p->n_tasks[shape];
    m.rows128 = p->rows128;
    m.rows64 = p->rows64;
    m.sound = p->d_sound;
    m.ws = ws;
    m.done = p->d_done;
    m.next = p->d_next;
    m.added = p->d_added;
    m.factor = p->d_factor;
    m.prepare_next = p->d_prep_next;
    m.n_mats = (uint32_t)p->mats.size();
    m.status = p->d_status;
    m.out = out;
    m.out_dtype = out_dtype;
    m.wait_limit = p->wait_limit;
    rc = kernel.launch(p, m, std::min<uint64_t>(p->n_full[shape], clusters), st);
    if (rc == ECQ_OK) p->unfinished = false;
    return rc;
}

bool finite(float x) { return x - x == 0.f; }

// Whether the plan's device is the current one: its addresses and the stream are that one's.
bool on_device(const ecq_muon* p) {
    int dev = 0;
    return cudaGetDevice(&dev) == cudaSuccess && dev == p->device;
}

// The tile lists that the plan's precision and tile choice need and that it does not have yet.
int build_tasks(ecq_muon* p) {
    for (int split = 0; split < 2; ++split) {
        if (p->long_sums ? !split : p->precision == (split ? ECQ_MUON_HALF : ECQ_MUON_SPLIT)) continue;
        const int shape = shape_of(choose_tiles(p, split), split);
        if (p->d_tasks[shape]) continue;
        TaskList list(p->mats, kShapes[shape], p->steps);
        uint64_t all = 0;
        for (uint32_t i = 0; i < p->mats.size(); ++i) all += list.all_tiles(i);
        if (all > 0x10000000ull) return ECQ_ERR_ARG;
        list.tasks.reserve(all);
        list.build();
        if (shape == 3) list.measure(p->n_sym, p->k_steps, p->chain);
        const uint64_t products = (list.products.size() * sizeof(MuonProduct) + 255) / 256 * 256;
        unsigned char* to = nullptr;
        if (cudaMalloc(&to, products + list.tasks.size() * sizeof(MuonTask)) != cudaSuccess) {
            cudaGetLastError();
            return ECQ_ERR_ALLOC;
        }
        if (cudaMemcpy(to, list.products.data(), list.products.size() * sizeof(MuonProduct), cudaMemcpyHostToDevice) != cudaSuccess ||
            cudaMemcpy(to + products, list.tasks.data(), list.tasks.size() * sizeof(MuonTask), cudaMemcpyHostToDevice) != cudaSuccess) {
            cudaFree(to);
            return ECQ_ERR_CUDA;
        }
        p->d_tasks[shape] = to;
        p->tasks_at[shape] = (uint32_t)products;
        p->n_tasks[shape] = (uint32_t)list.tasks.size();
    }
    return ECQ_OK;
}

int create(ecq_muon* p, uint32_t count, const uint64_t* offsets, const uint32_t* rows, const uint32_t* cols,
           const uint64_t* strides, const float* scales, uint32_t steps, const float* coefficients) {
    for (uint32_t k = 0; k < steps; ++k) {
        Step s = {3.4445f, -4.7750f, 2.0315f, 0.f};
        if (coefficients) s = {coefficients[3 * k], coefficients[3 * k + 1], coefficients[3 * k + 2], 0.f};
        if (!finite(s.a) || !finite(s.b) || !finite(s.c)) return ECQ_ERR_ARG;
        p->steps.push_back(s);
    }
    if (!steps_in_range(p->steps)) return ECQ_ERR_ARG;
    choose_shifts(p->steps);
    std::vector<MuonSpan> spans;
    std::vector<MuonTile> prep;
    for (uint32_t i = 0; i < count; ++i) {
        MuonMat mat = {};
        mat.offset = offsets[i];
        mat.rows = rows[i]; mat.cols = cols[i];
        mat.stride = strides ? strides[i] : cols[i];
        if (!mat.rows || !mat.cols || mat.rows > ECQ_MUON_MAX_SIDE || mat.cols > ECQ_MUON_MAX_SIDE ||
            std::min(mat.rows, mat.cols) > ECQ_MUON_MAX_RANK || mat.stride < mat.cols || mat.stride > (1ull << 40) ||
            mat.offset > (1ull << 48))
            return ECQ_ERR_ARG;
        mat.tall = mat.rows > mat.cols;
        mat.m = std::min(mat.rows, mat.cols); mat.n = std::max(mat.rows, mat.cols);
        p->long_sums |= mat.n > kHalfLongest;
        mat.pad = (uint32_t)round64(mat.m);
        mat.down = (mat.m + 127) / 128;
        mat.scale = scales ? scales[i] : 1.f;
        if (!finite(mat.scale)) return ECQ_ERR_ARG;
        mat.x_tile = (uint32_t)p->x_tiles; mat.m_tile = (uint32_t)p->m_tiles;
        p->x_tiles += round64(mat.n) / 64 * mat.down;
        p->padded[0] += (uint64_t)(mat.m + 127) / 128 * 128 * mat.n;
        p->padded[1] += (uint64_t)(mat.m + 255) / 256 * 256 * mat.n;
        p->m_tiles += (uint64_t)mat.pad / 64 * mat.down;
        if (workspace_tiles(p) > 0x0FFFFFFFull) return ECQ_ERR_ARG;    // pieces are TMA coordinates
        // spans of about kMuonSpan entries: flat where the rows lie end to end, else whole rows or parts of them
        mat.part0 = (uint32_t)spans.size();
        if (mat.stride == mat.cols) {
            const uint64_t all = (uint64_t)mat.rows * mat.cols;
            for (uint64_t at = 0; at < all; at += kMuonSpan)
                spans.push_back({mat.offset + at, 0, i, 1, (uint32_t)std::min<uint64_t>(kMuonSpan, all - at)});
        } else {
            const uint32_t per = std::max<uint32_t>(1, kMuonSpan / mat.cols);
            for (uint32_t r = 0; r < mat.rows; r += per)
                for (uint32_t c = 0; c < mat.cols; c += kMuonSpan)
                    spans.push_back({mat.offset + (uint64_t)r * mat.stride + c, mat.stride, i, std::min(per, mat.rows - r),
                                     std::min(kMuonSpan, mat.cols - c)});
        }
        mat.parts = (uint32_t)spans.size() - mat.part0;
        for (uint32_t r = 0; r * 64 < mat.rows; ++r)
            for (uint32_t c = 0; c * 64 < mat.cols; ++c) prep.push_back({i, (uint16_t)r, (uint16_t)c});
        p->mats.push_back(mat);
    }
    for (int s = 0; s < kShapeCount; ++s)
        for (const MuonMat& mat : p->mats)
            p->n_full[s] += (uint64_t)((mat.m + kShapes[s].cg * 128 - 1) / (kShapes[s].cg * 128)) *
                            ((mat.n + kShapes[s].tn - 1) / kShapes[s].tn);
    if (spans.size() + prep.size() > 0x7FFFFFFFull) return ECQ_ERR_ARG;

    uint64_t bytes = 0;
    auto place = [&](uint64_t n) { const uint64_t at = bytes; bytes += (n + 255) / 256 * 256; return at; };
    const uint64_t o_mats = place(count * sizeof(MuonMat)), o_spans = place(spans.size() * sizeof(MuonSpan));
    const uint64_t o_prep = place(prep.size() * sizeof(MuonTile));
    const uint64_t o_partial = place(spans.size() * 8), o_sound = place(count * 4ull), o_status = place(4);
    const uint64_t o_done = place(count * 8ull), o_next = place(8);
    const uint64_t o_added = place(count * 4ull), o_prep_next = place(4), o_factor = place(count * 8ull);
    std::vector<unsigned char> host(bytes, 0);
    memcpy(host.data() + o_mats, p->mats.data(), count * sizeof(MuonMat));
    memcpy(host.data() + o_spans, spans.data(), spans.size() * sizeof(MuonSpan));
    memcpy(host.data() + o_prep, prep.data(), prep.size() * sizeof(MuonTile));
    if (cudaGetDevice(&p->device) != cudaSuccess || p->device < 0 || p->device >= kMaxDevices ||
        cudaDeviceGetAttribute(&p->sms, cudaDevAttrMultiProcessorCount, p->device) != cudaSuccess)
        return ECQ_ERR_CUDA;
    if (cudaMalloc(&p->block, bytes) != cudaSuccess || cudaHostAlloc(&p->h_status, 4, cudaHostAllocDefault) != cudaSuccess) {
        cudaGetLastError();
        return ECQ_ERR_ALLOC;
    }
    if (cudaMemcpy(p->block, host.data(), bytes, cudaMemcpyHostToDevice) != cudaSuccess) return ECQ_ERR_CUDA;
    p->d_mats = reinterpret_cast<MuonMat*>(p->block + o_mats);
    p->d_spans = reinterpret_cast<MuonSpan*>(p->block + o_spans);
    p->d_prep = reinterpret_cast<MuonTile*>(p->block + o_prep);
    p->d_added = reinterpret_cast<uint32_t*>(p->block + o_added);
    p->d_factor = reinterpret_cast<unsigned long long*>(p->block + o_factor);
    p->d_prep_next = reinterpret_cast<uint32_t*>(p->block + o_prep_next);
    p->d_partial = reinterpret_cast<double*>(p->block + o_partial);
    p->d_sound = reinterpret_cast<uint32_t*>(p->block + o_sound);
    p->d_status = reinterpret_cast<uint32_t*>(p->block + o_status);
    p->d_done = reinterpret_cast<unsigned long long*>(p->block + o_done);
    p->d_next = reinterpret_cast<unsigned long long*>(p->block + o_next);
    p->reset_bytes = bytes - o_added;
    p->n_spans = (uint32_t)spans.size();
    p->n_prep = (uint32_t)prep.size();
    return build_tasks(p);
}

}  // namespace

extern "C" {

int ecq_muon_create(ecq_muon** out, uint32_t count, const uint64_t* offsets, const uint32_t* rows,
                    const uint32_t* cols, const uint64_t* strides, const float* scales, uint32_t steps,
                    const float* coefficients, int precision) {
    if (!out) return ECQ_ERR_ARG;
    *out = nullptr;
    if (!count || count > ECQ_MUON_MAX_COUNT || !offsets || !rows || !cols || !steps || steps > ECQ_MUON_MAX_STEPS ||
        precision < ECQ_MUON_AUTO || precision > ECQ_MUON_SPLIT)
        return ECQ_ERR_ARG;
    ecq_muon* p = new (std::nothrow) ecq_muon();
    if (!p) return ECQ_ERR_ALLOC;
    p->precision = precision;
    p->wait_limit = ECQ_WAIT_LIMIT_DEFAULT;
    int rc;
    try {
        rc = create(p, count, offsets, rows, cols, strides, scales, steps, coefficients);
    } catch (const std::bad_alloc&) {
        rc = ECQ_ERR_ALLOC;
    }
    if (rc != ECQ_OK) { ecq_muon_destroy(p); return rc; }
    *out = p;
    return ECQ_OK;
}

void ecq_muon_destroy(ecq_muon* p) {
    if (!p) return;
    if (p->block) cudaFree(p->block);
    for (unsigned char* tasks : p->d_tasks)
        if (tasks) cudaFree(tasks);
    if (p->h_status) cudaFreeHost(p->h_status);
    delete p;
}

int ecq_muon_set_tiles(ecq_muon* p, int tiles) {
    if (!p || tiles < ECQ_MUON_TILES_AUTO || tiles > ECQ_MUON_TILES_128X64) return ECQ_ERR_ARG;
    const int before = p->tiles;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaSetDevice(p->device) != cudaSuccess) return ECQ_ERR_CUDA;
    int rc;
    p->tiles = tiles;
    try {
        rc = build_tasks(p);
    } catch (const std::bad_alloc&) {
        rc = ECQ_ERR_ALLOC;
    }
    if (rc != ECQ_OK) p->tiles = before;
    cudaSetDevice(dev);
    return rc;
}

int ecq_muon_set_wait_limit(ecq_muon* p, uint32_t polls) {
    if (!p) return ECQ_ERR_ARG;
    p->wait_limit = polls;
    return ECQ_OK;
}

uint64_t ecq_muon_workspace_bytes(const ecq_muon* p) { return p ? kMuonTileBytes * workspace_tiles(p) : 0; }

int ecq_muon_bind(ecq_muon* p, void* workspace, uint64_t bytes, void* cuda_stream) {
    if (!p || !workspace || !aligned_to(workspace, 256) || bytes < kMuonTileBytes * workspace_tiles(p)) return ECQ_ERR_ARG;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaSetDevice(p->device) != cudaSuccess) return ECQ_ERR_CUDA;
    const bool mapped = tensor_map(&p->rows128, workspace, workspace_tiles(p), 16) &&
                        tensor_map(&p->rows64, workspace, workspace_tiles(p), 8);
    p->workspace = mapped ? static_cast<unsigned char*>(workspace) : nullptr;
    cudaSetDevice(dev);
    return mapped ? ECQ_OK : ECQ_ERR_CUDA;
}

int ecq_muon_orthogonalize(ecq_muon* p, const void* in, int in_dtype, void* out, int out_dtype, void* cuda_stream) {
    if (!p || !p->workspace || !in || !out || !dtype_bytes(in_dtype) || !dtype_bytes(out_dtype) || !aligned_to(in, 16) ||
        !aligned_to(out, 16) || (in == out && in_dtype != out_dtype) || !on_device(p))
        return ECQ_ERR_ARG;
    const MuonIn i = {in, nullptr, 0.f, 0};
    const MuonOut o = {nullptr, out, 1.f, 0.f, 0};
    return iterate(p, i, in_dtype, o, out_dtype, static_cast<cudaStream_t>(cuda_stream));
}

int ecq_muon_step(ecq_muon* p, const float* grad, float* momentum, float mu, int nesterov, float lr, float decay,
                  float* params, void* update, int update_dtype, void* cuda_stream) {
    if (!p || !p->workspace || !grad || !momentum || (!params && !update) || !aligned_to(grad, 16) ||
        !aligned_to(momentum, 16) || !aligned_to(params, 16) || !aligned_to(update, 16) ||
        (update && !dtype_bytes(update_dtype)))
        return ECQ_ERR_ARG;
    if (grad == momentum || (params && (params == grad || params == momentum || params == update)) ||
        update == static_cast<const void*>(grad) || update == momentum)
        return ECQ_ERR_ARG;
    if (!(mu >= 0.f && mu <= 1.f) || !(lr >= 0.f) || !(decay >= 0.f) || !finite(lr) || !finite(decay) ||
        !finite(lr * decay) || (nesterov != 0 && nesterov != 1) || !on_device(p))
        return ECQ_ERR_ARG;
    const MuonIn i = {grad, momentum, mu, nesterov};
    const MuonOut o = {params, update, 1.f - lr * decay, lr, 1};
    return iterate(p, i, ECQ_F32, o, update ? update_dtype : ECQ_F32, static_cast<cudaStream_t>(cuda_stream));
}

int ecq_muon_status(ecq_muon* p, void* cuda_stream) {
    if (!p || !on_device(p)) return ECQ_ERR_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (cudaMemcpyAsync(p->h_status, p->d_status, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaMemsetAsync(p->d_status, 0, 4, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
        return ECQ_ERR_CUDA;
    const uint32_t s = *p->h_status;
    return s & kStatusTimeout ? ECQ_ERR_TIMEOUT : s & kStatusNonFinite ? ECQ_ERR_NONFINITE : ECQ_OK;
}

}  // extern "C"
