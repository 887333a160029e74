// Log probabilities of given tokens from a language model's logits, with the entropy of each row
// and its best alternatives, and the backward pass to the logits.
#pragma once

#include <cfloat>
#include <cstdint>

#include "ecq_common.cuh"
#include "ecq_elem.cuh"

namespace ecq {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// ---- forward ---------------------------------------------------------------------------------
//
// With z_j = tau x_j (tau = 1 / temperature), m = max_j x_j, and in powers of two
// d_j = (x_j - m) tau log2(e), a row needs
//     s = sum_j 2^d_j,  t = sum_j 2^d_j d_j
//     lse = tau m + ln s,  log p_y = tau (x_y - m) - ln s,  H = ln 2 (log2 s - t / s).
// x_j - m is taken before the product with tau: near the maximum the difference is exact, and
// entries masked with the type's lowest value cannot overflow to a 0/0.
//
// One pass over the logits: every thread carries (m, s, t) of the entries it has seen and rescales
// s and t when a batch of its entries raises m; the threads' triples are merged by shuffles,
// through shared memory, and across the CTAs of a cluster when a row is split over one.
//
// The best `top` entries need no second pass over the row: threads are taken in kTokGroups groups,
// and the top-th largest of the groups' maxima is a bound that at least `top` entries reach, all of
// them in the groups whose maximum reaches it.  Only those groups' entries (about top / kTokGroups
// of the row) are read again, out of L2, and the few that reach the bound are ranked by counting.
// Entries are ordered by value, equal ones by index (the lower first); a 64-bit key holds both.

constexpr int kTokThreads = 256;         // of a CTA where rows are few, four of them an SM
constexpr int kTokStream = 128;          // where they are many, eight an SM: while some rank their best
                                         // entries the others keep the memory busy
constexpr int kTokGroups = 128;
constexpr int kTokUnroll = 4;            // 16-byte vectors in flight per thread
constexpr int kTokMaxTop = 32;
constexpr int kTokMaxCluster = 8;
constexpr int kTokCandidates = 1024;

struct TokenForward {
    const void* logits;
    uint64_t row_stride;
    const int64_t* targets;
    float* logprob;
    float* entropy;
    float* lse;
    float* top_logprob;
    int32_t* top_index;
    uint32_t vocab;
    uint32_t top;
    uint32_t cluster_log2;               // CTAs per row, a power of two
    float tau;
};

struct TokenSums { float m, s, t; };

// Sums relative to a larger maximum.  The exponent is held at -1e4 (2^-1e4 is 0) so that the
// initial m, the lowest finite value, and s = t = 0 give 0 and not 0 * inf.
__device__ __forceinline__ void token_rescale(TokenSums& a, float m, float k) {
    const float d = fmaxf(__fmul_rn(__fsub_rn(a.m, m), k), -1e4f);
    const float f = ex2(d);
    a.t = __fmul_rn(__fmaf_rn(a.s, d, a.t), f);
    a.s = __fmul_rn(a.s, f);
    a.m = m;
}

__device__ __forceinline__ void token_merge(TokenSums& a, TokenSums b, float k) {
    const float m = fmaxf(a.m, b.m);
    token_rescale(a, m, k);
    token_rescale(b, m, k);
    a.s = __fadd_rn(a.s, b.s);
    a.t = __fadd_rn(a.t, b.t);
}

// One entry.
template <bool ENT>
__device__ __forceinline__ void token_add(TokenSums& a, float x, float k) {
    if (x > a.m) token_rescale(a, x, k);
    const float d = __fmul_rn(__fsub_rn(x, a.m), k), e = ex2(d);
    a.s = __fadd_rn(a.s, e);
    // a masked entry has d = -inf and e = 0; it adds nothing to t
    if (ENT) a.t = __fmaf_rn(e, fmaxf(d, -1e4f), a.t);
}

// N vectors, two entries an instruction where there is one.
template <typename T, bool ENT, int N>
__device__ __forceinline__ void token_add(TokenSums& a, const uint4* raw, float k) {
    constexpr int E = Elem<T>::kPer16;
    float m = Elem<T>::largest(raw[0]);
#pragma unroll
    for (int u = 1; u < N; ++u) m = fmaxf(m, Elem<T>::largest(raw[u]));
    if (m > a.m) token_rescale(a, m, k);
    const uint64_t m2 = pack2(a.m, a.m), k2 = pack2(k, k);
    uint64_t s2 = 0, t2 = 0;                                          // two zeros
#pragma unroll
    for (int u = 0; u < N; ++u) {
        float x[E];
        Elem<T>::widen(raw[u], x);
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            float d0, d1;
            unpack2(mul2(sub2(pack2(x[i], x[i + 1]), m2), k2), d0, d1);
            const uint64_t e2 = pack2(ex2(d0), ex2(d1));
            s2 = add2(s2, e2);
            if (ENT) t2 = fma2(e2, pack2(fmaxf(d0, -1e4f), fmaxf(d1, -1e4f)), t2);
        }
    }
    float u, v;
    unpack2(s2, u, v);
    a.s = __fadd_rn(a.s, __fadd_rn(u, v));
    if (ENT) {
        unpack2(t2, u, v);
        a.t = __fadd_rn(a.t, __fadd_rn(u, v));
    }
}

// Larger keys are better: value first, then the lower index.  0 is below every entry's key.
__device__ __forceinline__ uint64_t token_key(float x, uint32_t index) {
    const uint32_t b = __float_as_uint(__fadd_rn(x, 0.f));                 // -0 and 0 are equal
    const uint32_t o = b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
    return ((uint64_t)o << 32) | (uint32_t)~index;
}
__device__ __forceinline__ float token_key_value(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ uint32_t token_key_index(uint64_t key) { return ~(uint32_t)key; }

// The part of a row that one CTA has: vectors [v0, v1) of the row's 16-byte aligned body, and
// the single entries before or behind the body where this CTA is the first or the last.
template <typename T>
struct TokenSpan {
    const T* row;
    uint32_t head, nv, vocab;            // entries before the body, vectors of the body
    uint32_t v0, v1;
    bool first, last;

    __device__ __forceinline__ uint32_t edge_index(uint32_t i, bool& have) const {
        // i-th of the up to 2 * (16 / sizeof(T) - 1) single entries
        constexpr uint32_t E = Elem<T>::kPer16;
        if (i < E) { have = first && i < head; return i; }
        const uint32_t j = head + nv * E + (i - E);
        have = last && j < vocab;
        return j;
    }
    __device__ __forceinline__ uint4 vec(uint32_t v) const {
        return __ldg(reinterpret_cast<const uint4*>(row + head) + v);
    }
    __device__ __forceinline__ uint32_t vec_index(uint32_t v) const { return head + v * Elem<T>::kPer16; }
};

struct TokenShared {
    uint64_t cand[kTokCandidates];
    uint64_t lists[kTokMaxCluster * kTokMaxTop];     // rank 0: every CTA's best entries, `top` of each
    uint64_t counts[kTokMaxCluster];                 // and how many they are
    TokenSums sums[kTokMaxCluster];                  // rank 0: every CTA's sums
    TokenSums warp_sums[8];
    __align__(16) float group_max[kTokGroups];
    uint32_t flagged[kTokMaxTop + kTokGroups];
    uint32_t n_tied, n_cand, warp_count[8];
    uint64_t best;
    float bound;
};

__device__ __forceinline__ void token_append(TokenShared& sm, uint64_t key) {
    const uint32_t at = atomicAdd(&sm.n_cand, 1u);
    if (at < (uint32_t)kTokCandidates) sm.cand[at] = key;
}

// Candidates of a CTA whose entries that reach the bound do not fit the list: a row of equal
// entries, or one whose few open entries stand before a mask of the lowest finite value.  Entries
// above the bound are collected first; if they fit, entries equal to it are taken in index order
// until there are enough.  Otherwise (all of them in few groups) the best are taken one by one.
template <typename T, int NT>
__device__ __noinline__ void token_collect_slow(TokenShared& sm, const TokenSpan<T>& sp, uint32_t top) {
    constexpr uint32_t E = Elem<T>::kPer16;
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float bound = sm.bound;
    float x[E];
    __syncthreads();
    if (tid == 0) sm.n_cand = 0;
    __syncthreads();
    for (uint32_t v = sp.v0 + tid; v < sp.v1; v += NT) {
        Elem<T>::widen(sp.vec(v), x);
        for (uint32_t i = 0; i < E; ++i)
            if (x[i] > bound) token_append(sm, token_key(x[i], sp.vec_index(v) + i));
    }
    if (tid < 2 * E) {
        bool have;
        const uint32_t j = sp.edge_index(tid, have);
        if (have) { const float y = Elem<T>::load(sp.row + j); if (y > bound) token_append(sm, token_key(y, j)); }
    }
    __syncthreads();
    uint32_t n = sm.n_cand;
    if (n <= (uint32_t)kTokCandidates - kTokMaxTop) {
        // ties in index order: head, body in chunks of one vector per thread, tail
        for (int part = 0; part < 3 && n < top; ++part) {
            const uint32_t begin = part == 1 ? sp.v0 : 0, end = part == 1 ? sp.v1 : 1;
            for (uint32_t base = begin; base < end && n < top; base += NT) {
                uint32_t mask = 0, index0 = 0;
                if (part == 1) {
                    if (base + tid < end) {
                        index0 = sp.vec_index(base + tid);
                        Elem<T>::widen(sp.vec(base + tid), x);
                        for (uint32_t i = 0; i < E; ++i) mask |= (x[i] == bound ? 1u : 0u) << i;
                    }
                } else if (tid < E) {
                    bool have;
                    index0 = sp.edge_index(part == 0 ? tid : E + tid, have);
                    mask = have && Elem<T>::load(sp.row + index0) == bound ? 1u : 0u;
                }
                const uint32_t mine = __popc(mask);
                uint32_t before = mine;                              // inclusive prefix over the warp
                for (int o = 1; o < 32; o <<= 1) {
                    const uint32_t u = __shfl_up_sync(~0u, before, o);
                    if (lane >= (uint32_t)o) before += u;
                }
                if (lane == 31) sm.warp_count[warp] = before;
                __syncthreads();
                uint32_t at = n + before - mine, all = 0;
                for (uint32_t w = 0; w < NT / 32; ++w) {
                    if (w < warp) at += sm.warp_count[w];
                    all += sm.warp_count[w];
                }
                for (uint32_t i = 0; i < E; ++i)
                    if ((mask >> i) & 1u) {
                        if (at < top) sm.cand[at] = token_key(bound, index0 + i);
                        ++at;
                    }
                n += all;
                __syncthreads();
            }
        }
        if (tid == 0) sm.n_cand = n < top ? n : (sm.n_cand > top ? sm.n_cand : top);
        __syncthreads();
        return;
    }
    uint64_t limit = ~0ull;
    uint32_t found = 0;
    for (; found < top; ++found) {
        uint64_t best = 0;
        for (uint32_t v = sp.v0 + tid; v < sp.v1; v += NT) {
            Elem<T>::widen(sp.vec(v), x);
            for (uint32_t i = 0; i < E; ++i) {
                const uint64_t key = x[i] >= -FLT_MAX ? token_key(x[i], sp.vec_index(v) + i) : 0;
                if (key < limit && key > best) best = key;
            }
        }
        if (tid < 2 * E) {
            bool have;
            const uint32_t j = sp.edge_index(tid, have);
            const float y = have ? Elem<T>::load(sp.row + j) : 0.f;
            const uint64_t key = have && y >= -FLT_MAX ? token_key(y, j) : 0;
            if (key < limit && key > best) best = key;
        }
        if (tid == 0) sm.best = 0;
        __syncthreads();
        if (best) atomicMax((unsigned long long*)&sm.best, (unsigned long long)best);
        __syncthreads();
        limit = sm.best;
        if (limit == 0) break;
        if (tid == 0) sm.cand[found] = limit;
        __syncthreads();
    }
    __syncthreads();
    if (tid == 0) sm.n_cand = found;
    __syncthreads();
}

// The CTA's best `top` entries into sm.cand (any order, sm.n_cand of them, more than needed).
template <typename T, int NT>
__device__ __forceinline__ void token_collect(TokenShared& sm, const TokenSpan<T>& sp, float m, uint32_t top) {
    constexpr uint32_t E = Elem<T>::kPer16;
    constexpr uint32_t L = NT / kTokGroups;                  // threads per group
    const uint32_t tid = threadIdx.x;
#pragma unroll
    for (uint32_t o = 1; o < L; o <<= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
    if (tid % L == 0) sm.group_max[tid / L] = m;
    if (tid == 0) { sm.n_cand = 0; sm.n_tied = 0; }
    __syncthreads();
    {                                                                 // L = 2 threads count for a group
        const uint32_t g0 = tid / L;
        const float mine = sm.group_max[g0];
        uint32_t rank = 0;
#pragma unroll 8
        for (uint32_t g = (tid % L) * 4; g < (uint32_t)kTokGroups; g += 4 * L) {
            const float4 o = *reinterpret_cast<const float4*>(&sm.group_max[g]);
            rank += (o.x > mine || (o.x == mine && g < g0)) ? 1u : 0u;
            rank += (o.y > mine || (o.y == mine && g + 1 < g0)) ? 1u : 0u;
            rank += (o.z > mine || (o.z == mine && g + 2 < g0)) ? 1u : 0u;
            rank += (o.w > mine || (o.w == mine && g + 3 < g0)) ? 1u : 0u;
        }
#pragma unroll
        for (uint32_t o = 1; o < L; o <<= 1) rank += __shfl_xor_sync(~0u, rank, o);
        if (rank == top - 1 && tid % L == 0) sm.bound = mine;
        // the groups that may reach the bound are those ranked before it
        if (rank < top && tid % L == 0) sm.flagged[rank] = g0;
        __syncthreads();
        if (rank >= top && tid % L == 0 && mine == sm.bound) sm.flagged[top + atomicAdd(&sm.n_tied, 1u)] = g0;
        __syncthreads();
    }
    const float bound = sm.bound;
    {
        // Groups whose maximum equals the bound but that rank behind it count, too: an entry of
        // theirs that equals it may come before others by index.
        const uint32_t steps = (sp.v1 - sp.v0 + NT - 1) / NT, per_group = steps * L;
        const uint32_t work = (top + sm.n_tied) * per_group;
        for (uint32_t i0 = tid; i0 < work; i0 += NT * kTokUnroll) {
            uint4 some[kTokUnroll];
            uint32_t at[kTokUnroll];
#pragma unroll
            for (int u = 0; u < kTokUnroll; ++u) {
                constexpr uint32_t none = Elem<T>::kMinusInf;
                const uint32_t i = i0 + u * NT, f = i / per_group, r = i - f * per_group;
                at[u] = i < work ? sp.v0 + (r / L) * NT + sm.flagged[f] * L + r % L : sp.v1;
                some[u] = at[u] < sp.v1 ? sp.vec(at[u]) : make_uint4(none, none, none, none);
            }
#pragma unroll
            for (int u = 0; u < kTokUnroll; ++u) {
                float x[E];
                Elem<T>::widen(some[u], x);
                if (Elem<T>::largest(some[u]) >= bound) {
#pragma unroll
                    for (uint32_t j = 0; j < E; ++j)
                        if (x[j] >= bound) token_append(sm, token_key(x[j], sp.vec_index(at[u]) + j));
                }
            }
        }
    }
    if (tid < 2 * E) {
        bool have;
        const uint32_t j = sp.edge_index(tid, have);
        if (have) { const float y = Elem<T>::load(sp.row + j); if (y >= bound) token_append(sm, token_key(y, j)); }
    }
    __syncthreads();
    if (sm.n_cand > (uint32_t)kTokCandidates) token_collect_slow<T, NT>(sm, sp, top);
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_addr(const void* p, uint32_t rank) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ void cluster_store(uint32_t addr, uint64_t v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ void cluster_store(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}

template <typename T, bool ENT, int NT>
__global__ void __launch_bounds__(NT, 1024 / NT) token_logprob_kernel(TokenForward P) {
    constexpr uint32_t E = Elem<T>::kPer16;
    __shared__ TokenShared sm;
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t C = 1u << P.cluster_log2, rank = blockIdx.x & (C - 1);
    const uint64_t row = blockIdx.x >> P.cluster_log2;
    if (C > 1) cluster_arrive();                                      // every CTA of the row has started

    TokenSpan<T> sp;
    sp.row = reinterpret_cast<const T*>(P.logits) + row * P.row_stride;
    const uint32_t odd = (uint32_t)((16u - (reinterpret_cast<uintptr_t>(sp.row) & 15u)) & 15u) / (uint32_t)sizeof(T);
    sp.vocab = P.vocab;
    sp.head = odd < P.vocab ? odd : P.vocab;
    sp.nv = (P.vocab - sp.head) / E;
    const uint32_t per = (sp.nv + C - 1) >> P.cluster_log2;
    sp.v0 = rank * per < sp.nv ? rank * per : sp.nv;
    sp.v1 = sp.v0 + per < sp.nv ? sp.v0 + per : sp.nv;
    sp.first = rank == 0;
    sp.last = rank == C - 1;

    // the target's logit, asked for before it is needed
    int64_t target = -1;
    float target_x = 0.f;
    if (P.logprob && rank == 0 && tid == 0) {
        target = P.targets[row];
        if (target >= 0 && target < (int64_t)P.vocab) target_x = Elem<T>::load(sp.row + target);
    }
    const float k = __fmul_rn(P.tau, kLog2e);
    TokenSums a = {-FLT_MAX, 0.f, 0.f};
    // batches of vectors; what is missing at the end is as if masked
    auto fetch = [&](uint32_t v) {
        constexpr uint32_t none = Elem<T>::kMinusInf;
        return v < sp.v1 ? sp.vec(v) : make_uint4(none, none, none, none);
    };
    for (uint32_t v = sp.v0 + tid; v < sp.v1 + tid; v += kTokUnroll * NT) {
        uint4 raw[kTokUnroll];
        if (v - tid + kTokUnroll * NT <= sp.v1) {
#pragma unroll
            for (int u = 0; u < kTokUnroll; ++u) raw[u] = sp.vec(v + u * NT);
        } else {
#pragma unroll
            for (int u = 0; u < kTokUnroll; ++u) raw[u] = fetch(v + u * NT);
        }
        token_add<T, ENT, kTokUnroll>(a, raw, k);
    }
    if (tid < 2 * E) {
        bool have;
        const uint32_t j = sp.edge_index(tid, have);
        if (have) token_add<ENT>(a, Elem<T>::load(sp.row + j), k);
    }

    const float own_max = a.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        token_merge(a, {__shfl_xor_sync(~0u, a.m, o), __shfl_xor_sync(~0u, a.s, o), __shfl_xor_sync(~0u, a.t, o)}, k);
    if (lane == 0) sm.warp_sums[warp] = a;
    if (P.top) token_collect<T, NT>(sm, sp, own_max, P.top);              // its barriers order warp_sums too
    else __syncthreads();
    if (C > 1) cluster_wait();

    if (warp == 0) {
        a = sm.warp_sums[lane & (NT / 32 - 1)];
#pragma unroll
        for (int o = NT / 64; o > 0; o >>= 1)
            token_merge(a, {__shfl_xor_sync(~0u, a.m, o), __shfl_xor_sync(~0u, a.s, o), __shfl_xor_sync(~0u, a.t, o)}, k);
    }
    if (tid == 0) {
        const uint32_t to = cluster_addr(&sm.sums[rank], 0);
        cluster_store(to, a.m); cluster_store(to + 4, a.s); cluster_store(to + 8, a.t);
    }
    if (P.top) {
        const uint32_t n = sm.n_cand;
        for (uint32_t i = n + tid; i < P.top; i += NT)
            cluster_store(cluster_addr(&sm.lists[rank * P.top + i], 0), (uint64_t)0);
        if (tid == 0) cluster_store(cluster_addr(&sm.counts[rank], 0), (uint64_t)(n < P.top ? n : P.top));
        for (uint32_t i = tid; i < n; i += NT) {
            const uint64_t key = sm.cand[i];
            uint32_t better = 0;
            for (uint32_t j = 0; j < n; ++j) better += sm.cand[j] > key ? 1u : 0u;
            if (better < P.top) cluster_store(cluster_addr(&sm.lists[rank * P.top + better], 0), key);
        }
    }
    if (C > 1) {
        cluster_arrive();
        cluster_wait();
        if (rank != 0) return;
    } else {
        __syncthreads();
    }

    a = sm.sums[0];
    for (uint32_t c = 1; c < C; ++c) token_merge(a, sm.sums[c], k);
    const bool empty = a.s == 0.f;                                    // nothing left by the mask
    const float ln_s = logf(a.s);                                     // -inf where empty, NaN where the row holds one
    if (tid == 0) {
        if (P.lse) P.lse[row] = empty ? -INFINITY : __fmaf_rn(a.m, P.tau, ln_s);
        if (ENT) P.entropy[row] = empty ? 0.f : __fsub_rn(ln_s, __fmul_rn(kLn2, __fdiv_rn(a.t, a.s)));
        if (P.logprob) {
            float lp = 0.f;
            if (target >= (int64_t)P.vocab) lp = NAN;
            else if (target >= 0)
                lp = empty ? -INFINITY : __fsub_rn(__fmul_rn(__fsub_rn(target_x, a.m), P.tau), ln_s);
            P.logprob[row] = lp;
        }
    }
    if (P.top) {
        const bool valid = a.s > 0.f;                                 // false for NaN as well
        if (tid < P.top && !valid) {
            P.top_logprob[row * P.top + tid] = empty ? -INFINITY : NAN;
            P.top_index[row * P.top + tid] = -1;
        }
        if (valid && C == 1 && tid < P.top) {
            const uint64_t key = sm.lists[tid];
            P.top_logprob[row * P.top + tid] =
                key ? __fsub_rn(__fmul_rn(__fsub_rn(token_key_value(key), a.m), P.tau), ln_s) : -INFINITY;
            P.top_index[row * P.top + tid] = key ? (int32_t)token_key_index(key) : -1;
        } else if (valid && tid < C * P.top) {
            // every CTA's list is in order: an entry's place is the number of better ones in each
            const uint64_t key = sm.lists[tid];
            uint32_t lo[kTokMaxCluster];
#pragma unroll
            for (int c = 0; c < kTokMaxCluster; ++c) lo[c] = 0;
#pragma unroll
            for (uint32_t step = kTokMaxTop; step > 0; step >>= 1) {
                if (step > P.top) continue;
#pragma unroll
                for (uint32_t c = 0; c < (uint32_t)kTokMaxCluster; ++c)
                    if (c < C && lo[c] + step <= P.top && sm.lists[c * P.top + lo[c] + step - 1] > key) lo[c] += step;
            }
            uint32_t better = 0;
#pragma unroll
            for (int c = 0; c < kTokMaxCluster; ++c) better += lo[c];
            if (key && better < P.top) {
                P.top_logprob[row * P.top + better] = __fsub_rn(__fmul_rn(__fsub_rn(token_key_value(key), a.m), P.tau), ln_s);
                P.top_index[row * P.top + better] = (int32_t)token_key_index(key);
            }
        }
        if (valid && C > 1 && tid < P.top) {                          // where the open entries run out
            uint64_t open = 0;
            for (uint32_t c = 0; c < C; ++c) open += sm.counts[c];
            if (tid >= open) {
                P.top_logprob[row * P.top + tid] = -INFINITY;
                P.top_index[row * P.top + tid] = -1;
            }
        }
    }
}

// ---- backward --------------------------------------------------------------------------------
//
// For a loss L with g = dL/d log p_y and e = dL/dH of a row, log p_j = tau x_j - lse,
//     dL/dx_j = tau (g [j = y] - p_j (g + e (log p_j + H))).
// One read of the logits, one write of their gradient; lse and H come from the forward pass.
//
// lse is tau max x + ln s rounded to 32 bits: 2^-24 |lse| of it is lost, and p is off by that part of
// itself.  A row of the lowest finite value, or one far from zero, loses all of ln s, and a row with
// tau max x out of range has an lse of -inf or inf.  Where the loss could pass a sixteenth of what the
// logits' type rounds to (for fp32: what the sums of the forward pass are off by), one CTA takes
// the whole row, adds s up again and takes log p_j = tau (x_j - m) - ln s.  All rows of that kind: 8192 x
// 50257 bf16 445 us against 264, 24 x 128001 41 against 8.  One CTA, because the row may be
// overwritten in place; by few registers (no unrolling), as its call counts for the whole kernel (with 64
// instead of 40 the ordinary rows take 301 us).

constexpr int kTokGradThreads = 256;
constexpr uint32_t kTokNoTarget = 0xFFFFFFFFu;
constexpr int kTokGradUnroll = 4;
template <typename T> constexpr float kTokLargeLse = sizeof(T) == 4 ? 128.f : 1024.f;

struct TokenBackward {
    const void* logits;
    void* d_logits;
    uint64_t rows, row_stride, d_row_stride;
    const int64_t* targets;
    const float* lse;
    const float* entropy;
    const float* d_logprob;
    const float* d_entropy;
    uint32_t vocab, chunks;              // CTAs' worth of vectors per row
    float tau;
};

struct TokenRow { float m, lse, w, u, hit; uint32_t target; bool empty; };   // of x - m

// MAX: m is not 0.  The target's entry is set by token_grad_target.
template <typename T, bool ENT, bool MAX, int N>
__device__ __forceinline__ void token_grad(const TokenRow& r, const TokenBackward& P, float* x) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float lp = __fmaf_rn(MAX ? __fsub_rn(x[i], r.m) : x[i], P.tau, -r.lse);
        const float p = ex2(__fmul_rn(lp, kLog2e));
        if (ENT) {
            lp = fmaxf(lp, -1e4f);                                    // where p is 0: 0, not 0 * inf, also for a large u
            x[i] = __fmul_rn(p, __fmaf_rn(r.u, lp, r.w));
        } else {
            x[i] = __fmul_rn(p, r.w);
        }
        if (r.empty) x[i] = 0.f;
    }
}

// What is known of a row whose lse is given relative to m.
template <bool ENT>
__device__ __forceinline__ TokenRow token_row(const TokenBackward& P, uint64_t row, float m, float lse) {
    TokenRow r;
    const int64_t y = P.targets ? P.targets[row] : -1;
    if (y >= (int64_t)P.vocab) lse = NAN;                             // as its log probability
    r.m = m;
    r.lse = lse;
    r.empty = lse == -INFINITY;
    const float g = P.d_logprob && y >= 0 ? P.d_logprob[row] : 0.f;
    r.target = y >= 0 && y < (int64_t)P.vocab && !r.empty ? (uint32_t)y : kTokNoTarget;
    r.hit = __fmul_rn(P.tau, g);
    if (ENT) {
        const float e = P.d_entropy[row];
        r.u = -__fmul_rn(P.tau, e);
        r.w = -__fmul_rn(P.tau, __fmaf_rn(e, P.entropy[row], g));
    } else {
        r.u = 0.f;
        r.w = -r.hit;
    }
    if (lse != lse) r.w = lse;                                        // a row with a NaN gives NaN
    return r;
}

// The target's entry from its logit: tau (g (1 - p) - e p (log p + H)).  A token that the model is sure of
// has p near 1, and all of its row's gradient is of the size of 1 - p: that is not to be a
// difference of rounded numbers (ex2's error alone is 2^-22).  Not inlined, for its registers.
template <typename T, bool ENT>
__device__ __noinline__ void token_grad_target(const TokenBackward& P, uint64_t row, float m, float lse, float x) {
    const uint64_t y = (uint64_t)P.targets[row];
    const float lp = __fmaf_rn(__fsub_rn(x, m), P.tau, -lse);
    const float g = P.d_logprob ? P.d_logprob[row] : 0.f;
    float d = -__fmul_rn(__fmul_rn(P.tau, g), expm1f(lp));
    if (ENT) {                                                        // the same as any entry's without g
        const float e = P.d_entropy[row], w = -__fmul_rn(P.tau, __fmul_rn(e, P.entropy[row]));
        d = __fadd_rn(d, __fmul_rn(ex2(__fmul_rn(lp, kLog2e)), __fmaf_rn(-__fmul_rn(P.tau, e), fmaxf(lp, -1e4f), w)));
    }
    Elem<T>::store(reinterpret_cast<T*>(P.d_logits) + row * P.d_row_stride + y, d);
}

// A whole row, with its sum taken anew.
template <typename T, bool ENT>
__device__ __noinline__ void token_grad_large(const TokenBackward& P, uint64_t row) {
    constexpr uint32_t E = Elem<T>::kPer16;
    __shared__ TokenSums sums[kTokGradThreads / 32];
    const uint32_t tid = threadIdx.x;
    const T* in = reinterpret_cast<const T*>(P.logits) + row * P.row_stride;
    T* out = reinterpret_cast<T*>(P.d_logits) + row * P.d_row_stride;
    const uint32_t odd = (uint32_t)((16u - (reinterpret_cast<uintptr_t>(in) & 15u)) & 15u) / (uint32_t)sizeof(T);
    const uint32_t head = odd < P.vocab ? odd : P.vocab;
    const uint32_t nv = (P.vocab - head) / E;
    const uint4* vin = reinterpret_cast<const uint4*>(in + head);
    const float k = __fmul_rn(P.tau, kLog2e);
    const uint32_t edge = tid < E ? tid : head + nv * E + (tid - E);  // this thread's single entry, if it has one
    const bool has_edge = tid < 2 * E && (tid < E ? tid < head : edge < P.vocab);

    TokenSums a = {-FLT_MAX, 0.f, 0.f};
#pragma unroll 1
    for (uint32_t v = tid; v < nv; v += kTokGradThreads) {
        const uint4 raw = vin[v];
        token_add<T, false, 1>(a, &raw, k);
    }
    if (has_edge) token_add<false>(a, Elem<T>::load(in + edge), k);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        token_merge(a, {__shfl_xor_sync(~0u, a.m, o), __shfl_xor_sync(~0u, a.s, o), 0.f}, k);
    __syncthreads();                                                  // the row before has read its sums
    if ((tid & 31) == 0) sums[tid >> 5] = a;
    __syncthreads();
    a = sums[0];
#pragma unroll
    for (int w = 1; w < kTokGradThreads / 32; ++w) token_merge(a, sums[w], k);

    const TokenRow r = token_row<ENT>(P, row, a.m, logf(a.s));        // -inf for an empty row
    // the thread that has the target's vector or edge, which it alone overwrites
    const uint32_t hit_v = (r.target - head) / E;
    const bool owner = r.target != kTokNoTarget &&
                       (r.target >= head && hit_v < nv ? hit_v % kTokGradThreads == tid : has_edge && edge == r.target);
    const float hit_x = owner ? Elem<T>::load(in + r.target) : 0.f;
#pragma unroll 1
    for (uint32_t v = tid; v < nv; v += kTokGradThreads) {
        float x[E];
        Elem<T>::widen(vin[v], x);
        token_grad<T, ENT, true, (int)E>(r, P, x);
        if (((reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) & 15u) == 0) {
            reinterpret_cast<uint4*>(out + head)[v] = Elem<T>::narrow(x);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < E; ++i) Elem<T>::store(out + head + v * E + i, x[i]);
        }
    }
    if (has_edge) {
        float x[1] = {Elem<T>::load(in + edge)};
        token_grad<T, ENT, true, 1>(r, P, x);
        Elem<T>::store(out + edge, x[0]);
    }
    if (owner) token_grad_target<T, ENT>(P, row, r.m, r.lse, hit_x);
}

template <typename T, bool ENT>
// (Left to itself the compiler takes 48 registers or more: 8192 x 50257 bf16 274 us against 264, 4096 x
// 50257 fp32 270 against 242.)
__global__ void __launch_bounds__(kTokGradThreads, 6) token_logprob_grad_kernel(const __grid_constant__ TokenBackward P) {
    constexpr uint32_t E = Elem<T>::kPer16;
    constexpr uint32_t kChunk = kTokGradThreads * kTokGradUnroll;
    const uint32_t tid = threadIdx.x;
    const uint64_t tasks = P.rows * P.chunks;
    bool large = false;                                               // a row is left for later
    for (uint64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
        const uint64_t row = task / P.chunks;
        const uint32_t chunk = (uint32_t)(task - row * P.chunks);
        const T* in = reinterpret_cast<const T*>(P.logits) + row * P.row_stride;
        T* out = reinterpret_cast<T*>(P.d_logits) + row * P.d_row_stride;
        const uint32_t odd = (uint32_t)((16u - (reinterpret_cast<uintptr_t>(in) & 15u)) & 15u) / (uint32_t)sizeof(T);
        const uint32_t head = odd < P.vocab ? odd : P.vocab;
        const uint32_t nv = (P.vocab - head) / E;
        const bool same = ((reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) & 15u) == 0;
        const uint4* vin = reinterpret_cast<const uint4*>(in + head);
        uint4 raw[kTokGradUnroll];
        const uint32_t v0 = chunk * kChunk + tid;
#pragma unroll
        for (int u = 0; u < kTokGradUnroll; ++u)
            if (v0 + u * kTokGradThreads < nv) raw[u] = vin[v0 + u * kTokGradThreads];

        const TokenRow r = token_row<ENT>(P, row, 0.f, P.lse[row]);
        if (fabsf(r.lse) >= kTokLargeLse<T>) {                        // not for NaN
            large |= chunk == 0;
            continue;
        }
        const uint32_t edge = tid < E ? tid : head + nv * E + (tid - E);
        const bool has_edge = chunk == P.chunks - 1 && tid < 2 * E && (tid < E ? tid < head : edge < P.vocab);
        // the thread that has the target's vector or edge, which it alone overwrites
        const uint32_t hit_v = (r.target - head) / E;
        const bool owner = r.target != kTokNoTarget &&
                           (r.target >= head && hit_v < nv ? hit_v / kChunk == chunk && hit_v % kTokGradThreads == tid
                                                           : has_edge && edge == r.target);
        const float hit_x = owner ? Elem<T>::load(in + r.target) : 0.f;

#pragma unroll
        for (int u = 0; u < kTokGradUnroll; ++u) {
            const uint32_t v = v0 + u * kTokGradThreads;
            if (v >= nv) break;
            float x[E];
            Elem<T>::widen(raw[u], x);
            token_grad<T, ENT, false, (int)E>(r, P, x);
            if (same) {
                reinterpret_cast<uint4*>(out + head)[v] = Elem<T>::narrow(x);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < E; ++i) Elem<T>::store(out + head + v * E + i, x[i]);
            }
        }
        if (has_edge) {
            float x[1] = {Elem<T>::load(in + edge)};
            token_grad<T, ENT, false, 1>(r, P, x);
            Elem<T>::store(out + edge, x[0]);
        }
        if (owner) token_grad_target<T, ENT>(P, row, 0.f, r.lse, hit_x);
    }
    // behind the loop, where nothing is held in registers across the call
    if (large)
        for (uint64_t task = blockIdx.x; task < tasks; task += gridDim.x)
            if (task % P.chunks == 0 && fabsf(P.lse[task / P.chunks]) >= kTokLargeLse<T>)
                token_grad_large<T, ENT>(P, task / P.chunks);
}

}  // namespace ecq
