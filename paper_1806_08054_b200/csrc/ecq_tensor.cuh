// What kernels that use the tensor cores (tcgen05) share: descriptors, tensor memory, pairs of CTAs, waits that give up,
// and how a kernel leaves after one.
#pragma once

#include <cstdint>

#include "ecq_common.cuh"
#include "ecq_ring.h"

namespace ecq {

// Shared-memory descriptor of an operand without swizzle: units of eight rows of 16 bytes, 128 bytes
// each.  `lead` is the byte distance from a unit to the next one along K, `step` to the next one
// along M or N.
__device__ __forceinline__ uint64_t umma_desc(uint32_t addr, uint32_t lead, uint32_t step) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(step >> 4) << 32) | (1ull << 46);
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

// All CTAs of a cluster, where no memory is handed over but barriers that were made visible by their own fence: a release would
// wait for results on their way to memory.
__device__ __forceinline__ void cluster_sync_relaxed() { asm volatile("barrier.cluster.arrive.relaxed;\n\tbarrier.cluster.wait;" ::: "memory"); }

// Waits that give up: the limit is per wait, and one that ran out ends all others soon.
__device__ __forceinline__ bool wait_or_stop(uint32_t bar, uint32_t parity, uint32_t limit, volatile uint32_t* stop) {
    for (uint32_t it = 0; it < limit; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if (*stop) return false;
    }
    *stop = 1;
    return false;
}
// The same where the other CTA of a pair arrives and its writes are read.
__device__ __forceinline__ bool wait_pair_or_stop(uint32_t bar, uint32_t parity, uint32_t limit, volatile uint32_t* stop) {
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
// What a CTA's warps leave for the case that a wait ran out.
struct RingEnd {
    uint32_t asked[2];                   // loads issued: left, right
    uint32_t multiplied, committed;      // of a pair's first CTA: steps whose products were issued, commits of accumulators
    uint32_t halted;                     // a wait ran out in a CTA of the cluster
};
__device__ __forceinline__ uint32_t peer_word(const volatile uint32_t& w, uint32_t cta) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(peer_addr(smem_u32(const_cast<const uint32_t*>(&w)), cta)) : "memory");
    return v;
}
// All threads of the cluster meet at its end; what a CTA whose wait ran out says then is known to all.  RELEASE: where
// arrivals on other CTAs' barriers may be on their way that nobody waits for.
template <bool RELEASE>
__device__ __forceinline__ bool ring_end(volatile RingEnd& end, bool stop, uint32_t ctas) {
    if (threadIdx.x == 0 && stop) {
        for (uint32_t c = 0; c < ctas; ++c)
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(peer_addr(smem_u32(const_cast<const uint32_t*>(&end.halted)), c)), "r"(1u) : "memory");
        asm volatile("fence.acq_rel.cluster;" ::: "memory");
    }
    if (RELEASE) pair_sync();
    else cluster_sync_relaxed();
    return end.halted != 0;
}
struct RingBars {
    uint32_t full;
    __device__ void arrive(uint32_t s, uint32_t bytes) { mbar_arrive_expect_tx(full + 8 * s, bytes); }
    __device__ void forgo(uint32_t s, uint32_t bytes) {
        asm volatile("mbarrier.complete_tx.relaxed.cluster.shared::cta.b64 [%0], %1;" ::"r"(full + 8 * s), "r"(bytes) : "memory");
    }
    __device__ void wait(uint32_t s, uint32_t parity) { mbar_wait(full + 8 * s, parity); }
};
// After a wait that ran out: every thread of the cluster comes here, and leaves when all that was issued for its CTAs has
// arrived, which these waits (with the built-in limit) see on the barriers where it is counted: loads, products,
// and what `others` waits for.  Other arrivals from CTAs are over when the cluster has met.  Barriers lie as the kernels
// have them: full and empty ones of the stages, then ACCS that accumulators are committed to in turn.
// CG CTAs share a ring.  (Inline: a call costs every launch 0.3 us, one token's product among them.)
template <int CG, uint32_t ACCS, typename Others>
__device__ __forceinline__ void ring_settle(const volatile RingEnd& end, const RingLoads& issued, uint32_t full, Others others) {
    pair_sync();
    if (threadIdx.x == 0) {
        const uint32_t stages = issued.stages, empty = full + 8 * stages, acc = empty + 8 * stages;
        const uint32_t rank = CG == 2 ? cta_rank() & 1u : 0, first = cta_rank() - rank;
        if (rank == 0) {
            const uint32_t l = end.asked[0], r = end.asked[1];
            const RingLoads loads = {stages, CG, {issued.bytes[0], issued.bytes[1]}, {issued.more[0], issued.more[1]}, issued.begin, issued.steps,
                                     {{l, r}, {CG == 2 ? peer_word(end.asked[0], first + 1) : l, CG == 2 ? peer_word(end.asked[1], first + 1) : r}}};
            RingBars bars = {full};
            ring_rest(loads, bars);
        }
        const uint32_t m = peer_word(end.multiplied, first), n = peer_word(end.committed, first);
#pragma unroll 1
        for (uint32_t j = m > stages ? m - stages : 0; j < m; ++j) mbar_wait(empty + 8 * (j % stages), (j / stages) & 1);
#pragma unroll 1
        for (uint32_t j = n > ACCS ? n - ACCS : 0; j < n; ++j) mbar_wait(acc + 8 * (j % ACCS), (j / ACCS) & 1);
        others();
    }
    pair_sync();
}

__device__ __forceinline__ uint4 lds16(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ void sts16(uint32_t addr, uint4 v) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// One lane of a converged warp, in a form from which the compiler can tell that it is one: TMA and
// tcgen05 instructions take their operands from uniform registers, and behind a plain comparison of
// the lane's number each of them costs about 0.1 us to issue.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

}  // namespace ecq
