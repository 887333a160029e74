// How a ring of loads is brought to rest after a wait ran out: arithmetic on counts, without a device, so that it
// compiles for the host too.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define ECQ_BOTH __host__ __device__
#else
#define ECQ_BOTH
#endif

namespace ecq {

// A ring of stages that two loaders fill, one for each operand.  Load j of an operand goes to stage j % stages; a stage's
// barrier ends phase j / stages when both loaders have arrived, each with the bytes that it expects, and all of
// them are there.  In a pair of CTAs each CTA loads its own part of an operand, bytes are counted on the
// first CTA's barriers, and the first CTA's loaders arrive there for both.
struct RingLoads {
    uint32_t stages, ctas;               // ctas: 1, or 2
    uint32_t bytes[2], more[2];          // of each operand and CTA in a step; and where scales come with it
    uint32_t begin, steps;               // steps along K of a tile: from `begin` on
    uint32_t asked[2][2];                // loads that were issued, of each CTA (one: given twice) and operand

    ECQ_BOTH uint32_t size(uint32_t operand, uint32_t j) const {
        const uint32_t k = begin + j % steps;
        return bytes[operand] + (k == begin || (k & 3) == 0 ? more[operand] : 0);
    }
};

// The loaders stopped where they were: some loads of a phase may be on their way and others not asked for, so that
// its barrier would wait for good, or does not expect what comes.  Here its arrivals and bytes are made up to
// what was issued: then the phase ends when the last byte has landed.  Loads are issued into stages
// whose phase before is over, so that phases further back than the ring is long are.
//   bars.arrive(stage, bytes)       arrives, expecting bytes
//   bars.forgo(stage, bytes)        takes back bytes that were expected
//   bars.wait(stage, parity)        (bounded)
template <typename Bars>
ECQ_BOTH inline void ring_rest(const RingLoads& r, Bars& bars) {
    const uint32_t left = r.asked[0][0] > r.asked[1][0] ? r.asked[0][0] : r.asked[1][0];
    const uint32_t right = r.asked[0][1] > r.asked[1][1] ? r.asked[0][1] : r.asked[1][1], most = left > right ? left : right;
    for (uint32_t j = most > r.stages ? most - r.stages : 0; j < most; ++j) {
        const uint32_t s = j % r.stages;
#pragma unroll
        for (uint32_t o = 0; o < 2; ++o) {
            const bool armed = j < r.asked[0][o], other = r.ctas == 2 && j < r.asked[1][o];
            if (!armed) bars.arrive(s, other ? r.size(o, j) : 0u);
            else if (r.ctas == 2 && !other) bars.forgo(s, r.size(o, j));
        }
        bars.wait(s, (j / r.stages) & 1u);
    }
}

}  // namespace ecq
