// A ring of loads on counters in place of barriers, stopped anywhere and brought to rest by csrc/ecq_ring.h.
#include <random>
#include <vector>

#include "ecq_ring.h"

using namespace ecq;

namespace {

struct Load { uint32_t stage, phase; long bytes; };

struct Model {
    RingLoads r;
    std::mt19937 rng;
    std::vector<uint32_t> phase, pending;
    std::vector<long> left;              // bytes expected and not there yet
    std::vector<Load> flying;
    uint32_t consumed = 0;
    int wrong = 0;

    Model(const RingLoads& loads, uint32_t seed) : r(loads), rng(seed), phase(loads.stages), pending(loads.stages, 2), left(loads.stages) {}

    void look(uint32_t s) {
        if (pending[s] || left[s]) return;
        for (const Load& f : flying) wrong += f.stage == s && f.phase <= phase[s];   // over before its bytes are there
        ++phase[s];
        pending[s] = 2;
    }
    void arrive(uint32_t s, uint32_t bytes) {
        if (!pending[s]) { ++wrong; return; }
        --pending[s];
        left[s] += bytes;
        look(s);
    }
    void forgo(uint32_t s, uint32_t bytes) { left[s] -= bytes; look(s); }
    bool land() {
        if (flying.empty()) return false;
        const uint32_t i = rng() % flying.size();
        const Load f = flying[i];
        flying.erase(flying.begin() + i);
        left[f.stage] -= f.bytes;
        look(f.stage);
        return true;
    }
    void wait(uint32_t s, uint32_t parity) {
        while ((phase[s] & 1u) == parity)
            if (!land()) { ++wrong; return; }                        // for good
    }
    bool load(uint32_t c, uint32_t o) {
        uint32_t& j = r.asked[c][o];
        if (j >= consumed + r.stages) return false;
        const uint32_t s = j % r.stages, b = r.size(o, j);
        if (c == 0) arrive(s, r.ctas * b);
        flying.push_back({s, j / r.stages, (long)b});
        ++j;
        return true;
    }
    void consume() { if (phase[consumed % r.stages] > consumed / r.stages) ++consumed; }
};

}  // namespace

// Runs `runs` rings, each stopped at a random point; how often something was wrong.
extern "C" int ring_model(uint32_t stages, uint32_t ctas, uint32_t begin, uint32_t steps, uint32_t seed, uint32_t runs, int rest) {
    int wrong = 0;
    for (uint32_t n = 0; n < runs; ++n) {
        Model m({stages, ctas, {1000, 700}, {50, 30}, begin, steps, {}}, seed + n);
        const uint32_t stop = m.rng() % 200;
        uint32_t off = 0;                                            // loaders that have stopped
        for (uint32_t t = 0; t < stop + 40; ++t) {
            const uint32_t what = m.rng() % 8, c = what & (ctas - 1), o = what >> 1 & 1;
            if (t > stop && m.rng() % 4 == 0) off |= 1u << (2 * c + o);
            if (what < 4) { if (!(off >> (2 * c + o) & 1)) m.load(c, o); }
            else if (what < 6) m.land();
            else if (t < stop) m.consume();
        }
        RingLoads r = m.r;
        if (ctas == 1) { r.asked[1][0] = r.asked[0][0]; r.asked[1][1] = r.asked[0][1]; }
        if (rest) ring_rest(r, m);
        wrong += m.wrong + (int)m.flying.size();
    }
    return wrong;
}
