// What the orthogonaliser's kernels do with their counters, for tests on fake_cudart.cpp.
#include "../paper_1806_08054_b200/csrc/ecq_host.h"
#include "../paper_1806_08054_b200/csrc/ecq_muon.cuh"

std::atomic<uint64_t> ecq::g_launches{0};

extern "C" bool fake_prepare(const void* args, unsigned grid) {
    const ecq::MuonPrepare& P = *static_cast<const ecq::MuonPrepare*>(args);
    if (P.what == 1) return true;
    const bool clean = !*P.next && !P.added[0] && !P.factor[0];
    if (P.what == 2) *P.next += grid;
    P.added[0] = 1;
    P.factor[0] = 1;
    return clean;
}

extern "C" void fake_iterate(const void* args) {
    const ecq::MuonIterate& P = *static_cast<const ecq::MuonIterate*>(args);
    *P.prepare_next = 0;
    for (uint32_t i = 0; i < P.n_mats; ++i) { P.added[i] = 0; P.factor[i] = 0; }
}
