// Host-side state shared by the library's translation units.
#pragma once

#include <atomic>
#include <cstdint>

namespace ecq {

extern std::atomic<uint64_t> g_launches;    // kernels launched in this process (ecq_launch_count)

// Per-device set-up (kernel attributes, the built-in scratch's address) is kept in tables
// indexed by the device ordinal; contexts on devices beyond them are refused.
constexpr int kMaxDevices = 64;

inline bool aligned_to(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Bytes of one element of an ECQ_F32 / ECQ_BF16 / ECQ_F16 array; 0 for an unknown type.
inline uint32_t dtype_bytes(int dtype) { return dtype == 0 ? 4u : dtype == 1 || dtype == 2 ? 2u : 0u; }

}  // namespace ecq
