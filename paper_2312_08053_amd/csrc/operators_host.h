// What the entry points of the operators beside a round check and launch with.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/kimad.h"

namespace kimad {

constexpr uint64_t MOST = 1ull << 40;                    // elements along an axis that the checks let through
constexpr uint64_t UNITS = 256;                         // compute units of the device
constexpr uint64_t GRID_MOST = 0x7FFFFFFFull, GRID_Y_MOST = 65535;
// a launch's workgroups along x: their threads are counted in 32 bits
inline bool grid_ok(uint64_t wgs, uint64_t threads) { return wgs <= GRID_MOST && wgs <= 0xFFFFFFFFull / threads; }

inline bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
inline int launched() { return hipGetLastError() == hipSuccess ? KIMAD_OK : KIMAD_ERR_HIP; }
inline uint64_t type_bytes(uint32_t type) { return type == KIMAD_VALUES_F32 ? 4 : 2; }

}  // namespace kimad
