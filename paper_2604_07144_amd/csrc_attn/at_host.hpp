// Checks and arithmetic that the C ABI's entry points share, on the host.
#ifndef AT_HOST_HPP
#define AT_HOST_HPP

#include <cstdint>

#include <hip/hip_runtime.h>

#include "autopoiesis_eval.h"

namespace {

constexpr uint64_t kMost = 1ull << 31;   // rows, columns and positions stay below
constexpr uint64_t kMostGroups = 1ull << 24;  // and workgroups (of 256 threads: a grid holds less than 2^32)

inline bool multiple(const void* p, uint64_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline bool stride_ok(int64_t s, int64_t n) { return s >= 0 && s % n == 0; }

// magic and shift of a division of numbers below 2^31 by `d`: n / d = ((2 n) * magic >> 32) >> shift
inline void divider(uint32_t d, uint32_t* magic, uint32_t* shift) {
    uint32_t l = 0;
    while ((1ull << l) < d) ++l;
    *shift = l;
    *magic = (uint32_t)(((1ull << (31 + l)) + d - 1) / d);
}

inline ap_status launched() { return hipGetLastError() == hipSuccess ? AP_OK : AP_ERR_DEVICE; }

}  // namespace

#endif  // AT_HOST_HPP
