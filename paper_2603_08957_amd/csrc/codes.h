// Codes of second moments in 8 bits, on the device and for tests on the host.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace tre {

constexpr int kBias2 = 23;  // of their exponents

__host__ __device__ inline int middle(int a, int b, int c) { return std::min(std::max(a, b), std::max(std::min(a, b), c)); }
// The code of a second moment times its block's power of two, y < 256.5.  `high` is
// what it is where E is not 0, `low` where it is; of these and the least code with E
// = 1 the right one lies in the middle.  `low` of a large value has no int: it is cut
// off above the largest `high` (less than 256), where it still is the largest.
template <bool CHANCE>
__host__ __device__ inline uint32_t second_code(float y, uint32_t word) {
    constexpr float kUnits = float(1u << (kBias2 + 2));  // of codes below 8
    constexpr uint32_t kNone = uint32_t(127 - kBias2) << 23;
    const uint32_t u = __builtin_bit_cast(uint32_t, y);
    if constexpr (CHANCE) {  // in steps of 2^-20 of a code
        const int w = middle(int(u - kNone), (8 << 20) - 1, int(__builtin_fminf(y * (kUnits * float(1u << 20)), 512.f * float(1u << 20))));
        return (uint32_t(w) + (word >> 12)) >> 20;
    } else {
        return uint32_t(middle(int(u - kNone + 0x7ffffu + (u >> 20 & 1)) >> 20, 8, int(__builtin_rintf(__builtin_fminf(y * kUnits, 512.f)))));
    }
}

}  // namespace tre
