// The whole-number arithmetic of the 8-bit product's integer sums (no CUDA
// needed: constant expressions).
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define REALQ_ANYWHERE __host__ __device__
#else
#define REALQ_ANYWHERE
#endif

namespace realq {

// sum_j x_j (c_j - z) from raw = sum_j x_j c_j modulo 2^32 and xsum = sum_j x_j,
// x in [-128, 127], at most 131071 columns.  raw may pass 32 bits and is kept
// unsigned, which wraps; the sum about the codes' middle `mid` = 2^(bits - 1)
// fits them (131071 x 128 x 128 < 2^31), and the zero point's distance from the
// middle is added in 64 bits.
REALQ_ANYWHERE constexpr int64_t centred_sum(uint32_t raw, int32_t xsum, int32_t mid, int32_t z) {
    const int32_t about = static_cast<int32_t>(raw - static_cast<uint32_t>(mid) * static_cast<uint32_t>(xsum));
    return about + static_cast<int64_t>(mid - z) * xsum;
}

// One more share of a raw sum
REALQ_ANYWHERE constexpr uint32_t add_share(uint32_t raw, int32_t share) { return raw + static_cast<uint32_t>(share); }

}  // namespace realq
