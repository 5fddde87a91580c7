// Bytes at any address, for rows whose width is no multiple of a load's.
#pragma once

#include "common.cuh"

namespace realq {

// 16 bytes from p on, those from `hi` on zero: aligned words where they lie
// inside [lo, hi), else single bytes.
__device__ __forceinline__ uint4 load16(const uint8_t *p, const uint8_t *lo, const uint8_t *hi) {
    const uint32_t mis = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 3);
    const uint8_t *a = p - mis;
    uint32_t v[4] = {0, 0, 0, 0};
    if (a >= lo && a + 20 <= hi) {
        uint32_t w[5];
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = __ldg(reinterpret_cast<const uint32_t *>(a) + i);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __funnelshift_r(w[i], w[i + 1], 8 * mis);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (p + i < hi) v[i >> 2] |= (uint32_t)__ldg(p + i) << (8 * (i & 3));
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// quotient and remainder, by 32-bit arithmetic where that is enough
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b, int64_t &rem) {
    if (((a | b) >> 32) == 0) {
        const uint32_t q = (uint32_t)a / (uint32_t)b;
        rem = (uint32_t)a - q * (uint32_t)b;
        return q;
    }
    const int64_t q = a / b;
    rem = a - q * b;
    return q;
}

}  // namespace realq
