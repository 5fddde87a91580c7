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

// 16 aligned bytes that are read once: they pass L1 by, which keeps what is read again.
__device__ __forceinline__ uint4 load_once(const uint8_t *p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}
// 16 aligned bytes, of which some may lie outside [lo, hi) (and read 0).
__device__ __forceinline__ uint4 load_piece(const uint8_t *p, const uint8_t *lo, const uint8_t *hi) {
    if (p >= lo && p + 16 <= hi) return load_once(p);
    uint32_t v[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (p + i >= lo && p + i < hi) v[i >> 2] |= (uint32_t)__ldg(p + i) << (8 * (i & 3));
    return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ uint4 shfl4(const uint4 &v, int src) {
    return make_uint4(__shfl_sync(0xFFFFFFFFu, v.x, src), __shfl_sync(0xFFFFFFFFu, v.y, src),
                      __shfl_sync(0xFFFFFFFFu, v.z, src), __shfl_sync(0xFFFFFFFFu, v.w, src));
}
// the 16 bytes from byte `mis` (0 to 15) on of the 32 in a, b
__device__ __forceinline__ uint4 realign(const uint4 &a, const uint4 &b, uint32_t mis) {
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t u[6], t[5];
#pragma unroll
    for (int i = 0; i < 6; ++i) u[i] = mis & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) t[i] = mis & 4 ? u[i + 1] : u[i];
    const uint32_t s = 8 * (mis & 3);
    return make_uint4(__funnelshift_r(t[0], t[1], s), __funnelshift_r(t[1], t[2], s), __funnelshift_r(t[2], t[3], s),
                      __funnelshift_r(t[3], t[4], s));
}
// A warp's consecutive 16 C bytes to a lane, at any address: lane l's begin at p
// = p(0) + 16 C l, all off the 16-byte boundary by the same amount.  Aligned
// pieces are loaded and the one that ends a lane's bytes comes from the next
// lane (`next`: that lane has bytes of its own).
template <int C>
__device__ __forceinline__ void load_chunks(const uint8_t *p, const uint8_t *lo, const uint8_t *hi, bool any, bool next,
                                            uint4 (&out)[C]) {
    const uint32_t mis = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15);
    uint4 ch[C + 1];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        ch[i] = make_uint4(0, 0, 0, 0);
        if (any) ch[i] = load_piece(p - mis + 16 * i, lo, hi);
    }
    ch[C] = shfl4(ch[0], ((threadIdx.x & 31) + 1) & 31);
    if (any && !next && mis) ch[C] = load_piece(p - mis + 16 * C, lo, hi);
#pragma unroll
    for (int i = 0; i < C; ++i) out[i] = realign(ch[i], ch[i + 1], mis);
}
__device__ __forceinline__ uint32_t byte_of(const uint4 &v, int b) {
    const uint32_t w = b < 8 ? (b < 4 ? v.x : v.y) : (b < 12 ? v.z : v.w);
    return (w >> (8 * (b & 3))) & 255u;
}
// The same in the other direction: the first `bytes` of a lane's 16 C go to p on
// (all lanes before `last` have all of theirs, those after it none).  Whole
// aligned pieces are stored, each by the lane in which it ends; the bytes before
// the warp's first and after its last one by a lane each.
template <int C>
__device__ __forceinline__ void store_chunks(uint8_t *p, const uint4 (&own)[C], int bytes, int last) {
    const int lane = threadIdx.x & 31, mis = (int)(reinterpret_cast<uintptr_t>(p) & 15), to = mis + bytes, end = to >> 4;
    const uint4 none = make_uint4(0, 0, 0, 0);
    uint4 before = shfl4(own[C - 1], (lane + 31) & 31), head = none, tail = none;
    uint8_t *a = p - mis;
#pragma unroll
    for (int j = 0; j <= C; ++j) {
        const uint4 cur = j < C ? own[j < C ? j : 0] : none;
        const uint4 v = mis ? realign(before, cur, 16 - mis) : cur;
        before = cur;
        if (j == 0) head = v;
        if (j == end) tail = v;
        if (j < C && j < end && bytes > 0 && (lane > 0 || j > 0 || mis == 0)) *reinterpret_cast<uint4 *>(a + 16 * j) = v;
    }
    uint8_t *first = a - 16 * C * lane;
    if (mis) {
        const uint4 v = shfl4(head, 0);
        const int to0 = __shfl_sync(0xFFFFFFFFu, to, 0);
        if (lane >= mis && lane < 16 && lane < to0) first[lane] = (uint8_t)byte_of(v, lane);
    }
    const uint4 v = shfl4(tail, last);
    const int tol = __shfl_sync(0xFFFFFFFFu, to, last);
    if (lane < (tol & 15) && !(mis && last == 0 && tol < 16))
        first[16 * C * last + (tol & ~15) + lane] = (uint8_t)byte_of(v, lane);
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
