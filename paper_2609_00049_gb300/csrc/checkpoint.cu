// Activation checkpoints in 8 bits: a layer's inputs X (T x n) kept for the
// backward pass as signed 8-bit codes with one power-of-two scale for each 32
// consecutive values of a token (the last block of a row may be shorter).
//
//   byte  b = biased fp32 exponent of the block's largest magnitude
//   code  q = clamp(rint(x 2^(133 - b)), -127, 127)
//   value x̂ = q 2^(b - 133)
//
// so the largest magnitude lies in [64, 128) steps, a value is off by at most
// half a step (a whole one where rounding would reach 128), and q with its
// sign fits bf16's eight significant bits: x̂ is a bf16 number and the
// products formed from it need no further rounding.  A block holding an
// infinity or a NaN gets byte 255 and reads back as NaN.
//
// Both directions read and write each byte once and are bound by HBM (16384 x
// 8192 in bf16: 64 us to pack, 6.3 TB/s; 58 us to unpack, 7.0 TB/s; in fp32 230
// us both ways, 5.9 TB/s).  A
// thread owns eight values (one 16-byte load of bf16, two of fp32) and four
// neighbouring lanes share a block, so its maximum takes two shuffles.  Widths
// that are not a multiple of 32 and unaligned buffers take 16 values to a lane
// and exchange aligned pieces between lanes.
#include "bytes.cuh"
#include "kernels.cuh"

namespace realq {
namespace {

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int THREADS = 256;
constexpr int UN = 2;   // groups of eight values per thread

__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }   // -126 <= e <= 127

// bits of |x|: ordered like the magnitudes, infinities and NaN above all numbers
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The code in the low byte.  x 2^(133 - b) in two exact steps (2^133 is no fp32
// number); adding 1.5 2^23 rounds it to the nearest even whole number, which
// then stands in the low mantissa bits.
__device__ __forceinline__ uint32_t code_of(float x, float s1, float s2) {
    const float y = fminf(fmaxf(x * s1 * s2, -127.f), 127.f);
    return __float_as_uint(__fadd_rn(y, 12582912.f));
}
__device__ __forceinline__ void scales_of(uint32_t b, float &s1, float &s2) {
    const int up = 133 - (int)b, h = up >> 1;
    s1 = pow2(h);
    s2 = pow2(up - h);
}
// 2^(b - 133), subnormal below b = 7; NaN for b = 255
__device__ __forceinline__ float step_of(uint32_t b) {
    if (b == 255u) return __int_as_float(0x7FC00000);
    return __uint_as_float(b >= 7u ? (b - 6u) << 23 : 1u << (b + 16u));
}

__device__ __forceinline__ void load8(const float *p, float (&v)[8]) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {   // every value is a bf16 number: the upper halves are exact
        w[i] = (__float_as_uint(v[2 * i]) >> 16) | (__float_as_uint(v[2 * i + 1]) & 0xFFFF0000u);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// Eight values of a thread and their way to codes.  bf16 stays in pairs up to
// the rounding (scaling by a power of two is exact in bf16 as well): taken one
// by one in fp32 the packing of bf16 was bound by its arithmetic (79 us for
// 16384 x 8192; 60 is HBM's share).
template <typename TX> struct Eight;
template <> struct Eight<float> {
    float v[8];
    __device__ __forceinline__ void load(const float *p) { load8(p, v); }
    __device__ __forceinline__ uint32_t top() const {   // bits of the largest magnitude
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, mag(v[i]));
        return m;
    }
    __device__ __forceinline__ uint2 codes(uint32_t b) const {
        float s1, s2;
        scales_of(b, s1, s2);
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) q[j] = code_of(v[4 * i + j], s1, s2);
            w[i] = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
        }
        return make_uint2(w[0], w[1]);
    }
};
template <> struct Eight<__nv_bfloat16> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        w[0] = a.x;
        w[1] = a.y;
        w[2] = a.z;
        w[3] = a.w;
    }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) m = __vmaxu2(m, w[i] & 0x7FFF7FFFu);
        return max(m << 16, m & 0xFFFF0000u);
    }
    __device__ __forceinline__ uint2 codes(uint32_t b) const {
        uint32_t out[2];
        if (b >= 6u) {
            const uint32_t s = (260u - b) << 7;   // 2^(133 - b)
            const __nv_bfloat162 scale = pair(s | s << 16), hi = pair(0x42FE42FEu), lo = pair(0xC2FEC2FEu);   // 127, -127
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t q[4];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const __nv_bfloat162 y = __hmin2(__hmax2(__hmul2(pair(w[2 * i + j]), scale), lo), hi);
                    const uint32_t u = *reinterpret_cast<const uint32_t *>(&y);
                    q[2 * j] = __float_as_uint(__fadd_rn(__uint_as_float(u << 16), 12582912.f));
                    q[2 * j + 1] = __float_as_uint(__fadd_rn(__uint_as_float(u & 0xFFFF0000u), 12582912.f));
                }
                out[i] = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
            }
        } else {   // 2^(133 - b) is no bf16 number
            Eight<float> f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f.v[2 * i] = __uint_as_float(w[i] << 16);
                f.v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
            return f.codes(b);
        }
        return make_uint2(out[0], out[1]);
    }
    static __device__ __forceinline__ __nv_bfloat162 pair(uint32_t u) { return *reinterpret_cast<__nv_bfloat162 *>(&u); }
};

// n a multiple of 32: rows end at block ends, so blocks are numbered through
// and a thread takes UN groups of eight values, a CTA's width apart, with all
// their loads in flight.
template <typename TX>
__global__ void __launch_bounds__(THREADS) pack_vec_kernel(int64_t groups, const TX *X, int8_t *codes, uint8_t *exps) {
    const int64_t g0 = (int64_t)blockIdx.x * (THREADS * UN) + threadIdx.x;
    Eight<TX> v[UN];
#pragma unroll
    for (int k = 0; k < UN; ++k)
        if (g0 + k * THREADS < groups) v[k].load(X + (g0 + k * THREADS) * 8);
#pragma unroll
    for (int k = 0; k < UN; ++k) {
        const int64_t g = g0 + k * THREADS;
        const bool in = g < groups;   // (4 groups a block: its lanes are all in or all out)
        uint32_t m = in ? v[k].top() : 0u;
        m = max(m, __shfl_xor_sync(FULL, m, 1));
        m = max(m, __shfl_xor_sync(FULL, m, 2));
        if (!in) continue;
        const uint32_t b = m >> 23;
        *reinterpret_cast<uint2 *>(codes + g * 8) = b < 255u ? v[k].codes(b) : make_uint2(0, 0);
        if ((threadIdx.x & 3) == 0) exps[g >> 2] = (uint8_t)b;
    }
}

template <typename TX>
__global__ void __launch_bounds__(THREADS) unpack_vec_kernel(int64_t groups, const int8_t *codes, const uint8_t *exps,
                                                             TX *X) {
    const int64_t g0 = (int64_t)blockIdx.x * (THREADS * UN) + threadIdx.x;
    uint2 w[UN];
    uint32_t b[UN];
#pragma unroll
    for (int k = 0; k < UN; ++k) {
        const int64_t g = g0 + k * THREADS;
        if (g < groups) {
            w[k] = __ldg(reinterpret_cast<const uint2 *>(codes) + g);
            b[k] = __ldg(exps + (g >> 2));
        }
    }
#pragma unroll
    for (int k = 0; k < UN; ++k) {
        const int64_t g = g0 + k * THREADS;
        if (g >= groups) continue;
        const float s = step_of(b[k]);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)((i < 4 ? w[k].x : w[k].y) >> (8 * (i & 3))) * s;
        store8(X + g * 8, v);
    }
}

// Any width and alignment: a warp takes segments of 16 neighbouring blocks of a
// row (nw to a row), a lane half a block.  Rows then begin at any address; aligned pieces
// are exchanged between neighbouring lanes (bytes.cuh).
__device__ __forceinline__ void take(Eight<float> (&v)[2], const uint4 (&q)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i >> 1].v[(i & 1) * 4] = __uint_as_float(q[i].x);
        v[i >> 1].v[(i & 1) * 4 + 1] = __uint_as_float(q[i].y);
        v[i >> 1].v[(i & 1) * 4 + 2] = __uint_as_float(q[i].z);
        v[i >> 1].v[(i & 1) * 4 + 3] = __uint_as_float(q[i].w);
    }
}
__device__ __forceinline__ void take(Eight<__nv_bfloat16> (&v)[2], const uint4 (&q)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[i].w[0] = q[i].x;
        v[i].w[1] = q[i].y;
        v[i].w[2] = q[i].z;
        v[i].w[3] = q[i].w;
    }
}
// values from the count-th on are zero
__device__ __forceinline__ void cut(Eight<float> &v, int count) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i >= count) v.v[i] = 0.f;
}
__device__ __forceinline__ void cut(Eight<__nv_bfloat16> &v, int count) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v.w[i] &= 2 * i + 1 < count ? ~0u : (2 * i < count ? 0xFFFFu : 0u);
}
__device__ __forceinline__ void give(const float (&v)[16], uint4 (&q)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        q[i] = make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]),
                          __float_as_uint(v[4 * i + 3]));
}
__device__ __forceinline__ void give(const float (&v)[16], uint4 (&q)[2]) {   // (bf16 numbers: their upper halves)
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __byte_perm(__float_as_uint(v[2 * i]), __float_as_uint(v[2 * i + 1]), 0x7632);
    q[0] = make_uint4(w[0], w[1], w[2], w[3]);
    q[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

// A lane's share of segment w (512 values of a row): its row, first column and
// count of values, and the last lane that has any.  (Two segments to a warp were
// slower: 140 us for 8192 x 8191 in bf16 both ways, against 124.)
struct Share {
    int64_t t, c;
    int count, last;
    bool next;
    __device__ __forceinline__ Share(int64_t w, int64_t n, int64_t nw) {
        const int lane = threadIdx.x & 31;
        t = divide(w, nw, c);
        const int64_t left = n - c * 512;   // values of the segment and what follows it, at least one
        c = c * 512 + lane * 16;
        count = (int)max((int64_t)0, min((int64_t)16, left - lane * 16));
        last = (int)min((int64_t)31, (left - 1) / 16);
        next = lane < last;
    }
};

template <typename TX>
__global__ void __launch_bounds__(THREADS) pack_row_kernel(int64_t T, int64_t n, int64_t nw, const TX *X,
                                                           int8_t *codes, uint8_t *exps) {
    constexpr int C = sizeof(TX);   // 16-byte pieces of 16 values
    const int64_t w = ((int64_t)blockIdx.x * THREADS + threadIdx.x) >> 5;
    if (w >= T * nw) return;
    const Share h(w, n, nw);
    const uint8_t *lo = reinterpret_cast<const uint8_t *>(X);
    uint4 q[C];
    load_chunks<C>(lo + (h.t * n + h.c) * C, lo, lo + T * n * C, h.count > 0, h.next, q);
    Eight<TX> v[2];
    take(v, q);
    if (h.count < 16) {
        cut(v[0], h.count);
        cut(v[1], h.count - 8);
    }
    uint32_t m = max(v[0].top(), v[1].top());
    m = max(m, __shfl_xor_sync(FULL, m, 1));
    const uint32_t b = m >> 23;
    uint4 out[1] = {make_uint4(0, 0, 0, 0)};
    if (b < 255u) {
        const uint2 a = v[0].codes(b), d = v[1].codes(b);
        out[0] = make_uint4(a.x, a.y, d.x, d.y);
    }
    store_chunks<1>(reinterpret_cast<uint8_t *>(codes) + h.t * n + h.c, out, h.count, h.last);
    if ((threadIdx.x & 1) == 0 && h.count > 0) exps[h.t * ((n + 31) / 32) + h.c / 32] = (uint8_t)b;
}

template <typename TX>
__global__ void __launch_bounds__(THREADS) unpack_row_kernel(int64_t T, int64_t n, int64_t nw, const int8_t *codes,
                                                             const uint8_t *exps, TX *X) {
    constexpr int C = sizeof(TX);
    const int64_t w = ((int64_t)blockIdx.x * THREADS + threadIdx.x) >> 5;
    if (w >= T * nw) return;
    const Share h(w, n, nw);
    const uint8_t *lo = reinterpret_cast<const uint8_t *>(codes);
    const float s = h.count > 0 ? step_of(__ldg(exps + h.t * ((n + 31) / 32) + h.c / 32)) : 0.f;
    uint4 q[1];
    load_chunks<1>(lo + h.t * n + h.c, lo, lo + T * n, h.count > 0, h.next, q);
    const uint32_t u[4] = {q[0].x, q[0].y, q[0].z, q[0].w};
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = (float)(int8_t)(u[i >> 2] >> (8 * (i & 3))) * s;
    uint4 out[C];
    give(v, out);
    store_chunks<C>(reinterpret_cast<uint8_t *>(X) + (h.t * n + h.c) * C, out, h.count * C, h.last);
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

template <typename TX>
static void pack_launch(cudaStream_t s, int64_t T, int64_t n, const TX *X, int8_t *codes, uint8_t *exps) {
    const int64_t nw = (n + 511) / 512, groups = T * n / 8;
    Launch L("checkpoint_pack", s);
    if (n % 32 == 0 && aligned16(X) && aligned16(codes))
        pack_vec_kernel<TX><<<(unsigned)((groups + THREADS * UN - 1) / (THREADS * UN)), THREADS, 0, s>>>(groups, X, codes, exps);
    else
        pack_row_kernel<TX><<<(unsigned)((T * nw * 32 + THREADS - 1) / THREADS), THREADS, 0, s>>>(T, n, nw, X, codes,
                                                                                                  exps);
}

template <typename TX>
static void unpack_launch(cudaStream_t s, int64_t T, int64_t n, const int8_t *codes, const uint8_t *exps, TX *X) {
    const int64_t nw = (n + 511) / 512, groups = T * n / 8;
    Launch L("checkpoint_unpack", s);
    if (n % 32 == 0 && aligned16(X) && aligned16(codes))
        unpack_vec_kernel<TX><<<(unsigned)((groups + THREADS * UN - 1) / (THREADS * UN)), THREADS, 0, s>>>(groups, codes, exps, X);
    else
        unpack_row_kernel<TX><<<(unsigned)((T * nw * 32 + THREADS - 1) / THREADS), THREADS, 0, s>>>(T, n, nw, codes,
                                                                                                    exps, X);
}

realq_status_t checkpoint_pack(cudaStream_t s, int64_t T, int64_t n, const void *X, realq_dtype_t dt, int8_t *codes,
                               uint8_t *exps) {
    if (dt == REALQ_BF16)
        pack_launch(s, T, n, static_cast<const __nv_bfloat16 *>(X), codes, exps);
    else
        pack_launch(s, T, n, static_cast<const float *>(X), codes, exps);
    return check_launch("checkpoint_pack");
}

realq_status_t checkpoint_unpack(cudaStream_t s, int64_t T, int64_t n, const int8_t *codes, const uint8_t *exps,
                                 void *X, realq_dtype_t dt) {
    if (dt == REALQ_BF16)
        unpack_launch(s, T, n, codes, exps, static_cast<__nv_bfloat16 *>(X));
    else
        unpack_launch(s, T, n, codes, exps, static_cast<float *>(X));
    return check_launch("checkpoint_unpack");
}

}  // namespace realq
