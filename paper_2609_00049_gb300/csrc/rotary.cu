// Rotary positions: (a, b) -> amplitude (a cos t - b sin t, b cos t + a sin t)
// for the first rot_dim values of every head of queries and keys, t =
// position inv_freq[i]; the transpose (angle -t) is the gradient.
//
// Angle: the frequency in turns per position is kept as a 64-bit fraction of a
// turn, so that position x frequency modulo one turn is the low half of an
// integer product, exact for any position (in fp32 a position of 10^6 would be
// off by up to 0.06 radians).  Its error is that of the double frequency, 2^-53
// of the angle, and of the last conversion to fp32, 2^-25 of a half turn at
// most; sincospif gives the rest.
//
// Bound by memory: every value is read and written once.  A CTA forms the
// cosines and sines of its tokens once in shared memory (a double product, an
// integer one and a sincospif for each pair and token; a head would take as long
// for them as for its values) and goes over all heads of q and k with 16-byte
// accesses.  16384 tokens of 64 + 8 heads of 128 in bf16, forward and gradient: 197
// us, 6.1 TB/s, 0.91 of a copy's rate; 8 tokens: 2.7 us a launch.
#include <cmath>

#include "kernels.cuh"

namespace realq {
namespace {

constexpr int THREADS = 256;

// the angle's cosine and sine for a position and a frequency in radians per position
__device__ __forceinline__ float2 turn(int64_t position, double inv_freq, float amplitude, bool back) {
    double rev = inv_freq * 0.15915494309189533577;   // 1 / (2 pi)
    rev -= floor(rev);
    const uint64_t step = __double2ull_rz(rev * 18446744073709551616.0);
    const uint64_t at = (uint64_t)position * step;
    // the nearest half turn is at most half of one away: a signed fraction
    const float half_turns = (float)(int32_t)(uint32_t)(at >> 32) * 4.656612873077393e-10f;   // 2^-31
    float s, c;
    sincospif(half_turns, &s, &c);
    return make_float2(amplitude * c, back ? -amplitude * s : amplitude * s);
}

template <class T> struct Vec;   // 16 bytes
template <> struct Vec<float> {
    static constexpr int N = 4;
    float v[4];
    __device__ __forceinline__ void load(const float *p) {
        const float4 x = *reinterpret_cast<const float4 *>(p);
        v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
    }
    __device__ __forceinline__ void store(float *p) const {
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    float v[8];
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) {
        const uint4 x = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <class T> struct One {   // any alignment and size
    static constexpr int N = 1;
    float v[1];
    __device__ __forceinline__ void load(const T *p) { v[0] = load_as_float(p, 0); }
    __device__ __forceinline__ void store(float *p) const { *p = v[0]; }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *p = __float2bfloat16_rn(v[0]); }
};
__device__ __forceinline__ float2 rotate(float a, float b, float2 cs) {
    return make_float2(a * cs.x - b * cs.y, b * cs.x + a * cs.y);
}

// One CTA: `tokens` tokens from blockIdx.x on, the heads blockIdx.y of gridDim.y parts.
// An item is one access (two, with half pairs) of one head of one token.
template <class T, class V, bool IL>
__global__ void __launch_bounds__(THREADS) rotary_kernel(RotaryArgs a, int tokens) {
    extern __shared__ float2 cs[];   // tokens x pairs
    const int pairs = a.rot_dim / 2;
    const int64_t t0 = (int64_t)blockIdx.x * tokens;
    const int nt = (int)min((int64_t)tokens, a.T - t0);
    for (int i = threadIdx.x; i < nt * pairs; i += THREADS)
        cs[i] = turn(a.positions[t0 + i / pairs], a.inv_freq[i % pairs], a.amplitude, a.transpose);
    __syncthreads();
    const int heads = a.n_q + a.n_k;
    const int h0 = (int)((int64_t)heads * blockIdx.y / gridDim.y), nh = (int)((int64_t)heads * (blockIdx.y + 1) / gridDim.y) - h0;
    // rotated accesses of a head (with IL V = One takes a pair at a time), then the copied ones
    const int rot = IL ? (V::N == 1 ? pairs : a.rot_dim / V::N) : pairs / V::N;
    const int items = rot + (a.copy_rest ? (a.head_dim - a.rot_dim) / V::N : 0);
    for (int i = threadIdx.x; i < nt * nh * items; i += THREADS) {
        const int j = i % items, h = h0 + i / items % nh, tl = i / (items * nh);
        const bool is_q = h < a.n_q;
        const int64_t t = t0 + tl;
        const T *src = is_q ? (const T *)a.q + t * a.q_ld + h * a.q_hs : (const T *)a.k + t * a.k_ld + (h - a.n_q) * a.k_hs;
        T *dst = is_q ? (T *)a.q_out + t * a.qo_ld + h * a.qo_hs : (T *)a.k_out + t * a.ko_ld + (h - a.n_q) * a.ko_hs;
        const float2 *c = cs + tl * pairs;
        V x, y;
        if (j >= rot) {
            const int d = a.rot_dim + (j - rot) * V::N;
            x.load(src + d);
            x.store(dst + d);
        } else if constexpr (IL && V::N > 1) {
            x.load(src + j * V::N);
#pragma unroll
            for (int e = 0; e < V::N; e += 2) {
                const float2 r = rotate(x.v[e], x.v[e + 1], c[(j * V::N + e) / 2]);
                x.v[e] = r.x, x.v[e + 1] = r.y;
            }
            x.store(dst + j * V::N);
        } else {
            const int d = IL ? 2 * j : j * V::N, d2 = IL ? d + 1 : d + pairs;
            x.load(src + d);
            y.load(src + d2);
#pragma unroll
            for (int e = 0; e < V::N; ++e) {
                const float2 r = rotate(x.v[e], y.v[e], c[IL ? j : d + e]);
                x.v[e] = r.x, y.v[e] = r.y;
            }
            x.store(dst + d);
            y.store(dst + d2);
        }
    }
}

template <class T> realq_status_t launch(cudaStream_t s, const RotaryArgs &a, int sms) {
    constexpr int N = Vec<T>::N;
    const bool inter = a.interleaved;
    const auto whole = [](int64_t v) { return v % N == 0; };
    const auto fits = [&](const void *p, int64_t ld, int64_t hs, int heads) {
        return heads == 0 || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && whole(ld) && whole(hs));
    };
    const bool wide = whole(inter ? a.rot_dim : a.rot_dim / 2) && whole(a.head_dim) && whole(a.rot_dim) &&
                      fits(a.q, a.q_ld, a.q_hs, a.n_q) && fits(a.q_out, a.qo_ld, a.qo_hs, a.n_q) &&
                      fits(a.k, a.k_ld, a.k_hs, a.n_k) && fits(a.k_out, a.ko_ld, a.ko_hs, a.n_k);
    // four tokens to a CTA once there are enough for all SMs (16384 tokens of 72 heads, both ways: 197 us, 217 with one;
    // 2432: 41 and 45), one where there are not (200: 3.3 us, 3.7 with four), then parts of the heads
    const int tokens = a.T >= 16ll * sms ? 4 : 1;
    const int64_t gx = (a.T + tokens - 1) / tokens;
    int parts = 1;
    while (gx * parts < 2 * sms && parts * 4 <= a.n_q + a.n_k) parts *= 2;
    const dim3 grid((unsigned)gx, (unsigned)parts);
    const size_t smem = (size_t)tokens * (a.rot_dim / 2) * sizeof(float2);
    Launch l("rotary", s);
    if (wide) {
        if (inter)
            rotary_kernel<T, Vec<T>, true><<<grid, THREADS, smem, s>>>(a, tokens);
        else
            rotary_kernel<T, Vec<T>, false><<<grid, THREADS, smem, s>>>(a, tokens);
    } else {
        if (inter)
            rotary_kernel<T, One<T>, true><<<grid, THREADS, smem, s>>>(a, tokens);
        else
            rotary_kernel<T, One<T>, false><<<grid, THREADS, smem, s>>>(a, tokens);
    }
    return check_launch("rotary");
}

}  // namespace

realq_status_t rotary(cudaStream_t s, const RotaryArgs &a, realq_dtype_t dt, int sms) {
    return dt == REALQ_BF16 ? launch<__nv_bfloat16>(s, a, sms) : launch<float>(s, a, sms);
}

void rotary_frequencies(int64_t R, double base, int scaling, double factor, double context, double low, double high,
                        double *out) {
    const double pi2 = 6.283185307179586477;
    if (scaling == REALQ_ROPE_BASE && R > 2) base *= std::pow(factor, (double)R / (double)(R - 2));
    for (int64_t i = 0; i < R / 2; ++i) {
        double f = std::pow(base, -2.0 * (double)i / (double)R);
        if (scaling == REALQ_ROPE_LINEAR) f /= factor;
        if (scaling == REALQ_ROPE_RAMP) {
            const double r = context * f / pi2;
            if (r <= low)
                f /= factor;
            else if (r < high) {
                const double w = (r - low) / (high - low);
                f *= w + (1.0 - w) / factor;
            }
        }
        out[i] = f;
    }
}

}  // namespace realq
