// Into and out of the 8-bit key/value cache: values are kept as
// scale (code - 128) with one scale for each block of tokens and head.
//
// Appending: a warp takes one block of one head of keys or values, reads its new
// values twice (their largest magnitude, then the codes: the second reading
// comes from the L1), and brings the codes that were there to the new scale
// where that grew.  Which block a warp has follows from its number alone: the
// blocks that sequence s touches are at most n / block + 2 for its n tokens, so
// numbers from starts[s] / block + 2 s on are free for them, and the sequence is
// found by bisection.
//
// Bound by memory: the new values are read and their codes written once.
#include "kernels.cuh"

namespace realq {
namespace {

constexpr int WARPS = 4;

// the last sequence s with key(s) <= i, key not decreasing
template <class Key> __device__ __forceinline__ int last_at_most(int n, int64_t i, Key key) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (key(mid) <= i)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

template <class T, int N> struct Piece {   // N values at a time
    __device__ static void load(const T *p, float (&v)[N]) {
        if constexpr (N == 1) {
            v[0] = load_as_float(p, 0);
        } else if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const float4 x = *reinterpret_cast<const float4 *>(p + i);
                v[i] = x.x, v[i + 1] = x.y, v[i + 2] = x.z, v[i + 3] = x.w;
            }
        } else {
            const uint4 x = *reinterpret_cast<const uint4 *>(p);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    __device__ static void store(T *p, const float (&v)[N]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; i += 4)
                *reinterpret_cast<float4 *>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
            *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
};

__device__ __forceinline__ uint32_t code_of(float x, float scale) {
    const float q = fminf(fmaxf(rintf(__fdiv_rn(x, scale)), -127.f), 127.f);
    return (uint32_t)((int)q + 128);
}

template <class T, int N>
__global__ void __launch_bounds__(32 * WARPS) append_kernel(KvAppendArgs a, int64_t units) {
    const int lane = threadIdx.x & 31;
    const int64_t unit = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5);
    if (unit >= units) return;
    const int per = 2 * a.c.n_kv, block = 1 << a.c.log_block;
    const int which = (int)(unit % per), head = which >> 1;
    const int64_t i = unit / per;
    const auto key = [&](int s) { return (int64_t)(a.starts[s] >> a.c.log_block) + 2ll * s; };
    const int s = last_at_most(a.n_seqs, i, key);
    const int64_t b = a.starts[s], e = a.starts[s + 1];
    if (b < 0 || e <= b || e > a.T) return;
    const int64_t first = a.positions[b];
    if (first < 0) return;
    const int64_t blk = (first >> a.c.log_block) + (i - key(s));   // of the sequence
    const int64_t p0 = blk << a.c.log_block;
    const int64_t from = max(first, p0), to = min(first + (e - b), p0 + block);
    if (i < key(s) || from >= to) return;
    const int64_t pi = p0 >> a.c.log_page;
    if (pi >= a.max_pages) return;
    const int pg = a.tables[s * a.max_pages + pi];
    if (pg < 0 || pg >= a.c.n_pages) return;

    const int D = a.c.head_dim;
    const int64_t tile = (int64_t)pg * a.c.n_kv + head;   // a page's tokens of one head
    const int place = (int)(p0 & ((1 << a.c.log_page) - 1));
    uint8_t *codes = ((which & 1) ? a.c.v_codes : a.c.k_codes) + ((tile << a.c.log_page) + place) * D;
    float *scale_at = ((which & 1) ? a.c.v_scale : a.c.k_scale) + (tile << (a.c.log_page - a.c.log_block)) + (place >> a.c.log_block);
    const int64_t ld = (which & 1) ? a.v_ld : a.k_ld, hs = (which & 1) ? a.v_hs : a.k_hs;
    const T *x = (const T *)((which & 1) ? a.v : a.k) + (b + (from - first)) * ld + head * hs;
    const int old = (int)(from - p0), cnt = (int)(to - from), row = D / N;

    uint32_t top = 0;   // of |x|, as bits: a NaN is above every number
    for (int j = lane; j < cnt * row; j += 32) {
        float v[N];
        Piece<T, N>::load(x + (int64_t)(j / row) * ld + (j % row) * N, v);
#pragma unroll
        for (int k = 0; k < N; ++k) top = max(top, __float_as_uint(v[k]) & 0x7FFFFFFFu);
    }
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    const float before = old > 0 ? *scale_at : 0.f;
    const bool bad = top >= 0x7F800000u || before != before;
    const float nan = __uint_as_float(0x7FC00000u);
    const float scale = bad ? nan : fmaxf(before, __fdiv_rn(__uint_as_float(top), 127.f));
    __syncwarp();
    if (lane == 0 && (old == 0 || !(scale == before))) *scale_at = scale;

    if (!bad && scale > before && before > 0.f) {   // what was there, in the new steps
        const float ratio = __fdiv_rn(before, scale);
        for (int j = lane; j < old * D / 16; j += 32) {
            uint4 *at = reinterpret_cast<uint4 *>(codes) + j;
            const uint4 w4 = *at;
            uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t r = 0;
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const float c = (float)((int)((w[k] >> (8 * m)) & 255u) - 128);
                    r |= (uint32_t)((int)rintf(__fmul_rn(c, ratio)) + 128) << (8 * m);
                }
                w[k] = r;
            }
            *at = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    uint8_t *out = codes + (int64_t)old * D;
    for (int j = lane; j < cnt * row; j += 32) {
        float v[N];
        Piece<T, N>::load(x + (int64_t)(j / row) * ld + (j % row) * N, v);
        if constexpr (N == 8) {
            uint32_t w[2] = {0, 0};
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k >> 2] |= (scale > 0.f ? code_of(v[k], scale) : 128u) << (8 * (k & 3));
            *reinterpret_cast<uint2 *>(out + (int64_t)j * 8) = make_uint2(w[0], w[1]);
        } else {
            out[j] = (uint8_t)(scale > 0.f ? code_of(v[0], scale) : 128u);
        }
    }
}

// a warp takes one token's keys or values of one head, 16 values to a lane
template <class T>
__global__ void __launch_bounds__(32 * WARPS) read_kernel(KvReadArgs a, int64_t units) {
    const int D = a.c.head_dim, lanes = D / 16;
    const int64_t i = (int64_t)blockIdx.x * (32 * WARPS) + threadIdx.x;
    if (i >= units * lanes) return;
    const int64_t unit = i / lanes;
    const int c = (int)(i % lanes), head = (int)(unit % a.c.n_kv);
    const int64_t t = unit / a.c.n_kv;
    const int s = last_at_most(a.n_seqs, t, [&](int q) { return (int64_t)a.starts[q]; });
    if (a.starts[s] < 0 || t < a.starts[s] || t >= a.starts[s + 1]) return;
    const int64_t p = a.positions[t], pi = p >> a.c.log_page;
    int pg = -1;
    if (p >= 0 && pi < a.max_pages) pg = a.tables[s * a.max_pages + pi];
    const bool there = pg >= 0 && pg < a.c.n_pages;
    const int64_t tile = (int64_t)pg * a.c.n_kv + head;
    const int place = (int)(p & ((1 << a.c.log_page) - 1));
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        T *out = (T *)(w ? a.v_out : a.k_out);
        if (out == nullptr) continue;
        float v[16], scale = __uint_as_float(0x7FC00000u);
        uint4 q = make_uint4(0, 0, 0, 0);
        if (there) {
            q = *reinterpret_cast<const uint4 *>((w ? a.c.v_codes : a.c.k_codes) + ((tile << a.c.log_page) + place) * D + 16 * c);
            scale = ((w ? a.c.v_scale : a.c.k_scale) + (tile << (a.c.log_page - a.c.log_block)))[place >> a.c.log_block];
        }
        const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = (float)((int)((u[k >> 2] >> (8 * (k & 3))) & 255u) - 128) * scale;
        out += unit * D + 16 * c;
        if (a.wide) {
            constexpr int N = 16 / sizeof(T);
#pragma unroll
            for (int k = 0; k < 16; k += N) {
                float r[N];
#pragma unroll
                for (int m = 0; m < N; ++m) r[m] = v[k + m];
                Piece<T, N>::store(out + k, r);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                if constexpr (sizeof(T) == 4)
                    out[k] = v[k];
                else
                    out[k] = __float2bfloat16_rn(v[k]);
            }
        }
    }
}

}  // namespace

realq_status_t kv_append(cudaStream_t s, const KvAppendArgs &a, realq_dtype_t dt) {
    const int64_t slots = (a.T >> a.c.log_block) + 2ll * a.n_seqs;
    const int64_t units = slots * 2 * a.c.n_kv;
    const auto even = [&](const void *p, int64_t ld, int64_t hs) {
        return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && hs % 8 == 0;
    };
    const bool wide = even(a.k, a.k_ld, a.k_hs) && even(a.v, a.v_ld, a.v_hs);
    const unsigned grid = (unsigned)((units + WARPS - 1) / WARPS);
    Launch l("kv_append", s);
    if (dt == REALQ_BF16) {
        if (wide)
            append_kernel<__nv_bfloat16, 8><<<grid, 32 * WARPS, 0, s>>>(a, units);
        else
            append_kernel<__nv_bfloat16, 1><<<grid, 32 * WARPS, 0, s>>>(a, units);
    } else {
        if (wide)
            append_kernel<float, 8><<<grid, 32 * WARPS, 0, s>>>(a, units);
        else
            append_kernel<float, 1><<<grid, 32 * WARPS, 0, s>>>(a, units);
    }
    return check_launch("kv_append");
}

realq_status_t kv_read(cudaStream_t s, const KvReadArgs &args, realq_dtype_t dt) {
    KvReadArgs a = args;
    const int64_t units = a.T * a.c.n_kv, threads = units * (a.c.head_dim / 16);
    a.wide = ((reinterpret_cast<uintptr_t>(a.k_out) | reinterpret_cast<uintptr_t>(a.v_out)) & 15) == 0;
    const unsigned grid = (unsigned)((threads + 32 * WARPS - 1) / (32 * WARPS));
    Launch l("kv_read", s);
    if (dt == REALQ_BF16)
        read_kernel<__nv_bfloat16><<<grid, 32 * WARPS, 0, s>>>(a, units);
    else
        read_kernel<float><<<grid, 32 * WARPS, 0, s>>>(a, units);
    return check_launch("kv_read");
}

}  // namespace realq
