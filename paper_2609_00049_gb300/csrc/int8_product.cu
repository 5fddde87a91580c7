// Y = diag(x_scale) (Xc - 128) (Wc - z)^T diag(w_scale): 8-bit token codes
// (T x n) times 8- or 4-bit channel codes (m x n), the product of the
// weight-activation setting run on the codes themselves.
//
// The sum over j is a whole number; the two scales are applied to it in fp32
// and the result is rounded once to Y's type.
//
// Streaming kernel (few tokens): bound by reading the weight codes once from
// HBM.  A warp owns R rows of W and up to eight tokens; each lane multiplies
// 16 bytes of codes at a time with dp4a, unsigned weight codes times signed
// token codes, exact in 32-bit integers; the zero point enters once per row:
// sum_j (w - z) x = sum_j w x - z sum_j x.  Integer sums do not depend on their
// order, so the warps of a row are joined through shared memory in any.
#include "kernels.cuh"

namespace realq {
namespace {

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int SW = 8;   // warps of a streaming CTA

__device__ __forceinline__ int dp4a_us(uint32_t a, uint32_t b, int c) {   // unsigned a, signed b
    int d;
    asm("dp4a.u32.s32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// Four code bytes at any address inside [lo, hi): two aligned words where they
// lie inside, else single bytes.
__device__ __forceinline__ uint32_t load_word(const uint8_t *p, const uint8_t *lo, const uint8_t *hi) {
    const uint32_t mis = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 3);
    const uint8_t *a = p - mis;
    if (mis == 0 && p + 4 <= hi) return __ldg(reinterpret_cast<const uint32_t *>(p));
    if (a >= lo && a + 8 <= hi) {
        const uint32_t w0 = __ldg(reinterpret_cast<const uint32_t *>(a));
        const uint32_t w1 = __ldg(reinterpret_cast<const uint32_t *>(a) + 1);
        return __funnelshift_r(w0, w1, 8 * mis);
    }
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (p + i < hi) w |= (uint32_t)__ldg(p + i) << (8 * i);
    return w;
}

// One word of weight codes times a token's codes.  8 bits: x[0] holds the four
// token codes; 4 bits: x[0] those of the even, x[1] those of the odd columns.
template <int WB>
__device__ __forceinline__ int mac(uint32_t w, const uint32_t (&x)[WB == 8 ? 1 : 2], int acc) {
    if constexpr (WB == 8) {
        return dp4a_us(w, x[0], acc);
    } else {
        return dp4a_us((w >> 4) & 0x0F0F0F0Fu, x[1], dp4a_us(w & 0x0F0F0F0Fu, x[0], acc));
    }
}
template <int WB>
__device__ __forceinline__ int sum_codes(const uint32_t (&x)[WB == 8 ? 1 : 2], int acc) {
    acc = dp4a_us(0x01010101u, x[0], acc);
    if constexpr (WB == 4) acc = dp4a_us(0x01010101u, x[1], acc);
    return acc;
}
// token codes as signed bytes in the order mac() takes them
template <int WB>
__device__ __forceinline__ void token_codes(const uint32_t *raw, uint32_t (&x)[WB == 8 ? 1 : 2]) {
    if constexpr (WB == 8) {
        x[0] = raw[0] ^ 0x80808080u;
    } else {
        x[0] = __byte_perm(raw[0], raw[1], 0x6420) ^ 0x80808080u;
        x[1] = __byte_perm(raw[0], raw[1], 0x7531) ^ 0x80808080u;
    }
}

// ALIGNED: rows of whole 16-byte vectors (n a multiple of 16, or of 32 for 4
// bits, and 16-byte aligned buffers).  Otherwise rows are walked in aligned
// 4-byte words, their first and last bytes singly; a warp's rows lie four
// apart, so they share their offset from the word boundary and with it the
// (unaligned) token words.
template <bool ALIGNED, int WB, int TT, int R, typename TY>
__global__ void __launch_bounds__(SW * 32)
    int8_stream_kernel(int64_t T, int64_t n, int64_t m, int kw, const uint8_t *X, const float *x_scale,
                       const uint8_t *W, const float *w_scale, const uint8_t *w_zero, TY *Y) {
    constexpr int XW = WB == 8 ? 1 : 2;
    __shared__ int part[SW][R * TT + TT];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = warp / kw, kpart = warp % kw, groups = SW / kw;
    const int64_t t0 = (int64_t)blockIdx.y * TT;
    const int64_t rb = WB == 8 ? n : (n + 1) / 2;   // bytes of a row of W
    // row of (group, j)
    const int64_t rbase = (int64_t)blockIdx.x * groups * R;
    auto row_of = [&](int j) -> int64_t {
        if (ALIGNED || R == 1) return rbase + group * R + j;
        return rbase + (group & 3) + 4 * (j + (int64_t)R * (group >> 2));   // groups is a multiple of 4 here
    };
    int acc[R][TT], xs[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        xs[t] = 0;
#pragma unroll
        for (int j = 0; j < R; ++j) acc[j][t] = 0;
    }
    const uint8_t *wrow[R];
#pragma unroll
    for (int j = 0; j < R; ++j)   // rows past m repeat the warp's first (same offset from the word boundary), unwritten
        wrow[j] = W + (row_of(j) < m ? row_of(j) : (row_of(0) < m ? row_of(0) : 0)) * rb;
    const uint8_t *xrow[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) xrow[t] = X + (t0 + t < T ? t0 + t : T - 1) * n;

    if constexpr (ALIGNED) {
        const int nv = (int)(rb / 16);
#pragma unroll 2
        for (int v = kpart * 32 + lane; v < nv; v += kw * 32) {
            uint32_t w[R][4];
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const uint4 q = __ldg(reinterpret_cast<const uint4 *>(wrow[j]) + v);
                w[j][0] = q.x; w[j][1] = q.y; w[j][2] = q.z; w[j][3] = q.w;
            }
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                uint32_t raw[4 * XW];
#pragma unroll
                for (int h = 0; h < XW; ++h) {
                    const uint4 q = __ldg(reinterpret_cast<const uint4 *>(xrow[t]) + v * XW + h);
                    raw[4 * h] = q.x; raw[4 * h + 1] = q.y; raw[4 * h + 2] = q.z; raw[4 * h + 3] = q.w;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t x[XW];
                    token_codes<WB>(raw + i * XW, x);
                    xs[t] = sum_codes<WB>(x, xs[t]);
#pragma unroll
                    for (int j = 0; j < R; ++j) acc[j][t] = mac<WB>(w[j][i], x, acc[j][t]);
                }
            }
        }
    } else {
        const uint8_t *xlo = X, *xhi = X + T * n;
        const int mis = (int)(reinterpret_cast<uintptr_t>(wrow[0]) & 3);
        const int64_t head = mis ? (4 - mis < rb ? 4 - mis : rb) : 0;
        const int64_t nw = (rb - head) / 4, tail = rb - head - 4 * nw;
        for (int64_t v = kpart * 32 + lane; v < nw; v += kw * 32) {
            uint32_t w[R];
#pragma unroll
            for (int j = 0; j < R; ++j) w[j] = __ldg(reinterpret_cast<const uint32_t *>(wrow[j] + head) + v);
            const int64_t c = (head + 4 * v) * XW;   // first column
            const bool last = WB == 4 && c + 8 > n;   // the byte of an odd width's last column holds one code
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                uint32_t raw[XW], x[XW];
#pragma unroll
                for (int h = 0; h < XW; ++h) raw[h] = load_word(xrow[t] + c + 4 * h, xlo, xhi);
                token_codes<WB>(raw, x);
                if (last) x[XW - 1] &= 0x00FFFFFFu;
                xs[t] = sum_codes<WB>(x, xs[t]);
#pragma unroll
                for (int j = 0; j < R; ++j) acc[j][t] = mac<WB>(w[j], x, acc[j][t]);
            }
        }
        // head and tail bytes, one to a lane of the first K part
        if (kpart == 0 && lane < head + tail) {
            const int64_t b = lane < head ? lane : rb - tail + (lane - head);
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int h = 0; h < XW; ++h) {
                    const int64_t c = b * XW + h;
                    if (c < n) {
                        const int xv = (int)__ldg(xrow[t] + c) - 128;
                        xs[t] += xv;
#pragma unroll
                        for (int j = 0; j < R; ++j) {
                            const int wv = __ldg(wrow[j] + b);
                            acc[j][t] += (WB == 8 ? wv : (h ? wv >> 4 : wv & 15)) * xv;
                        }
                    }
                }
        }
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        xs[t] = __reduce_add_sync(FULL, xs[t]);
#pragma unroll
        for (int j = 0; j < R; ++j) acc[j][t] = __reduce_add_sync(FULL, acc[j][t]);
    }
    if (kw > 1) {
        if (lane == 0) {
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                part[warp][R * TT + t] = xs[t];
#pragma unroll
                for (int j = 0; j < R; ++j) part[warp][j * TT + t] = acc[j][t];
            }
        }
        __syncthreads();
        if (kpart != 0) return;
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            for (int p = 1; p < kw; ++p) xs[t] += part[warp + p][R * TT + t];
#pragma unroll
            for (int j = 0; j < R; ++j)
                for (int p = 1; p < kw; ++p) acc[j][t] += part[warp + p][j * TT + t];
        }
    }
    // lane j TT + t writes (row j, token t)
    static_assert(R * TT <= 32, "one result to a lane");
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
        for (int t = 0; t < TT; ++t)
            if (lane == j * TT + t) {
                const int64_t i = row_of(j), tok = t0 + t;
                if (i < m && tok < T) {
                    const int z = w_zero ? w_zero[i] : (WB == 8 ? 128 : 8);
                    // (mod 2^32: the true sum fits, its two parts need not)
                    const int v = (int)((uint32_t)acc[j][t] - (uint32_t)z * (uint32_t)xs[t]);
                    store1(Y + tok * m + i, (float)v * x_scale[tok] * w_scale[i]);
                }
            }
}

template <bool ALIGNED, int WB, int TT, int R, typename TY>
realq_status_t stream_launch(cudaStream_t s, int64_t T, int64_t n, int64_t m, const uint8_t *X, const float *xs,
                             const uint8_t *W, const float *ws, const uint8_t *wz, TY *Y, int sms) {
    // Warps per group of R rows: as many as it takes to put 16 warps on each
    // SM, but no more than leave each its own 512-byte step of K.
    const int64_t rb = WB == 8 ? n : (n + 1) / 2;
    int kw = 1;
    const int kmax = ALIGNED || R == 1 ? SW : 2;   // (the unaligned rows need four groups per CTA)
    const int64_t ygroups = (T + TT - 1) / TT;
    while (kw < kmax && (m + R - 1) / R * kw * ygroups < (int64_t)sms * 16 && rb > 512 * kw) kw *= 2;
    const int64_t rows = (int64_t)(SW / kw) * R;
    {
        Launch L("int8_product_stream", s);
        int8_stream_kernel<ALIGNED, WB, TT, R, TY>
            <<<dim3((unsigned)((m + rows - 1) / rows), (unsigned)ygroups), SW * 32, 0, s>>>(T, n, m, kw, X, xs, W, ws,
                                                                                          wz, Y);
    }
    return check_launch("int8_product_stream");
}

template <bool ALIGNED, int WB, typename TY>
realq_status_t stream_tokens(cudaStream_t s, int64_t T, int64_t n, int64_t m, const uint8_t *X, const float *xs,
                             const uint8_t *W, const float *ws, const uint8_t *wz, TY *Y, int sms) {
    if (T == 1) {
        if (m < (int64_t)sms * 64) return stream_launch<ALIGNED, WB, 1, 1, TY>(s, T, n, m, X, xs, W, ws, wz, Y, sms);
        return stream_launch<ALIGNED, WB, 1, 4, TY>(s, T, n, m, X, xs, W, ws, wz, Y, sms);
    }
    if (T == 2) return stream_launch<ALIGNED, WB, 2, 4, TY>(s, T, n, m, X, xs, W, ws, wz, Y, sms);
    if (T <= 4) return stream_launch<ALIGNED, WB, 4, 4, TY>(s, T, n, m, X, xs, W, ws, wz, Y, sms);
    return stream_launch<ALIGNED, WB, 8, 4, TY>(s, T, n, m, X, xs, W, ws, wz, Y, sms);
}

template <int WB, typename TY>
realq_status_t stream(cudaStream_t s, int64_t T, int64_t n, int64_t m, const uint8_t *X, const float *xs,
                      const uint8_t *W, const float *ws, const uint8_t *wz, TY *Y, int sms) {
    const bool aligned = n % (WB == 8 ? 16 : 32) == 0 &&
                         ((reinterpret_cast<uintptr_t>(X) | reinterpret_cast<uintptr_t>(W)) & 15) == 0;
    return aligned ? stream_tokens<true, WB, TY>(s, T, n, m, X, xs, W, ws, wz, Y, sms)
                   : stream_tokens<false, WB, TY>(s, T, n, m, X, xs, W, ws, wz, Y, sms);
}

}  // namespace

constexpr int64_t STREAM_T = 8;   // tokens up to which the streaming kernel runs

size_t int8_product_ws_bytes(int64_t T, int64_t n, int64_t m, int w_bits, int sms) {
    return T <= STREAM_T ? 256 : int8_tc_ws_bytes(T, n, m, w_bits, sms);
}

realq_status_t int8_product(cudaStream_t s, int64_t T, int64_t n, int64_t m, const uint8_t *X, const float *x_scale,
                            const uint8_t *W, int w_bits, const float *w_scale, const uint8_t *w_zero, void *Y,
                            realq_dtype_t y_dtype, void *ws, int sms) {
    if (T > STREAM_T) {
        const int64_t rb = w_bits == 8 ? n : (n + 1) / 2;
        // (whole rows at an odd address go through the streaming kernel, eight tokens at a time)
        if (rb % 16 || (reinterpret_cast<uintptr_t>(W) & 15) == 0)
            return int8_product_tc(s, T, n, m, X, x_scale, W, w_bits, w_scale, w_zero, Y, y_dtype, ws, sms);
        if (T > 65535 * STREAM_T)
            return fail(REALQ_ERR_UNSUPPORTED, "int8_product: more than %lld tokens need 16-byte aligned W_codes",
                        (long long)(65535 * STREAM_T));
    }
    auto run = [&](auto *y) {
        return w_bits == 8 ? stream<8>(s, T, n, m, X, x_scale, W, w_scale, w_zero, y, sms)
                           : stream<4>(s, T, n, m, X, x_scale, W, w_scale, w_zero, y, sms);
    };
    return y_dtype == REALQ_BF16 ? run(static_cast<__nv_bfloat16 *>(Y)) : run(static_cast<float *>(Y));
}

}  // namespace realq
