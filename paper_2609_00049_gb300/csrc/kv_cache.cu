// Into and out of the 8-bit key/value cache: values are kept as
// scale (code - 128) with one scale for each block of tokens and head.
//
// Appending: a CTA takes one block of tokens, its warps the heads' keys and values in
// turn.  A warp holds a head's new values in registers (2048 bf16 values or 1024 fp32
// ones; more are read twice, the second time from the L1), finds their largest
// magnitude, brings the codes that were there to the new scale where that grew, and
// writes the new ones.  Which block a CTA has follows from its number alone: the
// blocks that sequence s touches are at most n / block + 2 for its n tokens, so
// numbers from starts[s] / block + 2 s on are free for them, and the sequence is
// found by a warp-wide search.
//
// What it cannot do without is memory: the new values are read and their codes written once.  Ragged
// prompts (30 thousand tokens of 8 heads of 128 in bf16) go in in 45 us, 3.5 TB/s with
// 0.69 of the issue slots used (a warp has nothing of its next block under way while it
// reduces and writes one), and come out in 32 us, 5.8 TB/s; one token of each
// of 64 sequences goes in and comes out in 7.4 us in a graph.
#include "kernels.cuh"

namespace realq {
namespace {

constexpr int WARPS = 8;

// the last sequence s of n with key(s) <= i, key not decreasing (the first where none is); a warp tries 32 at a time
template <class Key> __device__ __forceinline__ int last_at_most(int n, int64_t i, Key key) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, at = lo + lane * step;
        const uint32_t below = __ballot_sync(0xFFFFFFFFu, at < hi && key(at) <= i);
        lo += max(0, 31 - __clz(below)) * step;   // (a run of lanes from the first on)
        hi = min(hi, lo + step);
    }
    return lo;
}

template <class T> __device__ __forceinline__ void store16(T *p, const float *v) {   // 16 bytes of values
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
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

__device__ __forceinline__ uint32_t bytes4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// clamp(rint(x / scale), -127, 127) + 128
__device__ __forceinline__ uint32_t code_of(float x, float scale) {
    return scale > 0.f ? (uint32_t)((int)rintf(fminf(fmaxf(__fdiv_rn(x, scale), -127.f), 127.f)) + 128) : 128u;
}
// two fp32 numbers in a register pair
__device__ __forceinline__ uint64_t two(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 halves(uint64_t x) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// The codes of 4 numbers by division, as bytes.
__device__ __noinline__ uint32_t divided4(float x0, float x1, float x2, float x3, float scale) {
    return code_of(x0, scale) | code_of(x1, scale) << 8 | code_of(x2, scale) << 16 | code_of(x3, scale) << 24;
}
// The codes of 4 numbers, as bytes.  The quotient is taken as x inv, within 127 x 2^-22 of the fp32 quotient; adding
// 1.5 x 2^23 + 128 rounds it to a whole number, ties to even.  Where some quotient lies so near the middle between two
// codes that the division could decide otherwise, it decides.  (No quotient passes 127 by as much as rounding shows where
// scale is a normal number, at least the largest value over 127; elsewhere `plain` is false.)
__device__ __forceinline__ uint32_t codes4(float x0, float x1, float x2, float x3, float scale, uint64_t inv2, bool plain) {
    const uint64_t M = two(12583040.f, 12583040.f), m = two(-12583040.f, -12583040.f), minus = two(-1.f, -1.f);
    const uint64_t t0 = mul2(two(x0, x1), inv2), t1 = mul2(two(x2, x3), inv2);
    const uint64_t r0 = add2(t0, M), r1 = add2(t1, M);
    const float2 d0 = halves(add2(t0, mul2(add2(r0, m), minus))), d1 = halves(add2(t1, mul2(add2(r1, m), minus)));
    if (!plain || fmaxf(fmaxf(fabsf(d0.x), fabsf(d0.y)), fmaxf(fabsf(d1.x), fabsf(d1.y))) > 0.4999f) return divided4(x0, x1, x2, x3, scale);
    const float2 a = halves(r0), b = halves(r1);
    return bytes4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
}

// What a warp knows of the block it writes into: of sequence tokens p0 .. p0 + block - 1, `old` are there and `cnt` come.
struct Block {
    int64_t first_row;   // of k and v
    int64_t tile0;       // the page's first head
    int place, old, cnt; // of the block in its page
};
__device__ __forceinline__ bool find_block(const KvAppendArgs &a, int64_t i, Block &b) {
    const int block = 1 << a.c.log_block;
    const auto key = [&](int s) { return (int64_t)(a.starts[s] >> a.c.log_block) + 2ll * s; };
    const int s = last_at_most(a.n_seqs, i, key);
    const int64_t from_row = a.starts[s], to_row = a.starts[s + 1], k = key(s);
    if (from_row < 0 || to_row <= from_row || to_row > a.T || i < k) return false;
    const int64_t first = a.positions[from_row];
    if (first < 0 || first >= a.max_pages << a.c.log_page) return false;
    const int64_t p0 = ((first >> a.c.log_block) + (i - k)) << a.c.log_block;
    const int64_t from = max(first, p0), to = min(first + (to_row - from_row), p0 + block);
    const int64_t pi = p0 >> a.c.log_page;
    if (from >= to || pi >= a.max_pages) return false;
    const int pg = a.tables[s * a.max_pages + pi];
    if (pg < 0 || pg >= a.c.n_pages) return false;
    b.first_row = from_row + (from - first), b.tile0 = (int64_t)pg * a.c.n_kv;
    b.place = (int)(p0 & ((1 << a.c.log_page) - 1)), b.old = (int)(from - p0), b.cnt = (int)(to - from);
    return true;
}
// A block's new scale from the largest new magnitude (as bits); writes it where it changes.
__device__ __forceinline__ float new_scale(uint32_t top, float before, bool fresh, float *at) {
    const bool bad = top >= 0x7F800000u || before != before;
    const float scale = bad ? __uint_as_float(0x7FC00000u) : fmaxf(before, __fdiv_rn(__uint_as_float(top), 127.f));
    __syncwarp();
    if ((threadIdx.x & 31) == 0 && (fresh || !(scale == before))) *at = scale;
    return scale;
}
// The codes that were there, in the new steps.
__device__ __forceinline__ void rescale(uint8_t *codes, int bytes, float before, float scale) {
    if (!(scale > before && before > 0.f)) return;
    const float ratio = __fdiv_rn(before, scale);
#pragma unroll 1
    for (int j = threadIdx.x & 31; j < bytes / 16; j += 32) {
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

// 16 bytes of T as numbers
template <class T> struct Wide {
    static constexpr int N = 16 / sizeof(T);
    // its codes to `out`
    __device__ __forceinline__ static void put(uint8_t *out, const uint4 &r, float scale, uint64_t inv2, bool plain) {
        if constexpr (N == 8) {
            const auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
            const auto hi = [](uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); };
            *reinterpret_cast<uint2 *>(out) = make_uint2(codes4(lo(r.x), hi(r.x), lo(r.y), hi(r.y), scale, inv2, plain),
                                                         codes4(lo(r.z), hi(r.z), lo(r.w), hi(r.w), scale, inv2, plain));
        } else {
            *reinterpret_cast<uint32_t *>(out) =
                codes4(__uint_as_float(r.x), __uint_as_float(r.y), __uint_as_float(r.z), __uint_as_float(r.w), scale, inv2, plain);
        }
    }
    // the largest magnitude, as bits of fp32: a NaN is above every number
    __device__ __forceinline__ static uint32_t top(const uint4 &r, uint32_t t) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) t = N == 8 ? __vmaxu2(t, w[i] & 0x7FFF7FFFu) : max(t, w[i] & 0x7FFFFFFFu);
        return t;
    }
    __device__ __forceinline__ static uint32_t top_bits(uint32_t t) { return N == 8 ? max(t << 16, t & 0xFFFF0000u) : t; }
};

template <class T, bool WIDE>
__global__ void __launch_bounds__(32 * WARPS, 4) append_kernel(KvAppendArgs a) {
    constexpr int N = WIDE ? Wide<T>::N : 1, KEEP = 8;
    Block b;
    if (!find_block(a, blockIdx.x, b)) return;
    const int lane = threadIdx.x & 31, D = a.c.head_dim, row = D / N, n = b.cnt * row;
    const int token0 = lane / row, piece0 = lane - token0 * row, tokens32 = 32 / row, pieces32 = 32 - tokens32 * row;
    for (int unit = (threadIdx.x >> 5) + WARPS * blockIdx.y; unit < 2 * a.c.n_kv; unit += WARPS * gridDim.y) {
        const int head = unit >> 1;
        const bool is_v = unit & 1;
        const int64_t tile = b.tile0 + head, ld = is_v ? a.v_ld : a.k_ld;
        const T *x = (const T *)(is_v ? a.v : a.k) + b.first_row * ld + head * (is_v ? a.v_hs : a.k_hs);
        uint8_t *codes = (is_v ? a.c.v_codes : a.c.k_codes) + ((tile << a.c.log_page) + b.place) * D, *out = codes + (int64_t)b.old * D;
        float *scale_at = (is_v ? a.c.v_scale : a.c.k_scale) + (tile << (a.c.log_page - a.c.log_block)) + (b.place >> a.c.log_block);
        // the lane's pieces lane, lane + 32, ..: a token's lie together
        struct Walk {
            int token, piece;
        };
        const auto at = [&](const Walk &w) { return x + (int64_t)w.token * ld + w.piece * N; };
        const auto next = [&](Walk &w) {
            w.token += tokens32, w.piece += pieces32;
            if (w.piece >= row) w.piece -= row, ++w.token;
        };
        Walk w = {token0, piece0};
        const float before = b.old > 0 ? *scale_at : 0.f;
        uint32_t top = 0;
        if constexpr (WIDE) {
            // up to KEEP pieces a lane are read once, all of them under way; more a second time, from the L1
            uint4 kept[KEEP];
            const bool keep = n <= 32 * KEEP;
            if (keep) {
#pragma unroll
                for (int i = 0; i < KEEP; ++i) {
                    kept[i] = make_uint4(0, 0, 0, 0);
                    if (lane + 32 * i < n) kept[i] = *reinterpret_cast<const uint4 *>(at(w));
                    next(w);
                }
#pragma unroll
                for (int i = 0; i < KEEP; ++i) top = Wide<T>::top(kept[i], top);
            } else {
#pragma unroll 4
                for (int j = lane; j < n; j += 32, next(w)) top = Wide<T>::top(*reinterpret_cast<const uint4 *>(at(w)), top);
            }
            const float scale = new_scale(__reduce_max_sync(0xFFFFFFFFu, Wide<T>::top_bits(top)), before, b.old == 0, scale_at);
            rescale(codes, b.old * D, before, scale);
            const float inv = __fdiv_rn(1.f, scale);
            const uint64_t inv2 = two(inv, inv);
            const bool plain = scale >= 1.17549435e-38f;
            const auto put = [&](int j, const uint4 &r) { Wide<T>::put(out + (int64_t)j * N, r, scale, inv2, plain); };
            if (keep) {
#pragma unroll
                for (int i = 0; i < KEEP; ++i)
                    if (lane + 32 * i < n) put(lane + 32 * i, kept[i]);
            } else {
                w = {token0, piece0};
#pragma unroll 2
                for (int j = lane; j < n; j += 32, next(w)) put(j, *reinterpret_cast<const uint4 *>(at(w)));
            }
        } else {
            for (int j = lane; j < n; j += 32, next(w)) top = max(top, __float_as_uint(load_as_float(at(w), 0)) & 0x7FFFFFFFu);
            const float scale = new_scale(__reduce_max_sync(0xFFFFFFFFu, top), before, b.old == 0, scale_at);
            rescale(codes, b.old * D, before, scale);
            w = {token0, piece0};
            for (int j = lane; j < n; j += 32, next(w)) out[j] = (uint8_t)code_of(load_as_float(at(w), 0), scale);
        }
    }
}

// byte k of w less 128 as a float: behind the upper bytes of 2^23 it is a number's last bits (a conversion instruction
// runs at a quarter of an addition's rate)
__device__ __forceinline__ float code_value(uint32_t w, int k) {
    return __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7650 | k)) - 8388736.f;
}
// A warp takes a token, its lanes 16 bytes of values each of its heads' keys and values (`wide`: outputs that begin at 16
// bytes; a token's values are a multiple of that).
template <class T>
__global__ void __launch_bounds__(32 * WARPS) read_kernel(KvReadArgs a) {
    constexpr int N = 16 / sizeof(T);
    const int D = a.c.head_dim, per = D / N, lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5);
    if (t >= a.T) return;
    const int64_t p = a.positions[t], pi = p >> a.c.log_page;
    const int s = last_at_most(a.n_seqs, t, [&](int q) { return (int64_t)a.starts[q]; });
    if (a.starts[s] < 0 || t < a.starts[s] || t >= a.starts[s + 1] || a.starts[s + 1] > a.T) return;
    int pg = -1;
    if (p >= 0 && pi < a.max_pages) pg = a.tables[s * a.max_pages + pi];
    const bool there = pg >= 0 && pg < a.c.n_pages;
    const int place = (int)(p & ((1 << a.c.log_page) - 1)), all = a.c.n_kv * per;
    const int64_t tile0 = (int64_t)pg * a.c.n_kv;
#pragma unroll 4
    for (int i = lane; i < all; i += 32) {
        const int head = i / per, c = N * (i - head * per);
        const int64_t tile = tile0 + head;
        uint32_t q[2][N / 4];
        float scale[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            scale[w] = __uint_as_float(0x7FC00000u);
#pragma unroll
            for (int k = 0; k < N / 4; ++k) q[w][k] = 0;
            if (there && (w ? a.v_out : a.k_out) != nullptr) {
                const uint8_t *from = (w ? a.c.v_codes : a.c.k_codes) + ((tile << a.c.log_page) + place) * D + c;
                if constexpr (N == 8) {
                    const uint2 x = *reinterpret_cast<const uint2 *>(from);
                    q[w][0] = x.x, q[w][1] = x.y;
                } else {
                    q[w][0] = *reinterpret_cast<const uint32_t *>(from);
                }
                scale[w] = ((w ? a.c.v_scale : a.c.k_scale) + (tile << (a.c.log_page - a.c.log_block)))[place >> a.c.log_block];
            }
        }
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            T *out = (T *)(w ? a.v_out : a.k_out);
            if (out == nullptr) continue;
            float v[N];
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = code_value(q[w][k >> 2], k & 3) * scale[w];
            out += (t * a.c.n_kv + head) * D + c;
            if (a.wide) {
                store16(out, v);
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    if constexpr (sizeof(T) == 4)
                        out[k] = v[k];
                    else
                        out[k] = __float2bfloat16_rn(v[k]);
                }
            }
        }
    }
}

}  // namespace

realq_status_t kv_append(cudaStream_t s, const KvAppendArgs &a, realq_dtype_t dt, int sms) {
    const int64_t slots = (a.T >> a.c.log_block) + 2ll * a.n_seqs;
    const auto even = [&](const void *p, int64_t ld, int64_t hs) {
        const int64_t n = dt == REALQ_BF16 ? 8 : 4;
        return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % n == 0 && hs % n == 0;
    };
    const bool wide = even(a.k, a.k_ld, a.k_hs) && even(a.v, a.v_ld, a.v_hs);
    // a CTA takes all heads of a block; fewer, where there are few blocks (in and out of 200 tokens of one sequence: 9.1 us
    // in a graph, 12.3 with all heads to a CTA; of one token of each of 64: 7.4 and 8.3)
    int parts = 1;
    while (slots * parts < 4 * sms && parts * WARPS < 2 * a.c.n_kv) parts *= 2;
    const dim3 grid((unsigned)slots, (unsigned)parts);
    Launch l("kv_append", s);
    if (dt == REALQ_BF16) {
        if (wide)
            append_kernel<__nv_bfloat16, true><<<grid, 32 * WARPS, 0, s>>>(a);
        else
            append_kernel<__nv_bfloat16, false><<<grid, 32 * WARPS, 0, s>>>(a);
    } else {
        if (wide)
            append_kernel<float, true><<<grid, 32 * WARPS, 0, s>>>(a);
        else
            append_kernel<float, false><<<grid, 32 * WARPS, 0, s>>>(a);
    }
    return check_launch("kv_append");
}

realq_status_t kv_read(cudaStream_t s, const KvReadArgs &args, realq_dtype_t dt) {
    KvReadArgs a = args;
    a.wide = ((reinterpret_cast<uintptr_t>(a.k_out) | reinterpret_cast<uintptr_t>(a.v_out)) & 15) == 0;
    const unsigned grid = (unsigned)((a.T + WARPS - 1) / WARPS);
    Launch l("kv_read", s);
    if (dt == REALQ_BF16)
        read_kernel<__nv_bfloat16><<<grid, 32 * WARPS, 0, s>>>(a);
    else
        read_kernel<float><<<grid, 32 * WARPS, 0, s>>>(a);
    return check_launch("kv_read");
}

}  // namespace realq
