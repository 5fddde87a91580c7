// Attention of many query rows over the 8-bit cache (prompts) on the tensor
// cores: S = Q K^T and O = P V by tcgen05.mma kind::f16, scores and outputs in
// TMEM, P as the A operand from TMEM.
//
// A CTA takes up to 256 rows that share a key/value head (its query heads times
// the new tokens) as two tiles of 128, and goes over their cached tokens in tiles
// of 128.  Per tile of tokens the tensor cores take 4 x 512 cycles for the two row
// tiles' two products (at 128 channels), which bounds the kernel; beside them fit
//   - four producer warps: codes from the pages to fp16 in shared memory (exact:
//     a byte permute to 1024 + c, one subtraction of 1152), a tile ahead in
//     registers, K as the K-major and V as the MN-major B operand of the same layout: boxes of 64
//     channels, a token's 128-byte row swizzled;
//   - two softmax warpgroups, one to a row tile, a thread to a row: while one works
//     on its scores the tensor cores work for the other;
//   - one warp that issues the products.
// Per value of S a softmax thread spends a maximum, a multiply-add, an exponential, an addition and
// half a conversion: the block scales enter by the 16 tokens that share them.  With ks, vs a
// chunk's scales, lv = log2 vs and r the row's own scale (a power of two from
// scaling q into fp16's range, the softmax scale, log2 e),
//   p = 2^(S ks r + lv - M + 6),   sum += (sum of p in the chunk) / vs,
// so p already holds V's scale and O needs no other.  M is at least the running maximum less
// 8: it moves only when some row's maximum grew by more than that, and only then O is
// read, scaled and written back (the largest p stays below 2^14).  Scale blocks of fewer than 16
// tokens take one scale per token in the same formulas.  bf16 queries are exact in
// fp16 after scaling (down to 2^-29 of a row's largest value); fp32 queries and their p are two fp16
// parts each, which doubles the products.
//
// P lies over S in TMEM (its low part, with fp32, has columns of its own), so the next
// product into S is issued behind the product that reads P; the tensor cores run
// them in order.  Work is cut as for few rows (kv_schedule.cuh), partial results
// joined by the warpgroup that ends last.
#include <algorithm>

#include "kv_schedule.cuh"
#include "tc.cuh"

namespace realq {
namespace {

constexpr uint32_t FULL = 0xFFFFFFFFu;
constexpr int SOFT_WARPS = 8, PROD_WARPS = 4, THREADS = 32 * (SOFT_WARPS + PROD_WARPS + 1);
constexpr int SLOTS = 4;                 // of block scales
constexpr float NEG = -INFINITY, LIFT = 6.f, SLACK = 8.f;

template <int DP, bool F32> struct Shape {
    static constexpr int NM = DP == 256 ? 1 : 2;                                // row tiles
    static constexpr int ROWS = 128 * NM;
    static constexpr int KT = DP == 256 || (DP == 128 && F32) ? 64 : 128;       // tokens of a tile
    static constexpr int PARTS = F32 ? 2 : 1;
    static constexpr int STAGES = DP == 256 && F32 ? 1 : 2;                     // of K and of V
    static constexpr int BOXES = DP / 64;
    static constexpr int Q_BYTES = 128 * DP * 2;                                // one row tile, one part
    static constexpr int KV_BYTES = KT * DP * 2;
    static constexpr int SLOT_BYTES = 4 * KT * 4;
    static constexpr int RING = NM * PARTS * Q_BYTES, SCALES = RING + 2 * STAGES * KV_BYTES, BARS = SCALES + SLOTS * SLOT_BYTES;
    static constexpr int SMEM = BARS + 256 + 1024;
    static constexpr int NI = (KT / 8) * BOXES / PROD_WARPS;                    // 16-byte pieces of a tile to a producer
    static constexpr int PART = 128 * (DP + 2);                                 // numbers of a row tile's partial result
    // TMEM columns
    static constexpr int S(int i) { return i * KT; }
    static constexpr int O(int i) { return NM * KT + i * DP; }
    static constexpr int LO(int i) { return NM * (KT + DP) + i * (KT / 2); }
    static_assert(SMEM <= 232448 && NM * (KT + DP + (F32 ? KT / 2 : 0)) <= 512, "shared and tensor memory");
};

__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void group_sync(int id) { asm volatile("bar.sync %0, 128;" ::"r"(id) : "memory"); }
__device__ __forceinline__ void tmem_st_x16(uint32_t taddr, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

struct Ring {   // stage and phase of something that goes round
    int s = 0, n;
    uint32_t phase = 0;
    __device__ explicit Ring(int stages) : n(stages) {}
    __device__ __forceinline__ void next() {
        if (++s == n) s = 0, phase ^= 1u;
    }
};

// The units of a CTA's share, one after the other; every role walks them for itself.
template <int ROWS, int KT> struct Walk {
    const KvAttnArgs &a;
    Unit u;
    int tiles, from, count;    // of the unit, the share's first and how many
    int64_t unit0, at, end;
    __device__ Walk(const KvAttnArgs &args, const Unit &u0, int64_t first, int tiles0, int64_t at0, int64_t end0)
        : a(args), u(u0), tiles(tiles0), unit0(first), at(at0), end(end0) {
        set();
    }
    __device__ __forceinline__ void set() {
        from = (int)min(at - unit0, (int64_t)tiles - 1);
        count = (int)min(end - at, (int64_t)(tiles - from));
    }
    __device__ __forceinline__ bool more() const { return at < end; }
    __device__ void next() {
        at += count;
        if (at >= end) return;
        unit0 += tiles;
        u.r0 += ROWS;
        if (u.r0 >= u.m * a.group) {
            u.r0 = 0;
            if (++u.head >= a.c.n_kv) {
                u.head = 0;
                Seq q(a, u.seq);
                do {
                    if (++u.seq >= a.n_seqs) {   // (not reached unless lengths change meanwhile)
                        at = end;
                        return;
                    }
                    q = Seq(a, u.seq);
                } while (q.m == 0);
                u.q0 = q.q0, u.m = q.m, u.len = q.len;
            }
        }
        u.rows = min(ROWS, u.m * a.group - u.r0);
        span(a, u.m, u.len, u.r0, u.r0 + u.rows, &u.lo, &u.hi);
        tiles = tiles_of<KT>(u.lo, u.hi);
        set();
    }
};

template <int DP, bool F32, class T>
__global__ void __launch_bounds__(THREADS, 1) prompt_kernel(KvAttnArgs a, int *err) {
    using Sh = Shape<DP, F32>;
    constexpr int NM = Sh::NM, KT = Sh::KT, ROWS = Sh::ROWS;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ Window win;
    __shared__ int last_one[2];
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + Sh::BARS);
    uint64_t *k_full = bars, *k_empty = bars + 2, *v_full = bars + 4, *v_empty = bars + 6;
    uint64_t *q_full = bars + 8, *s_full = bars + 10, *p_full = bars + 12, *o_full = bars + 14, *done = bars + 16;
    uint32_t *tslot = reinterpret_cast<uint32_t *>(bars + 17);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tslot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int D = a.c.head_dim;

    dependents_may_start();
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(tc::smem_u32(k_full + i), 32 * PROD_WARPS);
            tc::mbar_init(tc::smem_u32(v_full + i), 32 * PROD_WARPS);
            tc::mbar_init(tc::smem_u32(k_empty + i), 1);
            tc::mbar_init(tc::smem_u32(v_empty + i), 1);
            tc::mbar_init(tc::smem_u32(q_full + i), 128);
            tc::mbar_init(tc::smem_u32(s_full + i), 1);
            tc::mbar_init(tc::smem_u32(p_full + i), 128);
            tc::mbar_init(tc::smem_u32(o_full + i), 1);
        }
        tc::mbar_init(tc::smem_u32(done), 1);
        *abort_flag = 0;
        tc::fence_barrier_init();
    }
    // the share and its first unit
    int64_t all = 0;
    for (int first = 0; first < a.n_seqs; first += SEQS) {
        fill_window<ROWS, KT, true>(a, win, first, all);
        all += win.sum[SEQS] * a.c.n_kv;
    }
    const Shares shares{all, min((int64_t)gridDim.x, all)};
    if (blockIdx.x >= shares.ctas) return;
    if (a.n_seqs > SEQS) fill_window<ROWS, KT, true>(a, win, 0, 0);
    const int64_t at0 = shares.begin(blockIdx.x), end0 = shares.begin(blockIdx.x + 1);
    Unit u0;
    int64_t first0;
    int tiles0;
    locate<ROWS, KT, true>(a, win, at0, u0, first0, tiles0);
    Walk<ROWS, KT> w(a, u0, first0, tiles0, at0, end0);

    if (warp == 0) tc::tmem_alloc(tc::smem_u32(tslot), 512);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = *tslot;
    bool ok = true;

    if (warp < SOFT_WARPS) {
        // ---------------- softmax: thread = row of row tile i ----------------
        const int i = warp >> 2, row = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_at = tmem + lanes + Sh::S(i), o_at = tmem + lanes + Sh::O(i), lo_at = tmem + lanes + Sh::LO(i);
        const bool fine = a.c.log_block < 4;
        uint8_t *qs = smem + i * Sh::PARTS * Sh::Q_BYTES;
        uint32_t s_phase = 0, o_phase = 0;
        int slot = 0;
        // the row's query into shared memory; returns what its scores are multiplied by
        const auto load_q = [&](const Unit &u) {
            const int r = u.r0 + 128 * i + row;
            const bool in = 128 * i + row < u.rows;
            const int qi = in ? r / a.group : 0;
            const T *q = (const T *)a.q + (int64_t)(u.q0 + qi) * a.q_ld + (int64_t)(u.head * a.group + (in ? r % a.group : 0)) * a.q_hs;
            const bool wide = ((reinterpret_cast<uintptr_t>(a.q) | (uintptr_t)(a.q_ld * sizeof(T)) | (uintptr_t)(a.q_hs * sizeof(T))) & 15) == 0;
            float top = 0.f;
            const auto values = [&](int d, float (&x)[8]) {   // q[d .. d + 7]
                if (!in) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = 0.f;
                } else if (wide) {
                    if constexpr (F32) {
                        const float4 v0 = *reinterpret_cast<const float4 *>(q + d), v1 = *reinterpret_cast<const float4 *>(q + d + 4);
                        x[0] = v0.x, x[1] = v0.y, x[2] = v0.z, x[3] = v0.w, x[4] = v1.x, x[5] = v1.y, x[6] = v1.z, x[7] = v1.w;
                    } else {
                        const uint4 v = *reinterpret_cast<const uint4 *>(q + d);
                        const uint32_t h[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            x[2 * e] = __uint_as_float(h[e] << 16), x[2 * e + 1] = __uint_as_float(h[e] & 0xFFFF0000u);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = load_as_float(q, d + e);
                }
            };
#pragma unroll 2
            for (int d = 0; d < D; d += 8) {
                float x[8];
                values(d, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
            }
            int k = 0;
            if (top > 0.f && top < INFINITY) k = 14 - ilogbf(top);
            const float sign = a.scale_log2 < 0.f ? -1.f : 1.f;   // the scores' factor is to be positive
            const float up0 = sign * scalbnf(1.f, k / 2), up1 = scalbnf(1.f, k - k / 2);
#pragma unroll 2
            for (int d = 0; d < D; d += 8) {
                float x[8];
                values(d, x);
                uint32_t h[4];
                const uint32_t to = (uint32_t)(d >> 6) * 16384u + row * 128 + ((((d >> 3) & 7) ^ (row & 7)) << 4);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = x[e] * up0 * up1;
#pragma unroll
                for (int e = 0; e < 4; ++e) h[e] = pack_half(x[2 * e], x[2 * e + 1]);
                *reinterpret_cast<uint4 *>(qs + to) = make_uint4(h[0], h[1], h[2], h[3]);
                if constexpr (F32) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) h[e] = pack_rest(x[2 * e], x[2 * e + 1], h[e]);
                    *reinterpret_cast<uint4 *>(qs + Sh::Q_BYTES + to) = make_uint4(h[0], h[1], h[2], h[3]);
                }
            }
            fence_async_smem();
            tc::mbar_arrive(tc::smem_u32(q_full + i));
            return fabsf(a.scale_log2) * scalbnf(1.f, -(k / 2)) * scalbnf(1.f, -(k - k / 2));
        };
        float rs = 0.f;
        bool loaded = false;
        while (w.more() && ok) {
            const Unit u = w.u;
            const int from = w.from, count = w.count, tiles = w.tiles;
            const int64_t unit0 = w.unit0;
            if (128 * i >= u.rows) {   // the row tile is empty: its tiles of tokens pass by
                slot = (slot + count) & (SLOTS - 1);
                w.next();
                continue;
            }
            if (!loaded) rs = load_q(u);
            const float factor = rs;
            const int r = u.r0 + 128 * i + row, qi = r / a.group, p = u.len - u.m + qi;
            const bool in = 128 * i + row < u.rows;
            const int row_hi = !in ? 0 : (a.causal ? min(u.len, p + 1) : u.len);
            const int row_lo = a.window > 0 ? (int)max((int64_t)0, (int64_t)p - a.window + 1) : 0;
            const int all_hi = __reduce_min_sync(FULL, in ? row_hi : INT32_MAX), all_lo = __reduce_max_sync(FULL, in ? row_lo : 0);
            float m = NEG, l = 0.f, bad = 0.f;   // bad: NaN once a value that the row sees is
            for (int t = 0; t < count && ok; ++t, slot = (slot + 1) & (SLOTS - 1)) {
                ok = __all_sync(FULL, tc::mbar_wait(tc::smem_u32(s_full + i), s_phase, abort_flag));
                s_phase ^= 1u;
                if (!ok) break;
                tc::fence_after_sync();
                const int k0 = (u.lo / KT + from + t) * KT;
                const bool masked = k0 + KT > all_hi || k0 < all_lo;
                const float *sc = reinterpret_cast<const float *>(smem + Sh::SCALES + slot * Sh::SLOT_BYTES);
                const auto seen = [&](int j) { return k0 + j < row_hi && k0 + j >= row_lo; };
                // the largest S ks r + lv
                float top = NEG;
#pragma unroll
                for (int c = 0; c < KT; c += 32) {
                    uint32_t v[32];
                    tc::tmem_ld_32x32b_x32(s_at + c, v);
                    if (masked) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (!seen(c + j)) v[j] = 0xFF800000u;
                    }
                    if (!fine) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float4 b = reinterpret_cast<const float4 *>(sc)[c / 16 + h];
                            float x = __uint_as_float(v[16 * h]);
#pragma unroll
                            for (int j = 1; j < 16; ++j) x = fmaxf(x, __uint_as_float(v[16 * h + j]));
                            top = fmaxf(top, fmaf(x, b.x * factor, b.y));
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const float4 ks = *reinterpret_cast<const float4 *>(sc + c + j), lv = *reinterpret_cast<const float4 *>(sc + KT + c + j);
                            top = fmaxf(top, fmaf(__uint_as_float(v[j]), ks.x * factor, lv.x));
                            top = fmaxf(top, fmaf(__uint_as_float(v[j + 1]), ks.y * factor, lv.y));
                            top = fmaxf(top, fmaf(__uint_as_float(v[j + 2]), ks.z * factor, lv.z));
                            top = fmaxf(top, fmaf(__uint_as_float(v[j + 3]), ks.w * factor, lv.w));
                        }
                    }
                }
                const bool grew = top > (m == NEG ? NEG : m + SLACK);
                if (__any_sync(FULL, grew)) {
                    const float now = fmaxf(m, top), f = now == NEG ? 1.f : exp2_fast(m - now);
                    m = now, l *= f;
                    if (t > 0) {   // (the products so far are done: S came behind them)
#pragma unroll 1
                        for (int c = 0; c < D; c += 16) {
                            uint32_t v[16];
                            tc::tmem_ld_32x32b_x16(o_at + c, v);
                            tc::tmem_wait_ld();
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * f);
                            tmem_st_x16(o_at + c, v);
                        }
                    }
                }
                const float base = LIFT - (m == NEG ? 0.f : m);
#pragma unroll
                for (int c = 0; c < KT; c += 32) {
                    uint32_t v[32], hi[16], lo[F32 ? 16 : 1];
                    tc::tmem_ld_32x32b_x32(s_at + c, v);
                    if (!fine) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float4 b = reinterpret_cast<const float4 *>(sc)[c / 16 + h];
                            const float c1 = b.x * factor, c0 = b.y + base;
                            float part = 0.f;
#pragma unroll
                            for (int j = 16 * h; j < 16 * h + 16; j += 2) {
                                float x0 = fmaf(__uint_as_float(v[j]), c1, c0), x1 = fmaf(__uint_as_float(v[j + 1]), c1, c0);
                                if (masked) {
                                    if (!seen(c + j)) x0 = NEG;
                                    if (!seen(c + j + 1)) x1 = NEG;
                                }
                                x0 = exp2_fast(x0), x1 = exp2_fast(x1);
                                part += x0 + x1;
                                hi[j / 2] = pack_half(x0, x1);
                                if constexpr (F32) lo[j / 2] = pack_rest(x0, x1, hi[j / 2]);
                            }
                            if (!(masked && part == 0.f))   // (unseen tokens' scales may be anything)
                                l = fmaf(part, b.z, l), bad = fmaf(part, b.w, bad);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const float4 ks = *reinterpret_cast<const float4 *>(sc + c + j), lv = *reinterpret_cast<const float4 *>(sc + KT + c + j);
                            const float4 iv = *reinterpret_cast<const float4 *>(sc + 2 * KT + c + j);
                            float x[4] = {fmaf(__uint_as_float(v[j]), ks.x * factor, lv.x + base), fmaf(__uint_as_float(v[j + 1]), ks.y * factor, lv.y + base),
                                          fmaf(__uint_as_float(v[j + 2]), ks.z * factor, lv.z + base), fmaf(__uint_as_float(v[j + 3]), ks.w * factor, lv.w + base)};
                            const float4 nv = *reinterpret_cast<const float4 *>(sc + 3 * KT + c + j);
                            const float inv[4] = {iv.x, iv.y, iv.z, iv.w}, nan[4] = {nv.x, nv.y, nv.z, nv.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if (masked && !seen(c + j + e)) x[e] = NEG;
                                x[e] = exp2_fast(x[e]);
                                if (!(masked && x[e] == 0.f)) l = fmaf(x[e], inv[e], l), bad = fmaf(x[e], nan[e], bad);
                            }
                            hi[j / 2] = pack_half(x[0], x[1]), hi[j / 2 + 1] = pack_half(x[2], x[3]);
                            if constexpr (F32) lo[j / 2] = pack_rest(x[0], x[1], hi[j / 2]), lo[j / 2 + 1] = pack_rest(x[2], x[3], hi[j / 2 + 1]);
                        }
                    }
                    tmem_st_x16(s_at + c / 2, hi);
                    if constexpr (F32) tmem_st_x16(lo_at + c / 2, lo);
                }
                tc::tmem_wait_st();
                tc::fence_before_sync();
                tc::mbar_arrive(tc::smem_u32(p_full + i));
            }
            if (!ok) break;
            // the next unit's queries while the last products run (this one's have been read: its last scores are there)
            w.next();
            loaded = w.more() && 128 * i < w.u.rows;
            if (loaded) rs = load_q(w.u);
            ok = __all_sync(FULL, tc::mbar_wait(tc::smem_u32(o_full + i), o_phase, abort_flag));
            o_phase ^= 1u;
            if (!ok) break;
            tc::fence_after_sync();

            const int64_t out_row = (int64_t)(u.q0 + qi) * a.n_heads + u.head * a.group + r % a.group;
            const bool aligned = (reinterpret_cast<uintptr_t>(a.out) & 15) == 0;
            const auto put = [&](int d, const float (&y)[4]) {   // out[d .. d + 3]
                T *o = (T *)a.out + out_row * D + d;
                if (!aligned) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (F32)
                            o[e] = y[e];
                        else
                            o[e] = __float2bfloat16_rn(y[e]);
                    }
                } else if constexpr (F32) {
                    *reinterpret_cast<float4 *>(o) = make_float4(y[0], y[1], y[2], y[3]);
                } else {
                    const __nv_bfloat162 h0 = __floats2bfloat162_rn(y[0], y[1]), h1 = __floats2bfloat162_rn(y[2], y[3]);
                    *reinterpret_cast<uint2 *>(o) = make_uint2(*reinterpret_cast<const uint32_t *>(&h0), *reinterpret_cast<const uint32_t *>(&h1));
                }
            };
            const auto put_lse = [&](float mm, float ll) {
                if (a.lse != nullptr) a.lse[out_row] = ll == 0.f ? NEG : (mm - LIFT + log2f(ll)) * 0.6931471805599453f;
            };
            const bool whole = count == tiles;
            const int first_cta = whole ? 0 : shares.owner(unit0), last_cta = whole ? 0 : shares.owner(unit0 + tiles - 1);
            const auto slot_of = [&](int c, bool begins) { return a.part + ((int64_t)(2 * c + (begins ? 1 : 0)) * NM + i) * Sh::PART; };
            float *mine = slot_of(blockIdx.x, from == 0);
            const float inv = l == 0.f ? 0.f : 1.f / l;   // (a row that sees nothing: zeros)
#pragma unroll 1
            for (int c = 0; c < D; c += 16) {
                uint32_t v[16];
                tc::tmem_ld_32x32b_x16(o_at + c, v);
                tc::tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; j += 4) {
                    float y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = __uint_as_float(v[j + e]) + bad;
                    if (whole) {
                        if (l == 0.f) y[0] = y[1] = y[2] = y[3] = 0.f;
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[e] *= inv;
                        if (in) put(c + j, y);
                    } else {
                        reinterpret_cast<float4 *>(mine)[(c + j) / 4 * 128 + row] = make_float4(y[0], y[1], y[2], y[3]);
                    }
                }
            }
            tc::fence_before_sync();
            if (whole) {
                if (in) put_lse(m, l);
                continue;
            }
            mine[128 * DP + row] = m, mine[128 * DP + 128 + row] = l;
            __threadfence();
            group_sync(1 + i);
            if (row == 0) {
                const unsigned others = (unsigned)(last_cta - first_cta);
                last_one[i] = atomicInc(reinterpret_cast<unsigned *>(a.counters) + 2 * first_cta + i, others) == others;
            }
            group_sync(1 + i);
            if (!last_one[i]) continue;
            __threadfence();
            float mm = NEG, ll = 0.f;
            for (int c = first_cta; c <= last_cta; ++c) mm = fmaxf(mm, __ldcg(slot_of(c, c == first_cta) + 128 * DP + row));
            for (int c = first_cta; c <= last_cta; ++c) {
                const float *s = slot_of(c, c == first_cta) + 128 * DP + row;
                const float mc = __ldcg(s), lc = __ldcg(s + 128);
                ll += mc == NEG ? lc * 0.f : lc * exp2_fast(mc - mm);   // (a NaN stays one)
            }
            const float all_inv = ll == 0.f ? 0.f : 1.f / ll;
            for (int d = 0; d < D; d += 4) {
                float y[4] = {0.f, 0.f, 0.f, 0.f};
                for (int c = first_cta; c <= last_cta; ++c) {
                    const float *s = slot_of(c, c == first_cta);
                    const float mc = __ldcg(s + 128 * DP + row), lc = __ldcg(s + 128 * DP + 128 + row);
                    if (lc == 0.f) continue;
                    const float f = mc == NEG ? 0.f : exp2_fast(mc - mm);
                    const float4 v = __ldcg(reinterpret_cast<const float4 *>(s) + d / 4 * 128 + row);
                    y[0] += v.x * f, y[1] += v.y * f, y[2] += v.z * f, y[3] += v.w * f;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] *= all_inv;
                if (in) put(d, y);
            }
            if (in) put_lse(mm, ll);
        }
        if (!ok) *abort_flag = 1;
    } else if (warp < SOFT_WARPS + PROD_WARPS) {
        // ---------------- producers: codes -> fp16 ----------------
        const int pw = warp - SOFT_WARPS, ptid = threadIdx.x - 32 * SOFT_WARPS;
        const int pieces = D / 16, token = lane & 7, piece0 = lane >> 3;
        const bool fine = a.c.log_block < 4;
        const int my_token = fine ? ptid : 16 * ptid;   // whose scales this thread brings
        Ring ring(Sh::STAGES);
        int slot = 0;
        while (w.more() && ok) {
            const Unit &u = w.u;
            const int tile0 = u.lo / KT + w.from;
            const int *table = a.tables + (int64_t)u.seq * a.max_pages;
            const auto page_of = [&](int tile) {   // of the tile's 8 tokens `lane`
                const int k0 = tile * KT + 8 * lane;
                if (lane >= KT / 8 || k0 >= u.hi || k0 + 8 <= u.lo) return -1;
                const int pg = table[k0 >> a.c.log_page];
                return pg >= 0 && pg < a.c.n_pages ? pg : -1;
            };
            const auto load = [&](const uint8_t *codes, int tile, int pages, uint4 (&x)[Sh::NI]) {
#pragma unroll
                for (int j = 0; j < Sh::NI; ++j) {
                    const int item = pw + PROD_WARPS * j, grp = item / Sh::BOXES, piece = item % Sh::BOXES * 4 + piece0;
                    const int pg = __shfl_sync(FULL, pages, grp);
                    const int place = (tile * KT + 8 * grp) & ((1 << a.c.log_page) - 1);
                    x[j] = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);
                    if (pg >= 0 && piece < pieces)
                        x[j] = __ldg(reinterpret_cast<const uint4 *>(
                            codes + ((((int64_t)pg * a.c.n_kv + u.head) << a.c.log_page) + place + token) * D + 16 * piece));
                }
            };
            const auto store = [&](uint8_t *to, const uint4 (&x)[Sh::NI]) {
#pragma unroll
                for (int j = 0; j < Sh::NI; ++j) {
                    const int item = pw + PROD_WARPS * j, grp = item / Sh::BOXES, box = item % Sh::BOXES;
                    if (box * 4 + piece0 >= pieces) continue;
                    uint8_t *line = to + box * (KT * 128) + (8 * grp + token) * 128;
                    *reinterpret_cast<uint4 *>(line + (((2 * piece0) ^ token) << 4)) =
                        make_uint4(codes01(x[j].x), codes23(x[j].x), codes01(x[j].y), codes23(x[j].y));
                    *reinterpret_cast<uint4 *>(line + (((2 * piece0 + 1) ^ token) << 4)) =
                        make_uint4(codes01(x[j].z), codes23(x[j].z), codes01(x[j].w), codes23(x[j].w));
                }
            };
            float ks = 0.f, vs = 0.f;
            bool there = false;
            const auto load_scales = [&](int tile, int pages) {
                const int pg = __shfl_sync(FULL, pages, (my_token >> 3) & 31);
                there = my_token < KT && pg >= 0;
                if (there) {
                    const int place = (tile * KT + my_token) & ((1 << a.c.log_page) - 1);
                    const int64_t at = (((int64_t)pg * a.c.n_kv + u.head) << (a.c.log_page - a.c.log_block)) + (place >> a.c.log_block);
                    ks = __ldg(a.c.k_scale + at), vs = __ldg(a.c.v_scale + at);
                }
            };
            uint4 kx[Sh::NI], vx[Sh::NI];
            int pages = page_of(tile0);
            load(a.c.k_codes, tile0, pages, kx);
            load_scales(tile0, pages);
            for (int t = 0; t < w.count; ++t, ring.next(), slot = (slot + 1) & (SLOTS - 1)) {
                const int next_pages = t + 1 < w.count ? page_of(tile0 + t + 1) : -1;
                load(a.c.v_codes, tile0 + t, pages, vx);
                ok = __all_sync(FULL, tc::mbar_wait(tc::smem_u32(k_empty + ring.s), ring.phase ^ 1u, abort_flag));
                if (!ok) break;
                tc::fence_after_sync();
                store(smem + Sh::RING + ring.s * Sh::KV_BYTES, kx);
                if (my_token < KT) {   // (the slot's last readers are behind the products that emptied this stage)
                    float *sc = reinterpret_cast<float *>(smem + Sh::SCALES + slot * Sh::SLOT_BYTES);
                    // a scale below 2^-100 counts as that; tokens without a page weigh nothing
                    const bool nan = there && vs != vs;   // (its part in the sum stays: the scores are not concerned)
                    const float lv = !there ? NEG : (nan ? 0.f : fmaxf(log2_fast(vs), -100.f)), iv = !there ? 0.f : exp2_fast(-lv);
                    const float k = there ? ks : 0.f, nv = nan ? vs : 0.f;
                    if (fine)
                        sc[my_token] = k, sc[KT + my_token] = lv, sc[2 * KT + my_token] = iv, sc[3 * KT + my_token] = nv;
                    else
                        reinterpret_cast<float4 *>(sc)[ptid] = make_float4(k, lv, iv, nv);
                }
                fence_async_smem();
                tc::mbar_arrive(tc::smem_u32(k_full + ring.s));
                load(a.c.k_codes, tile0 + t + 1, next_pages, kx);
                load_scales(tile0 + t + 1, next_pages);
                ok = __all_sync(FULL, tc::mbar_wait(tc::smem_u32(v_empty + ring.s), ring.phase ^ 1u, abort_flag));
                if (!ok) break;
                tc::fence_after_sync();
                store(smem + Sh::RING + (Sh::STAGES + ring.s) * Sh::KV_BYTES, vx);
                fence_async_smem();
                tc::mbar_arrive(tc::smem_u32(v_full + ring.s));
                pages = next_pages;
            }
            if (ok) w.next();
        }
        if (!ok) *abort_flag = 1;
    } else {
        // ---------------- products (the whole warp waits, one lane issues) ----------------
        const uint32_t idesc_s = tc::idesc_f16_f32(128, KT), idesc_o = tc::idesc_f16_f32(128, 0) | ((uint32_t)(D >> 3) << 17) | (1u << 16);
        const uint32_t base = tc::smem_u32(smem);
        const uint64_t q_desc = tc::smem_desc(base, 16, 1024, tc::SW_128B);
        const uint64_t k_desc = tc::smem_desc(base + Sh::RING, 16, 1024, tc::SW_128B);
        const uint64_t v_desc = tc::smem_desc(base + Sh::RING + Sh::STAGES * Sh::KV_BYTES, KT * 128, 1024, tc::SW_128B);
        const int steps = D / 16;
        uint32_t q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
        Ring kr(Sh::STAGES), vr(Sh::STAGES);
        const auto wait = [&](uint64_t *bar, uint32_t phase) {
            if (ok) ok = __all_sync(FULL, tc::mbar_wait(tc::smem_u32(bar), phase, abort_flag));
            if (ok) tc::fence_after_sync();
        };
        const auto scores = [&](int i) {   // S_i = Q_i K^T of the K stage
            if (tc::elect_one()) {
                for (int p = 0; p < Sh::PARTS; ++p) {
                    const uint64_t qd = q_desc + (uint32_t)((i * Sh::PARTS + p) * Sh::Q_BYTES >> 4);
                    const uint64_t kd = k_desc + (uint32_t)(kr.s * Sh::KV_BYTES >> 4);
#pragma unroll 4
                    for (int k = 0; k < steps; ++k)
                        tc::mma_f16_ss(tmem + Sh::S(i), qd + (k & 3) * 2 + (k >> 2) * 1024, kd + (k & 3) * 2 + (k >> 2) * (KT * 8), idesc_s,
                                       (p > 0 || k > 0) ? 1u : 0u);
                }
                tc::mma_commit(tc::smem_u32(s_full + i));
            }
            __syncwarp();
        };
        while (w.more() && ok) {
            const int nm = w.u.rows > 128 ? 2 : 1, count = w.count;
            for (int i = 0; i < nm; ++i) {
                wait(q_full + i, q_phase[i]);
                q_phase[i] ^= 1u;
                if (i == 0) wait(k_full + kr.s, kr.phase);
                if (ok) scores(i);
            }
            for (int t = 0; t < count && ok; ++t) {
                if (tc::elect_one()) tc::mma_commit(tc::smem_u32(k_empty + kr.s));   // (the scores of this tile are issued)
                __syncwarp();
                kr.next();
                wait(v_full + vr.s, vr.phase);
                for (int i = 0; i < nm && ok; ++i) {
                    wait(p_full + i, p_phase[i]);
                    p_phase[i] ^= 1u;
                    if (!ok) break;
                    if (tc::elect_one()) {
                        const uint64_t vd = v_desc + (uint32_t)(vr.s * Sh::KV_BYTES >> 4);
#pragma unroll
                        for (int p = 0; p < Sh::PARTS; ++p) {
                            const uint32_t pa = tmem + (p == 0 ? Sh::S(i) : Sh::LO(i));
#pragma unroll
                            for (int k = 0; k < KT / 16; ++k)
                                tc::mma_f16_ts(tmem + Sh::O(i), pa + k * 8, vd + k * 128, idesc_o, (t > 0 || p > 0 || k > 0) ? 1u : 0u);
                        }
                        if (t + 1 == count) tc::mma_commit(tc::smem_u32(o_full + i));
                    }
                    __syncwarp();
                    if (t + 1 < count) {
                        if (i == 0) wait(k_full + kr.s, kr.phase);
                        if (ok) scores(i);
                    }
                }
                if (ok && tc::elect_one()) tc::mma_commit(tc::smem_u32(v_empty + vr.s));
                __syncwarp();
                vr.next();
            }
            if (ok) w.next();
        }
        if (!ok) *abort_flag = 1;
        // every product issued has retired before TMEM is freed
        if (tc::elect_one()) tc::mma_commit(tc::smem_u32(done));
        __syncwarp();
        int never = 0;
        tc::mbar_wait(tc::smem_u32(done), 0u, &never, 100000000ull);
    }
    __syncwarp();
    if (!ok && lane == 0) atomicOr(err, (int)ST_TIMEOUT);
    tc::fence_before_sync();
    __syncthreads();
    if (warp == 0) tc::tmem_dealloc(tmem, 512);
}

template <int DP, class T> realq_status_t launch(cudaStream_t s, const KvAttnArgs &a, int *err, int sms) {
    using Sh = Shape<DP, sizeof(T) == 4>;
    const auto kernel = prompt_kernel<DP, sizeof(T) == 4, T>;
    REALQ_TRY(set_smem_limit((const void *)kernel, Sh::SMEM));
    Launch l("kv_attention_tc", s);
    kernel<<<(unsigned)sms, THREADS, Sh::SMEM, s>>>(a, err);
    return check_launch("kv_attention_tc");
}
template <class T> realq_status_t by_size(cudaStream_t s, const KvAttnArgs &a, int *err, int sms) {
    if (a.c.head_dim <= 64) return launch<64, T>(s, a, err, sms);
    if (a.c.head_dim <= 128) return launch<128, T>(s, a, err, sms);
    return launch<256, T>(s, a, err, sms);
}

}  // namespace

// Partial results: two a CTA, each of two row tiles of 128 x (128 + 2) numbers (one of 128 x (256 + 2) is fewer).
size_t kv_prompt_ws_bytes(int sms) {
    Carve c(nullptr);
    c.take<int>(2 * sms);
    c.take<float>((size_t)2 * sms * 2 * 128 * (128 + 2));
    return c.off;
}

realq_status_t kv_prompt(cudaStream_t s, const KvAttnArgs &args, realq_dtype_t dt, int *err, void *ws, int sms) {
    KvAttnArgs a = args;
    Carve c(ws);
    a.counters = c.take<int>(2 * sms);
    a.part = c.take<float>(0);
    return dt == REALQ_BF16 ? by_size<__nv_bfloat16>(s, a, err, sms) : by_size<float>(s, a, err, sms);
}

}  // namespace realq
