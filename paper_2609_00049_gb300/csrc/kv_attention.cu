// Attention of a few query rows over the 8-bit cache: single tokens, drafts.
//
// The rows that share a key/value head (its G query heads times the sequence's
// new tokens) are taken together, 8, 16 or 32 at a time (NT tiles of 8), against
// tiles of 64 cached tokens, 16 to a warp.  Bound by reading the codes once from
// HBM, so everything else has to fit under that:
//
// - Products by mma.sync m16n8k16 in fp16, transposed: S^T = K Q^T takes the
//   warp's 16 tokens as rows and 8 query rows as columns, so that a single query
//   head wastes seven columns of a cheap instruction, not fifteen rows of an
//   expensive one.  O^T = V^T P^T then takes 16 channels as rows.
// - Codes become fp16 exactly: a byte permute puts code c behind 0x64 (1024 + c),
//   one subtraction takes 1152 off.  The order of the channels inside a product
//   is free, so a lane uses the 16 consecutive bytes that it reads; V's bytes of
//   two tokens are interleaved by one more permute for two pairs.
// - Query rows are scaled by a power of two so that their largest value lies in
//   [2^14, 2^15): a bf16 row is exact in fp16 down to 2^-29 of its largest value, an fp32 row
//   is taken as the sum of two fp16 parts (22 bits).
// - The block scales of K multiply the scores in fp32, those of V the weights
//   before these become fp16: p = 2^(s - M) vscale with M = 14 less than the
//   running maximum of s + log2 vscale, so that the largest weight is about 2^14
//   and what fp16 cannot hold is 2^-38 of it.  With bf16 inputs p is rounded to
//   fp16 (2^-11 relative, an eighth of the output's own rounding); with fp32 ones it
//   is two fp16 parts.  The softmax's sum adds 2^(s - M - 14) in fp32.  log2 vscale
//   counts as -96 at least in the maximum, so that 2^31 tokens of zero values, 2^96
//   each, add up to 2^127.
// - A warp keeps its own maximum, sum and output; the four are joined at the end
//   of a CTA's share, and shares of one row tile by the CTA that ends last.
//
// Work is split evenly whatever the lengths: all (sequence, head, row tile)
// units' 64-token tiles in a row are cut into one share per resident CTA.  A
// unit that lies in one share is finished there; otherwise its CTAs leave
// (maximum, sum, output) in the workspace and the last to arrive adds them in
// the order of the shares, so results repeat bit by bit.  The arrival counter
// wraps to zero by itself.
//
// Measured: one token of each of 64 sequences of up to 16384, 64 heads to 8 of 128
// (1.24 GB of codes): 224 us, 5.5 TB/s, 0.81 of a copy's rate, with 0.63 of the issue
// slots used at three CTAs to an SM; one token over 131072: 64 us, of which 40 are
// the codes; one token over 1013, 16 heads: 10 us in a graph, all of it latency.
#include <algorithm>

#include "kv_schedule.cuh"

namespace realq {
namespace {

constexpr int WARPS = 4, THREADS = 32 * WARPS, GROUP = 16, TILE = GROUP * WARPS;
constexpr float NEG = -INFINITY, LIFT = 14.f, DOWN = 6.103515625e-05f;   // weights are 2^LIFT times what the sum adds; 2^-LIFT

__device__ __forceinline__ uint32_t transposed8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Sizes of the kernel for heads of up to DP channels and NT tiles of 8 rows.
template <int DP, int NT, bool F32> struct Shape {
    static constexpr int CH = DP / 16;                        // 16-byte pieces of a token's codes
    static constexpr int STEPS = DP / 16;                     // of the products over channels
    static constexpr int MT = DP / 16;                        // tiles of 16 channels of the output
    static constexpr int ROWS = 8 * NT;
    static constexpr int PARTS = F32 ? 2 : 1;                 // fp16 parts of a query
    static constexpr int SCALES = 2 * GROUP * 4;              // bytes
    static constexpr int STAGE = 2 * GROUP * DP + SCALES;     // a warp's 16 tokens
    static constexpr int STAGES = DP == 64 ? 6 : (DP == 128 ? 4 : 3);
    static constexpr int RING = STAGE * STAGES;               // per warp; its output at the end of a share
    static constexpr int QFRAG = STEPS * NT * PARTS * 32 * 8;
    static constexpr bool QREG = NT * STEPS * PARTS <= 16;    // held in registers
    static constexpr int SMEM = WARPS * RING + QFRAG;
    static_assert(ROWS * DP * 4 <= RING, "a warp's output fits its ring");
    // where a token's piece c lies in its row: spread so that neither the lanes of K (two tokens, four pieces) nor
    // those of V (four tokens, two pieces) meet in a bank
    __device__ static __forceinline__ int swizzle(int token, int c) {
        if constexpr (CH >= 8) return c ^ (((token >> 1) & 3) << 1) ^ ((token & 1) << 2);
        return c ^ ((token >> 1) & 3);
    }
};

template <int DP, int NT, bool F32, class T>
__global__ void __launch_bounds__(THREADS) decode_kernel(KvAttnArgs a) {
    using Sh = Shape<DP, NT, F32>;
    constexpr int ROWS = Sh::ROWS;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ Window win;
    __shared__ float row_scale[ROWS];
    __shared__ int row_lo[ROWS], row_hi[ROWS];
    __shared__ float join_m[WARPS][ROWS], join_l[WARPS][ROWS], row_m[ROWS], row_l[ROWS];
    __shared__ int last_one;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    uint8_t *ring = smem + warp * Sh::RING;
    uint2 *qfrag = reinterpret_cast<uint2 *>(smem + WARPS * Sh::RING);
    const int D = a.c.head_dim, pieces = D / 16;
    const bool wide = ((reinterpret_cast<uintptr_t>(a.q) | (uintptr_t)(a.q_ld * sizeof(T)) | (uintptr_t)(a.q_hs * sizeof(T))) & 15) == 0;
    float *const part = a.part;
    constexpr int PART = ROWS * (DP + 2);   // (a multiple of 16 bytes)

    // all tiles, and this CTA's share (up to 32 sequences without shared memory and its barriers: 16 heads over 1013
    // tokens 10.5 us in a graph, 10.7 with it; 32 sequences 116.5 and 118.7)
    const bool few = a.n_seqs <= 32;
    int64_t all = 0, least = 1;
    if (few) {
        const Lanes s = lanes_of<ROWS, TILE>(a);
        all = s.sum * a.c.n_kv, least = least_share(s.sum, s.units, 8);
    } else {
        for (int first = 0; first < a.n_seqs; first += SEQS) {
            fill_window<ROWS, TILE, false>(a, win, first, all);
            all += win.sum[SEQS] * a.c.n_kv;
        }
    }
    const Shares shares(all, max((int64_t)1, min((int64_t)gridDim.x, least == 1 ? all : all / least)));
    if (blockIdx.x >= shares.ctas) {
        wait_for_previous();
        return;
    }
    int64_t at = shares.begin(blockIdx.x);
    const int64_t end = shares.begin(blockIdx.x + 1);
    if (a.n_seqs > SEQS) fill_window<ROWS, TILE, false>(a, win, 0, 0);
    while (at < end) {
        Unit u;
        int64_t unit0;   // the unit's first tile
        int tiles;
        if (few)
            locate<ROWS, TILE>(a, lanes_of<ROWS, TILE>(a), at, u, unit0, tiles);   // (again: registers are short in the loop)
        else
            locate<ROWS, TILE, false>(a, win, at, u, unit0, tiles);
        const int from = (int)min(at - unit0, (int64_t)tiles - 1);
        const int count = (int)min(end - at, (int64_t)(tiles - from));
        const int tile0 = u.lo / TILE + from;
        at += count;

        // ---- this warp's 16 tokens of every tile ----
        const int *table = a.tables + (int64_t)u.seq * a.max_pages;
        const auto page_of = [&](int i) {   // of the warp's group i, -1 where there is none
            const int k0 = (tile0 + i) * TILE + warp * GROUP;   // (k0 + GROUP may be 2^31)
            if (i >= count || k0 >= u.hi || k0 + (GROUP - 1) < u.lo) return -1;
            const int pg = table[k0 >> a.c.log_page];
            return pg >= 0 && pg < a.c.n_pages ? pg : -1;
        };
        int pages = page_of(lane), pages_next = -1;   // of 32 groups, and of the next 32
        const auto page_at = [&](int i) { return __shfl_sync(0xFFFFFFFFu, pages, i & 31); };
        const auto load = [&](int i, int pg) {
            if (pg >= 0) {
                const int k0 = (tile0 + i) * TILE + warp * GROUP, place = k0 & ((1 << a.c.log_page) - 1);
                const int64_t tile = (int64_t)pg * a.c.n_kv + u.head;
                const int64_t src = ((tile << a.c.log_page) + place) * D;
                const uint32_t to = smem_addr(ring + (i % Sh::STAGES) * Sh::STAGE);
                for (int j = lane; j < GROUP * Sh::CH; j += 32) {
                    const int token = j / Sh::CH, c = j % Sh::CH;
                    if (c < pieces) {
                        const uint32_t off = token * DP + Sh::swizzle(token, c) * 16;
                        copy16(to + off, a.c.k_codes + src + token * D + 16 * c);
                        copy16(to + GROUP * DP + off, a.c.v_codes + src + token * D + 16 * c);
                    }
                }
                const int64_t sc = (tile << (a.c.log_page - a.c.log_block)) + ((place + (lane & 15)) >> a.c.log_block);
                copy4(to + 2 * GROUP * DP + 4 * lane, (lane < 16 ? a.c.k_scale : a.c.v_scale) + sc);
            }
            copies_end();
        };
        uint32_t have = 0;   // bit i % 32: group i has a page
        int loaded = 0;
        const auto load_next = [&]() {
            if (loaded < count) {
                if ((loaded & 31) == 0) {
                    if (loaded > 0) pages = pages_next;
                    pages_next = page_of(loaded + 32 + lane);
                }
                const int pg = page_at(loaded);
                have = (have & ~(1u << (loaded & 31))) | ((pg >= 0 ? 1u : 0u) << (loaded & 31));
                load(loaded, pg);
            } else {
                copies_end();
            }
            ++loaded;
        };
#pragma unroll 1
        for (int i = 0; i < Sh::STAGES - 1; ++i) load_next();

        // ---- queries (while the first codes come): a warp takes a tile of 8 rows ----
        for (int nt = warp; nt < NT; nt += WARPS) {
            const int r = u.r0 + 8 * nt + g;
            const bool row_in = 8 * nt + g < u.rows;
            const int qi = row_in ? r / a.group : 0;
            const T *q = (const T *)a.q + (int64_t)(u.q0 + qi) * a.q_ld + (int64_t)(u.head * a.group + (row_in ? r - qi * a.group : 0)) * a.q_hs;
            float v[DP / 4];
            float top = 0.f;
#pragma unroll
            for (int j = 0; j < DP / 64; ++j) {
                const int d = 16 * (t + 4 * j);   // (D is a multiple of 16)
                if (!row_in || d >= D) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[16 * j + e] = 0.f;
                } else if (!wide) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[16 * j + e] = load_as_float(q, d + e);
                } else if constexpr (F32) {
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const float4 x = *reinterpret_cast<const float4 *>(q + d + e);
                        v[16 * j + e] = x.x, v[16 * j + e + 1] = x.y, v[16 * j + e + 2] = x.z, v[16 * j + e + 3] = x.w;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 16; e += 8) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(q + d + e);
                        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            v[16 * j + e + 2 * k] = __uint_as_float(w[k] << 16), v[16 * j + e + 2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < DP / 4; ++e) top = fmaxf(top, fabsf(v[e]));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            // times 2^k: the largest lies in [2^14, 2^15) after that (a row below 2^-112 a little lower)
            const int ex = (int)(__float_as_uint(top) >> 23), k = ex == 255 ? 0 : min(126, 141 - ex);
            const float up = __uint_as_float((uint32_t)(127 + k) << 23);
#pragma unroll
            for (int step = 0; step < Sh::STEPS; ++step) {
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = v[4 * step + e] * up;
                const uint2 h = make_uint2(pack_half(x[0], x[1]), pack_half(x[2], x[3]));
                qfrag[((step * NT + nt) * Sh::PARTS) * 32 + lane] = h;
                if constexpr (F32)
                    qfrag[((step * NT + nt) * 2 + 1) * 32 + lane] = make_uint2(pack_rest(x[0], x[1], h.x), pack_rest(x[2], x[3], h.y));
            }
            if (t == 0) {
                const int p = u.len - u.m + qi;
                row_scale[8 * nt + g] = a.scale_log2 * __uint_as_float((uint32_t)(127 - k) << 23);
                row_hi[8 * nt + g] = !row_in ? 0 : min(a.room, a.causal ? p + 1 : u.len);
                row_lo[8 * nt + g] = a.window > 0 ? (int)max((int64_t)0, (int64_t)p - a.window + 1) : 0;
            }
        }
        __syncthreads();
        uint2 qreg[Sh::QREG ? Sh::STEPS * NT * Sh::PARTS : 1];
        if constexpr (Sh::QREG) {
#pragma unroll
            for (int i = 0; i < Sh::STEPS * NT * Sh::PARTS; ++i) qreg[i] = qfrag[i * 32 + lane];
        }
        float rs[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) rs[nt][0] = row_scale[8 * nt + 2 * t], rs[nt][1] = row_scale[8 * nt + 2 * t + 1];
        // tokens that every row sees
        const int p_first = u.len - u.m + u.r0 / a.group, p_last = u.len - u.m + (u.r0 + u.rows - 1) / a.group;
        const int clear_hi = min(a.room, a.causal ? p_first + 1 : u.len);
        const int64_t clear_lo = a.window > 0 ? (int64_t)p_last - a.window + 1 : 0;

        float o[Sh::MT][NT][4];
#pragma unroll
        for (int i = 0; i < Sh::MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) o[i][j][0] = o[i][j][1] = o[i][j][2] = o[i][j][3] = 0.f;
        float mx[NT][2], sum[NT][2];
#pragma unroll
        for (int j = 0; j < NT; ++j) mx[j][0] = mx[j][1] = NEG, sum[j][0] = sum[j][1] = 0.f;

#pragma unroll 1
        for (int i = 0; i < count; ++i) {
            copies_wait<Sh::STAGES - 2>();
            __syncwarp();
            load_next();   // into the stage that was read last
            if (!((have >> (i & 31)) & 1)) continue;
            const uint8_t *st = ring + (i % Sh::STAGES) * Sh::STAGE;
            const float *scales = reinterpret_cast<const float *>(st + 2 * GROUP * DP);
            const int k0 = (tile0 + i) * TILE + warp * GROUP;
            // scores
            float s[NT][4];
#pragma unroll
            for (int j = 0; j < NT; ++j) s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
#pragma unroll
            for (int j = 0; j < DP / 64; ++j) {
                const uint4 ka = *reinterpret_cast<const uint4 *>(st + g * DP + Sh::swizzle(g, t + 4 * j) * 16);
                const uint4 kb = *reinterpret_cast<const uint4 *>(st + (g + 8) * DP + Sh::swizzle(g + 8, t + 4 * j) * 16);
                const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t A[4] = {codes01(wa[w]), codes01(wb[w]), codes23(wa[w]), codes23(wb[w])};
                    const int step = 4 * j + w;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int pt = 0; pt < Sh::PARTS; ++pt) {
                            const int f = (step * NT + nt) * Sh::PARTS + pt;
                            const uint2 b = Sh::QREG ? qreg[Sh::QREG ? f : 0] : qfrag[f * 32 + lane];
                            mma16816(s[nt], A, b.x, b.y);
                        }
                }
            }
            float ksc[2] = {scales[g], scales[g + 8]}, vsc[2] = {scales[16 + g], scales[16 + g + 8]};
            const float lv0 = fmaxf(log2_fast(vsc[0]), -96.f), lv1 = fmaxf(log2_fast(vsc[1]), -96.f);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                s[nt][0] *= ksc[0] * rs[nt][0], s[nt][1] *= ksc[0] * rs[nt][1];
                s[nt][2] *= ksc[1] * rs[nt][0], s[nt][3] *= ksc[1] * rs[nt][1];
            }
            const bool masked = k0 + (GROUP - 1) >= clear_hi || k0 < clear_lo;
            if (masked) {
                const int ka = k0 + g, kb = k0 + g + 8;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int hi = row_hi[8 * nt + 2 * t + e], lo = row_lo[8 * nt + 2 * t + e];
                        if (ka >= hi || ka < lo) s[nt][e] = NEG;
                        if (kb >= hi || kb < lo) s[nt][2 + e] = NEG;
                    }
            }
            // the running maximum of s + log2 vscale over the warp's tokens, by query row
            float drop[NT][2];
            bool grew = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float m = fmaxf(s[nt][e] + lv0, s[nt][2 + e] + lv1);
                    m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
                    m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
                    m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
                    m = fmaxf(m, mx[nt][e]);
                    drop[nt][e] = m == NEG ? 0.f : mx[nt][e] - m;
                    grew = grew || m > mx[nt][e];
                    mx[nt][e] = m;
                }
            if (__any_sync(0xFFFFFFFFu, grew)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float f0 = exp2_fast(drop[nt][0]), f1 = exp2_fast(drop[nt][1]);
                    sum[nt][0] = lowered(sum[nt][0], drop[nt][0], f0), sum[nt][1] = lowered(sum[nt][1], drop[nt][1], f1);
#pragma unroll
                    for (int d = 0; d < Sh::MT; ++d) o[d][nt][0] *= f0, o[d][nt][1] *= f1, o[d][nt][2] *= f0, o[d][nt][3] *= f1;
                }
            }
            uint32_t pb[NT][Sh::PARTS][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float m = mx[nt][e & 1];
                    const float x = exp2_fast(s[nt][e] - (m == NEG ? 0.f : m - LIFT));
                    sum[nt][e & 1] = fmaf(x, DOWN, sum[nt][e & 1]);
                    p[e] = x * vsc[e >> 1];
                    if (masked && s[nt][e] == NEG) p[e] = 0.f;   // whatever the scale of a token that is not seen
                }
                __syncwarp();
                const uint32_t h0 = pack_half(p[0], p[1]), h1 = pack_half(p[2], p[3]);
                pb[nt][0][0] = transposed8x8(h0), pb[nt][0][1] = transposed8x8(h1);
                if constexpr (F32) {
                    pb[nt][1][0] = transposed8x8(pack_rest(p[0], p[1], h0));
                    pb[nt][1][1] = transposed8x8(pack_rest(p[2], p[3], h1));
                }
            }
            // output: a lane has tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9 of channels g DP / 8 ..
            const uint8_t *vt = st + GROUP * DP;
            const auto times_v = [&](int mt, uint32_t w0, uint32_t w1, uint32_t w8, uint32_t w9) {   // 4 channels: tiles mt, mt + 1
                const uint32_t a01 = __byte_perm(w0, w1, 0x5140), a23 = __byte_perm(w0, w1, 0x7362);
                const uint32_t b01 = __byte_perm(w8, w9, 0x5140), b23 = __byte_perm(w8, w9, 0x7362);
                const uint32_t A0[4] = {codes01(a01), codes23(a01), codes01(b01), codes23(b01)};
                const uint32_t A1[4] = {codes01(a23), codes23(a23), codes01(b23), codes23(b23)};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int pt = 0; pt < Sh::PARTS; ++pt) {
                        mma16816(o[mt][nt], A0, pb[nt][pt][0], pb[nt][pt][1]);
                        mma16816(o[mt + 1][nt], A1, pb[nt][pt][0], pb[nt][pt][1]);
                    }
            };
            const int tok[4] = {2 * t, 2 * t + 1, 2 * t + 8, 2 * t + 9};
            if constexpr (DP == 64) {
                uint2 w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    w[e] = *reinterpret_cast<const uint2 *>(vt + tok[e] * DP + Sh::swizzle(tok[e], g >> 1) * 16 + (g & 1) * 8);
                times_v(0, w[0].x, w[1].x, w[2].x, w[3].x);
                times_v(2, w[0].y, w[1].y, w[2].y, w[3].y);
            } else {
#pragma unroll
                for (int j = 0; j < DP / 128; ++j) {
                    uint4 w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        w[e] = *reinterpret_cast<const uint4 *>(vt + tok[e] * DP + Sh::swizzle(tok[e], g + 8 * j) * 16);
                    times_v(8 * j + 0, w[0].x, w[1].x, w[2].x, w[3].x);
                    times_v(8 * j + 2, w[0].y, w[1].y, w[2].y, w[3].y);
                    times_v(8 * j + 4, w[0].z, w[1].z, w[2].z, w[3].z);
                    times_v(8 * j + 6, w[0].w, w[1].w, w[2].w, w[3].w);
                }
            }
        }
        copies_wait<0>();
        __syncwarp();

        // ---- the four warps' shares: each leaves its output in its ring ----
        float *mine = reinterpret_cast<float *>(ring);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float l = sum[nt][e];
                l += __shfl_xor_sync(0xFFFFFFFFu, l, 4);
                l += __shfl_xor_sync(0xFFFFFFFFu, l, 8);
                l += __shfl_xor_sync(0xFFFFFFFFu, l, 16);
                const int r = 8 * nt + 2 * t + e;
                if (g == 0) join_m[warp][r] = mx[nt][e], join_l[warp][r] = l;
#pragma unroll
                for (int d = 0; d < Sh::MT; ++d) {   // tile d holds channels 2 d, 2 d + 1 of the lane's (of 16 j + .. with DP 256)
                    const int ch = DP == 64 ? 8 * g + 2 * d : 16 * (g + 8 * (d / 8)) + 2 * (d % 8);
                    *reinterpret_cast<float2 *>(mine + r * DP + ch) = make_float2(o[d][nt][e], o[d][nt][2 + e]);
                }
            }
        __syncthreads();
        const bool whole = count == tiles;
        const int first_cta = shares.owner(unit0), last_cta = shares.owner(unit0 + tiles - 1);
        float *slot = part + ((int64_t)2 * blockIdx.x + (from == 0 ? 1 : 0)) * PART;
        const auto finish = [&](int r, int d, const float4 &acc) {   // four values of row r, whose sum is row_l
            const int rr = u.r0 + r, qi = rr / a.group;
            const int64_t row = (int64_t)(u.q0 + qi) * a.n_heads + u.head * a.group + rr % a.group;
            const float m = row_m[r], l = row_l[r];
            const float inv = l == 0.f ? 0.f : 1.f / l * DOWN;   // (a sum of nothing: the row sees no token)
            const float y[4] = {acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv};
            T *o = (T *)a.out + row * D + d;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (F32)
                    o[e] = y[e];
                else
                    o[e] = __float2bfloat16_rn(y[e]);
            }
            if (d == 0 && a.lse != nullptr) a.lse[row] = l == 0.f ? NEG : (m + log2f(l)) * 0.6931471805599453f;
        };
        // (a share that saw nothing has maximum -inf, sum 0 and outputs 0; one that saw a NaN a sum of NaN)
        if (threadIdx.x < ROWS) {
            const int r = threadIdx.x;
            float m = NEG, l = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) m = fmaxf(m, join_m[w][r]);
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float mw = join_m[w][r], f = mw == NEG ? 0.f : exp2_fast(mw - m);
                l += lowered(join_l[w][r], mw - m, f);
                join_m[w][r] = f;
            }
            row_m[r] = m, row_l[r] = l;
            if (!whole) slot[ROWS * DP + r] = m, slot[ROWS * DP + ROWS + r] = l;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < u.rows * (DP / 4); i += THREADS) {
            const int r = i / (DP / 4), d = i % (DP / 4) * 4;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float4 v = reinterpret_cast<const float4 *>(smem + w * Sh::RING)[i];
                const float f = join_m[w][r];
                acc.x += v.x * f, acc.y += v.y * f, acc.z += v.z * f, acc.w += v.w * f;
            }
            if (!whole)
                reinterpret_cast<float4 *>(slot)[i] = acc;
            else if (d < D)
                finish(r, d, acc);
        }
        if (!whole) {
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0)
                last_one = atomicInc(reinterpret_cast<unsigned *>(a.counters) + first_cta, (unsigned)(last_cta - first_cta)) ==
                           (unsigned)(last_cta - first_cta);
            __syncthreads();
            if (last_one) {
                __threadfence();
                const auto slot_of = [&](int c) { return part + ((int64_t)2 * c + (c == first_cta ? 1 : 0)) * PART; };
                // The shares' maxima and sums, some shares at a time, into the rings; each row's maximum and sum over all of
                // them, a warp to a row; the shares' factors.
                constexpr int AT_ONCE = WARPS * Sh::RING / (ROWS * 8);
                const int parts = last_cta - first_cta + 1;
                float *const ms = reinterpret_cast<float *>(smem), *const ls = ms + AT_ONCE * ROWS;
                for (int pass = 0; pass < 2; ++pass)   // (of more shares than fit, the maxima go first)
                    for (int c0 = 0; c0 < parts; c0 += AT_ONCE) {
                        const int n = min(AT_ONCE, parts - c0);
                        if (parts <= AT_ONCE && pass == 1) break;
                        __syncthreads();
#pragma unroll 4
                        for (int i = threadIdx.x; i < n * ROWS; i += THREADS) {
                            const float *p = slot_of(first_cta + c0 + i / ROWS) + ROWS * DP + i % ROWS;
                            ms[i] = __ldcg(p), ls[i] = __ldcg(p + ROWS);
                        }
                        __syncthreads();
                        for (int r = warp; r < u.rows; r += WARPS) {
                            float m = c0 + pass == 0 ? NEG : row_m[r], l = c0 == 0 ? 0.f : row_l[r];
                            if (pass == 0) {
                                for (int c = lane; c < n; c += 32) m = fmaxf(m, ms[c * ROWS + r]);
#pragma unroll
                                for (int o = 16; o; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
                            }
                            if (pass == 1 || parts <= AT_ONCE) {
                                float some = 0.f;
                                for (int c = lane; c < n; c += 32) {
                                    const float mc = ms[c * ROWS + r], f = mc == NEG ? 0.f : exp2_fast(mc - m);
                                    some += lowered(ls[c * ROWS + r], mc - m, f);
                                    ms[c * ROWS + r] = f;
                                }
#pragma unroll
                                for (int o = 16; o; o /= 2) some += __shfl_xor_sync(0xFFFFFFFFu, some, o);
                                l += some;
                            }
                            if (lane == 0) row_m[r] = m, row_l[r] = l;
                        }
                    }
                __syncthreads();
                // the outputs in the order of the shares, several of them under way
                const bool ready = parts <= AT_ONCE;
                constexpr int DEEP = 8;   // (with more, the whole kernel takes registers that cost it a CTA to the SM)
                for (int i = threadIdx.x; i < u.rows * (DP / 4); i += THREADS) {
                    const int r = i / (DP / 4), d = i % (DP / 4) * 4;
                    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                    const float m = row_m[r];
#pragma unroll 1
                    for (int c0 = 0; c0 < parts; c0 += DEEP) {
                        float4 v[DEEP];
#pragma unroll
                        for (int k = 0; k < DEEP; ++k)
                            if (c0 + k < parts) v[k] = __ldcg(reinterpret_cast<const float4 *>(slot_of(first_cta + c0 + k)) + i);
#pragma unroll
                        for (int k = 0; k < DEEP; ++k)
                            if (c0 + k < parts) {
                                float f;
                                if (ready) {
                                    f = ms[(c0 + k) * ROWS + r];
                                } else {
                                    const float mc = __ldcg(slot_of(first_cta + c0 + k) + ROWS * DP + r);
                                    f = mc == NEG ? 0.f : exp2_fast(mc - m);
                                }
                                acc.x += v[k].x * f, acc.y += v[k].y * f, acc.z += v[k].z * f, acc.w += v[k].w * f;
                            }
                    }
                    if (d < D) finish(r, d, acc);
                }
            }
        }
        __syncthreads();   // the rings and the rows' numbers are free again
    }
    wait_for_previous();   // (the prompts' kernel, beside which this one may run: what comes after waits for both)
}

template <int DP, int NT, bool F32, class T> realq_status_t launch(cudaStream_t s, const KvAttnArgs &a, int sms) {
    using Sh = Shape<DP, NT, F32>;
    const auto kernel = decode_kernel<DP, NT, F32, T>;
    REALQ_TRY(set_smem_limit((const void *)kernel, Sh::SMEM));
    int per_sm = 0;
    REALQ_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, THREADS, Sh::SMEM));
    per_sm = std::max(1, std::min(per_sm, KV_MAX_CTAS_PER_SM));
    Launch l("kv_attention", s);
    // beside the prompts' kernel of the same call, which writes nothing that this one reads; else after what came before
    if (a.min_new == 1 && a.max_new < INT32_MAX)
        REALQ_CUDA_TRY(launch_overlapped(kernel, dim3((unsigned)(per_sm * sms)), dim3(THREADS), Sh::SMEM, s, a));
    else
        kernel<<<(unsigned)(per_sm * sms), THREADS, Sh::SMEM, s>>>(a);
    return check_launch("kv_attention");
}
template <int DP, bool F32, class T> realq_status_t by_rows(cudaStream_t s, const KvAttnArgs &a, int64_t rows, int sms) {
    if (rows <= 8) return launch<DP, 1, F32, T>(s, a, sms);
    if constexpr (DP == 256) {
        return launch<DP, 2, F32, T>(s, a, sms);
    } else {
        if (rows <= 16) return launch<DP, 2, F32, T>(s, a, sms);
        return launch<DP, 4, F32, T>(s, a, sms);
    }
}
template <class T> realq_status_t by_size(cudaStream_t s, const KvAttnArgs &a, int64_t rows, int sms) {
    constexpr bool F32 = sizeof(T) == 4;
    if (a.c.head_dim <= 64) return by_rows<64, F32, T>(s, a, rows, sms);
    if (a.c.head_dim <= 128) return by_rows<128, F32, T>(s, a, rows, sms);
    return by_rows<256, F32, T>(s, a, rows, sms);
}

}  // namespace

// Partial results: two a CTA of at most 32 rows of DP + 2 numbers each (16 rows of 256 + 2 are fewer).
size_t kv_decode_ws_bytes(int sms) {
    Carve c(nullptr);
    c.take<int>(KV_MAX_CTAS_PER_SM * sms);
    c.take<float>((size_t)2 * KV_MAX_CTAS_PER_SM * sms * 32 * (128 + 2));
    return c.off;
}

realq_status_t kv_decode(cudaStream_t s, const KvAttnArgs &args, realq_dtype_t dt, int64_t rows, void *ws, int sms) {
    KvAttnArgs a = args;
    Carve c(ws);
    a.counters = c.take<int>(KV_MAX_CTAS_PER_SM * sms);
    a.part = c.take<float>(0);
    return dt == REALQ_BF16 ? by_size<__nv_bfloat16>(s, a, rows, sms) : by_size<float>(s, a, rows, sms);
}

}  // namespace realq
