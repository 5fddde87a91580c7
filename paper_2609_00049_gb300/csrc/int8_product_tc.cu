// The 8-bit product for more than a few tokens, on the 5th-generation tensor
// cores: Y^T tiles of 128 output channels by up to 256 tokens.
//
// Code minus zero point is a whole number of at most nine bits, exact in fp16,
// and so are the products in fp32 and, while the running sum is below 2^24,
// their sums: kind::f16 gives the integer product at the bf16 rate (the int8
// rate of this GPU is far below it).  A running sum past 2^24 may lose about a
// unit in its last place at each accumulated MMA (16 of K), whatever the final
// sum.  Measured against the exact sums, with a plain fp32 product of the same
// values beside it: codes of one sign, n = 28672, off by 2.4e-7 of the result
// (3e-7); n = 131071, 7.2e-6 (7e-7); 28672 columns whose second half takes a sum
// of 4.6e8 away again, off by 7 (15).
//
// The weight codes are converted on their way in, so that they cross HBM and L2
// as bytes (or nibbles): TMA puts the codes of a K step (64, or 128 where a
// tile has at most 128 tokens and the waits between roles would cost more than
// the MMAs) in shared memory (swizzled by row length: a thread reads its row's 16-byte chunks
// without bank conflicts), eight converter warps, two groups taking turns, make
// fp16 pairs of them (the byte as the low mantissa bits of 1024, less
// 1024 + zero) and store them to TMEM as the MMA's A operand: lane = channel,
// a column to two of K.  Shared memory then carries only the tokens' plane,
// which a pass over the token codes writes as fp16 to the workspace; B is a
// K-major tile of it (128-byte swizzle).
//
// Roles (608 threads, one persistent CTA per SM): warps 0-7 convert, warps
// 8-15 drain the accumulator (lane = channel, so a warp's stores of one token
// are contiguous; two warps take turns at a lane quarter's 32-column blocks),
// warps 16 and 17 issue the TMA loads of tokens and codes, warp 18 the MMAs.  TMEM: an
// accumulator of up to 256 columns and eight A slots of 64 K, or two of up to
// 192 (a drain then overlaps the next tile) and four, or two of up to 128 and
// four of 128 K.  The codes have a ring
// of their own, freed by the converters, and run ahead of the tokens, whose
// stages (and the A slots) the MMAs free: a stage of either then covers one
// memory latency, not the conversion as well.  Tiles beyond whole
// waves over the SMs have their K range split; a second pass adds the
// parts in their order.
// Every wait is bounded; a tile whose wait gave up is written as NaN and the
// status word gets ST_TIMEOUT.
//
// Measured, 8192 tokens x 8192 x 8192: 568 us alone (1.94 PFLOP/s; the tensor
// pipe 82 % active at 2048 x 4096 x 9728), 36 us for the tokens' plane and 10 for
// the parts; a call 588 to 655 us among others, as the power cap has it, 575 to
// 602 with 4-bit weights.  Issued by one lane under a branch, with one ring for codes and
// tokens and the scales fetched while draining, it was 1.04 ms.
#include "bytes.cuh"
#include "kernels.cuh"
#include "tc.cuh"

#include <algorithm>

namespace realq {
namespace {

constexpr int TM = 128;                    // channels per tile
constexpr int TNMAX = 256;                 // tokens per tile
constexpr int MAX_STAGES = 8;              // of the tokens' ring and of A in TMEM
constexpr int MAX_WSTAGES = 16;            // of the codes' ring
constexpr int CONV_WARPS = 8, EPI_WARPS = 8;
constexpr int THREADS = (CONV_WARPS + EPI_WARPS + 3) * 32;
constexpr int RING_BYTES = 204800;
constexpr int SMEM_BYTES = RING_BYTES + 1024 + 512;
constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int MAX_SPLITS = 16;

__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

struct Shape {
    int64_t T, n, m;
    int N;            // tokens per tile, a multiple of 16
    int kstep;        // K per stage
    int acc, a0;      // TMEM: columns between the two accumulators (0: there is one), first column of the A slots
    int stages, wstages;   // ring lengths: tokens and A slots, codes
    int nti, ntj;     // tiles over channels, tokens
    int whole;        // tiles that keep their K range; the others are split
    int splits, per;  // K parts of those, K steps per part
    int ks;           // K steps
    int items;
};

struct Item {
    int ti, tj;       // channel tile, token tile
    int k0, nk;       // K steps
    int slot, z;      // split tiles: number among them and part (slot < 0: whole)
};

// Stage index and phase parity of a ring of S stages
struct Ring {
    int s = 0, S;
    uint32_t phase = 0;
    __device__ __forceinline__ explicit Ring(int stages) : S(stages) {}
    __device__ __forceinline__ void next() {
        if (++s == S) {
            s = 0;
            phase ^= 1u;
        }
    }
};

// Work item w: first the whole tiles, then the parts of the others (all first
// parts, all second parts, ...).  Tiles go in groups of 8 channel tiles, so that
// the CTAs running together share codes and tokens in L2.
__device__ __forceinline__ Item item_of(const Shape &sh, int w) {
    constexpr int G = 8;
    Item it;
    int t = w;
    if (w < sh.whole) {
        it.k0 = 0;
        it.nk = sh.ks;
        it.slot = -1;
        it.z = 0;
    } else {
        const int cut = sh.nti * sh.ntj - sh.whole;
        it.z = (w - sh.whole) / cut;
        it.slot = w - sh.whole - it.z * cut;
        it.k0 = it.z * sh.per;
        it.nk = min(sh.per, sh.ks - it.k0);
        t = sh.whole + it.slot;
    }
    const int g = t / (G * sh.ntj), r0 = g * G, rows = min(G, sh.nti - r0), k = t - g * G * sh.ntj;
    it.ti = r0 + k % rows;
    it.tj = k / rows;
    return it;
}

// Four bytes -> two fp16 pairs, eight nibbles of a word -> four pairs, less the zero point
__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

template <int WB, int KS, typename TY>
__global__ void __launch_bounds__(THREADS, 1)
    int8_tc_kernel(const __grid_constant__ CUtensorMap mapW, const __grid_constant__ CUtensorMap mapX, const Shape sh,
                   const float *x_scale, const float *w_scale, const uint8_t *w_zero, TY *Y, float *part, int *err) {
    constexpr int WROW = WB == 8 ? KS : KS / 2;   // bytes of a row of codes per stage
    constexpr int W_BYTES = TM * WROW;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t *xfull = reinterpret_cast<uint64_t *>(smem + RING_BYTES);
    uint64_t *ready = xfull + MAX_STAGES;        // A slot converted
    uint64_t *empty = ready + MAX_STAGES;        // tokens' stage and A slot read by the MMAs
    uint64_t *wfull = empty + MAX_STAGES;
    uint64_t *wempty = wfull + MAX_WSTAGES;      // codes' stage converted
    uint64_t *accf = wempty + MAX_WSTAGES;       // [2] accumulator complete
    uint64_t *acce = accf + 2;                   // [2] accumulator drained
    uint64_t *done = acce + 2;
    uint32_t *tslot = reinterpret_cast<uint32_t *>(done + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tslot + 1);

    dependents_may_start();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int x_bytes = sh.N * KS * 2;           // a multiple of 1024, as W_BYTES; KS / 64 boxes
    const int items = sh.items, S = sh.stages, SW = sh.wstages;
    uint8_t *wring = smem + S * x_bytes;
    const bool two = sh.acc > 0;                 // two accumulators

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            tc::mbar_init(tc::smem_u32(&xfull[s]), 1);
            tc::mbar_init(tc::smem_u32(&ready[s]), 4);
            tc::mbar_init(tc::smem_u32(&empty[s]), 1);
        }
        for (int s = 0; s < SW; ++s) {
            tc::mbar_init(tc::smem_u32(&wfull[s]), 1);
            tc::mbar_init(tc::smem_u32(&wempty[s]), 4);
        }
        for (int b = 0; b < 2; ++b) {
            tc::mbar_init(tc::smem_u32(&accf[b]), 1);
            tc::mbar_init(tc::smem_u32(&acce[b]), EPI_WARPS);
        }
        tc::mbar_init(tc::smem_u32(done), 1);
        *abort_flag = 0;
        tc::fence_barrier_init();
        tc::prefetch_tmap(&mapW);
        tc::prefetch_tmap(&mapX);
    }
    if (warp == 0) tc::tmem_alloc(tc::smem_u32(tslot), 512);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = *tslot;
    bool good = true;

    if (warp < CONV_WARPS) {
        // ---------------- converters: codes -> fp16 in TMEM ----------------
        const int group = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t a_base = tmem + (uint32_t)sh.a0 + ((uint32_t)((warp & 3) * 32) << 16);
        Ring r(S), rw(SW);   // over all of this CTA's items
        bool ok = true;
        int turn = 0;
        for (int w = blockIdx.x; w < items && ok; w += gridDim.x) {
            const Item im = item_of(sh, w);
            const int64_t gi = (int64_t)im.ti * TM + row;
            const int zero = w_zero && gi < sh.m ? __ldg(w_zero + gi) : (WB == 8 ? 128 : 8);
            // 1024 + z (and 64 + z for the upper nibble's position), exact in fp16
            const uint32_t hz = 0x6400u + (uint32_t)zero;
            const uint32_t base =
                WB == 8 ? hz | hz << 16 : hz | (uint32_t)__half_as_ushort(__int2half_rn(64 + zero)) << 16;
            for (int kk = 0; kk < im.nk; ++kk, r.next(), rw.next(), turn ^= 1) {
                if (turn != group) continue;
                const bool got = tc::mbar_wait(tc::smem_u32(&wfull[rw.s]), rw.phase, abort_flag) &&
                                 tc::mbar_wait(tc::smem_u32(&empty[r.s]), r.phase ^ 1u, abort_flag);
                if (!__all_sync(FULL, got)) {
                    *abort_flag = 1;
                    ok = false;
                    break;
                }
                tc::fence_after_sync();
                const uint8_t *src = wring + rw.s * W_BYTES + row * WROW;
                constexpr int CH = WB == 8 ? 4 : 2;   // 16-byte chunks to 64 of K
#pragma unroll
                for (int o = 0; o < KS / 64; ++o) {
                    uint32_t h[32];
#pragma unroll
                    for (int c = 0; c < CH; ++c) {
                        // the swizzle's place of the row's chunk: 128-byte rows, bits 4-6 ^= 7-9; 64, bits 4-5 ^= 7-8;
                        // 32, bit 4 ^= 7
                        const int cc = o * CH + c;
                        const int at = WROW == 128 ? cc ^ (row & 7) : (WROW == 64 ? cc ^ ((row >> 1) & 3) : cc ^ ((row >> 2) & 1));
                        const uint4 q = *reinterpret_cast<const uint4 *>(src + at * 16);
                        const uint32_t v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if constexpr (WB == 8) {
                                h[c * 8 + i * 2] = sub2(__byte_perm(v[i], 0x64646464u, 0x4140), base);
                                h[c * 8 + i * 2 + 1] = sub2(__byte_perm(v[i], 0x64646464u, 0x4342), base);
                            } else {
#pragma unroll
                                for (int b = 0; b < 4; ++b) {
                                    const uint32_t t = __byte_perm(v[i], 0u, 0x4040 | b | b << 8);
                                    h[c * 16 + i * 4 + b] = sub2((t & 0x00F0000Fu) | 0x54006400u, base);
                                }
                            }
                        }
                    }
                    tc::tmem_st_32x32b_x32(a_base + (uint32_t)(r.s * (KS / 2) + o * 32), h);
                }
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(tc::smem_u32(&wempty[rw.s]));
                tc::tmem_wait_st();
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(tc::smem_u32(&ready[r.s]));
            }
        }
    } else if (warp < CONV_WARPS + EPI_WARPS) {
        // ---------------- drain: accumulator -> Y or a part ----------------
        const int quarter = warp & 3, half = (warp - CONV_WARPS) >> 2;
        int lt = 0;
        for (int w = blockIdx.x; w < items; w += gridDim.x, ++lt) {
            const Item im = item_of(sh, w);
            const bool cut = im.slot >= 0;
            const int b = two ? lt & 1 : 0, round = two ? lt >> 1 : lt;
            const int64_t gi = (int64_t)im.ti * TM + quarter * 32 + lane;
            const int64_t t0 = (int64_t)im.tj * sh.N;
            const bool mine = gi < sh.m;
            const int nt = (int)min((int64_t)sh.N, sh.T - t0);   // tokens of this tile
            const float sw = mine ? __ldg(w_scale + gi) : 0.f;
            float sx[4];                                         // of this warp's four blocks, one token to a lane
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = (2 * j + half) * 32 + lane;
                sx[j] = t < nt ? __ldg(x_scale + t0 + t) : 0.f;
            }
            const int ncut = sh.nti * sh.ntj - sh.whole;
            auto part_of = [&](int z) {   // this lane's channel of a part: tokens TM apart
                return part + ((int64_t)z * ncut + im.slot) * sh.N * TM + quarter * 32 + lane;
            };
            if (good) {
                const bool got = tc::mbar_wait(tc::smem_u32(&accf[b]), (uint32_t)round & 1u, abort_flag);
                if (!__all_sync(FULL, got)) {
                    *abort_flag = 1;
                    good = false;   // this tile and the CTA's later ones are written as NaN
                }
            }
            tc::fence_after_sync();
            const uint32_t src = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(b * sh.acc);
            const int blocks = (sh.N + 31) / 32, mine_last = (blocks - 1 - half) / 2;   // blocks 2 j + half, j <= mine_last
            if (good && blocks <= half) {
                tc::fence_before_sync();
                if (lane == 0) tc::mbar_arrive(tc::smem_u32(&acce[b]));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c0 = (2 * j + half) * 32;
                if (c0 >= sh.N) continue;
                uint32_t v[32];
                if (good) {
                    // (a last block of 16 columns reads 16 more, which stay unused)
                    tc::tmem_ld_32x32b_x32(src + (uint32_t)c0, v);
                    if (j == mine_last) {
                        tc::fence_before_sync();
                        __syncwarp();
                        if (lane == 0) tc::mbar_arrive(tc::smem_u32(&acce[b]));
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < 32; ++q) v[q] = 0x7fc00000u;
                }
                const int nq = nt - c0;
                if (cut) {
                    float *p = part_of(im.z) + c0 * TM;
#pragma unroll
                    for (int q = 0; q < 32; ++q)
                        if (q < nq) p[q * TM] = __uint_as_float(v[q]);
                } else {
                    TY *y = Y + (t0 + c0) * sh.m + gi;
#pragma unroll
                    for (int q = 0; q < 32; ++q, y += sh.m) {
                        const float r = __uint_as_float(v[q]) * __shfl_sync(FULL, sx[j], q) * sw;
                        if (mine && q < nq) store1(y, r);
                    }
                }
            }
        }
    } else if (warp < CONV_WARPS + EPI_WARPS + 2) {
        if (lane == 0) {
            // ---------------- TMA producers: tokens, codes ----------------
            const bool codes = warp == CONV_WARPS + EPI_WARPS + 1;
            if (!codes) wait_for_previous();   // the tokens' plane (the codes are there)
            uint64_t *fulls = codes ? wfull : xfull, *empties = codes ? wempty : empty;
            uint8_t *ring = codes ? wring : smem;
            const int bytes = codes ? W_BYTES : x_bytes;
            const CUtensorMap *map = codes ? &mapW : &mapX;
            Ring r(codes ? SW : S);
            int it = 0;
            bool ok = true;
            for (int w = blockIdx.x; w < items && ok; w += gridDim.x) {
                const Item im = item_of(sh, w);
                const int dx = codes ? WROW : KS, y = codes ? im.ti * TM : im.tj * sh.N;
                int x = im.k0 * dx;
                for (int kk = 0; kk < im.nk; ++kk, ++it, r.next(), x += dx) {
                    ok = tc::mbar_wait(tc::smem_u32(&empties[r.s]), r.phase ^ 1u, abort_flag);
                    if (!ok) break;
                    const uint32_t fb = tc::smem_u32(&fulls[r.s]);
                    tc::mbar_arrive_expect_tx(fb, (uint32_t)bytes);
                    const uint32_t dst = tc::smem_u32(ring + r.s * bytes);
                    tc::tma_load_2d(dst, map, fb, x, y);
                    if (KS == 128 && !codes) tc::tma_load_2d(dst + (x_bytes >> 1), map, fb, x + 64, y);
                }
            }
            // on abort, let the copies already issued land before the CTA exits
            if (!ok || *abort_flag) {
                *abort_flag = 1;
                int never = 0;
                for (int k = (it > r.S ? it - r.S : 0); k < it; ++k)
                    tc::mbar_wait(tc::smem_u32(&fulls[k % r.S]), (uint32_t)(k / r.S) & 1u, &never, 100000000ull);
            }
        }
    } else {
        // ---------------- MMA issuer (the whole warp waits, one lane issues) ----------------
        const uint32_t idesc = tc::idesc_f16_f32(TM, 0) | ((uint32_t)(sh.N >> 3) << 17);
        const uint64_t desc0 = tc::smem_desc(tc::smem_u32(smem), 16, 1024, tc::SW_128B);
        Ring r(S);
        int lt = 0;
        bool ok = true;
        for (int w = blockIdx.x; w < items && ok; w += gridDim.x, ++lt) {
            const Item im = item_of(sh, w);
            const int b = two ? lt & 1 : 0, round = two ? lt >> 1 : lt;
            ok = __all_sync(FULL, tc::mbar_wait(tc::smem_u32(&acce[b]), ((uint32_t)round & 1u) ^ 1u, abort_flag));
            if (!ok) break;
            tc::fence_after_sync();
            const uint32_t d = tmem + (uint32_t)(b * sh.acc);
            for (int kk = 0; kk < im.nk; ++kk, r.next()) {
                ok = tc::mbar_wait(tc::smem_u32(&ready[r.s]), r.phase, abort_flag) &&
                     tc::mbar_wait(tc::smem_u32(&xfull[r.s]), r.phase, abort_flag);
                ok = __all_sync(FULL, ok);
                if (!ok) break;
                tc::fence_after_sync();
                const uint64_t desc = desc0 + (uint32_t)(r.s * x_bytes >> 4);
                const uint32_t a = tmem + (uint32_t)(sh.a0 + r.s * (KS / 2));
                if (tc::elect_one()) {
#pragma unroll
                    for (int k = 0; k < KS / 16; ++k)
                        tc::mma_f16_ts(d, a + k * 8, desc + (k & 3) * 2 + (k >> 2) * (uint32_t)(x_bytes >> 5), idesc,
                                       (kk > 0 || k > 0) ? 1u : 0u);
                    tc::mma_commit(tc::smem_u32(&empty[r.s]));
                }
                __syncwarp();
            }
            if (ok && tc::elect_one()) tc::mma_commit(tc::smem_u32(&accf[b]));
            __syncwarp();
        }
        if (!ok) *abort_flag = 1;
        // every MMA issued has retired before TMEM is freed
        if (tc::elect_one()) tc::mma_commit(tc::smem_u32(done));
        __syncwarp();
        int never = 0;
        tc::mbar_wait(tc::smem_u32(done), 0u, &never, 100000000ull);
    }
    __syncwarp();
    if (!good && lane == 0) atomicOr(err, ST_TIMEOUT);
    tc::fence_before_sync();
    __syncthreads();
    if (warp == 0) tc::tmem_dealloc(tmem, 512);
}

// The split tiles: parts added in their order, scaled and stored.  A block takes
// 8 tokens of a tile, a thread four neighbouring channels.
template <typename TY>
__global__ void __launch_bounds__(256) int8_reduce_kernel(const Shape sh, const float *part, const float *x_scale,
                                                          const float *w_scale, TY *Y) {
    wait_for_previous();
    const int cut = sh.nti * sh.ntj - sh.whole, slot = blockIdx.x;
    const Item im = item_of(sh, sh.whole + slot);
    const int t = blockIdx.y * 8 + (threadIdx.x >> 5), c = (threadIdx.x & 31) * 4;
    const int64_t tok = (int64_t)im.tj * sh.N + t, i = (int64_t)im.ti * TM + c;
    if (t >= sh.N || tok >= sh.T || i >= sh.m) return;
    const float4 *p = reinterpret_cast<const float4 *>(part + ((int64_t)slot * sh.N + t) * TM + c);
    const int64_t step = (int64_t)cut * sh.N * TM / 4;
    float4 a = load_after_wait(p);
#pragma unroll 4
    for (int z = 1; z < sh.splits; ++z) {
        const float4 b = load_after_wait(p + z * step);
        a.x += b.x;
        a.y += b.y;
        a.z += b.z;
        a.w += b.w;
    }
    const float sx = __ldg(x_scale + tok), v[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k < sh.m) store1(Y + tok * sh.m + i + k, v[k] * sx * __ldg(w_scale + i + k));
}

// Token codes -> fp16 plane of row stride ld (16 codes per thread where rows
// are whole vectors)
__device__ __forceinline__ void store_codes(uint4 *o, const uint4 &q, bool both) {
    const uint32_t v[4] = {q.x, q.y, q.z, q.w};
    uint32_t h[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        h[2 * j] = sub2(__byte_perm(v[j], 0x64646464u, 0x4140), 0x64806480u);
        h[2 * j + 1] = sub2(__byte_perm(v[j], 0x64646464u, 0x4342), 0x64806480u);
    }
    o[0] = make_uint4(h[0], h[1], h[2], h[3]);
    if (both) o[1] = make_uint4(h[4], h[5], h[6], h[7]);
}
__global__ void __launch_bounds__(256) int8_plane_vec_kernel(int64_t count, const uint8_t *X, uint32_t *plane) {
    dependents_may_start();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < count)
        store_codes(reinterpret_cast<uint4 *>(plane) + 2 * i, __ldg(reinterpret_cast<const uint4 *>(X) + i), true);
}
// any width and address; 16 codes a thread, ld a multiple of 8
__global__ void __launch_bounds__(256) int8_plane_kernel(int64_t T, int64_t n, const uint8_t *X, __half *plane,
                                                         int64_t ld) {
    dependents_may_start();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, pieces = (n + 15) / 16;
    if (i >= T * pieces) return;
    int64_t c;
    const int64_t t = divide(i, pieces, c);
    store_codes(reinterpret_cast<uint4 *>(plane + t * ld + c * 16), load16(X + t * n + c * 16, X, X + T * n),
                c * 16 + 8 < ld);
}
// rows of W at a stride of whole 16-byte pieces (what pads them lies outside the tensor map)
__global__ void __launch_bounds__(256) int8_pad_kernel(int64_t m, int64_t rb, const uint8_t *W, uint8_t *out,
                                                       int64_t ld) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, pieces = ld / 16;
    if (i >= m * pieces) return;
    int64_t c;
    const int64_t r = divide(i, pieces, c);
    reinterpret_cast<uint4 *>(out)[i] = load16(W + r * rb + c * 16, W, W + m * rb);
}

int64_t pad8(int64_t x) { return (x + 7) / 8 * 8; }
int64_t pad16(int64_t x) { return (x + 15) / 16 * 16; }
int64_t row_bytes(int64_t n, int w_bits) { return w_bits == 8 ? n : (n + 1) / 2; }

// One choice of token tiles: ntj of them, evenly filled, and its estimate in
// cycles.  Tiles that fill whole waves over the SMs keep their K range; the rest
// is cut into parts of at least four steps.  For 64 of K a tile of up to 128
// tokens takes 440 cycles (its conversions and waits), a larger one 2 N and 60,
// at least 520; its start and drain take 3500, or 800 where a second accumulator
// lets them overlap the next tile; the pass over the parts 5000 and the parts'
// bytes 3400 to a cycle, twice.
int64_t shape_for(Shape &sh, int64_t T, int64_t n, int64_t m, int64_t ntj, int w_bits, int sms) {
    sh.T = T;
    sh.n = n;
    sh.m = m;
    sh.N = (int)std::max<int64_t>(16, ((T + ntj - 1) / ntj + 15) / 16 * 16);
    sh.ntj = (int)((T + sh.N - 1) / sh.N);
    sh.nti = ceil_div(m, TM);
    sh.kstep = sh.N <= 128 ? 128 : 64;
    sh.acc = sh.N <= 128 ? 128 : (sh.N <= 192 ? 192 : 0);
    sh.a0 = sh.acc == 192 ? 384 : 256;
    const int KS = sh.kstep, xb = sh.N * KS * 2, wb = TM * (w_bits == 8 ? KS : KS / 2);
    sh.stages = std::min((512 - sh.a0) / (KS / 2), RING_BYTES / (xb + wb));
    sh.wstages = std::min(MAX_WSTAGES, (RING_BYTES - sh.stages * xb) / wb);
    sh.ks = ceil_div(n, KS);
    const int64_t tiles = (int64_t)sh.nti * sh.ntj, rest = tiles % sms;
    const int64_t step = sh.N <= 128 ? 880 : std::max(520, 2 * sh.N + 60), ends = sh.acc ? 800 : 3500;
    int parts = 1;
    int64_t cost = rest > 0 ? INT64_MAX : 0;
    for (int s = 1; s <= MAX_SPLITS && (s == 1 || sh.ks * KS / 64 / s >= 4) && s <= sh.ks && rest > 0 &&
                    (s == 1 || rest * s <= 2 * sms); ++s) {
        const int64_t c = (rest * s + sms - 1) / sms * ((sh.ks + s - 1) / s * step + ends) +
                          (s > 1 ? 5000 + 2 * rest * s * sh.N * TM * 4 / 3400 : 0);
        if (c < cost) {
            cost = c;
            parts = s;
        }
    }
    sh.per = (sh.ks + parts - 1) / parts;
    sh.splits = (sh.ks + sh.per - 1) / sh.per;
    sh.whole = (int)(sh.splits > 1 ? tiles - rest : tiles);
    sh.items = (int)(sh.whole + (tiles - sh.whole) * sh.splits);
    return cost + tiles / sms * (sh.ks * step + ends);
}

// The fastest of: tiles of up to 256 tokens, of up to 192 (two accumulators), and
// smaller ones where that leaves SMs idle.
Shape shape_of(int64_t T, int64_t n, int64_t m, int w_bits, int sms) {
    const int64_t fewest = (T + TNMAX - 1) / TNMAX, stride = std::max<int64_t>(1, fewest / 2);
    Shape best{}, sh{};
    int64_t best_cost = shape_for(best, T, n, m, fewest, w_bits, sms);
    auto offer = [&](int64_t ntj) {
        const int64_t cost = shape_for(sh, T, n, m, ntj, w_bits, sms);
        if (cost < best_cost) {
            best_cost = cost;
            best = sh;
        }
    };
    offer((T + 191) / 192);
    if ((int64_t)best.nti * fewest < 4 * sms)
        for (int64_t ntj = fewest + stride; ntj <= 4 * fewest; ntj += stride) offer(ntj);
    return best;
}

struct ProductWs {
    int *status;
    __half *x;
    uint8_t *w;
    float *part;
    size_t bytes;
    ProductWs(void *ws, const Shape &sh, int w_bits) {
        Carve c(ws);
        const int64_t rb = row_bytes(sh.n, w_bits);
        const int64_t cut = sh.splits > 1 ? (int64_t)sh.nti * sh.ntj - sh.whole : 0;
        status = c.take<int>(64);
        x = c.take<__half>((size_t)(sh.T * pad8(sh.n)));
        w = c.take<uint8_t>(rb % 16 ? (size_t)(sh.m * pad16(rb)) : 0);
        part = c.take<float>((size_t)(cut * sh.splits * sh.N * TM));
        bytes = c.off;
    }
};

template <int WB, int KS, typename TY>
realq_status_t tc_launch(cudaStream_t s, const Shape &sh, const CUtensorMap &mapW, const CUtensorMap &mapX,
                         const float *xs, const float *ws, const uint8_t *wz, TY *Y, const ProductWs &b, int sms) {
    const void *k = reinterpret_cast<const void *>(int8_tc_kernel<WB, KS, TY>);
    REALQ_TRY(set_smem_limit(k, SMEM_BYTES));
    {
        Launch L("int8_product_tc", s);
        REALQ_CUDA_TRY(launch_overlapped(int8_tc_kernel<WB, KS, TY>, dim3((unsigned)std::min(sh.items, sms)), dim3(THREADS),
                                         SMEM_BYTES, s, mapW, mapX, sh, xs, ws, wz, Y, b.part, b.status));
    }
    REALQ_TRY(check_launch("int8_product_tc"));
    if (sh.splits > 1) {
        Launch L("int8_product_reduce", s);
        REALQ_CUDA_TRY(launch_overlapped(int8_reduce_kernel<TY>,
                                         dim3((unsigned)(sh.nti * sh.ntj - sh.whole), (unsigned)((sh.N + 7) / 8)),
                                         dim3(256), 0, s, sh, (const float *)b.part, xs, ws, Y));
    }
    return check_launch("int8_product_reduce");
}

}  // namespace

size_t int8_tc_ws_bytes(int64_t T, int64_t n, int64_t m, int w_bits, int sms) {
    return ProductWs(nullptr, shape_of(T, n, m, w_bits, sms), w_bits).bytes;
}


realq_status_t int8_product_tc(cudaStream_t s, int64_t T, int64_t n, int64_t m, const uint8_t *X, const float *x_scale,
                               const uint8_t *W, int w_bits, const float *w_scale, const uint8_t *w_zero, void *Y,
                               realq_dtype_t y_dtype, void *ws, int sms) {
    const Shape sh = shape_of(T, n, m, w_bits, sms);
    const ProductWs b(ws, sh, w_bits);
    const int64_t ldx = pad8(n), rb = row_bytes(n, w_bits);
    const uint8_t *w = W;
    int64_t ldw = rb;
    if (rb % 16) {
        ldw = pad16(rb);
        w = b.w;
        Launch L("int8_product_pad", s);
        int8_pad_kernel<<<(unsigned)((m * (ldw / 16) + 255) / 256), 256, 0, s>>>(m, rb, W, b.w, ldw);
        REALQ_TRY(check_launch("int8_product_pad"));
    }
    {
        Launch L("int8_product_plane", s);
        if (n % 16 == 0 && (reinterpret_cast<uintptr_t>(X) & 15) == 0)
            int8_plane_vec_kernel<<<(unsigned)((T * n / 16 + 255) / 256), 256, 0, s>>>(
                T * n / 16, X, reinterpret_cast<uint32_t *>(b.x));
        else
            int8_plane_kernel<<<(unsigned)((T * ((n + 15) / 16) + 255) / 256), 256, 0, s>>>(T, n, X, b.x, ldx);
    }
    REALQ_TRY(check_launch("int8_product_plane"));
    const int wrow = w_bits == 8 ? sh.kstep : sh.kstep / 2;
    CUtensorMap mapW, mapX;
    CUresult cr = encode_tmap_2d_u8(&mapW, w, (uint64_t)rb, (uint64_t)m, (uint64_t)ldw, (uint32_t)wrow, TM,
                                    wrow == 128 ? 1 : (wrow == 64 ? 2 : 3));
    if (cr == CUDA_SUCCESS)
        cr = encode_tmap_2d_f16(&mapX, b.x, (uint64_t)n, (uint64_t)T, (uint64_t)ldx * 2, 64, (uint32_t)sh.N, 1);
    if (cr != CUDA_SUCCESS) return fail(REALQ_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)cr);
    auto run = [&](auto *y) {
        if (sh.kstep == 128)
            return w_bits == 8 ? tc_launch<8, 128>(s, sh, mapW, mapX, x_scale, w_scale, w_zero, y, b, sms)
                               : tc_launch<4, 128>(s, sh, mapW, mapX, x_scale, w_scale, w_zero, y, b, sms);
        return w_bits == 8 ? tc_launch<8, 64>(s, sh, mapW, mapX, x_scale, w_scale, w_zero, y, b, sms)
                           : tc_launch<4, 64>(s, sh, mapW, mapX, x_scale, w_scale, w_zero, y, b, sms);
    };
    return y_dtype == REALQ_BF16 ? run(static_cast<__nv_bfloat16 *>(Y)) : run(static_cast<float *>(Y));
}

}  // namespace realq
