// dW (+)= dY^T X̂ with X̂ read from its 8-bit checkpoint (T x n codes with one
// power-of-two scale byte per 32 values of a token): the weight gradient of a
// linear module whose inputs were kept in 8 bits.
//
// Arithmetic: a checkpoint value is a bf16 number, so X̂ is unpacked to a bf16
// plane without rounding; bf16 dY is used as it is and fp32 dY is split into
// three bf16 planes of eight significant bits each (hi + mid + lo = dY exactly,
// by truncation).  Products of bf16 numbers are exact in fp32, so the only
// rounding is the accumulation's.  The tensor core's accumulation loses about
// one unit in the last place per accumulated MMA, in one direction; it is
// promoted: two TMEM accumulators take CHUNK_STAGES x 64 tokens in turn and the
// drain warps add each into fp32 registers (IEEE additions) while the other
// fills.
//
// Two CTAs of a cluster work as a pair (cta_group::2) on a tile of dW of 256
// columns (X̂'s channels, the MMA's rows, 128 to each CTA) by 256 rows (dY's
// channels, the MMA's columns): each CTA loads its 128 channels of either
// operand, and the MMA takes B from both, so an operand byte in shared memory
// serves twice the products of a single CTA's tile (a 128 x 256 tile per CTA
// waited on L2: 806 cycles for 512 of MMA).  X̂'s channels lie on the TMEM lanes,
// so that a warp's stores of one row of dW are contiguous.  Both operands are
// token-major, i.e. MN-major for the MMA: a TMA box of 64 tokens x 64 channels
// (128-byte rows, 128-byte swizzle) is one canonical atom stack.  Persistent
// pairs walk the tiles; the accumulation lies in the drain warps' registers, so
// storing a tile overlaps the next one's MMAs.  Tiles beyond whole rounds over
// the pairs have their tokens split; a second pass adds the parts in their
// order.  Every wait is bounded; a tile whose wait gave up is written as NaN
// and the status word gets ST_TIMEOUT.
//
// Measured, 8192 tokens x 8192 x 8192 with bf16 dY: 596 us alone (1.85 PFLOP/s;
// the tensor pipe 80 % active at 4096 x 4864 x 8192), 38 us for X̂'s plane, which
// HBM bounds, and 10 for the parts; a call 632 to 720 us among others, as the
// power cap has it.  One CTA per tile took 1.09 ms.  With few tokens the stores
// of dW bound it (21 x 7936 x 28416: 170 us for 902 MB; 217 with bf16 and 329
// with fp32 dY for 21 x 7834 x 28327, where an odd n puts rows off the 32-byte
// sectors).  fp32 dY: 1999 x 1024 x 4096 45 us, 4000 x 5000 x 800 122.
#include "bytes.cuh"
#include "kernels.cuh"
#include "tc.cuh"

#include <algorithm>

namespace realq {
namespace {

constexpr int TC = 128;                          // channels of either operand per CTA
constexpr int TT = 2 * TC;                       // tile side
constexpr int KSTAGE = 64;                       // tokens per pipeline stage
constexpr int STAGES = 6;
constexpr int CHUNK_STAGES = 8;                  // stages per TMEM accumulator pass
constexpr int DRAIN_WARPS = 8;
constexpr int THREADS = (DRAIN_WARPS + 2) * 32;
constexpr int BOX_BYTES = 64 * KSTAGE * 2;
constexpr int OP_BYTES = TC * KSTAGE * 2;        // an operand's stage in one CTA: two boxes
constexpr int STAGE_BYTES = 2 * OP_BYTES;
constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + 1024 + 256;
constexpr uint32_t IDESC = tc::idesc_bf16_f32(TT, TT, 1, 1);
constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int MAX_SPLITS = 16;

struct Work {
    int64_t m, n, T;
    int64_t plane_rows;        // dY's planes lie this many rows apart
    int planes, nti, ntj;      // tiles over X̂'s channels, dY's channels
    int whole;                 // tiles that keep their token range; the others are split
    int splits;                // token parts of those
    int64_t tper;              // tokens per part, a multiple of KSTAGE
    int items;
};
struct Item {
    int i0, j0, nk;            // first channels, stages
    int slot, z;               // split tiles: number among them and part (slot < 0: whole)
    int64_t t0;
};
// Item k: first the whole tiles, then the parts of the others (all first parts,
// all second parts, ...).  Tiles go in groups of 8 tile rows, so that the pairs
// running together share operands in L2.
__host__ __device__ __forceinline__ Item item_of(const Work &w, int k) {
    constexpr int G = 8;
    Item it;
    it.slot = -1;
    it.z = 0;
    it.t0 = 0;
    int64_t tokens = w.T;
    int t = k;
    if (k >= w.whole) {
        const int cut = w.nti * w.ntj - w.whole;
        it.z = (k - w.whole) / cut;
        it.slot = k - w.whole - it.z * cut;
        it.t0 = it.z * w.tper;
        tokens = w.T - it.t0 < w.tper ? w.T - it.t0 : w.tper;
        t = w.whole + it.slot;
    }
    const int g = t / (G * w.ntj), r0 = g * G, left = w.nti - r0, rows = G < left ? G : left, u = t - g * G * w.ntj;
    it.i0 = (r0 + u % rows) * TT;
    it.j0 = (u / rows) * TT;
    it.nk = (int)((tokens + KSTAGE - 1) / KSTAGE) * w.planes;
    return it;
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
    weight_grad_kernel(const __grid_constant__ CUtensorMap mapX, const __grid_constant__ CUtensorMap mapY, const Work wk,
                       float *dW, int accumulate, float *part, int *err) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t *full = reinterpret_cast<uint64_t *>(smem + STAGES * STAGE_BYTES);   // the leader's: both CTAs' loads
    uint64_t *empty = full + STAGES;
    uint64_t *accf = empty + STAGES;             // [2] accumulator b holds a finished chunk
    uint64_t *acce = accf + 2;                   // [2] the leader's: accumulator b drained by both CTAs
    uint64_t *done = acce + 2;                   // every MMA issued has retired
    uint32_t *tslot = reinterpret_cast<uint32_t *>(done + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tslot + 1);

    dependents_may_start();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = tc::cluster_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            tc::mbar_init(tc::smem_u32(&full[s]), 1);
            tc::mbar_init(tc::smem_u32(&empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            tc::mbar_init(tc::smem_u32(&accf[b]), 1);
            tc::mbar_init(tc::smem_u32(&acce[b]), 2 * DRAIN_WARPS);
        }
        tc::mbar_init(tc::smem_u32(done), 1);
        *abort_flag = 0;
        tc::fence_barrier_init();
        tc::prefetch_tmap(&mapX);
        tc::prefetch_tmap(&mapY);
    }
    if (warp == 0) tc::tmem_alloc_pair(tc::smem_u32(tslot), 2 * TT);
    tc::fence_before_sync();
    __syncthreads();
    tc::cluster_sync();
    tc::fence_after_sync();
    const uint32_t tmem = *tslot;
    bool good = true;

    if (warp == DRAIN_WARPS) {
        if (lane == 0) {
            // ---------------- TMA producer: this CTA's channels ----------------
            wait_for_previous();   // the planes
            int s = 0, it = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int k = pair; k < wk.items && ok; k += pairs) {
                const Item im = item_of(wk, k);
                const int xi = im.i0 + (int)rank * TC, xj = im.j0 + (int)rank * TC;
                int y = (int)im.t0, p = 0;
                for (int i = 0; i < im.nk; ++i, ++it) {
                    ok = tc::mbar_wait(tc::smem_u32(&empty[s]), phase ^ 1u, abort_flag);
                    if (!ok) break;
                    const uint32_t fb = tc::map_rank(tc::smem_u32(&full[s]), 0);
                    if (rank == 0) tc::mbar_arrive_expect_tx(tc::smem_u32(&full[s]), 2 * STAGE_BYTES);
                    const uint32_t a = tc::smem_u32(smem + s * STAGE_BYTES);
                    const int yp = (int)(p * wk.plane_rows) + y;
                    tc::tma_load_2d_pair(a, &mapX, fb, xi, y);
                    tc::tma_load_2d_pair(a + BOX_BYTES, &mapX, fb, xi + 64, y);
                    tc::tma_load_2d_pair(a + OP_BYTES, &mapY, fb, xj, yp);
                    tc::tma_load_2d_pair(a + OP_BYTES + BOX_BYTES, &mapY, fb, xj + 64, yp);
                    if (++p == wk.planes) {   // the planes of 64 tokens follow one another
                        p = 0;
                        y += KSTAGE;
                    }
                    if (++s == STAGES) {
                        s = 0;
                        phase ^= 1u;
                    }
                }
            }
            if (!ok) *abort_flag = 1;
            // On abort, the copies already issued land before the pair's shared memory goes: the leader waits for
            // both CTAs' (its barriers count them), the other for the leader's exit below.
            if (*abort_flag && rank == 0) {
                int never = 0;
                for (int k = (it > STAGES ? it - STAGES : 0); k < it; ++k)
                    tc::mbar_wait(tc::smem_u32(&full[k % STAGES]), (uint32_t)(k / STAGES) & 1u, &never, 100000000ull);
            }
        }
    } else if (warp == DRAIN_WARPS + 1) {
        if (rank == 0) {
            // ---------------- MMA issuer (the whole warp waits, one lane issues) ----------------
            const uint64_t desc0 = tc::smem_desc(tc::smem_u32(smem), BOX_BYTES, 1024, tc::SW_128B);
            int s = 0, c = 0;   // stage; accumulator pass over all items
            uint32_t phase = 0;
            bool ok = true;
            for (int k = pair; k < wk.items && ok; k += pairs) {
                const Item im = item_of(wk, k);
                for (int i0 = 0; i0 < im.nk && ok; i0 += CHUNK_STAGES, ++c) {
                    const int b = c & 1;
                    ok = __all_sync(FULL, tc::mbar_wait(tc::smem_u32(&acce[b]), ((uint32_t)(c >> 1) & 1u) ^ 1u, abort_flag));
                    if (!ok) break;
                    tc::fence_after_sync();
                    const uint32_t d = tmem + (uint32_t)(b * TT);
                    const int cnt = min(CHUNK_STAGES, im.nk - i0);
                    for (int i = 0; i < cnt; ++i) {
                        ok = __all_sync(FULL, tc::mbar_wait(tc::smem_u32(&full[s]), phase, abort_flag));
                        if (!ok) break;
                        tc::fence_after_sync();
                        const uint64_t da = desc0 + (uint32_t)(s * STAGE_BYTES >> 4), db = da + (OP_BYTES >> 4);
                        if (tc::elect_one()) {
#pragma unroll
                            for (int q = 0; q < KSTAGE / 16; ++q)
                                tc::mma_f16_ss_pair(d, da + q * (2048 >> 4), db + q * (2048 >> 4), IDESC,
                                                    (i > 0 || q > 0) ? 1u : 0u);
                            tc::mma_commit_pair(tc::smem_u32(&empty[s]));
                        }
                        __syncwarp();
                        if (++s == STAGES) {
                            s = 0;
                            phase ^= 1u;
                        }
                    }
                    if (ok && tc::elect_one()) tc::mma_commit_pair(tc::smem_u32(&accf[b]));
                    __syncwarp();
                }
            }
            if (!ok) *abort_flag = 1;
            // every MMA issued has retired before either CTA frees its TMEM
            if (tc::elect_one()) tc::mma_commit_pair(tc::smem_u32(done));
            __syncwarp();
            int never = 0;
            tc::mbar_wait(tc::smem_u32(done), 0u, &never, 100000000ull);
        }
    } else {
        // ------- drain warps: TMEM passes -> fp32 registers (lane quarter, column half) -> dW -------
        const uint32_t src = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)((warp >> 2) * 128);
        int c = 0;
        for (int k = pair; k < wk.items; k += pairs) {
            const Item im = item_of(wk, k);
            float acc[128];
#pragma unroll
            for (int q = 0; q < 128; ++q) acc[q] = 0.f;
            for (int i0 = 0; i0 < im.nk && good; i0 += CHUNK_STAGES, ++c) {
                const int b = c & 1;
                if (!__all_sync(FULL, tc::mbar_wait(tc::smem_u32(&accf[b]), (uint32_t)(c >> 1) & 1u, abort_flag))) {
                    *abort_flag = 1;
                    good = false;   // this tile and the pair's later ones are written as NaN
                    break;
                }
                tc::fence_after_sync();
#pragma unroll
                for (int c0 = 0; c0 < 128; c0 += 16) {
                    uint32_t v[16];
                    tc::tmem_ld_32x32b_x16(src + (uint32_t)(b * TT + c0), v);
                    tc::tmem_wait_ld();
#pragma unroll
                    for (int q = 0; q < 16; ++q) acc[c0 + q] += __uint_as_float(v[q]);
                }
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive_cluster(tc::map_rank(tc::smem_u32(&acce[b]), 0));
            }
            const int tc0 = (int)rank * TC + (warp & 3) * 32 + lane, tr0 = (warp >> 2) * 128;   // in the tile
            if (im.slot >= 0) {   // a part: the whole tile, 256 x 256
                float *o = part + (((int64_t)im.z * (wk.nti * wk.ntj - wk.whole) + im.slot) * TT + tr0) * TT + tc0;
#pragma unroll
                for (int q = 0; q < 128; ++q) o[q * TT] = good ? acc[q] : __int_as_float(0x7fc00000);
            } else if (im.i0 + tc0 < wk.n) {
                const int64_t row = im.j0 + tr0;
                float *o = dW + row * wk.n + im.i0 + tc0;
                const int rows = (int)min((int64_t)128, wk.m - row);
#pragma unroll
                for (int q = 0; q < 128; ++q, o += wk.n)
                    if (q < rows) {
                        const float v = good ? acc[q] : __int_as_float(0x7fc00000);
                        *o = accumulate ? *o + v : v;
                    }
            }
        }
    }
    __syncwarp();
    if (!good && lane == 0) atomicOr(err, ST_TIMEOUT);
    tc::fence_before_sync();
    __syncthreads();
    if (rank == 1 && warp == 0) {   // the leader's last arrival here, after all its others
        int never = 0;
        tc::mbar_wait(tc::smem_u32(done), 0u, &never);
    }
    __syncwarp();
    tc::cluster_sync();   // neither CTA's shared memory, barriers or TMEM are in use by the other any more
    if (warp == 0) tc::tmem_dealloc_pair(tmem, 2 * TT);
}

// The split tiles: parts added in their order.  A block takes four rows of a
// tile, a thread four neighbouring columns.
__global__ void __launch_bounds__(256) weight_grad_reduce(const Work wk, const float *part, float *dW, int accumulate) {
    wait_for_previous();
    const int slot = blockIdx.x, cut = wk.nti * wk.ntj - wk.whole;
    const Item im = item_of(wk, wk.whole + slot);
    const int r = blockIdx.y * 4 + (threadIdx.x >> 6), c = (threadIdx.x & 63) * 4;
    const int64_t row = im.j0 + r, col = im.i0 + c;
    if (row >= wk.m || col >= wk.n) return;
    const float4 *p = reinterpret_cast<const float4 *>(part + ((int64_t)slot * TT + r) * TT + c);
    const int64_t step = (int64_t)cut * TT * TT / 4;
    float4 v = load_after_wait(p);
#pragma unroll 4
    for (int z = 1; z < wk.splits; ++z) {
        const float4 b = load_after_wait(p + z * step);
        v.x += b.x;
        v.y += b.y;
        v.z += b.z;
        v.w += b.w;
    }
    const float a[4] = {v.x, v.y, v.z, v.w};
    float *o = dW + row * wk.n + col;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (col + k < wk.n) o[k] = accumulate ? o[k] + a[k] : a[k];
}

// 2^(b - 133), subnormal below b = 7; NaN for b = 255
__device__ __forceinline__ float step_of(uint32_t b) {
    if (b == 255u) return __int_as_float(0x7FC00000);
    return __uint_as_float(b >= 7u ? (b - 6u) << 23 : 1u << (b + 16u));
}
// two fp32 numbers that are bf16 numbers, as a bf16 pair
__device__ __forceinline__ uint32_t upper2(float lo, float hi) {
    return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
}

// fp32 v = hi + mid + lo, each of eight significant bits, by truncation (an
// infinity or NaN stays in hi; a NaN whose payload lies in the lower half must
// not become an infinity)
__device__ __forceinline__ void split3(float v, float &hi, float &mid, float &lo) {
    const bool num = (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u;
    hi = num ? __uint_as_float(__float_as_uint(v) & 0xFFFF0000u) : __bfloat162float(__float2bfloat16_rn(v));
    const float r = num ? v - hi : 0.f;
    mid = __uint_as_float(__float_as_uint(r) & 0xFFFF0000u);
    lo = r - mid;
}

// The operands' planes, in one launch: the first xblocks blocks unpack X̂ to
// bf16 (row stride ldx), 16 values a thread; the others bring dY to its planes
// (row stride ldy): bf16 copied, 16 bytes a thread, or fp32 split in three, four
// values a thread.  FLAT: rows follow one another at whole pieces (n a multiple
// of 32, m of 8), so pieces are numbered through.  Columns past the widths lie
// outside the tensor maps.
struct Planes {
    int64_t T, n, m, ldx, ldy;
    unsigned xblocks;
    const int8_t *codes;
    const uint8_t *exps;
    __nv_bfloat16 *x;
    const void *dY;
    int dy_f32;
    __nv_bfloat16 *dy;
};
template <bool FLATX, bool FLATY>
__global__ void __launch_bounds__(256) grad_planes_kernel(const Planes p) {
    dependents_may_start();
    if (blockIdx.x < p.xblocks) {
        const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, pieces = (p.n + 15) / 16;
        if (i >= p.T * pieces) return;
        uint4 q;
        uint32_t b;
        uint4 *o;
        bool both = true;
        if (FLATX) {
            q = __ldg(reinterpret_cast<const uint4 *>(p.codes) + i);
            b = __ldg(p.exps + (i >> 1));
            o = reinterpret_cast<uint4 *>(p.x) + 2 * i;
        } else {
            int64_t c;
            const int64_t t = divide(i, pieces, c);
            const uint8_t *lo = reinterpret_cast<const uint8_t *>(p.codes);
            q = load16(lo + t * p.n + c * 16, lo, lo + p.T * p.n);
            b = __ldg(p.exps + t * ((p.n + 31) / 32) + (c >> 1));
            o = reinterpret_cast<uint4 *>(p.x + t * p.ldx + c * 16);
            both = c * 16 + 8 < p.ldx;
        }
        const float s = step_of(b);
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
        uint32_t h[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            h[k] = upper2((float)(int8_t)(w[k >> 1] >> (16 * (k & 1))) * s,
                          (float)(int8_t)(w[k >> 1] >> (16 * (k & 1) + 8)) * s);
        o[0] = make_uint4(h[0], h[1], h[2], h[3]);
        if (both) o[1] = make_uint4(h[4], h[5], h[6], h[7]);
        return;
    }
    const int64_t i = (int64_t)(blockIdx.x - p.xblocks) * 256 + threadIdx.x, plane = p.T * p.ldy;
    if (p.dy_f32) {
        const int64_t pieces = (p.m + 3) / 4;
        if (i >= p.T * pieces) return;
        float a[4];
        int64_t at;
        if (FLATY) {
            const float4 v = __ldg(reinterpret_cast<const float4 *>(p.dY) + i);
            a[0] = v.x;
            a[1] = v.y;
            a[2] = v.z;
            a[3] = v.w;
            at = 4 * i;
        } else {
            int64_t c;
            const int64_t t = divide(i, pieces, c);
            const float *src = static_cast<const float *>(p.dY) + t * p.m + c * 4;
#pragma unroll
            for (int k = 0; k < 4; ++k) a[k] = c * 4 + k < p.m ? __ldg(src + k) : 0.f;
            at = t * p.ldy + c * 4;
        }
        float h[3][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) split3(a[k], h[0][k], h[1][k], h[2][k]);
#pragma unroll
        for (int k = 0; k < 3; ++k)
            *reinterpret_cast<uint2 *>(p.dy + k * plane + at) =
                make_uint2(upper2(h[k][0], h[k][1]), upper2(h[k][2], h[k][3]));
    } else {
        const int64_t pieces = p.ldy / 8;
        if (i >= p.T * pieces) return;
        int64_t c;
        const int64_t t = divide(i, pieces, c);
        const uint8_t *lo = static_cast<const uint8_t *>(p.dY);
        reinterpret_cast<uint4 *>(p.dy)[i] = load16(lo + (t * p.m + c * 8) * 2, lo, lo + p.T * p.m * 2);
    }
}

int64_t pad8(int64_t x) { return (x + 7) / 8 * 8; }

// Tiles that fill whole rounds over the pairs of SMs keep their token range; the
// rest is cut into the count of parts that is estimated the fastest, in cycles: a
// stage takes 512 (the MMAs), a tile's start and end 3000, the pass over the
// parts 5000 and the parts' bytes 3400 to a cycle, twice; a part keeps at least
// four stages.
Work work_of(int64_t T, int64_t m, int64_t n, int planes, int sms) {
    Work w{};
    w.m = m;
    w.n = n;
    w.T = T;
    w.plane_rows = T;
    w.planes = planes;
    w.nti = ceil_div(n, TT);
    w.ntj = ceil_div(m, TT);
    const int64_t pairs = sms / 2, tiles = (int64_t)w.nti * w.ntj, rest = tiles % pairs, ks = (T + KSTAGE - 1) / KSTAGE;
    int best = 1;
    int64_t cost = INT64_MAX;
    for (int s = 1; s <= MAX_SPLITS && (s == 1 || ks * planes / s >= 4) && s <= ks && rest > 0; ++s) {
        const int64_t c = (rest * s + pairs - 1) / pairs * ((ks + s - 1) / s * planes * 512 + 3000) +
                          (s > 1 ? 5000 + 2 * rest * s * TT * TT * 4 / 3400 : 0);
        if (c < cost) {
            cost = c;
            best = s;
        }
    }
    w.tper = (ks + best - 1) / best * KSTAGE;
    w.splits = (int)((T + w.tper - 1) / w.tper);
    w.whole = (int)(w.splits > 1 ? tiles - rest : tiles);
    w.items = (int)(w.whole + (tiles - w.whole) * w.splits);
    return w;
}

struct GradWs {
    int *status;
    __nv_bfloat16 *x, *dy;
    float *part;
    size_t bytes;
    GradWs(void *ws, const Work &w, realq_dtype_t dt) {
        Carve c(ws);
        status = c.take<int>(64);
        x = c.take<__nv_bfloat16>((size_t)(w.T * pad8(w.n)));
        dy = c.take<__nv_bfloat16>((size_t)(w.T * pad8(w.m)) * (dt == REALQ_F32 ? 3 : (w.m % 8 ? 1 : 0)));
        part = c.take<float>((size_t)(w.items - w.whole) * TT * TT);
        bytes = c.off;
    }
};

}  // namespace

size_t checkpoint_grad_ws_bytes(int64_t T, int64_t m, int64_t n, realq_dtype_t dt, int sms) {
    return GradWs(nullptr, work_of(T, m, n, dt == REALQ_F32 ? 3 : 1, sms), dt).bytes;
}

realq_status_t checkpoint_grad(cudaStream_t s, int64_t T, int64_t m, int64_t n, const void *dY, realq_dtype_t dt,
                               const int8_t *codes, const uint8_t *exps, float *dW, int accumulate, void *ws, int sms) {
    const int planes = dt == REALQ_F32 ? 3 : 1;
    const Work wk = work_of(T, m, n, planes, sms);
    const GradWs w(ws, wk, dt);
    const bool direct = dt == REALQ_BF16 && m % 8 == 0;   // dY read where it lies
    const int64_t ldx = pad8(n), ldy = pad8(m);
    const bool xv = n % 32 == 0 && (reinterpret_cast<uintptr_t>(codes) & 15) == 0, yv = dt == REALQ_F32 && m % 8 == 0;
    Planes p{T, n, m, ldx, ldy, (unsigned)((T * ((n + 15) / 16) + 255) / 256), codes, exps, w.x, dY,
             dt == REALQ_F32, w.dy};
    const int64_t ypieces = T * (dt == REALQ_F32 ? (m + 3) / 4 : ldy / 8);
    const unsigned blocks = p.xblocks + (direct ? 0u : (unsigned)((ypieces + 255) / 256));
    {
        Launch L("checkpoint_grad_planes", s);
        if (xv && yv)
            grad_planes_kernel<true, true><<<blocks, 256, 0, s>>>(p);
        else if (xv)
            grad_planes_kernel<true, false><<<blocks, 256, 0, s>>>(p);
        else if (yv)
            grad_planes_kernel<false, true><<<blocks, 256, 0, s>>>(p);
        else
            grad_planes_kernel<false, false><<<blocks, 256, 0, s>>>(p);
    }
    REALQ_TRY(check_launch("checkpoint_grad_planes"));
    CUtensorMap mapY, mapX;
    CUresult cr = encode_tmap_2d_bf16(&mapY, direct ? dY : (const void *)w.dy, (uint64_t)m, (uint64_t)(planes * T),
                                      (uint64_t)ldy * 2, 64, KSTAGE, 1);
    if (cr == CUDA_SUCCESS)
        cr = encode_tmap_2d_bf16(&mapX, w.x, (uint64_t)n, (uint64_t)T, (uint64_t)ldx * 2, 64, KSTAGE, 1);
    if (cr != CUDA_SUCCESS) return fail(REALQ_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)cr);
    REALQ_TRY(set_smem_limit(reinterpret_cast<const void *>(weight_grad_kernel), SMEM_BYTES));
    {
        Launch L("checkpoint_weight_grad", s);
        REALQ_CUDA_TRY(launch_overlapped(weight_grad_kernel, dim3((unsigned)(2 * std::min(wk.items, sms / 2))),
                                         dim3(THREADS), SMEM_BYTES, s, mapX, mapY, wk, dW, accumulate, w.part,
                                         w.status));
    }
    REALQ_TRY(check_launch("checkpoint_weight_grad"));
    if (wk.splits > 1) {
        Launch L("checkpoint_grad_reduce", s);
        REALQ_CUDA_TRY(launch_overlapped(weight_grad_reduce, dim3((unsigned)(wk.nti * wk.ntj - wk.whole), TT / 4),
                                         dim3(256), 0, s, wk, (const float *)w.part, dW, accumulate));
        REALQ_TRY(check_launch("checkpoint_grad_reduce"));
    }
    return REALQ_OK;
}

}  // namespace realq
