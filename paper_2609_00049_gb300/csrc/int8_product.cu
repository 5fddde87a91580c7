// Y = diag(x_scale) (Xc - 128) (Wc - z)^T diag(w_scale): 8-bit token codes
// (T x n) times 8- or 4-bit channel codes (m x n), the product of the
// weight-activation setting run on the codes themselves.
//
// The sum over j is a whole number; the two scales are applied to it in fp32
// and the result is rounded once to Y's type.
//
// Streaming kernel (few tokens): bound by reading the weight codes once from
// HBM.  A warp takes RT x 16 channels and all tokens (NT x 8) over a share of K
// with mma.sync m16n8k16 in fp16 (dp4a needs no conversion, but runs at 16 lanes
// a cycle on an SM here: from four tokens on it took longer than the codes' way
// from HBM).  The order of K inside the product is free as long as both operands
// share it, so a lane reads 16 bytes of codes of a channel at a time and uses
// them where they are:
//   - an unsigned code c in the low mantissa bits of an fp16 is the subnormal
//     c 2^-24, so weight codes become A with one byte permute per pair, nibbles
//     with one mask per pair (upper nibbles read as c 2^-20);
//   - the tokens' codes become fp16 whole numbers x (those that meet upper
//     nibbles x / 16), exactly;
//   - the zero point enters once: sum (c - z) x = sum c x - z sum x, where an A
//     of ones gives sum x on the way.
// Products and sums are whole multiples of 2^-24 and exact while below 2^24 of
// them; the sums are moved to 32-bit integers before they can get there
// (FLUSH), so the result is the exact integer sum whatever the codes.  The
// eight warps of a CTA, and up to eight CTAs of a cluster where channels alone
// do not fill the SMs evenly, add their shares of K as integers.
//
// Measured, 8 tokens x 8192 x 28672, among calls (in a captured graph): 41.7 us
// (38.1) with 8-bit weights, 235 MB at 5.6 TB/s (6.2, 0.91 of the copy rate);
// 28.7 us (25.6) with 4-bit ones, 118 MB at 4.1 TB/s (4.6).  With 4 bits no unit
// is full (issue slots 54 %, ALU pipe 56 %, tensor pipe 39 %, DRAM 0.61 to 0.68
// of the copy rate): half the bytes take the same conversions and products, of
// which about a third are the tokens' own, repeated for every channel tile.
// 1 token x 1024 x 2048: 2.4 us in a graph, a launch.  Unaligned rows, 1 token x
// 8191 x 28672: 75 us with 8-bit weights, 55 with 4-bit ones (floors 35 and 17).
#include <cooperative_groups.h>

#include <algorithm>

#include "bytes.cuh"
#include "code_sums.cuh"
#include "kernels.cuh"

namespace cg = cooperative_groups;

namespace realq {
namespace {

constexpr int SW = 8;             // warps of a CTA
constexpr int MAX_CLUSTER = 8;

__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// the first `count` bytes of w, the others the code of zero
__device__ __forceinline__ uint32_t first_bytes(uint32_t w, int count) {
    const uint32_t keep = count >= 4 ? ~0u : (count <= 0 ? 0u : (1u << 8 * count) - 1u);
    return (w & keep) | (0x80808080u & ~keep);
}

__device__ __forceinline__ uint32_t word_of(const uint4 &v, int i) {
    return i == 0 ? v.x : (i == 1 ? v.y : (i == 2 ? v.z : v.w));
}

// Lane's 16 bytes of weight codes as A pairs: word i gives pairs 2 i, 2 i + 1
// (bytes 0 1, 2 3) or 4 i .. 4 i + 3 (nibbles 0 4, 1 5, 2 6, 3 7).
template <int WB>
__device__ __forceinline__ uint32_t weight_pair(uint32_t w, int j) {
    if constexpr (WB == 8) {
        return j == 0 ? __byte_perm(w, 0u, 0x4140) : __byte_perm(w, 0u, 0x4342);
    } else {
        const uint32_t v = j < 2 ? w : w >> 8;
        return j & 1 ? v & 0x00F000F0u : v & 0x000F000Fu;
    }
}
// The tokens' pairs in the same order, for one word of weight codes.
template <int WB>
__device__ __forceinline__ void token_pairs(const uint4 *k, int i, uint32_t *x) {
    if constexpr (WB == 8) {
        const uint32_t w = word_of(k[0], i);
        x[0] = sub2(__byte_perm(w, 0x64646464u, 0x4140), 0x64806480u);   // 1024 + c less 1152
        x[1] = sub2(__byte_perm(w, 0x64646464u, 0x4342), 0x64806480u);
    } else {
        const uint32_t w0 = word_of(k[i >> 1], (i & 1) * 2), w1 = word_of(k[i >> 1], (i & 1) * 2 + 1);
        const uint32_t a = __byte_perm(w0, w1, 0x5140), b = __byte_perm(w0, w1, 0x7362);   // columns 0 4 1 5, 2 6 3 7
        x[0] = sub2(__byte_perm(a, 0x64646464u, 0x4140), 0x64806480u);
        x[1] = sub2(__byte_perm(a, 0x54545454u, 0x4342), 0x54805480u);   // 64 + c / 16 less 72
        x[2] = sub2(__byte_perm(b, 0x64646464u, 0x4140), 0x64806480u);
        x[3] = sub2(__byte_perm(b, 0x54545454u, 0x4342), 0x54805480u);
    }
}

// 16 bytes global -> shared without a register, or zeros
template <bool KEEP>
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there) {
    const int bytes = there ? 16 : 0;
    if constexpr (KEEP)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
    else
        asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// A warp's sums over its share of K.
template <int WB, int NT, int RT> struct Sums {
    static constexpr int XP = WB == 8 ? 1 : 2;    // 16-byte pieces of token codes to one of weight codes
    static constexpr int WP = WB == 8 ? 2 : 4;    // pairs of a word
    // steps between flushes: 8 bits, 64 codes of at most 255 x 128 each; 4 bits, 128 codes of 15 x 128
    static constexpr int FLUSH = WB == 8 ? 8 : 64;
    float acc[RT][NT][4] = {}, xacc[NT][4] = {};
    uint32_t sum[RT][NT][4] = {};   // modulo 2^32
    int since = 0;

    __device__ __forceinline__ void flush() {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sum[r][t][e] = add_share(sum[r][t][e], __float2int_rn(acc[r][t][e] * 16777216.f));
                    acc[r][t][e] = 0.f;
                }
        since = 0;
    }
    // one step: this lane's 16 bytes of 2 RT channels, and the codes of NT tokens that meet them
    __device__ __forceinline__ void step(const uint4 (&wq)[RT][2], const uint4 (&k)[NT][XP]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {             // words of the 16 bytes
            uint32_t x[NT][WP];
#pragma unroll
            for (int t = 0; t < NT; ++t) token_pairs<WB>(k[t], i, x[t]);
#pragma unroll
            for (int j = 0; j < WP; j += 2) {     // a product takes two pairs
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    uint32_t a[4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t w = word_of(wq[r][h], i);
                        a[h] = weight_pair<WB>(w, j);
                        a[2 + h] = weight_pair<WB>(w, j + 1);
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t) mma16816(acc[r][t], a, x[t][j], x[t][j + 1]);
                }
                // ones (16 where the pair holds x / 16)
                const uint32_t one[4] = {0x3C003C00u, 0x3C003C00u, WB == 8 ? 0x3C003C00u : 0x4C004C00u,
                                         WB == 8 ? 0x3C003C00u : 0x4C004C00u};
#pragma unroll
                for (int t = 0; t < NT; ++t) mma16816(xacc[t], one, x[t][j], x[t][j + 1]);
            }
        }
        if (++since == FLUSH) flush();
    }
};

// ALIGNED: rows of whole 16-byte pieces of codes (n a multiple of 16, or of 32
// for 4 bits) at 16-byte aligned addresses.  Each lane then copies the pieces it
// will use into a ring of its own in shared memory, several steps ahead, so that
// the loads in flight cost no registers (held in registers they left 16 warps on
// an SM and 64 KB in flight at best: 29 us for 8 tokens x 8192 x 28672 with 4-bit
// weights).  Other rows are loaded to registers, realigned between lanes.
template <int WB, int NT, int RT> struct Ring {
    static constexpr int XP = WB == 8 ? 1 : 2;
    static constexpr int SLOT = (2 * RT + NT * XP) * 512;                // bytes of a warp's step
    static constexpr int STAGES = 104 * 1024 / (SW * SLOT) < 8 ? 104 * 1024 / (SW * SLOT) : 8;
    static constexpr int BYTES = SW * SLOT * STAGES;
};

template <bool ALIGNED, int WB, int NT, int RT, typename TY>
__global__ void __launch_bounds__(SW * 32, 2)
    int8_stream_kernel(int64_t T, int64_t n, int64_t m, const uint8_t *X, const float *x_scale, const uint8_t *W,
                       const float *w_scale, const uint8_t *w_zero, TY *Y) {
    using S = Sums<WB, NT, RT>;
    using R = Ring<WB, NT, RT>;
    constexpr int XP = S::XP, ROWS = RT * 16, TOK = NT * 8, OUT = ROWS * TOK;
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ uint32_t red[SW * OUT];
    __shared__ uint32_t xred[SW * TOK];
    const int64_t tok0 = (int64_t)blockIdx.y * TOK;   // this CTA's group of tokens
    T -= tok0;
    X += tok0 * n;
    x_scale += tok0;
    Y += tok0 * m;
    cg::cluster_group cluster = cg::this_cluster();
    const int CL = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int64_t rb = WB == 8 ? n : (n + 1) / 2;   // bytes of a row of W
    const int pieces = (int)((rb + 15) / 16);
    const int steps = (pieces + 3) / 4;             // four neighbouring pieces (64 bytes of each row) to a step
    const int64_t tiles = (m + ROWS - 1) / ROWS;
    const int64_t clusters = gridDim.x / CL;

    const uint8_t *xrow[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) xrow[t] = X + min((int64_t)(t * 8 + g), T - 1) * n;
    auto rows_of = [&](int64_t tile, const uint8_t *(&wrow)[RT][2]) {   // (rows past m repeat the last, unwritten)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h) wrow[r][h] = W + min(tile * ROWS + r * 16 + h * 8 + g, m - 1) * rb;
    };
    const uint4 zeros = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);   // codes of x = 0

    // ALIGNED: the warps of the cluster take a tile's steps in turn, `turns` each (some beyond the end, which read as
    // zeros); the copies run ahead across tiles.
    const int turns = (steps + CL * SW - 1) / (CL * SW);
    int64_t ftile = blockIdx.x / CL;
    int fturn = 0, fslot = 0, slot = 0;
    const uint8_t *frow[RT][2];
    const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(ring)) + warp * R::SLOT + lane * 16;
    auto fetch = [&] {
        if (ftile < tiles) {
            const int64_t v = ((int64_t)(fturn * CL + rank) * SW + warp) * 4 + q;
            const bool there = v < pieces;
            const int64_t at = there ? v * 16 : 0;
            const uint32_t dst = mine + fslot * (SW * R::SLOT);
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h) copy16<false>(dst + (2 * r + h) * 512, frow[r][h] + at, there);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int p = 0; p < XP; ++p)
                    copy16<true>(dst + (2 * RT + t * XP + p) * 512, xrow[t] + at * XP + p * 16, there);
            if (++fturn == turns) {
                fturn = 0;
                ftile += clusters;
                rows_of(ftile, frow);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++fslot == R::STAGES) fslot = 0;
    };
    if constexpr (ALIGNED) {
        rows_of(ftile, frow);
#pragma unroll
        for (int k = 0; k < R::STAGES - 1; ++k) fetch();
    }

    for (int64_t tile = blockIdx.x / CL; tile < tiles; tile += clusters) {
        S sums;
        if constexpr (ALIGNED) {
            for (int k = 0; k < turns; ++k) {
                fetch();
                asm volatile("cp.async.wait_group %0;" ::"n"(R::STAGES - 1) : "memory");
                const uint4 *src = reinterpret_cast<const uint4 *>(ring + (slot * SW + warp) * R::SLOT) + lane;
                uint4 wq[RT][2], kq[NT][XP];
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h) wq[r][h] = src[(2 * r + h) * 32];
                const bool there = ((k * CL + rank) * SW + warp) * 4 + q < pieces;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int p = 0; p < XP; ++p) kq[t][p] = there ? src[(2 * RT + t * XP + p) * 32] : zeros;
                sums.step(wq, kq);
                if (++slot == R::STAGES) slot = 0;
            }
        } else {
            // Pairs of neighbouring steps in turn: a lane loads aligned pieces and has the following one
            // from the next lane (the pair's last lane loads it itself).
            const uint8_t *whi = W + m * rb, *xhi = X + T * n, *wrow[RT][2];
            rows_of(tile, wrow);
            for (int s0 = 2 * (rank * SW + warp); s0 < steps; s0 += 2 * CL * SW) {
                uint4 wq[2][RT][2], next[RT][2];
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint8_t *p =
                            wrow[r][h] - (reinterpret_cast<uintptr_t>(wrow[r][h]) & 15) + ((int64_t)s0 * 4 + q) * 16;
                        wq[0][r][h] = load_piece(p, W, whi);
                        wq[1][r][h] = load_piece(p + 64, W, whi);
                        if (q == 3) next[r][h] = load_piece(p + 80, W, whi);
                    }
                const int src = (lane & ~3) | ((q + 1) & 3);
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t mis = (uint32_t)(reinterpret_cast<uintptr_t>(wrow[r][h]) & 15);
                        const uint4 n0 = shfl4(q == 0 ? wq[1][r][h] : wq[0][r][h], src), n1 = shfl4(wq[1][r][h], src);
                        wq[0][r][h] = realign(wq[0][r][h], n0, mis);
                        wq[1][r][h] = realign(wq[1][r][h], q == 3 ? next[r][h] : n1, mis);
                    }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if (s0 + u >= steps) break;   // (the same for the whole warp)
                    uint4 kq[NT][XP];
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int p = 0; p < XP; ++p) {
                            const int64_t c = (((int64_t)s0 + u) * 4 + q) * (16 * XP) + p * 16;   // first column
                            kq[t][p] = zeros;
                            if (c < n) {
                                kq[t][p] = load16(xrow[t] + c, X, xhi);
                                if (c + 16 > n) {   // columns from n on take no part
                                    const int left = (int)(n - c);
                                    kq[t][p] =
                                        make_uint4(first_bytes(kq[t][p].x, left), first_bytes(kq[t][p].y, left - 4),
                                                   first_bytes(kq[t][p].z, left - 8), first_bytes(kq[t][p].w, left - 12));
                                }
                            }
                        }
                    sums.step(wq[u], kq);
                }
            }
        }
        sums.flush();

#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    red[warp * OUT + (t * 8 + 2 * q + (e & 1)) * ROWS + r * 16 + (e >> 1) * 8 + g] = sums.sum[r][t][e];
        if (g == 0) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    xred[warp * TOK + t * 8 + 2 * q + e] = (uint32_t)__float2int_rn(sums.xacc[t][e]);
        }
        __syncthreads();
        // the warps' shares, then the cluster's; modulo 2^32, so any order is the same
        for (int k = threadIdx.x; k < OUT + TOK; k += SW * 32) {
            uint32_t *p = k < OUT ? red + k : xred + k - OUT;
            const int step = k < OUT ? OUT : TOK;
            uint32_t a = p[0];
#pragma unroll
            for (int w = 1; w < SW; ++w) a += p[w * step];
            p[0] = a;
        }
        if (CL > 1) {
            cluster.sync();
            if (rank == 0) {
                for (int k = threadIdx.x; k < OUT + TOK; k += SW * 32) {
                    uint32_t *p = k < OUT ? red + k : xred + k - OUT;
                    uint32_t a = p[0];
                    for (int c = 1; c < CL; ++c) a += *cluster.map_shared_rank(p, c);
                    p[0] = a;
                }
            }
            cluster.sync();   // the other CTAs' sums have been read
        } else {
            __syncthreads();
        }
        if (rank == 0) {
            for (int k = threadIdx.x; k < OUT; k += SW * 32) {
                const int64_t i = tile * ROWS + k % ROWS, t = k / ROWS;
                if (i < m && t < T) {
                    const int z = w_zero ? w_zero[i] : (WB == 8 ? 128 : 8);
                    const int64_t v = centred_sum(red[k], (int32_t)xred[k / ROWS], WB == 8 ? 128 : 8, z);
                    store1(Y + t * m + i, (float)v * __ldg(x_scale + t) * __ldg(w_scale + i));
                }
            }
        }
        __syncthreads();   // the sums have been read
    }
    if constexpr (ALIGNED) asm volatile("cp.async.wait_all;" ::: "memory");
}

template <bool ALIGNED, int WB, int NT, int RT, typename TY>
realq_status_t stream_launch(cudaStream_t s, int64_t T, int64_t n, int64_t m, const uint8_t *X, const float *xs,
                             const uint8_t *W, const float *ws, const uint8_t *wz, TY *Y, int sms) {
    // Clusters walk the tiles of RT x 16 channels; CTAs over K: the count whose
    // turns take the fewest steps of a warp, a tile's end counted as two, each
    // warp keeping at least two steps.
    const int64_t rb = WB == 8 ? n : (n + 1) / 2, tiles = (m + RT * 16 - 1) / (RT * 16), steps = (rb + 63) / 64;
    const int64_t groups = (T + NT * 8 - 1) / (NT * 8), slots = std::max<int64_t>(2 * sms / groups, MAX_CLUSTER);
    int cl = 1;
    int64_t best = INT64_MAX;
    for (int c = 1; c <= MAX_CLUSTER && (c == 1 || steps >= 2 * SW * c); c *= 2) {
        const int64_t held = slots / c;   // clusters at once
        const int64_t cost = (tiles + held - 1) / held * ((steps + SW * c - 1) / (SW * c) + 2);
        if (cost < best) {
            best = cost;
            cl = c;
        }
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(std::min(tiles, slots / cl) * cl), (unsigned)groups);
    cfg.blockDim = dim3(SW * 32);
    cfg.dynamicSmemBytes = ALIGNED ? Ring<WB, NT, RT>::BYTES : 0;
    cfg.stream = s;
    if (ALIGNED)
        REALQ_TRY(set_smem_limit(reinterpret_cast<const void *>(int8_stream_kernel<ALIGNED, WB, NT, RT, TY>),
                                 Ring<WB, NT, RT>::BYTES));
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cl;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cl > 1 ? 1 : 0;
    {
        Launch L("int8_product_stream", s);
        REALQ_CUDA_TRY(cudaLaunchKernelEx(&cfg, int8_stream_kernel<ALIGNED, WB, NT, RT, TY>, T, n, m, X, xs, W, ws, wz, Y));
    }
    return check_launch("int8_product_stream");
}

template <bool ALIGNED, int WB, typename TY>
realq_status_t stream_tokens(cudaStream_t s, int64_t T, int64_t n, int64_t m, const uint8_t *X, const float *xs,
                             const uint8_t *W, const float *ws, const uint8_t *wz, TY *Y, int sms) {
    // 32 channels to a warp halve the work on the tokens' codes, where there are enough of them; unaligned tokens are
    // more work, so there a quarter of that is enough where rows are long (1 x 15767 x 3927: 26 us against 33)
    const int64_t rb = WB == 8 ? n : (n + 1) / 2;
    const bool wide = m >= (int64_t)sms * 32 || (!ALIGNED && m >= (int64_t)sms * 8 && rb >= 4096);
    if (T <= 8)
        return wide ? stream_launch<ALIGNED, WB, 1, 2, TY>(s, T, n, m, X, xs, W, ws, wz, Y, sms)
                    : stream_launch<ALIGNED, WB, 1, 1, TY>(s, T, n, m, X, xs, W, ws, wz, Y, sms);
    return wide ? stream_launch<ALIGNED, WB, 2, 2, TY>(s, T, n, m, X, xs, W, ws, wz, Y, sms)
                : stream_launch<ALIGNED, WB, 2, 1, TY>(s, T, n, m, X, xs, W, ws, wz, Y, sms);
}

template <int WB, typename TY>
realq_status_t stream(cudaStream_t s, int64_t T, int64_t n, int64_t m, const uint8_t *X, const float *xs,
                      const uint8_t *W, const float *ws, const uint8_t *wz, TY *Y, int sms) {
    const bool aligned = n % (WB == 8 ? 16 : 32) == 0 &&
                         ((reinterpret_cast<uintptr_t>(X) | reinterpret_cast<uintptr_t>(W)) & 15) == 0;
    return aligned ? stream_tokens<true, WB, TY>(s, T, n, m, X, xs, W, ws, wz, Y, sms)
                   : stream_tokens<false, WB, TY>(s, T, n, m, X, xs, W, ws, wz, Y, sms);
}

// Whether the streaming kernel runs: for up to 16 tokens (8192 -> 28672: 16
// tokens take 44 us here, 47 in the tensor-core product with 8-bit weights, 40
// and 47 with 4-bit ones), and for up to 64 where reading the codes once for
// every 16 of them is less than the other product's planes, launches and ramps
// (1024 -> 2048: 64 tokens 5.4 and 7.8 us, 128 tokens 9.2 and 8.8).
constexpr int64_t GROUP = 16, MOST_GROUPED = 64, STREAM_BYTES = 24 << 20;
bool streams(int64_t T, int64_t n, int64_t m, int w_bits) {
    const int64_t bytes = m * (w_bits == 8 ? n : (n + 1) / 2);
    return T <= GROUP || (T <= MOST_GROUPED && (T + GROUP - 1) / GROUP * bytes <= STREAM_BYTES);
}

}  // namespace

size_t int8_product_ws_bytes(int64_t T, int64_t n, int64_t m, int w_bits, int sms) {
    return streams(T, n, m, w_bits) ? 256 : int8_tc_ws_bytes(T, n, m, w_bits, sms);
}

realq_status_t int8_product(cudaStream_t s, int64_t T, int64_t n, int64_t m, const uint8_t *X, const float *x_scale,
                            const uint8_t *W, int w_bits, const float *w_scale, const uint8_t *w_zero, void *Y,
                            realq_dtype_t y_dtype, void *ws, int sms) {
    // (whole 16-byte rows at an odd address cannot be a tensor map's, and are
    // streamed for 16 tokens at a time)
    const bool odd = (w_bits == 8 ? n : (n + 1) / 2) % 16 == 0 && (reinterpret_cast<uintptr_t>(W) & 15) != 0;
    if (!odd && !streams(T, n, m, w_bits))
        return int8_product_tc(s, T, n, m, X, x_scale, W, w_bits, w_scale, w_zero, Y, y_dtype, ws, sms);
    auto run = [&](auto *y) -> realq_status_t {
        constexpr int64_t MOST = GROUP * 65535;   // a grid's
        for (int64_t t = 0; t < T; t += MOST) {
            const int64_t k = std::min(MOST, T - t);
            REALQ_TRY(w_bits == 8 ? stream<8>(s, k, n, m, X + t * n, x_scale + t, W, w_scale, w_zero, y + t * m, sms)
                                  : stream<4>(s, k, n, m, X + t * n, x_scale + t, W, w_scale, w_zero, y + t * m, sms));
        }
        return REALQ_OK;
    };
    return y_dtype == REALQ_BF16 ? run(static_cast<__nv_bfloat16 *>(Y)) : run(static_cast<float *>(Y));
}

}  // namespace realq
