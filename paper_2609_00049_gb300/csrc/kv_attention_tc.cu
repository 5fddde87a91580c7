// Attention of many query rows over the 8-bit cache (prompts) on the tensor
// cores: S = Q K^T and O = P V by tcgen05.mma kind::f16, scores and outputs in
// TMEM, P as the A operand from TMEM.
//
// A CTA takes up to 256 rows that share a key/value head (its query heads times
// the new tokens) as two tiles of 128, and goes over their cached tokens in tiles
// of 128.  Per tile of tokens the tensor cores take 4 x 512 cycles for the two row
// tiles' two products (at 128 channels), which bounds the kernel; beside them fit
//   - two loader warps, for K with the scales and for V: page numbers, bulk copies of the codes into rings of their own;
//   - eight converter warps, four for K and four for V: codes to fp16 (exact: a byte permute to 1024 + c, one
//     subtraction of 1152), K as the K-major and V as the MN-major B operand of the
//     same layout: boxes of 64 channels, a token's 128-byte row swizzled;
//   - sixteen softmax warps, eight to a row tile, a thread to half of a row: while those of
//     one row tile work on its scores the tensor cores work for the other;
//   - one warp that issues the products.
// Per value of S a softmax thread spends a maximum, a multiply-add, an exponential, an addition and
// half a conversion: the block scales enter by the 16 tokens that share them.  With ks, vs a
// chunk's scales, lv = log2 vs and r the row's own scale (a power of two from
// scaling q into fp16's range, the softmax scale, log2 e),
//   p = 2^(S ks r + lv - M + 6),   sum += (sum of p in the chunk) 2^-6 / vs,
// so p already holds V's scale and O needs no other.  M is at least the running maximum less
// 8: it moves only when some row's maximum grew by more than that, and only then O is
// read, scaled and written back (the largest p stays below 2^14).  lv is at least -88, so that
// 2^31 tokens of zero values, 2^(88 + 8) each, add up to 2^127 at most.  Beside values of
// a scale 2^60 larger a chunk's p may be too small for any number while its weights are not:
// the sum then takes 2^(S ks r - M) by an exponential of its own, in tiles marked by the loader.  Scale blocks of fewer than 16
// tokens take one scale per token in the same formulas.  bf16 queries are exact in
// fp16 after scaling (down to 2^-29 of a row's largest value); fp32 queries and their p are two fp16
// parts each, which doubles the products: 22 bits of a p near the largest, which is 2^6 to 2^14, and
// to 2^-25 in any (a weight 2^-20 of its row's largest may have only its upper part).  V's scale enters
// as 2^lv with lv from lg2.approx, off by 2^-22 of itself (the sum takes the same lv out again).
// Measured for heads of 128 above all; those of 256 have one ring slot (and with fp32 one stage), so
// that loading, converting and products take turns there.
//
// P lies over S in TMEM (its low part, with fp32, has columns of its own), so the next
// product into S is issued behind the product that reads P; the tensor cores run
// them in order.  Work is cut as for few rows (kv_schedule.cuh), partial results
// joined by the warps that end last.
//
// Measured (bf16, 128 channels, 8 heads to a key/value head): a prompt of 8192 tokens
// 1570 us, 0.70 PFLOP/s, 0.37 of the measured bf16 rate; 5 ragged chunks of up to 1500
// tokens over up to 12000, 32 heads to 8, 578 us.  No unit is busy throughout: the
// schedulers issue in 0.66 of their cycles, some 3500 times for each 256 x 128 scores, the
// ALU works in 0.50 of them, the tensor cores in 0.39, shared memory in 0.55 (0.30 for
// threads, 0.25 for the tensor cores' operands).  Instructions alone do not bound it: of an
// earlier version with 20 warps 56 % of them could be taken out for 17 % of the cycles.
// Scores, maximum, weights and product of a row tile follow one another, as P lies
// over S; that chain and shared memory are what is left to explain the rest.  Slower
// were: tiles of 64 tokens with two parts of
// scores in TMEM (1965 us), one pass with the old maximum and P in registers (1602),
// more registers for the softmax warps from the others (1595).
#include <algorithm>
#include <type_traits>

#include "kv_schedule.cuh"
#include "tc.cuh"

namespace realq {
namespace {

constexpr uint32_t FULL = 0xFFFFFFFFu;
constexpr int SOFT_WARPS = 16, CONV_WARPS = 4;   // (softmax: eight to a row tile; converters: four for K and four for V)
constexpr int MMA_WARP = SOFT_WARPS + 2 * CONV_WARPS, LOAD_WARP = MMA_WARP + 1, THREADS = 32 * (MMA_WARP + 4);   // (loaders of K and of V; one is idle)
constexpr int UNIT = 32;                 // tokens whose codes come and are converted together
constexpr int SLOTS = 4;                 // of block scales
constexpr float NEG = -INFINITY, LIFT = 6.f, DOWN = 0.015625f, SLACK = 8.f;   // (DOWN: 2^-LIFT)
constexpr int FAR = 60;                  // log2 of two scales' quotient from which on the smaller one's weights are summed by themselves
constexpr float OWN = 24.f, OWN_DOWN = 5.9604645e-08f;   // (these are 2^OWN times what the sum takes)

template <int DP, bool F32> struct Shape {
    static constexpr int NM = DP == 256 ? 1 : 2;                                // row tiles
    static constexpr int ROWS = 128 * NM;
    static constexpr int KT = DP == 256 || (DP == 128 && F32) ? 64 : 128;       // tokens of a tile
    static constexpr int PARTS = F32 ? 2 : 1;
    static constexpr int STAGES = DP == 256 && F32 ? 1 : 2;                     // of K and of V
    static constexpr int BOXES = DP / 64;
    static constexpr int Q_BYTES = 128 * DP * 2;                                // one row tile, one part
    static constexpr int KV_BYTES = KT * DP * 2;
    static constexpr int SLOT_BYTES = 3 * KT * 4;
    static constexpr int UNITS = KT / UNIT, RAW_BYTES = UNIT * DP, RAW_SLOTS = DP == 256 ? 1 : 3;   // of K's and of V's codes each
    static constexpr int RING = NM * PARTS * Q_BYTES, RAW = RING + 2 * STAGES * KV_BYTES, SCALES = RAW + 2 * RAW_SLOTS * RAW_BYTES,
                         BARS = SCALES + SLOTS * SLOT_BYTES;
    static constexpr int SMEM = BARS + 512 + 1024;
    static constexpr int PART = 128 * (DP + 2);                                 // numbers of a row tile's partial result
    // TMEM columns
    static constexpr int S(int i) { return i * KT; }
    static constexpr int O(int i) { return NM * KT + i * DP; }
    static constexpr int LO(int i) { return NM * (KT + DP) + i * (KT / 2); }
    static_assert(SMEM + 512 + 1024 * NM <= 232448 && (int)sizeof(Window) <= 2 * RAW_SLOTS * RAW_BYTES && NM * (KT + DP + (F32 ? KT / 2 : 0)) <= 512, "shared and tensor memory");
};

__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tmem_st_x16(uint32_t taddr, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

__device__ __forceinline__ void tmem_ld_x8(uint32_t taddr, uint32_t (&r)[8]) {   // complete after tmem_wait_ld
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr));
}
__device__ __forceinline__ void tmem_st_x8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
                 "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// two fp32 values in one register pair
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
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// `bytes` consecutive bytes global -> shared, counted on `bar` (all three multiples of 16)
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

// tc::mbar_wait by the SM's clock, the thread asleep meanwhile (a warp that polls takes issue slots from the others).
// Gives up after about two seconds.
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(1000000u)   // ns, at most
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *abort) {
    if (try_wait(bar, parity)) return true;
    const int64_t t0 = clock64();
    for (uint32_t it = 1;; ++it) {
        if (try_wait(bar, parity)) return true;
        if ((it & 63u) == 0 && (*abort || clock64() - t0 > 4000000000ll)) return false;
    }
}

__device__ __forceinline__ void tmem_ld_x32(uint32_t taddr, uint32_t *r) {   // complete after tmem_wait_ld
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}

// A barrier of some warps, one arrival each, that gives up as every wait here does (a warp that gave up elsewhere does
// not come).  Whole warps come to it, and to every tcgen05 instruction: lanes that have parted meet before.
struct Meet {
    uint32_t bar, phase = 0;
    __device__ explicit Meet(uint64_t *b) : bar(tc::smem_u32(b)) {}
    __device__ __forceinline__ bool operator()(volatile int *abort) {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) tc::mbar_arrive(bar);
        const bool ok = __all_sync(FULL, bar_wait(bar, phase, abort));
        phase ^= 1u;
        return ok;
    }
};

struct Ring {   // stage and phase of something that goes round
    int s = 0, n;
    uint32_t phase = 0;
    __device__ explicit Ring(int stages) : n(stages) {}
    __device__ __forceinline__ void next() {
        if (++s == n) s = 0, phase ^= 1u;
    }
};

// The units of a CTA's share, one after the other.  Each role has its own in shared memory (registers are
// short), which one of its threads moves on.
template <int ROWS, int KT> struct Walk {
    Unit u;
    int tiles, from, count;    // of the unit, the share's first and how many
    int64_t unit0, at, end;
    __device__ __forceinline__ void set() {
        from = (int)min(at - unit0, (int64_t)tiles - 1);
        count = (int)min(end - at, (int64_t)(tiles - from));
    }
    __device__ void start(const Unit &u0, int64_t first, int tiles0, int64_t at0, int64_t end0) {
        u = u0, tiles = tiles0, unit0 = first, at = at0, end = end0;
        set();
    }
    __device__ __forceinline__ bool more() const { return at < end; }
    __device__ __forceinline__ void next(const KvAttnArgs &a) {
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

// The sum's part of 2^(S ks r - M) for the tokens among a thread's `cols` whose scale lies far below others (no weight of
// theirs is in P).  Not inlined: no instruction of the usual tiles makes room for it.
__device__ __noinline__ float far_weights(uint32_t s_at, const float *sc, int stride, int cols, int step, int lo, int hi, float factor, float lift) {
    float sum = 0.f;
#pragma unroll 1
    for (int c = 0; c < cols; c += 8) {
        uint32_t v[8];
        tmem_ld_x8(s_at + c, v);
        tc::tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float *at = step ? sc + c + j : sc + (c & ~15) / 4;
            if (c + j >= lo && c + j < hi && at[2 * stride] == 0.f && at[stride] > NEG) sum += exp2_fast(fmaf(__uint_as_float(v[j]), at[0] * factor, lift));
        }
        __syncwarp();
    }
    return sum * OWN_DOWN;
}

template <int DP, bool F32, class T>
__global__ void __launch_bounds__(THREADS, 1) prompt_kernel(const __grid_constant__ KvAttnArgs a, int *err) {
    using Sh = Shape<DP, F32>;
    constexpr int NM = Sh::NM, KT = Sh::KT, ROWS = Sh::ROWS;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Window &win = *reinterpret_cast<Window *>(smem + Sh::RAW);   // (before the first codes come)
    __shared__ int last_one[2];
    __shared__ Shares shares;
    __shared__ int far_scales[SLOTS];   // of the scales' slots: some lies far below others
    __shared__ Walk<ROWS, KT> walks[7];   // row tiles, K's and V's converters, products, loaders
    __shared__ float swap[2][NM][128];   // between the threads of a row
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + Sh::BARS);
    uint64_t *k_full = bars, *k_empty = bars + 2, *v_full = bars + 4, *v_empty = bars + 6;
    uint64_t *q_full = bars + 8, *s_full = bars + 10, *p_full = bars + 12, *o_full = bars + 14, *done = bars + 16;
    uint64_t *raw_full = bars + 17, *raw_empty = raw_full + 2 * Sh::RAW_SLOTS;   // K's slots, V's slots
    uint64_t *pairs = raw_empty + 2 * Sh::RAW_SLOTS, *tiles_meet = pairs + 8, *convs_meet = tiles_meet + 2;
    uint32_t *tslot = reinterpret_cast<uint32_t *>(convs_meet + 2);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tslot + 1);
    uint32_t *raw_there = tslot + 2;   // of each slot's groups of 16 tokens, those that have a page
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int D = a.c.head_dim;

    dependents_may_start();
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(tc::smem_u32(k_full + i), CONV_WARPS + 1);   // and the scales
            tc::mbar_init(tc::smem_u32(v_full + i), CONV_WARPS);
            tc::mbar_init(tc::smem_u32(k_empty + i), 1);
            tc::mbar_init(tc::smem_u32(v_empty + i), 1);
            tc::mbar_init(tc::smem_u32(q_full + i), 8);
            tc::mbar_init(tc::smem_u32(s_full + i), 1);
            tc::mbar_init(tc::smem_u32(p_full + i), 8);
            tc::mbar_init(tc::smem_u32(o_full + i), 1);
        }
        for (int i = 0; i < 2 * Sh::RAW_SLOTS; ++i) {
            tc::mbar_init(tc::smem_u32(raw_full + i), 1);
            tc::mbar_init(tc::smem_u32(raw_empty + i), CONV_WARPS);
        }
        for (int i = 0; i < 8; ++i) tc::mbar_init(tc::smem_u32(pairs + i), 2);
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(tc::smem_u32(tiles_meet + i), 8);
            tc::mbar_init(tc::smem_u32(convs_meet + i), CONV_WARPS);
        }
        tc::mbar_init(tc::smem_u32(done), 1);
        *abort_flag = 0;
        tc::fence_barrier_init();
    }
    // the share and its first unit
    int64_t all = 0, units = 0;
    for (int first = 0; first < a.n_seqs; first += SEQS) {
        fill_window<ROWS, KT, true>(a, win, first, all);
        all += win.sum[SEQS] * a.c.n_kv, units += win.units * a.c.n_kv;
    }
    const int64_t least = least_share(all, units, 4);
    const Shares sh(all, max((int64_t)1, min((int64_t)gridDim.x, least == 1 ? all : all / least)));
    if (blockIdx.x >= sh.ctas) return;
    if (a.n_seqs > SEQS) fill_window<ROWS, KT, true>(a, win, 0, 0);
    {
        const int64_t at0 = sh.begin(blockIdx.x);
        Unit u0;
        int64_t first0;
        int tiles0;
        locate<ROWS, KT, true>(a, win, at0, u0, first0, tiles0);
        fence_async_smem();   // (the codes' copies come over win)
        __syncthreads();
        if (threadIdx.x < 7) walks[threadIdx.x].start(u0, first0, tiles0, at0, sh.begin(blockIdx.x + 1));
        if (threadIdx.x == 0) shares = sh;
    }
    Walk<ROWS, KT> &w = walks[warp >= LOAD_WARP ? min(warp - LOAD_WARP, 1) + 5 : (warp < SOFT_WARPS ? warp >> 3 : (warp - SOFT_WARPS) / 4 + 2)];

    __syncwarp();
    if (warp == 0) tc::tmem_alloc(tc::smem_u32(tslot), 512);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = *tslot;
    bool ok = true;

    if (warp < SOFT_WARPS) {
        // ---------------- softmax: a thread has half of a row of row tile i ----------------
        const int i = warp >> 3, half = (warp >> 2) & 1, row = threadIdx.x & 127;
        Meet pair(pairs + (warp & 3) + 4 * i), all_rows(tiles_meet + i);   // the two warps that share 32 rows; a row tile's eight
        constexpr int COLS = KT / 2;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_at = tmem + lanes + Sh::S(i) + half * COLS, o_at = tmem + lanes + Sh::O(i), lo_at = tmem + lanes + Sh::LO(i) + half * (COLS / 2);
        const bool fine = a.c.log_block < 4;
        uint8_t *qs = smem + i * Sh::PARTS * Sh::Q_BYTES;
        uint32_t s_phase = 0, o_phase = 0;
        int slot = 0;
        // The row tile's queries into shared memory; returns what this thread's row's scores are multiplied by.  LANES
        // lanes take a row, 8 values each, a warp 16 of the rows; the rows' factors go by shared memory.
        constexpr int LANES = DP / 8, AT_ONCE = 32 / LANES, BATCH = 4;
        const bool wide = ((reinterpret_cast<uintptr_t>(a.q) | (uintptr_t)(a.q_ld * sizeof(T)) | (uintptr_t)(a.q_hs * sizeof(T))) & 15) == 0;
        const auto load_q = [&](const Unit &u) {
            const int d = lane % LANES * 8, sub = lane / LANES;
            int rw = (warp & 3) * 32 + half * 16 + sub;                 // row of the tile: token qi, head g of the group
            int qi = (u.r0 + 128 * i + rw) / a.group, g = u.r0 + 128 * i + rw - qi * a.group;
#pragma unroll 1
            for (int j0 = 0; j0 < LANES / 2; j0 += BATCH) {
                uint4 raw[BATCH][F32 ? 2 : 1];
                const int rw0 = rw;
#pragma unroll
                for (int j = 0; j < BATCH; ++j) {
                    const T *q = (const T *)a.q + (int64_t)(u.q0 + qi) * a.q_ld + (int64_t)(u.head * a.group + g) * a.q_hs + d;
#pragma unroll
                    for (int e = 0; e < (F32 ? 2 : 1); ++e) raw[j][e] = make_uint4(0, 0, 0, 0);
                    if (128 * i + rw < u.rows && d < D) {
                        if (wide) {
#pragma unroll
                            for (int e = 0; e < (F32 ? 2 : 1); ++e) raw[j][e] = reinterpret_cast<const uint4 *>(q)[e];
                        } else if constexpr (F32) {
                            const uint32_t *w = reinterpret_cast<const uint32_t *>(q);
                            raw[j][0] = make_uint4(w[0], w[1], w[2], w[3]), raw[j][1] = make_uint4(w[4], w[5], w[6], w[7]);
                        } else {
                            const uint16_t *w = reinterpret_cast<const uint16_t *>(q);
                            raw[j][0] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
                        }
                    }
                    rw += AT_ONCE;
                    for (g += AT_ONCE; g >= a.group; g -= a.group) ++qi;
                }
#pragma unroll
                for (int j = 0; j < BATCH; ++j) {
                    float x[8];
                    if constexpr (F32) {
                        const uint32_t w[8] = {raw[j][0].x, raw[j][0].y, raw[j][0].z, raw[j][0].w, raw[j][1].x, raw[j][1].y, raw[j][1].z, raw[j][1].w};
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(w[e]);
                    } else {
                        const uint32_t w[4] = {raw[j][0].x, raw[j][0].y, raw[j][0].z, raw[j][0].w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[2 * e] = __uint_as_float(w[e] << 16), x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
                    }
                    float top = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
#pragma unroll
                    for (int o = 1; o < LANES; o *= 2) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
                    // times 2^k: the largest lies in [2^14, 2^15) after that (a row below 2^-112 a little lower)
                    const int e = (int)(__float_as_uint(top) >> 23), k = e == 255 ? 0 : min(126, 141 - e);
                    float up = __uint_as_float((uint32_t)(127 + k) << 23);
                    const float back = fabsf(a.scale_log2) * __uint_as_float((uint32_t)(127 - k) << 23);
                    if (a.scale_log2 < 0.f) up = -up;   // (the scores' factor is to be positive)
                    if (lane % LANES == 0) swap[0][i][rw0 + j * AT_ONCE] = back;
                    if (d < D) {
                        uint32_t h[4];
                        const int r = rw0 + j * AT_ONCE;
                        uint8_t *to = qs + (d >> 6) * 16384 + r * 128 + ((((d >> 3) & 7) ^ (r & 7)) << 4);
#pragma unroll
                        for (int n = 0; n < 8; ++n) x[n] *= up;
#pragma unroll
                        for (int n = 0; n < 4; ++n) h[n] = pack_half(x[2 * n], x[2 * n + 1]);
                        *reinterpret_cast<uint4 *>(to) = make_uint4(h[0], h[1], h[2], h[3]);
                        if constexpr (F32) {
#pragma unroll
                            for (int n = 0; n < 4; ++n) h[n] = pack_rest(x[2 * n], x[2 * n + 1], h[n]);
                            *reinterpret_cast<uint4 *>(to + Sh::Q_BYTES) = make_uint4(h[0], h[1], h[2], h[3]);
                        }
                    }
                }
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(tc::smem_u32(q_full + i));
            ok = pair(abort_flag) && ok;
            const float mine = swap[0][i][row];
            ok = pair(abort_flag) && ok;
            return mine;
        };
        float rs = 0.f;
        bool loaded = false;
        const auto advance = [&]() {
            ok = all_rows(abort_flag) && ok;
            if ((threadIdx.x & 255) == 0) w.next(a);
            ok = all_rows(abort_flag) && ok;
        };
        while (w.more() && ok) {
            const int count = w.count;
            if (128 * i >= w.u.rows) {   // the row tile is empty: its tiles of tokens pass by
                slot = (slot + count) & (SLOTS - 1);
                advance();
                continue;
            }
            if (!loaded) rs = load_q(w.u);
            const float factor = rs;
            const bool in = 128 * i + row < w.u.rows;
            int row_hi = 0, row_lo = 0;
            int64_t out_row;
            {
                const int r = w.u.r0 + 128 * i + row, qi = r / a.group, p = w.u.len - w.u.m + qi;
                if (in) row_hi = min(a.room, a.causal ? p + 1 : w.u.len);
                if (a.window > 0) row_lo = (int)max((int64_t)0, (int64_t)p - a.window + 1);
                out_row = (int64_t)(w.u.q0 + qi) * a.n_heads + w.u.head * a.group + (r - qi * a.group);
            }
            const int all_hi = __reduce_min_sync(FULL, in ? row_hi : INT32_MAX), all_lo = __reduce_max_sync(FULL, in ? row_lo : 0);
            int k0 = (w.u.lo / KT + w.from) * KT + half * COLS;   // this thread's first token of a tile
            float m = NEG, l = 0.f, bad = 0.f;   // bad: NaN once a value that the row sees is
            for (int t = 0; t < count && ok; ++t, k0 += KT, slot = (slot + 1) & (SLOTS - 1)) {
                ok = __all_sync(FULL, bar_wait(tc::smem_u32(s_full + i), s_phase, abort_flag));
                s_phase ^= 1u;
                if (!ok) break;
                tc::fence_after_sync();
                const bool masked = k0 + (COLS - 1) >= all_hi || k0 < all_lo;
                const int far = far_scales[slot];
                const float *sc = reinterpret_cast<const float *>(smem + Sh::SCALES + slot * Sh::SLOT_BYTES) + half * (fine ? COLS : COLS / 4);
                const auto seen = [&](int j) { return k0 + j < row_hi && k0 + j >= row_lo; };
                // the largest S ks r + lv
                float top = NEG;
                const auto largest = [&](auto masks, auto fines, int c, uint32_t *v) {
                    if constexpr (masks) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] = seen(c + j) ? v[j] : 0xFF800000u;
                    }
                    if constexpr (!fines) {
                        const float4 b = reinterpret_cast<const float4 *>(sc)[c / 16];
                        float x[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            x[j] = max3(__uint_as_float(v[3 * j]), __uint_as_float(v[3 * j + 1]), __uint_as_float(v[3 * j + 2]));
                        const float y = max3(x[0], __uint_as_float(v[12]), __uint_as_float(v[13])), z = max3(x[1], __uint_as_float(v[14]), __uint_as_float(v[15]));
                        top = fmaxf(top, fmaf(fmaxf(max3(y, x[2], x[3]), z), b.x * factor, b.y));
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; j += 4) {
                            const float4 ks = *reinterpret_cast<const float4 *>(sc + c + j), lv = *reinterpret_cast<const float4 *>(sc + KT + c + j);
                            top = fmaxf(top, fmaf(__uint_as_float(v[j]), ks.x * factor, lv.x));
                            top = fmaxf(top, fmaf(__uint_as_float(v[j + 1]), ks.y * factor, lv.y));
                            top = fmaxf(top, fmaf(__uint_as_float(v[j + 2]), ks.z * factor, lv.z));
                            top = fmaxf(top, fmaf(__uint_as_float(v[j + 3]), ks.w * factor, lv.w));
                        }
                    }
                };
                using yes = std::true_type;
                using no = std::false_type;
                const auto over_few = [&](auto f) {   // (the rarer kinds of tiles: short loops, for the instruction cache)
                    uint32_t v[16];
#pragma unroll 1
                    for (int c = 0; c < COLS; c += 16) {
                        tc::tmem_ld_32x32b_x16(s_at + c, v);
                        tc::tmem_wait_ld();
                        f(c, v);
                    }
                };
                // the row's maximum from both its threads, and what that changes
                float base = 0.f;
                const auto agree = [&]() {
                    swap[half][i][row] = top;
                    ok = pair(abort_flag) && ok;
                    top = fmaxf(top, swap[half ^ 1][i][row]);
                    const bool grew = far != 0 || top > (m == NEG ? NEG : m + SLACK);
                    if (__any_sync(FULL, grew)) {
                        const float now = fmaxf(m, top), drop = now == NEG ? 0.f : m - now, f = exp2_fast(drop);
                        m = now, l = lowered(l, drop, f);
                        if (t > 0) {   // (the products so far are done: S came behind them)
    #pragma unroll 1
                            for (int c = 16 * half; c < D; c += 32) {
                                uint32_t v[16];
                                tc::tmem_ld_32x32b_x16(o_at + c, v);
                                tc::tmem_wait_ld();
    #pragma unroll
                                for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * f);
                                tmem_st_x16(o_at + c, v);
                            }
                        }
                        if (far != 0) l += far_weights(s_at, sc, fine ? KT : 1, COLS, fine, row_lo - k0, row_hi - k0, factor, OWN - (m == NEG ? 0.f : m));
                    }
                    base = LIFT - (m == NEG ? 0.f : m);
                };
                // (16 columns become 8 of P, over ones that have been read)
                const auto weights = [&](auto masks, auto fines, int c, uint32_t *v) {
                    uint32_t hi[8];
                    [[maybe_unused]] uint32_t lo[F32 ? 8 : 1];
                    if constexpr (!fines) {
                        const float4 b = reinterpret_cast<const float4 *>(sc)[c / 16];
                        const float c1 = b.x * factor, c0 = b.y + base;
                        const uint64_t c11 = two(c1, c1), c00 = two(c0, c0);
                        uint64_t part2 = 0;
#pragma unroll
                        for (int j = 0; j < 16; j += 2) {
                            float2 x = halves(fma2(two(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), c11, c00));
                            if constexpr (masks) {
                                x.x = seen(c + j) ? x.x : NEG;
                                x.y = seen(c + j + 1) ? x.y : NEG;
                            }
                            x.x = exp2_fast(x.x), x.y = exp2_fast(x.y);
                            part2 = add2(part2, two(x.x, x.y));
                            hi[j / 2] = pack_half(x.x, x.y);
                            if constexpr (F32) lo[j / 2] = pack_rest(x.x, x.y, hi[j / 2]);
                        }
                        const float2 ph = halves(part2);
                        const float part = ph.x + ph.y;
                        // (unseen tokens' scales may be anything; a seen NaN counts, however small its weight)
                        if (!masks || (k0 + c < row_hi && k0 + c + 15 >= row_lo)) l = fmaf(part, b.z, l), bad = fmaf(part, b.w, bad);
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; j += 4) {
                            const float4 ks = *reinterpret_cast<const float4 *>(sc + c + j), lv = *reinterpret_cast<const float4 *>(sc + KT + c + j);
                            const float4 iv = *reinterpret_cast<const float4 *>(sc + 2 * KT + c + j);   // with a minus: the value is NaN
                            float x[4] = {fmaf(__uint_as_float(v[j]), ks.x * factor, lv.x + base), fmaf(__uint_as_float(v[j + 1]), ks.y * factor, lv.y + base),
                                          fmaf(__uint_as_float(v[j + 2]), ks.z * factor, lv.z + base), fmaf(__uint_as_float(v[j + 3]), ks.w * factor, lv.w + base)};
                            const float inv[4] = {iv.x, iv.y, iv.z, iv.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                x[e] = exp2_fast(seen(c + j + e) ? x[e] : NEG);
                                const bool some = seen(c + j + e);
                                l = fmaf(x[e], some ? fabsf(inv[e]) : 0.f, l);
                                if (some && signbit(inv[e])) bad = __uint_as_float(0x7FC00000u);
                            }
                            hi[j / 2] = pack_half(x[0], x[1]), hi[j / 2 + 1] = pack_half(x[2], x[3]);
                            if constexpr (F32) lo[j / 2] = pack_rest(x[0], x[1], hi[j / 2]), lo[j / 2 + 1] = pack_rest(x[2], x[3], hi[j / 2 + 1]);
                        }
                    }
                    if constexpr (masks) __syncwarp();
                    tmem_st_x8(s_at + c / 2, hi);
                    if constexpr (F32) tmem_st_x8(lo_at + c / 2, lo);
                };
                if (!fine && !masked) {
                    uint32_t v[32];
#pragma unroll 1
                    for (int c = 0; c < COLS; c += 32) {
                        tmem_ld_x32(s_at + c, v);
                        tc::tmem_wait_ld();
                        largest(no{}, no{}, c, v);
                        largest(no{}, no{}, c + 16, v + 16);
                    }
                    agree();
#pragma unroll 1
                    for (int c = 0; c < COLS; c += 32) {
                        tmem_ld_x32(s_at + c, v);
                        tc::tmem_wait_ld();
                        weights(no{}, no{}, c, v);
                        weights(no{}, no{}, c + 16, v + 16);
                    }
                } else if (!fine) {
                    over_few([&](int c, uint32_t *v) { largest(yes{}, no{}, c, v); });
                    agree();
                    over_few([&](int c, uint32_t *v) { weights(yes{}, no{}, c, v); });
                } else {
                    over_few([&](int c, uint32_t *v) { largest(yes{}, yes{}, c, v); });
                    agree();
                    over_few([&](int c, uint32_t *v) { weights(yes{}, yes{}, c, v); });
                }
                tc::tmem_wait_st();
                if (!ok) break;
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(tc::smem_u32(p_full + i));
            }
            if (!ok) break;
            const bool whole = count == w.tiles, begins = w.from == 0;
            int first_cta = 0, last_cta = 0;
            if (!whole) first_cta = shares.owner(w.unit0), last_cta = shares.owner(w.unit0 + w.tiles - 1);
            // the next unit's queries while the last products run (this one's have been read: its last scores are there)
            advance();
            if (!ok) break;
            loaded = w.more() && 128 * i < w.u.rows;
            if (loaded) rs = load_q(w.u);
            ok = __all_sync(FULL, bar_wait(tc::smem_u32(o_full + i), o_phase, abort_flag));
            o_phase ^= 1u;
            if (!ok) break;
            tc::fence_after_sync();

            const bool aligned = (reinterpret_cast<uintptr_t>(a.out) & 15) == 0;
            const auto put = [&](int d, const float (&y)[8]) {   // out[d .. d + 7]
                T *o = (T *)a.out + out_row * D + d;
                if (!aligned) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if constexpr (F32)
                            o[e] = y[e];
                        else
                            o[e] = __float2bfloat16_rn(y[e]);
                    }
                } else if constexpr (F32) {
                    *reinterpret_cast<float4 *>(o) = make_float4(y[0], y[1], y[2], y[3]);
                    *reinterpret_cast<float4 *>(o + 4) = make_float4(y[4], y[5], y[6], y[7]);
                } else {
                    uint32_t h[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const __nv_bfloat162 b = __floats2bfloat162_rn(y[2 * e], y[2 * e + 1]);
                        h[e] = *reinterpret_cast<const uint32_t *>(&b);
                    }
                    *reinterpret_cast<uint4 *>(o) = make_uint4(h[0], h[1], h[2], h[3]);
                }
            };
            const auto put_lse = [&](float mm, float ll) {
                if (a.lse != nullptr) a.lse[out_row] = ll == 0.f ? NEG : (mm + log2f(ll)) * 0.6931471805599453f;
            };
            const auto slot_of = [&](int c, bool begins) { return a.part + ((int64_t)(2 * c + (begins ? 1 : 0)) * NM + i) * Sh::PART; };
            float *mine = slot_of(blockIdx.x, begins);
            swap[half][i][row] = l;
            ok = pair(abort_flag) && ok;
            l += swap[half ^ 1][i][row];
            ok = pair(abort_flag) && ok;
            swap[half][i][row] = bad;
            ok = pair(abort_flag) && ok;
            bad += swap[half ^ 1][i][row];
            ok = pair(abort_flag) && ok;   // (the next scores' maximum goes there)
            if (!ok) break;
            const float inv = DOWN / l;
#pragma unroll 1
            for (int c = 16 * half; c < D; c += 32) {
                uint32_t v[16];
                tc::tmem_ld_32x32b_x16(o_at + c, v);
                tc::tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; j += 8) {
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = __uint_as_float(v[j + e]) + bad;
                    if (whole) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = l == 0.f ? 0.f : y[e] * inv;   // (a row that sees nothing: zeros)
                        if (in) put(c + j, y);
                    } else {
                        float4 *to = reinterpret_cast<float4 *>(mine) + (c + j) / 4 * 128 + row;
                        to[0] = make_float4(y[0], y[1], y[2], y[3]), to[128] = make_float4(y[4], y[5], y[6], y[7]);
                    }
                }
                __syncwarp();
            }
            tc::fence_before_sync();
            if (whole) {
                if (in && half == 0) put_lse(m, l);
                continue;
            }
            if (half == 0) mine[128 * DP + row] = m, mine[128 * DP + 128 + row] = l;
            __threadfence();
            ok = all_rows(abort_flag);
            if (!ok) break;
            if ((threadIdx.x & 255) == 0) {
                const unsigned others = (unsigned)(last_cta - first_cta);
                last_one[i] = atomicInc(reinterpret_cast<unsigned *>(a.counters) + 2 * first_cta + i, others) == others;
            }
            ok = all_rows(abort_flag);
            if (!ok) break;
            if (!last_one[i]) continue;
            __threadfence();
            float mm = NEG, ll = 0.f;
            const int parts = last_cta - first_cta + 1;
#pragma unroll 4
            for (int c = 0; c < parts; ++c) mm = fmaxf(mm, __ldcg(slot_of(first_cta + c, c == 0) + 128 * DP + row));
#pragma unroll 4
            for (int c = 0; c < parts; ++c) {
                const float *s = slot_of(first_cta + c, c == 0) + 128 * DP + row;
                const float mc = __ldcg(s), lc = __ldcg(s + 128);
                ll += lowered(lc, mc - mm, mc == NEG ? 0.f : exp2_fast(mc - mm));   // (a NaN stays one)
            }
            const float all_inv = ll == 0.f ? 0.f : DOWN / ll;
#pragma unroll 1
            for (int d = 8 * half; d < D; d += 16) {
                float y[8] = {};
#pragma unroll 4
                for (int c = 0; c < parts; ++c) {   // (where a share saw nothing its outputs are 0)
                    const float *s = slot_of(first_cta + c, c == 0);
                    const float mc = __ldcg(s + 128 * DP + row);
                    const float4 *p4 = reinterpret_cast<const float4 *>(s) + d / 4 * 128 + row;
                    const float4 v0 = __ldcg(p4), v1 = __ldcg(p4 + 128);
                    const float f = mc == NEG ? 0.f : exp2_fast(mc - mm);
                    y[0] += v0.x * f, y[1] += v0.y * f, y[2] += v0.z * f, y[3] += v0.w * f;
                    y[4] += v1.x * f, y[5] += v1.y * f, y[6] += v1.z * f, y[7] += v1.w * f;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] *= all_inv;
                if (in) put(d, y);
            }
            if (in && half == 0) put_lse(mm, ll);
        }
        if (!ok) *abort_flag = 1;
    } else if (warp < MMA_WARP) {
        // ---------------- converters of K or of V: codes -> fp16, 32 tokens at a time ----------------
        // Eight lanes take four pieces of 16 channels of two neighbouring tokens, in different boxes where there are
        // several: neither the reading nor the writing (rows of odd and even tokens swizzled apart) meets in a bank.
        const bool is_v = warp >= SOFT_WARPS + CONV_WARPS;
        const int cw = warp & (CONV_WARPS - 1), piece = lane & 3, sel = (lane >> 2) & 1;
        const int token0 = 8 * cw + 2 * (lane >> 3) + sel, pieces = D / 16;
        const int to0 = token0 * 128 + (((2 * piece) ^ (token0 & 7)) << 4), to1 = token0 * 128 + (((2 * piece + 1) ^ (token0 & 7)) << 4);
        uint8_t *const stages = smem + Sh::RING + (is_v ? Sh::STAGES * Sh::KV_BYTES : 0);
        uint64_t *const empty = is_v ? v_empty : k_empty, *const filled = is_v ? v_full : k_full;
        uint64_t *const raw_in = raw_full + (is_v ? Sh::RAW_SLOTS : 0), *const raw_out = raw_empty + (is_v ? Sh::RAW_SLOTS : 0);
        const uint8_t *const raws = smem + Sh::RAW + (is_v ? Sh::RAW_SLOTS * Sh::RAW_BYTES : 0) + token0 * D + 16 * piece;
        uint32_t *const theres = raw_there + (is_v ? Sh::RAW_SLOTS : 0);
        Meet meet(convs_meet + is_v);
        Ring ring(Sh::STAGES), raw(Sh::RAW_SLOTS);
        while (w.more() && ok) {
            const int units = Sh::UNITS * w.count;
#pragma unroll 1
            for (int h = 0; h < units; ++h) {
                const int part = h % Sh::UNITS;
                if (part == 0) ok = __all_sync(FULL, bar_wait(tc::smem_u32(empty + ring.s), ring.phase ^ 1u, abort_flag));
                if (ok) ok = __all_sync(FULL, bar_wait(tc::smem_u32(raw_in + raw.s), raw.phase, abort_flag));
                if (!ok) break;
                const uint8_t *from = raws + raw.s * Sh::RAW_BYTES;
                uint8_t *to = stages + ring.s * Sh::KV_BYTES + part * UNIT * 128;
                const bool there = (theres[raw.s] >> (token0 >> 4)) & 1u;
                uint4 x[Sh::BOXES];
#pragma unroll
                for (int k = 0; k < Sh::BOXES; ++k) {
                    const int box = Sh::BOXES > 1 ? k ^ sel : 0;
                    x[k] = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);
                    if (4 * box + piece < pieces && there) x[k] = *reinterpret_cast<const uint4 *>(from + 64 * box);
                }
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(tc::smem_u32(raw_out + raw.s));   // the next codes may come
#pragma unroll
                for (int k = 0; k < Sh::BOXES; ++k) {
                    const int box = Sh::BOXES > 1 ? k ^ sel : 0;
                    uint8_t *line = to + box * (KT * 128);
                    if (4 * box + piece < pieces) {
                        *reinterpret_cast<uint4 *>(line + to0) = make_uint4(codes01(x[k].x), codes23(x[k].x), codes01(x[k].y), codes23(x[k].y));
                        *reinterpret_cast<uint4 *>(line + to1) = make_uint4(codes01(x[k].z), codes23(x[k].z), codes01(x[k].w), codes23(x[k].w));
                    }
                }
                raw.next();
                if (part == Sh::UNITS - 1) {
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(tc::smem_u32(filled + ring.s));
                    ring.next();
                }
            }
            if (!ok || !meet(abort_flag)) {
                ok = false;
                break;
            }
            if ((threadIdx.x & 127) == 0) w.next(a);
            ok = meet(abort_flag);
        }
        if (!ok) *abort_flag = 1;
    } else {
        if (warp == LOAD_WARP || warp == LOAD_WARP + 1) {
        // ---------------- loaders of K, with the scales, and of V: pages, codes by bulk copies of 16 tokens ----------------
        const bool is_v = warp != LOAD_WARP, fine = a.c.log_block < 4;
        uint64_t *const raw_in = raw_full + (is_v ? Sh::RAW_SLOTS : 0), *const raw_out = raw_empty + (is_v ? Sh::RAW_SLOTS : 0);
        uint8_t *const raws = smem + Sh::RAW + (is_v ? Sh::RAW_SLOTS * Sh::RAW_BYTES : 0);
        uint32_t *const theres = raw_there + (is_v ? Sh::RAW_SLOTS : 0);
        const uint8_t *const codes = is_v ? a.c.v_codes : a.c.k_codes;
        Ring kring(Sh::STAGES), raw(Sh::RAW_SLOTS);
        uint32_t fills = 0;
        int slot = 0;
        while (w.more() && ok) {
            int top = -128;   // log2 of the largest scale of values so far
            const int count = w.count, lo = w.u.lo, hi = w.u.hi, head = w.u.head;
            const int *table = a.tables + (int64_t)w.u.seq * a.max_pages;
            const int base = (lo / KT + w.from) * KT;
            const auto page_of = [&](int t) {   // of the tile's 16 tokens `lane`
                if (t >= count || lane >= KT / 16) return -1;
                const int k0 = base + t * KT + 16 * lane;   // (k0 + 16 may be 2^31)
                return k0 < hi && k0 + 15 >= lo ? __ldg(table + (k0 >> a.c.log_page)) : -1;
            };
            float ks = 0.f, vs = 0.f;
            bool there_s = false;
            const auto scales_of = [&](int t, int pg16, int n) {   // of the tile's token or 16 tokens n
                const int token = fine ? n : 16 * n, pg = __shfl_sync(FULL, pg16, (token >> 4) & 31);
                there_s = token < KT && pg >= 0 && pg < a.c.n_pages;
                if (there_s) {
                    const int pl = (base + t * KT + token) & ((1 << a.c.log_page) - 1);
                    const int64_t s = (((int64_t)pg * a.c.n_kv + head) << (a.c.log_page - a.c.log_block)) + (pl >> a.c.log_block);
                    ks = __ldg(a.c.k_scale + s), vs = __ldg(a.c.v_scale + s);
                }
            };
            int page = page_of(0), next_page = page_of(1);
#pragma unroll 1
            for (int t = 0; t < count && ok; ++t, kring.next(), slot = (slot + 1) & (SLOTS - 1)) {
                const bool good = page >= 0 && page < a.c.n_pages;
                const uint32_t there = __ballot_sync(FULL, good);
                const int k0 = base + t * KT + 16 * (lane & (KT / 16 - 1)), place = k0 & ((1 << a.c.log_page) - 1);
                const int64_t tile = (int64_t)page * a.c.n_kv + head;
                const uint8_t *src = codes + ((tile << a.c.log_page) + place) * D;
                if (!is_v && !fine) scales_of(t, page, lane);   // (under way with the codes)
#pragma unroll 1
                for (int h = 0; h < Sh::UNITS; ++h, raw.next()) {
                    ok = __all_sync(FULL, bar_wait(tc::smem_u32(raw_out + raw.s), raw.phase ^ 1u, abort_flag));
                    if (!ok) break;
                    const uint32_t mine = there >> (2 * h) & 3u, full = tc::smem_u32(raw_in + raw.s);
                    if (lane == 0) {
                        theres[raw.s] = mine;
                        tc::mbar_arrive_expect_tx(full, __popc(mine) * 16 * D);
                    }
                    ++fills;
                    __syncwarp();
                    if (good && lane / 2 == h) bulk_load(tc::smem_u32(raws + raw.s * Sh::RAW_BYTES + (lane & 1) * 16 * D), src, 16 * D, full);
                    __syncwarp();
                }
                if (!is_v && ok) {
                    // The tile's scales, once the stage is free: then three tiles before have their weights, and with them
                    // the slot's last readers are done, and the stage's barrier is in the phase of this tile.
                    ok = __all_sync(FULL, bar_wait(tc::smem_u32(k_empty + kring.s), kring.phase ^ 1u, abort_flag));
                    if (!ok) break;
                    float *sc = reinterpret_cast<float *>(smem + Sh::SCALES + slot * Sh::SLOT_BYTES);
                    const int entries = fine ? KT : KT / 16;
                    // (a scale that is no number counts for nothing; an infinite one, behind a sequence's end, for 2^127)
                    const auto largest = [&]() { top = max(top, __reduce_max_sync(FULL, there_s && vs > 0.f ? (int)ceilf(fminf(log2_fast(vs), 127.f)) : -128)); };
                    if (fine) {
#pragma unroll 1
                        for (int n = lane; n < KT; n += 32) {
                            scales_of(t, page, n);
                            largest();
                        }
                    } else {
                        largest();
                    }
                    bool marked = false;
#pragma unroll 1
                    for (int n0 = 0; n0 < entries; n0 += 32) {
                        const int n = n0 + lane;
                        if (n0 > 0 || fine) scales_of(t, page, n);
                        // tokens without a page weigh nothing; a scale below 2^-88 counts as that; a NaN's part in the sum
                        // stays (the scores are not concerned)
                        const bool nan = there_s && vs != vs;
                        const float k = there_s ? ks : 0.f, nv = nan ? vs : 0.f;
                        const float lv = !there_s ? NEG : (nan ? 0.f : fmaxf(log2_fast(vs), -88.f));
                        const bool far = there_s && lv < (float)(top - FAR);
                        const float iv = !there_s || far ? 0.f : exp2_fast(-lv) * DOWN;
                        marked = marked || far;
                        if (n < entries) {
                            if (fine)
                                sc[n] = k, sc[KT + n] = lv, sc[2 * KT + n] = nan ? -iv : iv;
                            else
                                reinterpret_cast<float4 *>(sc)[n] = make_float4(k, lv, iv, nv);
                        }
                    }
                    marked = __any_sync(FULL, marked);
                    if (lane == 0) far_scales[slot] = marked;
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(tc::smem_u32(k_full + kring.s));
                }
                page = next_page;
                next_page = page_of(t + 2);
            }
            __syncwarp();
            if (ok && lane == 0) w.next(a);
            __syncwarp();
        }
        if (!ok) {   // copies under way land before the CTA ends
            *abort_flag = 1;
            int never = 0;
            for (uint32_t k = fills > Sh::RAW_SLOTS ? fills - Sh::RAW_SLOTS : 0; k < fills; ++k)
                tc::mbar_wait(tc::smem_u32(raw_in + k % Sh::RAW_SLOTS), k / Sh::RAW_SLOTS & 1u, &never, 100000000ull);
        }
        } else if (warp == MMA_WARP) {
        // ---------------- products ----------------
        const uint32_t idesc_s = tc::idesc_f16_f32(128, KT), idesc_o = tc::idesc_f16_f32(128, 0) | ((uint32_t)(D >> 3) << 17) | (1u << 16);
        const uint32_t base = tc::smem_u32(smem);
        const uint64_t q_desc = tc::smem_desc(base, 16, 1024, tc::SW_128B);
        const uint64_t k_desc = tc::smem_desc(base + Sh::RING, 16, 1024, tc::SW_128B);
        const uint64_t v_desc = tc::smem_desc(base + Sh::RING + Sh::STAGES * Sh::KV_BYTES, KT * 128, 1024, tc::SW_128B);
        const int steps = D / 16;
        uint32_t phases = 0;   // bit i: of q_full, bit 2 + i: of p_full
        Ring kr(Sh::STAGES), vr(Sh::STAGES);
        if (tc::elect_one()) {   // (one thread for everything: between two products there is little time)
            const auto wait = [&](uint64_t *bar, uint32_t phase) {
                ok = ok && bar_wait(tc::smem_u32(bar), phase, abort_flag);
                tc::fence_after_sync();
            };
            while (w.more() && ok) {
                const int nm = w.u.rows > 128 ? 2 : 1, count = w.count;
                // step t: the outputs of tile t (none at -1), the scores of tile t + 1
#pragma unroll 1
                for (int t = -1; t < count && ok; ++t) {
                    if (t >= 0) wait(v_full + vr.s, vr.phase);
#pragma unroll 1
                    for (int i = 0; i < nm && ok; ++i) {
                        if (t < 0) {
                            wait(q_full + i, phases >> i & 1u);
                            phases ^= 1u << i;
                        } else {   // O_i += P_i V
                            wait(p_full + i, phases >> (2 + i) & 1u);
                            phases ^= 4u << i;
                            if (!ok) break;
#pragma unroll 1
                            for (int p = 0; p < Sh::PARTS; ++p) {
                                const uint64_t vd = v_desc + (uint32_t)(vr.s * Sh::KV_BYTES >> 4);
                                // (P's halves lie over the halves of S)
                                const uint32_t pa = tmem + (p == 0 ? Sh::S(i) : Sh::LO(i)), up = p == 0 ? KT / 4 : 0;
#pragma unroll
                                for (int k = 0; k < KT / 16; ++k)
                                    tc::mma_f16_ts(tmem + Sh::O(i), pa + k * 8 + (k >= KT / 32 ? up : 0), vd + k * 128, idesc_o, (k > 0 || p > 0 || t > 0) ? 1u : 0u);
                            }
                            if (t + 1 == count) tc::mma_commit(tc::smem_u32(o_full + i));
                        }
                        if (t + 1 < count) {   // S_i = Q_i K^T of the K stage
                            if (i == 0) wait(k_full + kr.s, kr.phase);
                            if (!ok) break;
#pragma unroll 1
                            for (int p = 0; p < Sh::PARTS; ++p) {
                                const uint64_t qd = q_desc + (uint32_t)((i * Sh::PARTS + p) * Sh::Q_BYTES >> 4);
                                const uint64_t kd = k_desc + (uint32_t)(kr.s * Sh::KV_BYTES >> 4);
#pragma unroll
                                for (int k = 0; k < DP / 16; ++k)
                                    if (k < steps)
                                        tc::mma_f16_ss(tmem + Sh::S(i), qd + (k & 3) * 2 + (k >> 2) * 1024, kd + (k & 3) * 2 + (k >> 2) * (KT * 8), idesc_s,
                                                       (p > 0 || k > 0) ? 1u : 0u);
                            }
                            tc::mma_commit(tc::smem_u32(s_full + i));
                        }
                    }
                    if (!ok) break;
                    if (t >= 0) {
                        tc::mma_commit(tc::smem_u32(v_empty + vr.s));
                        vr.next();
                    }
                    if (t + 1 < count) {
                        tc::mma_commit(tc::smem_u32(k_empty + kr.s));
                        kr.next();
                    }
                }
                if (ok) w.next(a);
            }
            if (!ok) *abort_flag = 1;
            tc::mma_commit(tc::smem_u32(done));
        }
        __syncwarp();
        ok = *abort_flag == 0;
        // every product issued has retired before TMEM is freed
        int never = 0;
        tc::mbar_wait(tc::smem_u32(done), 0u, &never, 100000000ull);
        }
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
