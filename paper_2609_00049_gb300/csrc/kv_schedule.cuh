// How the attention kernels cut their work: one unit is a sequence, a key/value
// head and a tile of ROWS query rows (the head's query heads times the new
// tokens, token by token); its cached tokens are taken in tiles of TILE.  All
// units' tiles in a row are cut into one share per CTA.
#pragma once

#include "kernels.cuh"

namespace realq {
namespace {

constexpr int SEQS = 512;                 // sequences whose tile counts are held at a time

// a / b for numbers that nearly always have 32 bits (a division of 64 takes longer than a read of global memory)
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// Shares of `all` tiles among `ctas` CTAs that differ by one tile at most, the larger ones first.
struct Shares {
    int64_t all, ctas, each, more;
    __device__ Shares() {}
    __device__ __forceinline__ Shares(int64_t tiles, int64_t most) : all(tiles), ctas(min(most, tiles)) {
        each = ctas > 0 ? quotient(all, ctas) : 0, more = all - each * ctas;
    }
    __device__ __forceinline__ int64_t begin(int64_t c) const { return c * each + min(c, more); }
    __device__ __forceinline__ int owner(int64_t x) const {   // of tile x
        const int64_t large = more * (each + 1);
        return (int)(x < large ? quotient(x, each + 1) : more + quotient(x - large, each));
    }
};

// The fewest tiles that a CTA takes: the shares of a unit of many tiles cost more to join than they save, those of units of
// few would only straddle them.  Units of up to `per` tiles on average are cut into single ones, of 4 x `per` or more into
// fours.  Measured with 32 heads to 8 (one tile, two, four, eight): 8 tokens over 2000 by the kernel of few rows, 32 tiles
// to a unit, 42, 33, 26, 31 us; 16 tokens over 2000 by that of many, 16 tiles, 47, 37, 33, 39; 8 single tokens over up to
// 1013, 8 tiles, 12.5, 16.5, 17, 25.
__device__ __forceinline__ int64_t least_share(int64_t tiles, int64_t units, int per) {
    const int64_t n = units * per;
    return tiles >= 4 * n ? 4 : (tiles >= 3 * n ? 3 : (tiles >= 2 * n ? 2 : 1));
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// sum 2^d, d <= 0, with f = 2^d: maxima hold the values' scales too, so that a sum may be 2^96 and belong to a maximum
// that lies 2^-150 below (zero values beside large ones), where f is no number: in two steps there.
__device__ __forceinline__ float lowered(float sum, float d, float f) {
    return d < -120.f ? sum * 7.523163845e-37f * exp2_fast(d + 120.f) : sum * f;
}
__device__ __forceinline__ float log2_fast(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t hsub2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
// what pack_half left of (lo, hi)
__device__ __forceinline__ uint32_t pack_rest(float lo, float hi, uint32_t h) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
    return pack_half(lo - f.x, hi - f.y);
}
// bytes 0 1 / 2 3 of w as two fp16 whole numbers c - 128
__device__ __forceinline__ uint32_t codes01(uint32_t w) { return hsub2(__byte_perm(w, 0x64646464u, 0x4140), 0x64806480u); }
__device__ __forceinline__ uint32_t codes23(uint32_t w) { return hsub2(__byte_perm(w, 0x64646464u, 0x4342), 0x64806480u); }

struct Unit {        // one sequence, key/value head and row tile
    int seq, head;
    int q0, m;       // the sequence's first query token and their number
    int len;         // its tokens (those beyond the table's row, which no one sees, among them)
    int r0, rows;    // rows of the tile: r0 .. r0 + rows - 1 of m x G
    int lo, hi;      // cached tokens that any row sees: [lo, hi)
};

// The cached tokens [lo, hi) that rows r0 .. r1 - 1 of a sequence see; their tiles (at least one: rows that see nothing
// are written too).
__device__ __forceinline__ void span(const KvAttnArgs &a, int m, int len, int r0, int r1, int *lo, int *hi) {
    const int p0 = len - m + r0 / a.group, p1 = len - m + (r1 - 1) / a.group;
    *hi = max(0, min(a.room, a.causal ? p1 + 1 : len));
    *lo = a.window > 0 ? (int)min((int64_t)*hi, max((int64_t)0, (int64_t)p0 - a.window + 1)) : 0;
}
template <int TILE> __device__ __forceinline__ int tiles_of(int lo, int hi) {
    return hi > lo ? (hi - 1) / TILE - lo / TILE + 1 : 1;
}

struct Seq {
    int q0, m, len;
    __device__ Seq(const KvAttnArgs &a, int s) {
        const int64_t b = a.starts[s], e = a.starts[s + 1];
        const bool ok = b >= 0 && e > b && e <= a.T;
        q0 = ok ? (int)b : 0, m = ok ? (int)(e - b) : 0;
        len = max(a.lengths[s], 0);
        if (m > 0 && !a.takes(m)) m = 0;   // another kernel's
    }
};
template <int ROWS, int TILE> __device__ __forceinline__ int row_tiles(const KvAttnArgs &a, const Seq &q, int r0) {
    int lo, hi;
    span(a, q.m, q.len, r0, min(r0 + ROWS, q.m * a.group), &lo, &hi);
    return tiles_of<TILE>(lo, hi);
}
template <int ROWS, int TILE> __device__ int64_t seq_tiles(const KvAttnArgs &a, int s) {   // of one head
    const Seq q(a, s);
    int64_t n = 0;
    for (int r = 0; r < q.m * a.group; r += ROWS) n += row_tiles<ROWS, TILE>(a, q, r);
    return n;
}

// The tile counts of SEQS sequences from `first` on, as a running sum (of one head).
struct Window {
    int first;
    int64_t base;               // tiles of all heads before them
    int64_t sum[SEQS + 1];
    int64_t warp_sum[4];        // (of the warps that add up)
    unsigned long long units;   // of one head (LONG)
};
// All threads of the CTA call it; the first 128 add up.  A sequence's row tiles are gone
// over by one thread, or, for prompts of many (LONG), by a warp.
template <int ROWS, int TILE, bool LONG> __device__ void fill_window(const KvAttnArgs &a, Window &w, int first, int64_t base) {
    constexpr int COUNT = 128, PER = SEQS / COUNT;
    const bool counts = threadIdx.x < COUNT;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t mine[PER], total = 0;
    if constexpr (LONG) {
        unsigned long long units = 0;
        __syncthreads();   // (the window before has been read)
        if (threadIdx.x == 0) w.units = 0;
        __syncthreads();
        for (int i = warp; i < SEQS; i += blockDim.x / 32) {
            int64_t n = 0;   // (a prompt of millions of tokens has more tiles than 32 bits count)
            if (first + i < a.n_seqs) {
                const Seq q(a, first + i);
                units += (q.m * a.group + ROWS - 1) / ROWS;
                for (int r = lane * ROWS; r < q.m * a.group; r += 32 * ROWS) n += row_tiles<ROWS, TILE>(a, q, r);
#pragma unroll
                for (int d = 16; d; d /= 2) n += __shfl_xor_sync(0xFFFFFFFFu, n, d);
            }
            if (lane == 0) w.sum[i] = n;
        }
        if (lane == 0 && units > 0) atomicAdd(&w.units, units);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int k = threadIdx.x * PER + i;
        if constexpr (LONG)
            mine[i] = counts ? w.sum[k] : 0;
        else
            mine[i] = counts && first + k < a.n_seqs ? seq_tiles<ROWS, TILE>(a, first + k) : 0;
        total += mine[i];
    }
    int64_t x = total;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int64_t y = __shfl_up_sync(0xFFFFFFFFu, x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();
    if (counts && lane == 31) w.warp_sum[warp] = x;
    __syncthreads();
    if (counts) {
        int64_t at = x - total;
        for (int i = 0; i < warp; ++i) at += w.warp_sum[i];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            w.sum[threadIdx.x * PER + i] = at;
            at += mine[i];
        }
        if (threadIdx.x == COUNT - 1) w.sum[SEQS] = at;
    }
    if (threadIdx.x == 0) w.first = first, w.base = base;
    __syncthreads();
}

// Up to 32 sequences: every warp holds them all, a lane to a sequence, and needs no shared memory.
struct Lanes {
    int q0, m, len;
    int64_t from, to;   // the lane's sequence's tiles of one head, in the running count
    int64_t sum;        // of all
    int64_t units;      // of all
};
template <int ROWS, int TILE> __device__ __forceinline__ Lanes lanes_of(const KvAttnArgs &a) {
    const int lane = threadIdx.x & 31;
    Lanes r = {0, 0, 0, 0, 0, 0, 0};
    int64_t n = 0;
    int units = 0;
    if (lane < a.n_seqs) {
        const Seq q(a, lane);
        r.q0 = q.q0, r.m = q.m, r.len = q.len;
        units = (q.m * a.group + ROWS - 1) / ROWS;
        for (int r0 = 0; r0 < q.m * a.group; r0 += ROWS) n += row_tiles<ROWS, TILE>(a, q, r0);
    }
    int64_t x = n;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int64_t y = __shfl_up_sync(0xFFFFFFFFu, x, d);
        if (lane >= d) x += y;
    }
    r.from = x - n, r.to = x, r.sum = __shfl_sync(0xFFFFFFFFu, x, 31);
    r.units = __reduce_add_sync(0xFFFFFFFFu, units);   // (at most 2^30 rows in all)
    return r;
}
template <int ROWS, int TILE>
__device__ __forceinline__ void locate(const KvAttnArgs &a, const Lanes &s, int64_t at, Unit &u, int64_t &unit0, int &tiles) {
    const uint32_t behind = __ballot_sync(0xFFFFFFFFu, s.to * a.c.n_kv > at);
    u.seq = behind ? __ffs(behind) - 1 : 0;
    u.q0 = __shfl_sync(0xFFFFFFFFu, s.q0, u.seq), u.m = __shfl_sync(0xFFFFFFFFu, s.m, u.seq), u.len = __shfl_sync(0xFFFFFFFFu, s.len, u.seq);
    const int64_t from = __shfl_sync(0xFFFFFFFFu, s.from, u.seq), per_head = max((int64_t)1, __shfl_sync(0xFFFFFFFFu, s.to, u.seq) - from);
    int64_t off = at - from * a.c.n_kv;
    u.head = (int)min(quotient(off, per_head), (int64_t)a.c.n_kv - 1);
    unit0 = at - off + u.head * per_head;
    off -= u.head * per_head;
    const int rows_all = u.m * a.group;
    for (u.r0 = 0;; u.r0 += ROWS) {
        u.rows = min(ROWS, rows_all - u.r0);
        span(a, u.m, u.len, u.r0, u.r0 + u.rows, &u.lo, &u.hi);
        tiles = tiles_of<TILE>(u.lo, u.hi);
        if (off < tiles || u.r0 + ROWS >= rows_all) break;
        off -= tiles, unit0 += tiles;
    }
}

// The unit that holds tile `at` (at least the window's base), where it begins and how many tiles it has.  Called by
// whole warps.
template <int ROWS, int TILE, bool LONG>
__device__ __forceinline__ void locate(const KvAttnArgs &a, Window &win, int64_t at, Unit &u, int64_t &unit0, int &tiles) {
    // (lengths that another stream changes meanwhile give wrong results; the loops end all the same)
    while (at >= win.base + win.sum[SEQS] * a.c.n_kv && win.first + SEQS < a.n_seqs)
        fill_window<ROWS, TILE, LONG>(a, win, win.first + SEQS, win.base + win.sum[SEQS] * a.c.n_kv);
    int lo = 0, hi = SEQS - 1;   // the last sequence that begins at or before the tile
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (win.base + win.sum[mid] * a.c.n_kv <= at)
            lo = mid;
        else
            hi = mid - 1;
    }
    u.seq = win.first + lo;
    const int64_t per_head = max((int64_t)1, win.sum[lo + 1] - win.sum[lo]);
    int64_t off = at - (win.base + win.sum[lo] * a.c.n_kv);
    u.head = (int)min(quotient(off, per_head), (int64_t)a.c.n_kv - 1);
    unit0 = at - off + u.head * per_head;
    off -= u.head * per_head;
    const Seq q(a, u.seq);
    u.q0 = q.q0, u.m = q.m, u.len = q.len, u.r0 = 0;
    const int rows_all = q.m * a.group, lane = threadIdx.x & 31;
    if (LONG && rows_all > ROWS) {
        for (;; u.r0 += 32 * ROWS) {   // 32 row tiles at a time
            const int r = u.r0 + lane * ROWS;
            const int n = r < rows_all ? row_tiles<ROWS, TILE>(a, q, r) : 0;
            int x = n;   // (32 times at most 2^25)
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int y = __shfl_up_sync(0xFFFFFFFFu, x, d);
                if (lane >= d) x += y;
            }
            const int sum = __shfl_sync(0xFFFFFFFFu, x, 31);
            if (off >= sum && u.r0 + 32 * ROWS < rows_all) {
                off -= sum, unit0 += sum;
                continue;
            }
            const uint32_t over = __ballot_sync(0xFFFFFFFFu, x > off);
            const int j = over ? __ffs(over) - 1 : (rows_all - 1 - u.r0) / ROWS;
            const int before = __shfl_sync(0xFFFFFFFFu, x - n, j);
            u.r0 += j * ROWS, unit0 += before;
            break;
        }
        u.rows = min(ROWS, rows_all - u.r0);
        span(a, q.m, q.len, u.r0, u.r0 + u.rows, &u.lo, &u.hi);
        tiles = tiles_of<TILE>(u.lo, u.hi);
        return;
    }
    for (;; u.r0 += ROWS) {
        u.rows = min(ROWS, rows_all - u.r0);
        span(a, q.m, q.len, u.r0, u.r0 + u.rows, &u.lo, &u.hi);
        tiles = tiles_of<TILE>(u.lo, u.hi);
        if (off < tiles || u.r0 + ROWS >= rows_all) break;
        off -= tiles, unit0 += tiles;
    }
}

}  // namespace
}  // namespace realq
