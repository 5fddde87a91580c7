// Token log probabilities of rows of logits, with the row's entropy and its k
// likeliest tokens, and the gradient of all of them.
//
// Forward, for a row x of V logits with maximum m, s = sum e^(x_j - m) and
// u = sum e^(x_j - m) (x_j - m):
//   log p_y = (x_y - m) - log s,     H = log s - u / s,
// so one pass with running (m, s, u) gives all three.  The row is read once
// from HBM, which bounds the kernel.  A CTA owns a row; when there are too few
// rows to fill the SMs, a cluster of up to eight CTAs shares one and joins its
// parts through distributed shared memory in a fixed order.
//
// The k likeliest in the same pass: each thread notes the maximum of every
// 64-byte run it reads (runs merged so that it has at most 32 notes).  The four
// largest thread maxima of each of the 8 warps (the eight largest of each of 4,
// in a CTA of 128 threads) are 32 different elements of the row, so the k-th
// largest of them is a lower bound tau of the k-th largest element.  Only runs whose note reaches tau are read again (from L2),
// their elements >= tau collected and ranked by (value, lower index).  Where
// more than CAP elements reach tau (rows of equal values), k ordered passes
// over the row take their place.
//
// Gradient, with p_j = e^((x_j - m) - log s), c the row's coefficient of
// log p_y plus those of its alternatives:
//   d_j = c_y [j = y] + sum_i c_i [j = id_i] - p_j (c + c_H (log p_j + H)).
// The dense part is elementwise (one read and one write per logit, bound by
// HBM); the at most k + 1 listed positions are rewritten by the CTA that owns
// their columns.
//
// All sums are fp32 per thread (a few hundred terms), joined pairwise.
//
// Measured, 4096 rows x 128256 in bf16: 181 us with 5 alternatives (5.8 TB/s),
// 168 without (6.3 TB/s); the rows' ends, where the candidates are ranked, are
// the difference.  Taking the arithmetic's clamp or its packing away does not
// change it, more CTAs per SM (five or six, 40 to 48 registers) make it slower
// (208 to 217 us).  The gradient: 315 us (6.7 TB/s).  One row with 20
// alternatives: 9 us, of which the launch and reading it take 4.
#include <cooperative_groups.h>

#include "kernels.cuh"

namespace cg = cooperative_groups;

namespace realq {
namespace {

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr int U = 4;          // 16-byte loads in flight per thread
constexpr int NOTES = 32;     // run maxima kept per thread
constexpr int CAP = 1024;     // collected candidates
constexpr int RUNS = 256;     // runs that are read again
constexpr int KMAX = 32;
constexpr int MAX_CLUSTER = 8;

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xFF800000); }
__device__ __forceinline__ float nan_f() { return __int_as_float(0x7FC00000); }
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <typename TX> struct Vec;
template <> struct Vec<float> {
    static constexpr int E = 4;
    static __device__ __forceinline__ uint4 fill() {
        return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u);
    }
    static __device__ __forceinline__ void split(const uint4 &r, float (&v)[4]) {
        v[0] = __uint_as_float(r.x);
        v[1] = __uint_as_float(r.y);
        v[2] = __uint_as_float(r.z);
        v[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ uint4 join(const float (&v)[4]) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
    static __device__ __forceinline__ float top(const uint4 (&r)[U]) {
        float m = neg_inf();
#pragma unroll
        for (int q = 0; q < U; ++q)
            m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(r[q].x), __uint_as_float(r[q].y)),
                               fmaxf(__uint_as_float(r[q].z), __uint_as_float(r[q].w))));
        return m;
    }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int E = 8;
    static __device__ __forceinline__ uint4 fill() {
        return make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u);
    }
    static __device__ __forceinline__ void split(const uint4 &r, float (&v)[8]) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ uint4 join(const float (&v)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float top(const uint4 (&r)[U]) {   // pairwise in bf16, exact
        __nv_bfloat162 m = __halves2bfloat162(__ushort_as_bfloat16(0xFF80), __ushort_as_bfloat16(0xFF80));
#pragma unroll
        for (int q = 0; q < U; ++q) {
            const __nv_bfloat162 *h = reinterpret_cast<const __nv_bfloat162 *>(&r[q]);
            m = __hmax2(m, __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
        }
        return fmaxf(__low2float(m), __high2float(m));
    }
};
__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// A row as `head` single elements up to the first 16-byte boundary, nv
// vectors and `tail` single elements.
template <typename TX> struct Row {
    const TX *p;
    int head, nv, tail;
    __device__ __forceinline__ Row(const TX *row, int V) : p(row) {
        const int mis = (int)(reinterpret_cast<uintptr_t>(row) & 15);
        head = min(V, mis ? (16 - mis) / (int)sizeof(TX) : 0);
        nv = (V - head) / Vec<TX>::E;
        tail = V - head - nv * Vec<TX>::E;
    }
    __device__ __forceinline__ uint4 vec(int i) const {
        return __ldg(reinterpret_cast<const uint4 *>(p + head) + i);
    }
};

// Running (m, s, u) in units of log 2 for u; m = -inf with s = 0 (or NaN) when
// nothing finite has been met.
struct Stat {
    float m, s, u;
};
__device__ __forceinline__ void raise(Stat &a, float m) {   // a's sums relative to a larger maximum
    const bool none = a.m == neg_inf();
    // (2^-200 is 0 here; the bound keeps an infinite difference out of the product)
    const float d = none ? 0.f : fmaxf((a.m - m) * LOG2E, -200.f), c = ex2(d);
    a.u = c * (a.s == 0.f ? 0.f : a.u + a.s * d);
    a.s *= c;
    a.m = m;
}
// two fp32 numbers in one register pair
__device__ __forceinline__ uint64_t pack2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t r, float &a, float &b) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r));
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
// two logits into pairs of partial sums (nbase = minus the maximum, twice)
__device__ __forceinline__ void add_pair(uint64_t &s, uint64_t &u, float x0, float x1, uint64_t nbase) {
    const uint64_t t = mul2(add2(pack2(x0, x1), nbase), pack2(LOG2E, LOG2E));
    float t0, t1;
    unpack2(t, t0, t1);
    const uint64_t e = pack2(ex2(t0), ex2(t1));
    s = add2(s, e);
    // (e is 0 below -200: -inf and the type's lowest value stay out of the product)
    u = fma2(e, pack2(fmaxf(t0, -200.f), fmaxf(t1, -200.f)), u);
}

// The warp's largest value (no NaN among them): one reduction of integers in the order of the floats.
__device__ __forceinline__ float warp_max(float v) {
    const int b = __float_as_int(v), m = __reduce_max_sync(FULL, b ^ ((b >> 31) & 0x7FFFFFFF));
    return __int_as_float(m ^ ((m >> 31) & 0x7FFFFFFF));
}
// the warp's joined sums, on each lane
__device__ __forceinline__ Stat join_warp(Stat a) {
    const float m = warp_max(a.m);
    if (a.m < m) raise(a, m);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a.s += __shfl_xor_sync(FULL, a.s, o);
        a.u += __shfl_xor_sync(FULL, a.u, o);
    }
    a.m = m;
    return a;
}

// A candidate as one number: larger values first, equal ones by the lower index.
__device__ __forceinline__ uint64_t key_of(float v, int i) {
    const uint32_t b = __float_as_uint(v + 0.f);   // (-0 counts as 0)
    return (uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (uint32_t)(INT32_MAX - i);
}
__device__ __forceinline__ float key_value(uint64_t k) {
    const uint32_t b = (uint32_t)(k >> 32);
    return __uint_as_float(b & 0x80000000u ? b & 0x7FFFFFFFu : ~b);
}
__device__ __forceinline__ int key_index(uint64_t k) { return INT32_MAX - (int)(uint32_t)k; }

__device__ __forceinline__ bool before(float va, int ia, float vb, int ib) { return va > vb || (va == vb && ia < ib); }

template <int NT> struct FwdSmem {   // NT: threads of a forward CTA
    float note[NOTES][NT];
    uint64_t cand[CAP];
    uint64_t top[KMAX];       // keys, 0 where there is none
    uint64_t cluster_top[MAX_CLUSTER * KMAX];   // on the cluster's first CTA: every CTA's
    Stat cluster_total[MAX_CLUSTER];
    uint32_t run[RUNS];       // runs that reach tau: note << 16 | thread
    int runs;
    float wmax[32];
    Stat part[NT / 32];
    Stat total;
    uint64_t best[NT / 32];
    float tau;
    int count;
};
// the place of key among n others (none equal)
__device__ __forceinline__ int place_of(const uint64_t *keys, int n, uint64_t key) {
    int above = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) above += keys[j] > key;
    return above;
}

template <typename TX, int NT>
__global__ void __launch_bounds__(NT, 1024 / NT)
    logprobs_kernel(int V, int64_t ld, const TX *X, const int64_t *targets, float *logprob, float *norm,
                    float *entropy, int k, int64_t *top_ids, float *top_lp) {
    constexpr int E = Vec<TX>::E;
    constexpr int PER_WARP = 1024 / NT;   // thread maxima that each warp gives for tau (32 in all)
    __shared__ FwdSmem<NT> sm;
    cg::cluster_group cluster = cg::this_cluster();
    const int CL = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    // (waited for before the first CTA's shared memory is written: by then it has to have started)
    if (CL > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    const int64_t r = blockIdx.x / CL;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Row<TX> row(X + r * ld, V);
    const int v0 = (int)((int64_t)row.nv * rank / CL), v1 = (int)((int64_t)row.nv * (rank + 1) / CL);
    const int iters = (v1 - v0 + NT * U - 1) / (NT * U);
    int shift = 0;
    while (iters > 0 && ((iters - 1) >> shift) >= NOTES) ++shift;

    // the row's single elements: head on the first CTA, tail on the last
    int scol = -1;
    if (rank == 0 && tid < row.head) scol = tid;
    if (rank == CL - 1 && tid >= NT - row.tail) scol = V - (NT - tid);
    const float sx = scol >= 0 ? load_as_float(row.p, scol) : neg_inf();

    int64_t y = -1;   // the target, fetched early
    float xy = 0.f;
    if (logprob && rank == 0 && tid == 0) {
        y = targets[r];
        if (y >= 0 && y < V) xy = load_as_float(row.p, y);
    }

    Stat st{neg_inf(), 0.f, 0.f};
    float note = neg_inf();
    if (scol >= 0) {   // e^0 = 1; a NaN or +inf is kept in s as a NaN, with or without its maximum
        st.m = sx == sx ? sx : neg_inf();
        st.s = sx == neg_inf() ? 0.f : 1.f + (sx - sx);
    }
    uint4 raw[U];
    auto load = [&](int it) {
        const int b = v0 + it * (NT * U) + tid;
#pragma unroll
        for (int q = 0; q < U; ++q) raw[q] = b + q * NT < v1 ? row.vec(b + q * NT) : Vec<TX>::fill();
    };
    if (iters > 0) load(0);
    for (int it = 0; it < iters; ++it) {
        uint4 cur[U];
#pragma unroll
        for (int q = 0; q < U; ++q) cur[q] = raw[q];
        if (it + 1 < iters) load(it + 1);   // in flight during this one's arithmetic
        const float cm = Vec<TX>::top(cur);
        if (cm > st.m) raise(st, cm);
        const float nb = st.m == neg_inf() ? 0.f : -st.m;
        const uint64_t nbase = pack2(nb, nb);
        uint64_t s2 = pack2(st.s, 0.f), u2 = pack2(st.u, 0.f);
#pragma unroll
        for (int q = 0; q < U; ++q) {
            float x[E];
            Vec<TX>::split(cur[q], x);
#pragma unroll
            for (int e = 0; e < E; e += 2) add_pair(s2, u2, x[e], x[e + 1], nbase);
        }
        float a, b;
        unpack2(s2, a, b);
        st.s = a + b;
        unpack2(u2, a, b);
        st.u = a + b;
        note = fmaxf(note, cm);
        if (k > 0 && (it + 1 == iters || ((it + 1) >> shift) != (it >> shift))) {
            sm.note[it >> shift][tid] = note;
            note = neg_inf();
        }
    }

    // ---- join the threads' sums ----
    const Stat joined = join_warp(st);
    if (lane == 0) sm.part[warp] = joined;
    if (k > 0) {   // (st.m is the thread's maximum)
        float v = st.m, top = joined.m;
#pragma unroll
        for (int p = 0; p < PER_WARP; ++p) {
            if (p > 0) top = warp_max(v);
            if (lane == 0) sm.wmax[PER_WARP * warp + p] = top;
            if (lane == __ffs(__ballot_sync(FULL, v == top)) - 1) v = neg_inf();
        }
        if (tid < KMAX) sm.top[tid] = 0;
        if (tid == 0) sm.count = sm.runs = 0;
    }
    __syncthreads();
    if (warp == 0) {
        const Stat t = join_warp(lane < NT / 32 ? sm.part[lane] : Stat{neg_inf(), 0.f, 0.f});
        if (lane == 0) sm.total = t;
    } else if (warp == 1 && k > 0) {
        const float v = sm.wmax[lane];
        int above = 0;
#pragma unroll
        for (int j = 0; j < 32; ++j) above += before(sm.wmax[j], j, v, lane);
        if (above == k - 1) sm.tau = v;
    }
    __syncthreads();

    // ---- this CTA's k likeliest ----
    if (k > 0) {
        const float tau = sm.tau;
        auto offer = [&](float x, int col) {
            if (x >= tau && x > neg_inf()) {
                const int at = atomicAdd(&sm.count, 1);
                if (at < CAP) sm.cand[at] = key_of(x, col);
            }
        };
        if (scol >= 0) offer(sx, scol);
        const int nn = iters > 0 ? ((iters - 1) >> shift) + 1 : 0;
        if (iters == 1) {   // the only run is still in registers
            if (sm.note[0][tid] >= tau) {
#pragma unroll
                for (int q = 0; q < U; ++q) {
                    float x[E];
                    Vec<TX>::split(raw[q], x);
#pragma unroll
                    for (int e = 0; e < E; ++e) offer(x[e], row.head + (v0 + q * NT + tid) * E + e);   // (past the end: -inf)
                }
            }
        } else {
            for (int n = 0; n < nn; ++n) {
                const float top = sm.note[n][tid];
                if (top >= tau && top > neg_inf()) {
                    const int at = atomicAdd(&sm.runs, 1);
                    if (at < RUNS) sm.run[at] = (uint32_t)(n << 16 | tid);
                }
            }
            __syncthreads();
            // a run's 64 bytes by a warp, one value to a lane, several runs in flight
            constexpr int PER = 4, VALUES = U * E;
            const int R = sm.runs;
            if (R > RUNS) {
                if (tid == 0) sm.count = CAP + 1;
            } else {
                for (int i0 = warp; i0 < R; i0 += PER * (NT / 32)) {
                    for (int half = 0; half < 1 << shift; ++half) {
                        float x[PER];
                        int col[PER];
#pragma unroll
                        for (int p = 0; p < PER; ++p) {
                            const int i = i0 + p * (NT / 32);
                            x[p] = neg_inf();
                            col[p] = 0;
                            if (i < R && lane < VALUES) {
                                const uint32_t run = sm.run[i];
                                const int it = ((int)(run >> 16) << shift) + half;
                                const int v = v0 + it * (NT * U) + lane / E * NT + (int)(run & 0xFFFFu);
                                if (it < iters && v < v1) {
                                    col[p] = row.head + v * E + lane % E;
                                    x[p] = load_as_float(row.p, col[p]);
                                }
                            }
                        }
#pragma unroll
                        for (int p = 0; p < PER; ++p) offer(x[p], col[p]);
                    }
                }
            }
        }
        __syncthreads();
        const int C = sm.count;
        if (C <= CAP) {
            for (int i = tid; i < C; i += NT) {
                const uint64_t key = sm.cand[i];
                const int at = place_of(sm.cand, C, key);
                if (at < k) sm.top[at] = key;
            }
        } else {
            // too many equal values: the k first of the row's order, one at a time
            uint64_t last = ~0ull;
            for (int j = 0; j < k; ++j) {
                uint64_t best = 0;
                auto see = [&](float x, int col) {
                    const uint64_t key = key_of(x, col);
                    if (x > neg_inf() && key < last && key > best) best = key;
                };
                if (scol >= 0) see(sx, scol);
                for (int v = v0 + tid; v < v1; v += NT) {
                    float x[E];
                    Vec<TX>::split(row.vec(v), x);
#pragma unroll
                    for (int e = 0; e < E; ++e) see(x[e], row.head + v * E + e);
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(FULL, best, o));
                if (lane == 0) sm.best[warp] = best;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < NT / 32; ++w) best = max(best, sm.best[w]);
                __syncthreads();
                if (best == 0) break;   // (the same on every thread)
                if (tid == 0) sm.top[j] = best;
                last = best;
            }
        }
        __syncthreads();
    }

    // ---- join the cluster's parts on its first CTA, into which every CTA writes its own ----
    if (CL > 1) {
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        FwdSmem<NT> *first = cluster.map_shared_rank(&sm, 0);
        if (tid == 0) first->cluster_total[rank] = sm.total;
        if (tid < k) first->cluster_top[rank * k + tid] = sm.top[tid];
        cluster.sync();
        if (rank != 0) return;
        if (warp == NT / 32 - 1) {
            const Stat t = join_warp(lane < CL ? sm.cluster_total[lane] : Stat{neg_inf(), 0.f, 0.f});
            if (lane == 0) sm.total = t;
        }
        if (tid < k) sm.top[tid] = 0;
        __syncthreads();
        // a key's place: eight lanes count the larger keys, each in one CTA's list, which is in order
        for (int u0 = 0; u0 < CL * k * MAX_CLUSTER; u0 += NT) {
            const int i = (u0 + tid) / MAX_CLUSTER, list = tid % MAX_CLUSTER;
            const uint64_t key = i < CL * k ? sm.cluster_top[i] : 0;
            int above = 0;
            if (key && list < CL) {
                for (int step = KMAX / 2; step > 0; step >>= 1)   // (above < k always leaves a key to look at)
                    if (above + step <= k && sm.cluster_top[list * k + above + step - 1] > key) above += step;
                if (above < k && sm.cluster_top[list * k + above] > key) ++above;
            }
#pragma unroll
            for (int o = 1; o < MAX_CLUSTER; o <<= 1) above += __shfl_xor_sync(FULL, above, o);
            if (key && list == 0 && above < k) sm.top[above] = key;
        }
        __syncthreads();
    }

    const Stat t = sm.total;
    const bool empty = t.m == neg_inf() && t.s == 0.f;   // nothing but -inf
    const bool bad = !(t.s == t.s);                      // a NaN or +inf in the row
    const float m = bad ? nan_f() : t.m, ls = bad ? nan_f() : (empty ? 0.f : logf(t.s));
    if (tid == 0) {
        if (norm) {
            norm[2 * r] = m;
            norm[2 * r + 1] = ls;
        }
        if (entropy) {
            const float H = empty ? 0.f : ls - t.u / t.s * LN2;
            entropy[r] = bad ? nan_f() : (H < 0.f ? 0.f : H);
        }
        if (logprob) {
            float lp = 0.f;
            if (y >= V)
                lp = nan_f();
            else if (y >= 0)
                lp = empty ? neg_inf() : (xy - m) - ls;
            logprob[r] = lp;
        }
    }
    if (tid < k) {
        const uint64_t key = bad ? 0 : sm.top[tid];
        top_ids[r * k + tid] = key ? key_index(key) : -1;
        if (top_lp) top_lp[r * k + tid] = bad ? nan_f() : (key ? (key_value(key) - m) - ls : neg_inf());
    }
}

// ----------------------------------------------------------------- gradient ---
constexpr int BT = 256;
constexpr int BU = 4;

struct RowGrad {
    float m, ls, c, ch, H;
    __device__ __forceinline__ float dense(float x) const {   // -p (c + c_H (log p + H))
        const float lp = (x - m) - ls, p = ex2(lp * LOG2E);
        return p > 0.f ? -p * (c + ch * (lp + H)) : (p == p ? 0.f : p);
    }
};

template <typename TX>
__global__ void __launch_bounds__(BT)
    logprobs_grad_kernel(int V, int chunks, int64_t ld, const TX *X, const int64_t *targets, const float *norm,
                         const float *d_logprob, const float *entropy, const float *d_entropy, int k,
                         const int64_t *top_ids, const float *d_top, int64_t ldd, TX *D) {
    constexpr int E = Vec<TX>::E, CV = BT * BU;   // vectors per chunk
    const int64_t r = blockIdx.x / chunks;
    const int chunk = (int)(blockIdx.x % chunks);
    const int tid = threadIdx.x, lane = tid & 31;
    const TX *xr = X + r * ld;
    TX *dr = D + r * ldd;
    // vectors only where both rows are off the 16-byte boundary by the same amount
    const bool same = ((reinterpret_cast<uintptr_t>(xr) ^ reinterpret_cast<uintptr_t>(dr)) & 15) == 0;
    Row<TX> row(xr, V);
    const int span = CV * E;
    // columns [c0, c1) of this chunk: the head goes with the first, the tail with the last
    const int nch = same ? max(1, (row.nv + CV - 1) / CV) : (V + span - 1) / span;
    if (chunk >= nch) return;
    const int c0 = same ? (chunk == 0 ? 0 : row.head + chunk * span) : chunk * span;
    const int c1 = same ? (chunk == nch - 1 ? V : row.head + (chunk + 1) * span) : min(V, c0 + span);

    RowGrad g;
    g.m = norm[2 * r];
    g.ls = norm[2 * r + 1];
    const bool empty = g.m == neg_inf();
    const int64_t y64 = d_logprob ? targets[r] : -1;
    const int y = y64 >= 0 && y64 < V ? (int)y64 : -1;
    float cy = y64 >= 0 ? d_logprob[r] : 0.f;
    if (y64 >= V) cy = nan_f();
    g.ch = d_entropy ? d_entropy[r] : 0.f;
    g.H = d_entropy ? entropy[r] : 0.f;
    // coefficients of the alternatives, summed in a fixed order
    const int64_t id64 = lane < k ? top_ids[r * k + lane] : -1;
    const int id = id64 >= 0 && id64 < V ? (int)id64 : -1;
    const float ct = lane < k && id >= 0 ? d_top[r * k + lane] : 0.f;
    float sum = ct;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(FULL, sum, o);
    g.c = cy + sum;
    if (empty) {   // no token has a probability: no gradient
        g.m = 0.f;
        g.c = g.ch = 0.f;
    }

    // the listed positions inside this chunk: their logits before anything is written (D may be X)
    int at = -1, at_y = -1;
    float fix = 0.f, fix_y = 0.f;
    if (tid < 32) {
        const int cand = id >= c0 && id < c1 ? id : -1;
        float add = 0.f;
        for (int j = 0; j < k; ++j) {
            const int oj = __shfl_sync(FULL, id, j);
            const float cj = __shfl_sync(FULL, ct, j);
            if (oj == cand) add += cj;
        }
        if (cand == y) add += cy;
        at = cand;
        if (at >= 0) fix = g.dense(load_as_float(xr, at)) + add;
        const bool listed = __any_sync(FULL, id >= 0 && id == y);
        if (lane == 0 && !listed && y >= c0 && y < c1) {
            at_y = y;
            fix_y = g.dense(load_as_float(xr, y)) + cy;
        }
    }
    if (empty) at = at_y = -1;
    const int any = __syncthreads_or(at >= 0 || at_y >= 0);

    if (same) {
        const int b = chunk * CV + tid;
        const uint4 *px = reinterpret_cast<const uint4 *>(xr + row.head);
        uint4 *pd = reinterpret_cast<uint4 *>(dr + row.head);
        uint4 raw[BU];
#pragma unroll
        for (int q = 0; q < BU; ++q)
            if (b + q * BT < row.nv) raw[q] = px[b + q * BT];
#pragma unroll
        for (int q = 0; q < BU; ++q)
            if (b + q * BT < row.nv) {
                float x[E];
                Vec<TX>::split(raw[q], x);
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = g.dense(x[e]);
                pd[b + q * BT] = Vec<TX>::join(x);
            }
        if (chunk == 0 && tid < row.head) store1(dr + tid, g.dense(load_as_float(xr, tid)));
        if (chunk == nch - 1 && tid >= BT - row.tail) {
            const int c = V - (BT - tid);
            store1(dr + c, g.dense(load_as_float(xr, c)));
        }
    } else {
        for (int c = c0 + tid; c < c1; c += BT) store1(dr + c, g.dense(load_as_float(xr, c)));
    }
    if (any) {
        __syncthreads();
        if (at >= 0) store1(dr + at, fix);
        if (at_y >= 0) store1(dr + at_y, fix_y);
    }
}

// More rows than CTAs of 256 threads fit, and short ones: CTAs of 128, so that
// more rows are under way (seven to an SM, by their 28 KB of shared memory and
// the 1 KB that each CTA takes; registers would let eight).  With 5 alternatives,
// 128 threads against 256: 3469 x 4236 in fp32 30.7 and 35.1 us, 4000 x 32000 in
// bf16 61.7 and 65.6; longer rows are slower so: 2250 x 16774 in fp32 48 and 41.
constexpr int64_t SMALL_ROW = 65536;   // bytes

template <typename TX, int NT>
realq_status_t fwd_launch_nt(cudaStream_t s, int64_t T, int64_t V, int64_t ld, const void *X, const int64_t *targets,
                          float *logprob, float *norm, float *entropy, int k, int64_t *top_ids, float *top_lp,
                          int sms) {
    // 1024 threads fit an SM.  A row gets as many CTAs (a power of two up to 8) as
    // leave no second wave; each should still have a full pass of vectors.
    int cl = 1;
    while (cl < MAX_CLUSTER && T * cl * 2 <= 1024 / NT * (int64_t)sms && V / (2 * cl) >= (int64_t)NT * Vec<TX>::E) cl *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(T * cl));
    cfg.blockDim = dim3(NT);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cl;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cl > 1 ? 1 : 0;
    {
        Launch L("token_logprobs", s);
        REALQ_CUDA_TRY(cudaLaunchKernelEx(&cfg, logprobs_kernel<TX, NT>, (int)V, ld, static_cast<const TX *>(X), targets,
                                          logprob, norm, entropy, k, top_ids, top_lp));
    }
    return check_launch("token_logprobs");
}

template <typename TX>
realq_status_t fwd_launch(cudaStream_t s, int64_t T, int64_t V, int64_t ld, const void *X, const int64_t *targets,
                          float *logprob, float *norm, float *entropy, int k, int64_t *top_ids, float *top_lp,
                          int sms) {
    if (T > 4 * sms && V * (int64_t)sizeof(TX) <= SMALL_ROW)
        return fwd_launch_nt<TX, 128>(s, T, V, ld, X, targets, logprob, norm, entropy, k, top_ids, top_lp, sms);
    return fwd_launch_nt<TX, 256>(s, T, V, ld, X, targets, logprob, norm, entropy, k, top_ids, top_lp, sms);
}

template <typename TX>
realq_status_t grad_launch(cudaStream_t s, int64_t T, int64_t V, int64_t ld, const void *X, const int64_t *targets,
                           const float *norm, const float *d_logprob, const float *entropy, const float *d_entropy,
                           int k, const int64_t *top_ids, const float *d_top, int64_t ldd, void *D) {
    const int64_t span = (int64_t)BT * BU * Vec<TX>::E;
    const int64_t chunks = (V + span - 1) / span;
    {
        Launch L("token_logprobs_grad", s);
        logprobs_grad_kernel<TX><<<(unsigned)(T * chunks), BT, 0, s>>>(
            (int)V, (int)chunks, ld, static_cast<const TX *>(X), targets, norm, d_logprob, entropy, d_entropy, k,
            top_ids, d_top, ldd, static_cast<TX *>(D));
    }
    return check_launch("token_logprobs_grad");
}

}  // namespace

realq_status_t token_logprobs(cudaStream_t s, int64_t T, int64_t V, int64_t ld, const void *X, realq_dtype_t dt,
                              const int64_t *targets, float *logprob, float *norm, float *entropy, int k,
                              int64_t *top_ids, float *top_lp, int sms) {
    return dt == REALQ_BF16
               ? fwd_launch<__nv_bfloat16>(s, T, V, ld, X, targets, logprob, norm, entropy, k, top_ids, top_lp, sms)
               : fwd_launch<float>(s, T, V, ld, X, targets, logprob, norm, entropy, k, top_ids, top_lp, sms);
}

realq_status_t token_logprobs_grad(cudaStream_t s, int64_t T, int64_t V, int64_t ld, const void *X, realq_dtype_t dt,
                                   const int64_t *targets, const float *norm, const float *d_logprob,
                                   const float *entropy, const float *d_entropy, int k, const int64_t *top_ids,
                                   const float *d_top, int64_t ldd, void *D) {
    return dt == REALQ_BF16 ? grad_launch<__nv_bfloat16>(s, T, V, ld, X, targets, norm, d_logprob, entropy, d_entropy,
                                                         k, top_ids, d_top, ldd, D)
                            : grad_launch<float>(s, T, V, ld, X, targets, norm, d_logprob, entropy, d_entropy, k,
                                                 top_ids, d_top, ldd, D);
}

}  // namespace realq
