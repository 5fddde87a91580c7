// Token log probabilities of rows of logits, with the row's entropy and its k
// likeliest tokens, and the gradient of all of them.
//
// Forward, for a row x of V logits with maximum m, s = sum e^(x_j - m) and
// u = sum e^(x_j - m) (x_j - m):
//   log p_y = (x_y - m) - log s,     H = log s - u / s,
// so one pass with running (m, s, u) gives all three.  The row is read once
// from HBM, which bounds the kernel.  A CTA owns a row; when there are too few
// rows to fill the SMs, a cluster of up to eight CTAs shares one and joins its
// parts through distributed shared memory in rank order.
//
// The k likeliest in the same pass: each thread notes the maximum of every
// 64-byte run it reads (runs merged so that it has at most 16 notes).  The two
// largest thread maxima of each of the 16 warps are 32 different elements of
// the row, so the k-th largest of them is a lower bound tau of the k-th
// largest element.  Only runs whose note reaches tau are read again (from L2),
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
#include <cooperative_groups.h>

#include "kernels.cuh"

namespace cg = cooperative_groups;

namespace realq {
namespace {

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr int NT = 512;       // threads of a forward CTA (16 warps: 32 maxima for tau)
constexpr int U = 4;          // 16-byte loads in flight per thread
constexpr int NOTES = 16;     // run maxima kept per thread
constexpr int CAP = 1024;     // collected candidates
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
    static __device__ __forceinline__ float round1(float v) { return v; }
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
__device__ __forceinline__ Stat join(Stat a, Stat b) {
    const float m = fmaxf(a.m, b.m);
    if (a.m < m) raise(a, m);
    if (b.m < m) raise(b, m);
    return Stat{m, a.s + b.s, a.u + b.u};
}
__device__ __forceinline__ void add(Stat &a, float x, float base) {
    const float t = (x - base) * LOG2E, e = ex2(t);
    a.s += e;
    a.u += e * fmaxf(t, -200.f);   // e is 0 there; -inf and the type's lowest value stay out of the product
}

__device__ __forceinline__ bool before(float va, int ia, float vb, int ib) { return va > vb || (va == vb && ia < ib); }

struct FwdSmem {
    float note[NOTES][NT];
    float cv[CAP];
    int ci[CAP];
    float topv[KMAX];
    int topi[KMAX];
    float wmax[32];
    Stat part[16];
    Stat total;
    float rv[16];
    int ri[16];
    float tau;
    int count;
};

template <typename TX>
__global__ void __launch_bounds__(NT, 2)
    logprobs_kernel(int V, int64_t ld, const TX *X, const int64_t *targets, float *logprob, float *norm,
                    float *entropy, int k, int64_t *top_ids, float *top_lp) {
    constexpr int E = Vec<TX>::E;
    __shared__ FwdSmem sm;
    cg::cluster_group cluster = cg::this_cluster();
    const int CL = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
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

    Stat st{neg_inf(), 0.f, 0.f};
    float tmax = sx, note = neg_inf();
    if (scol >= 0) {
        st.m = sx;
        add(st, sx, sx == neg_inf() ? 0.f : sx);
        if (!(sx == sx)) st.m = neg_inf();   // a NaN is kept in s alone
    }
    if (!(tmax == tmax)) tmax = neg_inf();
    for (int it = 0; it < iters; ++it) {
        uint4 raw[U];
        const int b = v0 + it * (NT * U) + tid;
#pragma unroll
        for (int q = 0; q < U; ++q) raw[q] = b + q * NT < v1 ? row.vec(b + q * NT) : Vec<TX>::fill();
        float x[U][E];
        float cm = neg_inf();
#pragma unroll
        for (int q = 0; q < U; ++q) {
            Vec<TX>::split(raw[q], x[q]);
#pragma unroll
            for (int e = 0; e < E; ++e) cm = fmaxf(cm, x[q][e]);
        }
        if (cm > st.m) raise(st, cm);
        const float base = st.m == neg_inf() ? 0.f : st.m;
#pragma unroll
        for (int q = 0; q < U; ++q)
#pragma unroll
            for (int e = 0; e < E; ++e) add(st, x[q][e], base);
        note = fmaxf(note, cm);
        tmax = fmaxf(tmax, cm);
        if (k > 0 && (it + 1 == iters || ((it + 1) >> shift) != (it >> shift))) {
            sm.note[it >> shift][tid] = note;
            note = neg_inf();
        }
    }

    // ---- join the threads' sums ----
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Stat b;
        b.m = __shfl_xor_sync(FULL, st.m, o);
        b.s = __shfl_xor_sync(FULL, st.s, o);
        b.u = __shfl_xor_sync(FULL, st.u, o);
        st = join(st, b);
    }
    if (lane == 0) sm.part[warp] = st;
    if (k > 0) {
        float w1 = tmax;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) w1 = fmaxf(w1, __shfl_xor_sync(FULL, w1, o));
        const int holder = __ffs(__ballot_sync(FULL, tmax == w1)) - 1;
        float w2 = lane == holder ? neg_inf() : tmax;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) w2 = fmaxf(w2, __shfl_xor_sync(FULL, w2, o));
        if (lane == 0) {
            sm.wmax[2 * warp] = w1;
            sm.wmax[2 * warp + 1] = w2;
        }
        if (tid < KMAX) {
            sm.topv[tid] = neg_inf();
            sm.topi[tid] = -1;
        }
        if (tid == 0) sm.count = 0;
    }
    __syncthreads();
    if (warp == 0) {
        if (lane == 0) {
            Stat t = sm.part[0];
            for (int w = 1; w < NT / 32; ++w) t = join(t, sm.part[w]);
            sm.total = t;
        }
        if (k > 0) {
            const float v = sm.wmax[lane];
            int above = 0;
            for (int j = 0; j < 32; ++j) {
                const float o = __shfl_sync(FULL, v, j);
                above += before(o, j, v, lane);
            }
            if (above == k - 1) sm.tau = v;
        }
    }
    __syncthreads();

    // ---- this CTA's k likeliest ----
    if (k > 0) {
        const float tau = sm.tau;
        auto offer = [&](float x, int col) {
            if (x >= tau && x > neg_inf()) {
                const int at = atomicAdd(&sm.count, 1);
                if (at < CAP) {
                    sm.cv[at] = x;
                    sm.ci[at] = col;
                }
            }
        };
        if (scol >= 0) offer(sx, scol);
        const int nn = iters > 0 ? ((iters - 1) >> shift) + 1 : 0;
        for (int n = 0; n < nn; ++n) {
            const float top = sm.note[n][tid];
            if (!(top >= tau && top > neg_inf())) continue;
            for (int it = n << shift; it < min(iters, (n + 1) << shift); ++it)
                for (int q = 0; q < U; ++q) {
                    const int v = v0 + it * (NT * U) + q * NT + tid;
                    if (v >= v1) continue;
                    float x[E];
                    Vec<TX>::split(row.vec(v), x);
#pragma unroll
                    for (int e = 0; e < E; ++e) offer(x[e], row.head + v * E + e);
                }
        }
        __syncthreads();
        const int C = sm.count;
        if (C <= CAP) {
            for (int i = tid; i < C; i += NT) {
                const float v = sm.cv[i];
                const int c = sm.ci[i];
                int above = 0;
                for (int j = 0; j < C; ++j) above += before(sm.cv[j], sm.ci[j], v, c);
                if (above < k) {
                    sm.topv[above] = v;
                    sm.topi[above] = c;
                }
            }
        } else {
            // too many equal values: the k first of the row's order, one at a time
            float pv = __int_as_float(0x7F800000);
            int pi = -1;
            for (int j = 0; j < k; ++j) {
                float bv = neg_inf();
                int bi = INT32_MAX;
                auto see = [&](float x, int col) {
                    if (x > neg_inf() && before(pv, pi, x, col) && before(x, col, bv, bi)) {
                        bv = x;
                        bi = col;
                    }
                };
                if (scol >= 0) see(sx, scol);
                for (int v = v0 + tid; v < v1; v += NT) {
                    float x[E];
                    Vec<TX>::split(row.vec(v), x);
#pragma unroll
                    for (int e = 0; e < E; ++e) see(x[e], row.head + v * E + e);
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    const float ov = __shfl_xor_sync(FULL, bv, o);
                    const int oi = __shfl_xor_sync(FULL, bi, o);
                    if (before(ov, oi, bv, bi)) {
                        bv = ov;
                        bi = oi;
                    }
                }
                if (lane == 0) {
                    sm.rv[warp] = bv;
                    sm.ri[warp] = bi;
                }
                __syncthreads();
                bv = sm.rv[0];
                bi = sm.ri[0];
                for (int w = 1; w < NT / 32; ++w)
                    if (before(sm.rv[w], sm.ri[w], bv, bi)) {
                        bv = sm.rv[w];
                        bi = sm.ri[w];
                    }
                __syncthreads();
                if (bv == neg_inf()) break;   // (the same on every thread)
                if (tid == 0) {
                    sm.topv[j] = bv;
                    sm.topi[j] = bi;
                }
                pv = bv;
                pi = bi;
            }
        }
        __syncthreads();
    }

    // ---- join the cluster's parts on its first CTA ----
    if (CL > 1) {
        cluster.sync();
        if (rank == 0) {
            if (tid == 0) {
                Stat t = sm.total;
                for (int c = 1; c < CL; ++c) t = join(t, *cluster.map_shared_rank(&sm.total, c));
                sm.total = t;
            }
            const bool mine = tid < CL * k;
            if (mine) {
                const FwdSmem *o = cluster.map_shared_rank(&sm, tid / k);
                sm.cv[tid] = o->topv[tid % k];
                sm.ci[tid] = o->topi[tid % k];
            }
            __syncthreads();
            if (k > 0 && tid < k) {
                sm.topv[tid] = neg_inf();
                sm.topi[tid] = -1;
            }
            __syncthreads();
            if (mine && sm.ci[tid] >= 0) {
                int above = 0;
                for (int j = 0; j < CL * k; ++j)
                    above += sm.ci[j] >= 0 && before(sm.cv[j], sm.ci[j], sm.cv[tid], sm.ci[tid]);
                if (above < k) {
                    sm.topv[above] = sm.cv[tid];
                    sm.topi[above] = sm.ci[tid];
                }
            }
            __syncthreads();
        }
        cluster.sync();   // the other CTAs' shared memory has been read
        if (rank != 0) return;
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
            const int64_t y = targets[r];
            float lp = 0.f;
            if (y >= V)
                lp = nan_f();
            else if (y >= 0)
                lp = empty ? neg_inf() : (load_as_float(row.p, y) - m) - ls;
            logprob[r] = lp;
        }
    }
    if (tid < k) {
        const int id = bad ? -1 : sm.topi[tid];
        top_ids[r * k + tid] = id;
        if (top_lp) top_lp[r * k + tid] = bad ? nan_f() : (id >= 0 ? (sm.topv[tid] - m) - ls : neg_inf());
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

template <typename TX>
realq_status_t fwd_launch(cudaStream_t s, int64_t T, int64_t V, int64_t ld, const void *X, const int64_t *targets,
                          float *logprob, float *norm, float *entropy, int k, int64_t *top_ids, float *top_lp,
                          int sms) {
    // Two CTAs fit an SM.  A row gets as many CTAs (a power of two up to 8) as
    // leave no second wave; each should still have a full pass of vectors.
    int cl = 1;
    while (cl < MAX_CLUSTER && T * cl * 2 <= 2 * (int64_t)sms && V / (2 * cl) >= (int64_t)NT * Vec<TX>::E) cl *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(T * cl));
    cfg.blockDim = dim3(NT);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cl;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    {
        Launch L("token_logprobs", s);
        REALQ_CUDA_TRY(cudaLaunchKernelEx(&cfg, logprobs_kernel<TX>, (int)V, ld, static_cast<const TX *>(X), targets,
                                          logprob, norm, entropy, k, top_ids, top_lp));
    }
    return check_launch("token_logprobs");
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
