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
// One CTA owns a 128 x 256 tile of dW (rows of dY's width, columns of X̂'s) and
// a range of tokens.  Both operands are token-major, i.e. MN-major for the
// MMA: a TMA box of 64 tokens x 64 channels (128-byte rows, 128-byte swizzle)
// is one canonical atom stack, two boxes make A and four make B.  Tokens are
// split over CTAs when the tiles alone do not fill the SMs; the parts are
// summed in a fixed order.
#include "kernels.cuh"
#include "tc.cuh"

#include <algorithm>

namespace realq {
namespace {

constexpr int TM = 128;
constexpr int TN = 256;
constexpr int KSTAGE = 64;                       // tokens per pipeline stage
constexpr int STAGES = 4;
constexpr int CHUNK_STAGES = 16;                 // stages per TMEM accumulator pass
constexpr int DRAIN_WARPS = 8;
constexpr int THREADS = (DRAIN_WARPS + 2) * 32;
constexpr int BOX_BYTES = 64 * KSTAGE * 2;
constexpr int A_BYTES = TM * KSTAGE * 2;
constexpr int B_BYTES = TN * KSTAGE * 2;
constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + 1024 + 256;
constexpr uint32_t IDESC = tc::idesc_bf16_f32(TM, TN, 1, 1);
constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int MAX_SPLITS = 8;

// Tile t of the nti x ntj grid, in groups of 8 row tiles: the CTAs resident
// together cover a compact block of dW and share operands through L2.
__device__ __forceinline__ void tile_of(int t, int nti, int ntj, int &ti, int &tj) {
    constexpr int G = 8;
    const int g = t / (G * ntj), r0 = g * G, rows = min(G, nti - r0), k = t - g * G * ntj;
    ti = r0 + k % rows;
    tj = k / rows;
}

// planes: token rows [p T_pad, p T_pad + T) of A hold dY's plane p
__global__ void __launch_bounds__(THREADS, 1)
    weight_grad_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, int planes,
                       int64_t plane_rows, int64_t m, int64_t n, int64_t T, int64_t tper, float *dW, int accumulate,
                       float *part, int *err) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t *full = reinterpret_cast<uint64_t *>(smem + STAGES * STAGE_BYTES);
    uint64_t *empty = full + STAGES;
    uint64_t *accf = empty + STAGES;             // [2] accumulator b holds a finished chunk
    uint64_t *acce = accf + 2;                   // [2] accumulator b has been drained
    uint64_t *done = acce + 2;                   // every MMA issued has retired
    uint32_t *tslot = reinterpret_cast<uint32_t *>(done + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tslot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int ti, tj;
    tile_of((int)blockIdx.x, (int)((m + TM - 1) / TM), (int)((n + TN - 1) / TN), ti, tj);
    const int i0 = ti * TM, j0 = tj * TN;
    const int64_t t_begin = (int64_t)blockIdx.y * tper;
    const int64_t t_end = min(T, t_begin + tper);
    const int nkp = t_end > t_begin ? (int)((t_end - t_begin + KSTAGE - 1) / KSTAGE) : 0;   // stages per plane
    const int nk = nkp * planes;
    const int nch = (nk + CHUNK_STAGES - 1) / CHUNK_STAGES;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            tc::mbar_init(tc::smem_u32(&full[s]), 1);
            tc::mbar_init(tc::smem_u32(&empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            tc::mbar_init(tc::smem_u32(&accf[b]), 1);
            tc::mbar_init(tc::smem_u32(&acce[b]), DRAIN_WARPS);
        }
        tc::mbar_init(tc::smem_u32(done), 1);
        *abort_flag = 0;
        tc::fence_barrier_init();
        tc::prefetch_tmap(&mapA);
        tc::prefetch_tmap(&mapB);
    }
    if (warp == 0) tc::tmem_alloc(tc::smem_u32(tslot), 2 * TN);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = *tslot;

    float acc[128];
#pragma unroll
    for (int c = 0; c < 128; ++c) acc[c] = 0.f;
    bool good = true;

    if (warp == DRAIN_WARPS) {
        if (lane == 0) {
            // ---------------- TMA producer ----------------
            // the planes of a token range follow one another stage by stage
            int it = 0;
            for (; it < nk; ++it) {
                const int s = it % STAGES;
                const uint32_t r = (uint32_t)(it / STAGES);
                if (!tc::mbar_wait(tc::smem_u32(&empty[s]), (r & 1u) ^ 1u, abort_flag)) {
                    *abort_flag = 1;
                    break;
                }
                const uint32_t fb = tc::smem_u32(&full[s]);
                tc::mbar_arrive_expect_tx(fb, STAGE_BYTES);
                const int p = it % planes;
                const int y = (int)(t_begin + (int64_t)(it / planes) * KSTAGE);
                const int ya = (int)(p * plane_rows) + y;
                const uint32_t a = tc::smem_u32(smem + s * STAGE_BYTES);
                tc::tma_load_2d(a, &mapA, fb, i0, ya);
                tc::tma_load_2d(a + BOX_BYTES, &mapA, fb, i0 + 64, ya);
#pragma unroll
                for (int q = 0; q < 4; ++q) tc::tma_load_2d(a + A_BYTES + q * BOX_BYTES, &mapB, fb, j0 + 64 * q, y);
            }
            // on abort, let the copies already issued land before the CTA exits
            if (*abort_flag) {
                int never = 0;
                for (int k = (it > STAGES ? it - STAGES : 0); k < it; ++k)
                    tc::mbar_wait(tc::smem_u32(&full[k % STAGES]), (uint32_t)(k / STAGES) & 1u, &never,
                                  100000000ull);
            }
        }
    } else if (warp == DRAIN_WARPS + 1) {
        // ---------------- MMA issuer (the whole warp waits, one lane issues) ----------------
        const uint64_t desc0 = tc::smem_desc(tc::smem_u32(smem), BOX_BYTES, 1024, tc::SW_128B);
        int s = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int c = 0; c < nch && ok; ++c) {
            const int b = c & 1;
            if (c >= 2) {
                ok = __all_sync(FULL, tc::mbar_wait(tc::smem_u32(&acce[b]), (uint32_t)((c >> 1) - 1) & 1u, abort_flag));
                if (!ok) break;
            }
            tc::fence_after_sync();
            const uint32_t d = tmem + (uint32_t)(b * TN);
            const int cnt = min(CHUNK_STAGES, nk - c * CHUNK_STAGES);
            for (int i = 0; i < cnt; ++i) {
                ok = __all_sync(FULL, tc::mbar_wait(tc::smem_u32(&full[s]), phase, abort_flag));
                if (!ok) break;
                tc::fence_after_sync();
                const uint64_t da = desc0 + (uint32_t)(s * STAGE_BYTES >> 4), db = da + (A_BYTES >> 4);
                if (tc::elect_one()) {
#pragma unroll
                    for (int k = 0; k < KSTAGE / 16; ++k)
                        tc::mma_bf16_ss(d, da + k * (2048 >> 4), db + k * (2048 >> 4), IDESC, (i > 0 || k > 0) ? 1u : 0u);
                    tc::mma_commit(tc::smem_u32(&empty[s]));
                }
                __syncwarp();
                if (++s == STAGES) {
                    s = 0;
                    phase ^= 1u;
                }
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
    } else {
        // ------- drain warps: TMEM chunk -> fp32 registers (lane quarter, column half) -------
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t col_base = (uint32_t)((warp >> 2) * 128);
        for (int c = 0; c < nch; ++c) {
            const int b = c & 1;
            const bool ok = tc::mbar_wait(tc::smem_u32(&accf[b]), (uint32_t)(c >> 1) & 1u, abort_flag);
            if (!__all_sync(FULL, ok)) {
                good = false;
                *abort_flag = 1;
                break;
            }
            tc::fence_after_sync();
#pragma unroll
            for (int c0 = 0; c0 < 128; c0 += 32) {
                uint32_t v[32];
                tc::tmem_ld_32x32b_x32(tmem + lane_base + (uint32_t)(b * TN) + col_base + (uint32_t)c0, v);
#pragma unroll
                for (int q = 0; q < 32; ++q) acc[c0 + q] += __uint_as_float(v[q]);
            }
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(tc::smem_u32(&acce[b]));
        }
    }
    __syncwarp();
    const bool all_good = __syncthreads_and(good && !*abort_flag) != 0;

    if (warp < DRAIN_WARPS) {
        const int64_t gi = i0 + (warp & 3) * 32 + lane;
        const int64_t gj0 = j0 + (warp >> 2) * 128;
        if (gi < m) {
            float *out = part ? part + (int64_t)blockIdx.y * m * n : dW;
            const bool add = !part && accumulate;
#pragma unroll
            for (int q = 0; q < 128; ++q)
                if (gj0 + q < n) {
                    const float v = all_good ? acc[q] : __int_as_float(0x7fc00000);
                    float *o = out + gi * n + gj0 + q;
                    *o = add ? *o + v : v;
                }
        }
    }
    if (!all_good && threadIdx.x == 0) atomicOr(err, ST_TIMEOUT);
    tc::fence_before_sync();
    __syncthreads();
    if (warp == 0) tc::tmem_dealloc(tmem, 2 * TN);
}

__global__ void __launch_bounds__(256) weight_grad_reduce(int64_t count, int splits, const float *part, float *dW,
                                                          int accumulate) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    float v = part[i];
    for (int z = 1; z < splits; ++z) v += part[z * count + i];
    dW[i] = accumulate ? dW[i] + v : v;
}

// X̂ as a bf16 plane of row stride ldx (columns from n on are not written and
// lie outside the tensor map).  A thread unpacks 16 values (half a block) where
// rows are whole blocks, else a warp a block.
__device__ __forceinline__ float step_of(uint32_t b) {
    if (b == 255u) return __int_as_float(0x7FC00000);
    return __uint_as_float(b >= 7u ? (b - 6u) << 23 : 1u << (b + 16u));
}
__global__ void __launch_bounds__(256) unpack_plane_vec_kernel(int64_t count, const uint4 *codes, const uint8_t *exps,
                                                               uint4 *X) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    const uint4 q = __ldg(codes + i);
    const float s = step_of(__ldg(exps + (i >> 1)));
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    uint32_t h[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {   // (bf16 numbers: the upper halves are exact)
        const float lo = (float)(int8_t)(w[k >> 1] >> (16 * (k & 1))) * s;
        const float hi = (float)(int8_t)(w[k >> 1] >> (16 * (k & 1) + 8)) * s;
        h[k] = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
    }
    X[2 * i] = make_uint4(h[0], h[1], h[2], h[3]);
    X[2 * i + 1] = make_uint4(h[4], h[5], h[6], h[7]);
}
__global__ void __launch_bounds__(256) unpack_plane_kernel(int64_t T, int64_t n, int64_t nb, const int8_t *codes,
                                                           const uint8_t *exps, __nv_bfloat16 *X, int64_t ldx) {
    const int lane = threadIdx.x & 31;
    const int64_t w = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 5;
    if (w >= T * nb) return;
    const int64_t t = w / nb, c = (w % nb) * 32 + lane;
    if (c < n) X[t * ldx + c] = __float2bfloat16_rn((float)codes[t * n + c] * step_of(exps[w]));
}

// dY's planes: bf16 copied to an aligned row stride, fp32 as three bf16 planes
__global__ void __launch_bounds__(256) copy_plane_kernel(int64_t T, int64_t m, const __nv_bfloat16 *dY,
                                                         __nv_bfloat16 *out, int64_t ld) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= T * m) return;
    out[i / m * ld + i % m] = dY[i];
}
__global__ void __launch_bounds__(256) split_plane_kernel(int64_t T, int64_t m, const float *dY, __nv_bfloat16 *out,
                                                          int64_t ld) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= T * m) return;
    const float v = dY[i];
    const bool num = (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u;
    const uint32_t hi = __float_as_uint(v) & 0xFFFF0000u;
    const float r1 = num ? v - __uint_as_float(hi) : 0.f;   // infinities and NaN stay in the first plane
    const uint32_t mid = __float_as_uint(r1) & 0xFFFF0000u;
    const uint32_t lo = __float_as_uint(r1 - __uint_as_float(mid)) & 0xFFFF0000u;
    const int64_t at = i / m * ld + i % m, plane = T * ld;
    // (a NaN whose payload lies in the lower half must not become an infinity)
    out[at] = num ? __ushort_as_bfloat16((unsigned short)(hi >> 16)) : __float2bfloat16_rn(v);
    out[at + plane] = __ushort_as_bfloat16((unsigned short)(mid >> 16));
    out[at + 2 * plane] = __ushort_as_bfloat16((unsigned short)(lo >> 16));
}

int64_t pad8(int64_t x) { return (x + 7) / 8 * 8; }

// Token ranges: with fewer tiles than SMs, as many as fill them without
// leaving a range under four stages.
int grad_splits(int64_t T, int64_t m, int64_t n, int sms) {
    const int64_t tiles = (int64_t)ceil_div(m, TM) * ceil_div(n, TN);
    int64_t s = sms / tiles;
    s = std::min<int64_t>(s, T / (4 * KSTAGE));
    return (int)std::max<int64_t>(1, std::min<int64_t>(s, MAX_SPLITS));
}

struct GradWs {
    int *status;
    __nv_bfloat16 *x, *dy;
    float *part;
    size_t bytes;
    GradWs(void *ws, int64_t T, int64_t m, int64_t n, realq_dtype_t dt, int splits) {
        Carve c(ws);
        status = c.take<int>(64);
        x = c.take<__nv_bfloat16>((size_t)(T * pad8(n)));
        dy = c.take<__nv_bfloat16>((size_t)(T * pad8(m)) * (dt == REALQ_F32 ? 3 : (m % 8 ? 1 : 0)));
        part = c.take<float>(splits > 1 ? (size_t)splits * m * n : 0);
        bytes = c.off;
    }
};

}  // namespace

size_t checkpoint_grad_ws_bytes(int64_t T, int64_t m, int64_t n, realq_dtype_t dt, int sms) {
    return GradWs(nullptr, T, m, n, dt, grad_splits(T, m, n, sms)).bytes;
}

realq_status_t checkpoint_grad(cudaStream_t s, int64_t T, int64_t m, int64_t n, const void *dY, realq_dtype_t dt,
                               const int8_t *codes, const uint8_t *exps, float *dW, int accumulate, void *ws, int sms) {
    int splits = grad_splits(T, m, n, sms);
    const GradWs w(ws, T, m, n, dt, splits);
    REALQ_CUDA_TRY(cudaMemsetAsync(w.status, 0, sizeof(int), s));
    const int64_t nb = (n + 31) / 32, ldx = pad8(n);
    {
        Launch L("checkpoint_grad_unpack", s);
        if (n % 32 == 0 && (reinterpret_cast<uintptr_t>(codes) & 15) == 0)
            unpack_plane_vec_kernel<<<(unsigned)((T * n / 16 + 255) / 256), 256, 0, s>>>(
                T * n / 16, reinterpret_cast<const uint4 *>(codes), exps, reinterpret_cast<uint4 *>(w.x));
        else
            unpack_plane_kernel<<<(unsigned)((T * nb * 32 + 255) / 256), 256, 0, s>>>(T, n, nb, codes, exps, w.x, ldx);
    }
    REALQ_TRY(check_launch("checkpoint_grad_unpack"));
    const bool direct = dt == REALQ_BF16 && m % 8 == 0;
    const int planes = dt == REALQ_F32 ? 3 : 1;
    const int64_t ldy = pad8(m);
    if (!direct) {
        Launch L("checkpoint_grad_planes", s);
        const unsigned g = (unsigned)((T * m + 255) / 256);
        if (dt == REALQ_BF16)
            copy_plane_kernel<<<g, 256, 0, s>>>(T, m, static_cast<const __nv_bfloat16 *>(dY), w.dy, ldy);
        else
            split_plane_kernel<<<g, 256, 0, s>>>(T, m, static_cast<const float *>(dY), w.dy, ldy);
        REALQ_TRY(check_launch("checkpoint_grad_planes"));
    }
    CUtensorMap mapA, mapB;
    CUresult cr = encode_tmap_2d_bf16(&mapA, direct ? dY : (const void *)w.dy, (uint64_t)m, (uint64_t)(planes * T),
                                      (uint64_t)ldy * 2, 64, KSTAGE, 1);
    if (cr == CUDA_SUCCESS)
        cr = encode_tmap_2d_bf16(&mapB, w.x, (uint64_t)n, (uint64_t)T, (uint64_t)ldx * 2, 64, KSTAGE, 1);
    if (cr != CUDA_SUCCESS) return fail(REALQ_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)cr);
    int64_t tper = (T + splits - 1) / splits;
    tper = (tper + KSTAGE - 1) / KSTAGE * KSTAGE;
    splits = (int)((T + tper - 1) / tper);
    REALQ_TRY(set_smem_limit(reinterpret_cast<const void *>(weight_grad_kernel), SMEM_BYTES));
    const int64_t tiles = (int64_t)ceil_div(m, TM) * ceil_div(n, TN);
    {
        Launch L("checkpoint_weight_grad", s);
        weight_grad_kernel<<<dim3((unsigned)tiles, (unsigned)splits), THREADS, SMEM_BYTES, s>>>(
            mapA, mapB, planes, T, m, n, T, tper, dW, accumulate, splits > 1 ? w.part : nullptr, w.status);
    }
    REALQ_TRY(check_launch("checkpoint_weight_grad"));
    if (splits > 1) {
        Launch L("checkpoint_grad_reduce", s);
        weight_grad_reduce<<<(unsigned)((m * n + 255) / 256), 256, 0, s>>>(m * n, splits, w.part, dW, accumulate);
        REALQ_TRY(check_launch("checkpoint_grad_reduce"));
    }
    return REALQ_OK;
}

}  // namespace realq
