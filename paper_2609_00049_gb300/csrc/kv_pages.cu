// Pages of the key/value cache: taking, sharing, giving up and compacting them.
//
// The bookkeeping (reference counts, tables, lengths: a few numbers per page and
// row) runs as one cluster of eight CTAs, whose hardware barrier orders the
// steps of a call, so that a call is one launch however many steps it has; a
// page's contents are then copied by a second launch over all SMs, which reads
// on the device how many copies there are.  Free pages are those whose count is
// 0; they are taken in ascending order, found by counting them in eight parts
// of the pool and then listing the first few.
//
// Bound by latency (the bookkeeping: a few steps of global reads and atomics)
// and by memory (the copies: each byte read and written once).  56 branches of
// eight prompts take 10 us to fork and 13.5 to reserve a token each, with copies of
// 10 us; compacting 2048 pages of 8 layers, half in use, 13.5 us for the plan and
// 66 for 403 MB, 6.1 TB/s, 0.9 of a copy's rate.
#include <algorithm>

#include "kernels.cuh"
#include "tc.cuh"

namespace realq {
namespace {

constexpr int CTAS = 8, THREADS = 1024, WARPS = THREADS / 32, ALL = CTAS * THREADS;

// Workspace of the page operators.
struct PageWs {
    int *head;          // [0] status, [1] copies to make, [2] failed, [8 + c] counts of part c, [16 + c] others
    int *list;          // n_pages: free pages in ascending order; compact: holes
    int *writers;       // n_pages: rows of the call that write into a shared page
    int *latest;        // n_pages: the last of them (+ 1)
    int *src, *dst;     // max(n_rows, n_pages): copies to make
    int *winner;        // n_rows
    int *need;          // n_rows: pages a row takes, then where its first lies in the list
    int *stage;         // n_rows x (max_pages + 1): fork's rows as they were
};

size_t carve(void *ws, int64_t n_pages, int64_t n_rows, int64_t max_pages, PageWs *out) {
    Carve c(ws);
    PageWs w;
    w.head = c.take<int>(64);
    w.list = c.take<int>(n_pages);
    w.writers = c.take<int>(n_pages);
    w.latest = c.take<int>(n_pages);
    w.src = c.take<int>(std::max(n_rows, n_pages));
    w.dst = c.take<int>(std::max(n_rows, n_pages));
    w.winner = c.take<int>(n_rows);
    w.need = c.take<int>(n_rows);
    w.stage = c.take<int>((size_t)n_rows * (max_pages + 1));
    if (out) *out = w;
    return c.off;
}

__device__ __forceinline__ int rank() { return (int)tc::cluster_rank(); }
// all threads of the cluster; what they wrote to global memory before is seen after (the barrier releases and acquires)
__device__ __forceinline__ void meet() { tc::cluster_sync(); }
// memory that other CTAs of the cluster write during the kernel: past the L1
__device__ __forceinline__ int peek(const int *p) { return __ldcg(p); }

// the CTA's sum of v
__device__ __forceinline__ int block_sum(int v) {
    __shared__ int part[WARPS];
    v = __reduce_add_sync(0xFFFFFFFFu, v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    int t = part[threadIdx.x & 31];
    return __reduce_add_sync(0xFFFFFFFFu, t);
}
// exclusive prefix of v over the CTA's threads; *total their sum
template <class I> __device__ __forceinline__ I block_scan(I v, I *total) {
    __shared__ I part[WARPS];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    I x = v;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const I y = __shfl_up_sync(0xFFFFFFFFu, x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 31) part[w] = x;
    __syncthreads();
    I p = part[lane];
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const I y = __shfl_up_sync(0xFFFFFFFFu, p, d);
        if (lane >= d) p += y;
    }
    *total = __shfl_sync(0xFFFFFFFFu, p, 31);
    const I base = w == 0 ? 0 : __shfl_sync(0xFFFFFFFFu, p, w - 1);
    return base + x - v;
}

__device__ __forceinline__ bool in_pool(int page, int n_pages) { return page >= 0 && page < n_pages; }

// This CTA's share of the pool's pages.
struct Part {
    int lo, hi;
    __device__ explicit Part(int n) {
        const int per = (n + CTAS - 1) / CTAS;
        lo = min(n, rank() * per), hi = min(n, lo + per);
    }
};
template <class Pred> __device__ __forceinline__ void count_part(const Part &part, int *counts, Pred pred) {
    int mine = 0;
    for (int p = part.lo + threadIdx.x; p < part.hi; p += THREADS) mine += pred(p) ? 1 : 0;
    mine = block_sum(mine);
    if (threadIdx.x == 0) counts[rank()] = mine;
}
// of the eight counts, those of the parts before this one and of all
__device__ __forceinline__ int2 counted(const int *counts) {
    int2 r = make_int2(0, 0);
    for (int c = 0; c < CTAS; ++c) {
        const int v = peek(counts + c);
        r.x += c < rank() ? v : 0, r.y += v;
    }
    return r;
}
// put(r, p) for the pages p of this part that pred holds for, r counting from `at`, as far as r < limit
template <class Pred, class Put>
__device__ __forceinline__ void list_part(const Part &part, int at, int limit, Pred pred, Put put) {
    for (int base = part.lo; base < part.hi && at < limit; base += THREADS) {
        const int p = base + threadIdx.x;
        const bool yes = p < part.hi && pred(p);
        int total;
        const int r = at + block_scan(yes ? 1 : 0, &total);
        if (yes && r < limit) put(r, p);
        at += total;
    }
}

// --------------------------------------------------------------- reserve ---
struct Row {            // a row's part of the call
    int64_t len, add;   // its tokens before, the new ones
    int first, after;   // table entries that need a new page: [first, after)
    int last;           // a partly filled last page, or -1
    bool ok;
};
__device__ __forceinline__ Row row_of(const KvPagesView &v, const int *starts, int log_page, int s, int64_t T) {
    Row r;
    const int64_t b = starts[s], e = starts[s + 1], page = 1ll << log_page;
    r.len = v.lengths[s], r.add = e - b;
    r.ok = b >= 0 && e >= b && e <= T && r.len >= 0 && r.len + r.add <= INT32_MAX;
    const int64_t first = (r.len + page - 1) >> log_page, after = (r.len + r.add + page - 1) >> log_page;
    r.ok = r.ok && (r.add == 0 || after <= v.max_pages);
    r.first = (int)first, r.after = r.ok && r.add > 0 ? (int)after : (int)first;
    r.last = -1;
    if (r.ok && r.add > 0 && (r.len & (page - 1)) != 0) {
        r.last = v.tables[s * v.max_pages + (r.len >> log_page)];
        if (!in_pool(r.last, v.n_pages)) r.ok = false, r.last = -1;
    }
    return r;
}

__global__ void __cluster_dims__(CTAS, 1, 1) __launch_bounds__(THREADS)
reserve_kernel(KvPagesView v, const int *starts, int64_t T, int64_t *positions, int log_page, PageWs w) {
    dependents_may_start();   // (the copies wait for this kernel's end)
    const int tid = rank() * THREADS + threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int n_rows = (int)v.n_rows;
    const Part part((int)v.n_pages);
    const auto is_free = [&](int p) { return v.used[p] <= 0; };
    for (int s = tid; s < n_rows; s += ALL) {
        const Row r = row_of(v, starts, log_page, s, T);
        if (r.last >= 0) w.writers[r.last] = 0, w.latest[r.last] = 0;
    }
    if (tid == 0) w.head[1] = 0, w.head[2] = starts[0] != 0 ? 1 : 0;
    count_part(part, w.head + 8, is_free);
    meet();
    for (int s = tid; s < n_rows; s += ALL) {
        const Row r = row_of(v, starts, log_page, s, T);
        if (!r.ok) w.head[2] = 1;
        if (r.last >= 0 && v.used[r.last] > 1) {
            atomicAdd(w.writers + r.last, 1);
            atomicMax(w.latest + r.last, s + 1);
        }
    }
    meet();
    // How many pages each row takes and where its first lies in the list of free ones: every CTA goes over all rows
    // for the sum, the first one notes it.  A shared last page is copied unless the row is the last of its holders.
    bool refused = peek(w.head + 2) != 0;
    const int2 free_pages = counted(w.head + 8);
    int64_t wanted = 0;   // (1024 rows of up to 2^24 pages pass 32 bits)
    for (int base = 0; base < n_rows && !refused; base += THREADS) {
        const int s = base + threadIdx.x;
        int64_t n = 0;
        bool copy = false;
        if (s < n_rows) {
            const Row r = row_of(v, starts, log_page, s, T);
            if (r.last >= 0) {
                const int held = v.used[r.last];
                copy = held > 1 && !(peek(w.latest + r.last) == s + 1 && peek(w.writers + r.last) >= held);
            }
            n = r.after - r.first + (copy ? 1 : 0);
        }
        int64_t total;
        const int64_t r = block_scan(n, &total);
        if (s < n_rows && rank() == 0) w.need[s] = (int)(wanted + r), w.winner[s] = copy ? 1 : 0;   // (below 2^30 unless refused)
        refused = total > free_pages.y - wanted;
        wanted += total;
    }
    if (!refused) list_part(part, free_pages.x, (int)wanted, is_free, [&](int r, int p) { w.list[r] = p; });
    meet();
    if (refused) {   // (every CTA has counted the same)
        if (tid == 0) atomicOr(w.head, (int)ST_NO_PAGES);
        for (int64_t t = tid; t < T; t += ALL) positions[t] = -1;
        return;
    }
    // Nothing below reads what another row changes: the choices are made.
    for (int s = warp; s < n_rows; s += ALL / 32) {
        const Row r = row_of(v, starts, log_page, s, T);
        __syncwarp();
        if (r.add == 0) continue;
        int at = peek(w.need + s);
        int *row = v.tables + s * v.max_pages;
        if (peek(w.winner + s)) {
            if (lane == 0) {
                const int p = peek(w.list + at), k = atomicAdd(w.head + 1, 1);
                w.src[k] = r.last, w.dst[k] = p;
                row[r.len >> log_page] = p;
                v.used[p] = 1;
                atomicSub(v.used + r.last, 1);
            }
            ++at;
        }
        for (int j = r.first + lane; j < r.after; j += 32) {
            const int p = peek(w.list + at + (j - r.first)), before = row[j];
            if (in_pool(before, (int)v.n_pages)) atomicSub(v.used + before, 1);   // (left by a sequence put back to fewer tokens)
            row[j] = p;
            v.used[p] = 1;
        }
        const int64_t b = starts[s];
        for (int64_t i = lane; i < r.add; i += 32) positions[b + i] = r.len + i;
        if (lane == 0) v.lengths[s] = (int)(r.len + r.add);
    }
    for (int64_t t = starts[n_rows] + tid; t < T; t += ALL) positions[t] = -1;
}

// ------------------------------------------------------------------ fork ---
__global__ void __cluster_dims__(CTAS, 1, 1) __launch_bounds__(THREADS)
fork_kernel(KvPagesView v, int n, const int *src, const int *dst, PageWs w) {
    const int tid = rank() * THREADS + threadIdx.x, warp = tid >> 5, lane = tid & 31, n_rows = (int)v.n_rows;
    const int M = (int)v.max_pages;
    const auto valid = [&](int i) { return src[i] >= 0 && src[i] < n_rows && dst[i] >= 0 && dst[i] < n_rows; };
    for (int i = tid; i < n; i += ALL)
        if (valid(i)) w.winner[dst[i]] = 0;
    meet();
    for (int i = tid; i < n; i += ALL)
        if (valid(i)) atomicMax(w.winner + dst[i], i + 1);
    meet();
    // the sources' rows as they are, put aside by destination; the pages' counts meanwhile
    const auto counts = [&](int i) { return valid(i) && peek(w.winner + dst[i]) == i + 1; };
    for (int i = warp; i < n; i += ALL / 32) {
        if (!counts(i)) continue;
        const int *from = v.tables + (int64_t)src[i] * M, *old = v.tables + (int64_t)dst[i] * M;
        int *stage = w.stage + (int64_t)dst[i] * (M + 1);
        for (int j = lane; j < M; j += 32) {
            const int a = from[j], b = old[j];
            stage[j] = a;
            if (a == b) continue;
            if (in_pool(a, (int)v.n_pages)) atomicAdd(v.used + a, 1);
            if (in_pool(b, (int)v.n_pages)) atomicSub(v.used + b, 1);
        }
        if (lane == 0) stage[M] = v.lengths[src[i]];
    }
    meet();
    for (int i = warp; i < n; i += ALL / 32) {
        if (!counts(i) || src[i] == dst[i]) continue;
        int *to = v.tables + (int64_t)dst[i] * M;
        const int *stage = w.stage + (int64_t)dst[i] * (M + 1);
        for (int j = lane; j < M; j += 32) to[j] = peek(stage + j);
        if (lane == 0) v.lengths[dst[i]] = peek(stage + M);
    }
}

// --------------------------------------------------------------- release ---
// (an entry is exchanged for -1, so a row listed twice gives its pages up once)
__global__ void __launch_bounds__(256) release_kernel(KvPagesView v, const int *rows) {
    const int s = rows[blockIdx.x];
    if (s < 0 || s >= v.n_rows) return;
    int *row = v.tables + (int64_t)s * v.max_pages;
    for (int64_t j = threadIdx.x; j < v.max_pages; j += 256) {
        const int p = atomicExch(row + j, -1);
        if (in_pool(p, (int)v.n_pages)) atomicSub(v.used + p, 1);
    }
    if (threadIdx.x == 0) v.lengths[s] = 0;
}

// --------------------------------------------------------------- compact ---
__global__ void __cluster_dims__(CTAS, 1, 1) __launch_bounds__(THREADS)
compact_kernel(const int *used, int n_pages, int *used_out, int *moved_to, PageWs w) {
    dependents_may_start();
    const int tid = rank() * THREADS + threadIdx.x;
    const Part part(n_pages);
    count_part(part, w.head + 8, [&](int p) { return used[p] > 0; });
    meet();
    const int live = counted(w.head + 8).y;
    const auto hole = [&](int p) { return p < live && used[p] <= 0; };
    const auto moves = [&](int p) { return p >= live && used[p] > 0; };
    count_part(part, w.head + 16, hole);
    count_part(part, w.head + 24, moves);
    meet();
    const int2 holes = counted(w.head + 16), moved = counted(w.head + 24);   // (as many of both)
    list_part(part, holes.x, n_pages, hole, [&](int r, int p) { w.dst[r] = p; });
    list_part(part, moved.x, n_pages, moves, [&](int r, int p) { w.src[r] = p; });
    for (int p = part.lo + threadIdx.x; p < part.hi; p += THREADS) moved_to[p] = used[p] > 0 ? p : -1;
    if (tid == 0) w.head[1] = moved.y;
    meet();
    // used_out may be used: a page that stays and a free one behind are their own, a moved one and its hole go together
    for (int p = part.lo + threadIdx.x; p < part.hi; p += THREADS) {
        const int u = used[p];
        if (p < live ? u > 0 : u <= 0) used_out[p] = p < live ? u : 0;
    }
    meet();
    for (int k = tid; k < moved.y; k += ALL) {
        const int from = peek(w.src + k), to = peek(w.dst + k);
        const int u = used[from];
        moved_to[from] = to;
        used_out[to] = u;
        used_out[from] = 0;
    }
}

// ---------------------------------------------------------------- copies ---
struct CopyArgs {
    KvView c;
    int64_t n_layers;
    const int *src, *dst, *count;   // count NULL: n
    int64_t n;
    const int *tables, *moved_to;   // table entries to follow the pages, or NULL
    int *tables_out;
    int64_t entries;
};
constexpr int COPY_THREADS = 256, COPY_DEEP = 4, CHUNK = 16 * COPY_THREADS * COPY_DEEP;

__global__ void __launch_bounds__(COPY_THREADS) copy_kernel(CopyArgs a) {
    wait_for_previous();
    const int64_t n = a.count ? min((int64_t)*a.count, a.n) : a.n;
    const int64_t bytes = (int64_t)a.c.n_kv * a.c.head_dim << a.c.log_page;           // of a page's codes, a multiple of 256
    const int64_t scales = (int64_t)a.c.n_kv << (a.c.log_page - a.c.log_block);
    const int64_t chunks = (bytes + CHUNK - 1) / CHUNK, per = 2 * chunks;
    for (int64_t i = blockIdx.x; i < n * a.n_layers * per; i += gridDim.x) {
        const int64_t c = i % per, l = i / per % a.n_layers, k = i / (per * a.n_layers);
        const int from = a.src[k], to = a.dst[k];
        if (!in_pool(from, a.c.n_pages) || !in_pool(to, a.c.n_pages) || from == to) continue;
        const bool v = c >= chunks;
        const int64_t off = (c % chunks) * CHUNK, layer = l * a.c.n_pages;
        const uint8_t *s = (v ? a.c.v_codes : a.c.k_codes) + (layer + from) * bytes + off;
        uint8_t *d = (v ? a.c.v_codes : a.c.k_codes) + (layer + to) * bytes + off;
        uint4 r[COPY_DEEP];
#pragma unroll
        for (int m = 0; m < COPY_DEEP; ++m) {
            const int64_t o = 16 * (threadIdx.x + COPY_THREADS * m);
            if (off + o < bytes) r[m] = __ldcs(reinterpret_cast<const uint4 *>(s + o));
        }
#pragma unroll
        for (int m = 0; m < COPY_DEEP; ++m) {
            const int64_t o = 16 * (threadIdx.x + COPY_THREADS * m);
            if (off + o < bytes) __stcs(reinterpret_cast<uint4 *>(d + o), r[m]);
        }
        if (c % chunks == 0) {
            const float *fs = (v ? a.c.v_scale : a.c.k_scale) + (layer + from) * scales;
            float *fd = (v ? a.c.v_scale : a.c.k_scale) + (layer + to) * scales;
            for (int64_t j = threadIdx.x; j < scales; j += COPY_THREADS) fd[j] = fs[j];
        }
    }
    if (a.tables == nullptr) return;
    for (int64_t i = (int64_t)blockIdx.x * COPY_THREADS + threadIdx.x; i < a.entries; i += (int64_t)gridDim.x * COPY_THREADS) {
        const int p = a.tables[i];
        a.tables_out[i] = in_pool(p, a.c.n_pages) ? a.moved_to[p] : p;
    }
}

realq_status_t copies(cudaStream_t s, const CopyArgs &a, int sms) {
    const int64_t bytes = (int64_t)a.c.n_kv * a.c.head_dim << a.c.log_page;
    const int64_t items = std::max<int64_t>(a.n * a.n_layers * 2 * ((bytes + CHUNK - 1) / CHUNK), a.entries / COPY_THREADS + 1);
    const unsigned grid = (unsigned)std::min<int64_t>(items, 8ll * sms);
    Launch l("pages_copy", s);
    REALQ_CUDA_TRY(launch_overlapped(copy_kernel, dim3(grid), dim3(COPY_THREADS), 0, s, a));
    return check_launch("pages_copy");
}

}  // namespace

size_t pages_ws_bytes(int64_t n_pages, int64_t n_rows, int64_t max_pages) {
    return carve(nullptr, n_pages, n_rows, max_pages, nullptr);
}

realq_status_t pages_reserve(cudaStream_t s, const KvPagesView &v, const int *starts, int64_t T, int64_t *positions,
                             const KvView &c, int64_t n_layers, void *ws, int sms) {
    PageWs w;
    carve(ws, v.n_pages, v.n_rows, v.max_pages, &w);
    {
        Launch l("pages_reserve", s);
        reserve_kernel<<<CTAS, THREADS, 0, s>>>(v, starts, T, positions, c.log_page, w);
        REALQ_TRY(check_launch("pages_reserve"));
    }
    return copies(s, CopyArgs{c, n_layers, w.src, w.dst, w.head + 1, v.n_rows, nullptr, nullptr, nullptr, 0}, sms);
}

realq_status_t pages_fork(cudaStream_t s, const KvPagesView &v, int64_t n, const int *src, const int *dst, void *ws) {
    PageWs w;
    carve(ws, v.n_pages, v.n_rows, v.max_pages, &w);
    Launch l("pages_fork", s);
    fork_kernel<<<CTAS, THREADS, 0, s>>>(v, (int)n, src, dst, w);
    return check_launch("pages_fork");
}

realq_status_t pages_release(cudaStream_t s, const KvPagesView &v, int64_t n, const int *rows) {
    Launch l("pages_release", s);
    release_kernel<<<(unsigned)n, 256, 0, s>>>(v, rows);
    return check_launch("pages_release");
}

realq_status_t pages_compact(cudaStream_t s, const KvPagesView &v, const KvView &c, int64_t n_layers, int *used_out,
                             int *tables_out, int *moved_to, void *ws, int sms) {
    PageWs w;
    carve(ws, v.n_pages, v.n_rows, v.max_pages, &w);
    {
        Launch l("pages_compact", s);
        compact_kernel<<<CTAS, THREADS, 0, s>>>(v.used, (int)v.n_pages, used_out, moved_to, w);
        REALQ_TRY(check_launch("pages_compact"));
    }
    return copies(s, CopyArgs{c, n_layers, w.src, w.dst, w.head + 1, v.n_pages, v.tables, moved_to, tables_out,
                              v.n_rows * v.max_pages}, sms);
}

realq_status_t pages_copy(cudaStream_t s, const KvView &c, int64_t n_layers, int64_t n, const int *src, const int *dst,
                          int sms) {
    return copies(s, CopyArgs{c, n_layers, src, dst, nullptr, n, nullptr, nullptr, nullptr, 0}, sms);
}

}  // namespace realq
