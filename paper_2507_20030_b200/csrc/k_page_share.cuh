// Pages that several requests name: requests that begin as copies of others (fork), pages given back by finished requests
// (release), and the pages in use moved to the front of the pool (compact).
//
// The block tables are the only record of who holds a page; there are no counters to keep in step with them.  A page is in use
// exactly while a row of the table names it, which takes one pass over the tables to find out, and every result has one order:
// forks in the order of the call, pages given back in the order of the rows, moved pages in ascending order.
#pragma once
#include "common.cuh"
#include "k_pages.cuh"

namespace faedkv {
namespace pages {

constexpr unsigned int kBadRow = 0x106;                   // a row of the block table that there is not, or that may not be written
constexpr int kCluster = 16;                              // CTAs that meet in one launch: the most there are,
constexpr int kClusterAnywhere = 8;                       // and what every GPU or part of one has room for

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// All threads of the cluster; what was written to global memory before is seen after.
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int height_of(const int32_t *n_free, int n_pages, unsigned int *status, bool report) {
    const int h = *n_free;
    if (h >= 0 && h <= n_pages) return h;
    if (report) flag(status, kBadFreeList);
    return h < 0 ? 0 : n_pages;
}
__device__ __forceinline__ int length_of(const int32_t *len, int b, long long cap, unsigned int *status) {
    const int t = len[b];
    if (t >= 0 && t <= cap) return t;
    flag(status, kBadLength);
    return t < 0 ? 0 : (int)cap;
}

// ---- fork ---------------------------------------------------------------------------------------------

struct ForkArgs {
    const int32_t *src, *dst, *len, *free_pages, *n_free; // len may be NULL
    int32_t *kv_len, *table, *n_free_out, *ws;            // ws[i]: fork i's fresh page, -1 none needed, -2 nothing is done; ws[n + b]: marks of row b
    uint8_t *codes[2];
    float *scale[2];
    int n, B, W, H, n_pages, page_shift;
    unsigned int *status;
};

// Tokens that fork i takes from row s: the row's length, cut to what the table holds and to len[i].  (Whether a fork is refused is its callers' to say.)
__device__ __forceinline__ int fork_length(const ForkArgs &a, int i, int s, bool report) {
    const long long cap = (long long)a.W << a.page_shift;
    const int t = a.kv_len[s];
    int n = t < 0 ? 0 : (int)min((long long)t, cap);
    if (report && (t < 0 || t > cap)) flag(a.status, kBadLength);
    if (a.len != nullptr) {
        const int most = a.len[i];
        if (report && most < 0) flag(a.status, kBadLength);
        n = min(n, max(most, 0));
    }
    return n;
}
__device__ __forceinline__ bool fork_rows(const ForkArgs &a, int i, int &s, int &d) {
    s = a.src[i];
    d = a.dst[i];
    return s >= 0 && s < a.B && d >= 0 && d < a.B;
}

// What is done for one fork, by `threads` of them in turn: the first entries of the table row, and the open page's rows (K and V of all heads).
__device__ __forceinline__ void fork_copy(const ForkArgs &a, int s, int d, int n, int fresh, int tid, int threads) {
    const int whole = n >> a.page_shift, rest = n & ((1 << a.page_shift) - 1);
    const int32_t *from = a.table + (size_t)s * a.W;
    int32_t *to = a.table + (size_t)d * a.W;
    const int open = rest == 0 ? 0 : from[whole];
    for (int p = tid; p < whole; p += threads) to[p] = from[p];
    if (rest == 0 || !FAEDKV_IN_BOUNDS(kTagPageShare, whole < a.W && fresh >= 0 && fresh < a.n_pages)) return;
    if (tid == 0) to[whole] = fresh;
    if (open < 0 || open >= a.n_pages) {
        if (tid == 0) flag(a.status, kBadPage);
        return;
    }
    const size_t unit = (size_t)8 << a.page_shift;        // 16-byte pieces of a page of one head
    const int each = rest * 8, all = 2 * a.H * each;       // < 2^23
    const uint32_t inv = 0xffffffffu / (uint32_t)each + 1; // (u * inv >> 32 = u / each: u * each is less than 2^32 ...)
    auto place = [&](int u, size_t &piece) {               // which tensor, and where in the page
        int th = (int)__umulhi((uint32_t)u, inv);
        if (th * each > u) --th;                           // (... but for the last rows of thousands of heads)
        piece = (size_t)(th >> 1) * unit + (u - th * each);
        return th & 1;
    };
    const size_t x0 = (size_t)open * a.H * unit, y0 = (size_t)fresh * a.H * unit;
    for (int u0 = tid; u0 < all; u0 += 8 * threads) {
        uint4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            size_t piece;
            if (u0 + k * threads < all) v[k] = reinterpret_cast<const uint4 *>(place(u0 + k * threads, piece) ? a.codes[1] : a.codes[0])[x0 + piece];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            size_t piece;
            if (u0 + k * threads < all) reinterpret_cast<uint4 *>(place(u0 + k * threads, piece) ? a.codes[1] : a.codes[0])[y0 + piece] = v[k];
        }
    }
    for (int th = tid; th < 2 * a.H; th += threads) {
        float *scale = th & 1 ? a.scale[1] : a.scale[0];
        scale[(size_t)fresh * a.H + (th >> 1)] = scale[(size_t)open * a.H + (th >> 1)];
    }
}

// Few forks among few rows: every CTA finds out for itself which forks before its own take a page; one launch, and no workspace (8 forks: 15.7 us a call
// with a plan in one CTA before the copies, 10.7 so; 16 rows into 256: 10 and 9 us on the device, of which the bytes are 2).  Grid (forks, parts of a fork's copy).  COPY = false, one CTA: the height of the stack alone, where it is written over the one that all have to read.
constexpr int kForkSmall = 1024, kForkRows = 4096;
template <bool COPY>
static __global__ void __launch_bounds__(256) k_page_fork(const ForkArgs a, const bool height_too) {
    __shared__ int32_t mark[kForkRows];                    // of a row: the first fork into it, -1 if one takes from it
    __shared__ int counts[8];
    if (!COPY) pdl_wait();
    const int tid = threadIdx.x, me = COPY ? (int)blockIdx.x : a.n, page = 1 << a.page_shift;
    const bool report = COPY && blockIdx.x == 0 && blockIdx.y == 0;
    const int height = height_of(a.n_free, a.n_pages, a.status, tid == 0 && report);
    int src[kForkSmall / 256], dst[kForkSmall / 256];
    bool valid[kForkSmall / 256];
    for (int b = tid; b < a.B; b += 256) mark[b] = 0x7fffffff;
#pragma unroll
    for (int k = 0; k < kForkSmall / 256; ++k) {
        const int i = tid + 256 * k;
        valid[k] = i < a.n && fork_rows(a, i, src[k], dst[k]);
        if (report && i < a.n && !valid[k] && src[k] >= 0) flag(a.status, kBadRow);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kForkSmall / 256; ++k)
        if (valid[k]) {
            atomicMin(mark + dst[k], tid + 256 * k);
            atomicMin(mark + src[k], -1);
        }
    __syncthreads();
    // pages that the forks before this CTA's take, and all
    int before = 0, all = 0;
#pragma unroll
    for (int k = 0; k < kForkSmall / 256; ++k) {
        const int i = tid + 256 * k;
        if (!valid[k]) continue;
        if (mark[dst[k]] != i) {
            if (report) flag(a.status, kBadRow);
            continue;
        }
        const bool need = (fork_length(a, i, src[k], report) & (page - 1)) != 0;
        before += need && i < me;
        all += need;
    }
    const int both = __reduce_add_sync(0xffffffffu, before << 16 | all);
    if ((tid & 31) == 0) counts[tid >> 5] = both;
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) sum += counts[w];
    if (height_too && tid == 0 && (!COPY || report)) *a.n_free_out = height - min(sum & 0xffff, height);
    if (!COPY) return;
    int s, d;
    if (!fork_rows(a, me, s, d) || mark[d] != me) return;
    const int n = fork_length(a, me, s, false), nth = (sum >> 16) + 1;
    const bool need = (n & (page - 1)) != 0;
    int fresh = -1;
    bool ok = !need || nth <= height;
    if (ok && need) {
        fresh = a.free_pages[height - nth];
        if (fresh < 0 || fresh >= a.n_pages) {
            if (tid == 0) flag(a.status, kBadPage);
            ok = false;
        }
    }
    if (blockIdx.y == 0 && tid == 0) a.kv_len[d] = ok ? n : 0;
    if (ok) fork_copy(a, s, d, n, fresh, blockIdx.y * 256 + tid, gridDim.y * 256);
}

// Many: one CTA finds which forks are done, their fresh pages, lengths.  A row that is both taken from and written, and all but the first
// fork into a row, are refused: a mark for each row finds them (the smallest fork that writes it, -1 if one takes from it).
static __global__ void __launch_bounds__(kPlanThreads) k_page_fork_plan(const ForkArgs a) {
    __shared__ long long warp_sums[32];
    const int tid = threadIdx.x, page = 1 << a.page_shift;
    const int height = height_of(a.n_free, a.n_pages, a.status, tid == 0);
    int32_t *mark = a.ws + a.n;
    int s, d;
    for (int i = tid; i < a.n; i += kPlanThreads)
        if (fork_rows(a, i, s, d)) mark[s] = mark[d] = 0x7fffffff;
        else if (s >= 0) flag(a.status, kBadRow);
    __syncthreads();
    for (int i = tid; i < a.n; i += kPlanThreads)
        if (fork_rows(a, i, s, d)) {
            atomicMin(mark + d, i);
            atomicMin(mark + s, -1);
        }
    __syncthreads();
    long long before = 0;
    for (int i0 = 0; i0 < a.n; i0 += kPlanThreads) {
        const int i = i0 + tid;
        bool valid = i < a.n && fork_rows(a, i, s, d);
        if (valid && __ldcg(mark + d) != i) {
            flag(a.status, kBadRow);
            valid = false;
        }
        const int n = valid ? fork_length(a, i, s, true) : 0;
        const bool need = (n & (page - 1)) != 0;
        long long total;
        const long long upto = before + block_scan(need ? 1 : 0, warp_sums, &total);
        before += total;
        int fresh = -1;
        bool ok = valid && (!need || upto <= height);
        if (ok && need) {
            fresh = a.free_pages[height - upto];
            if (fresh < 0 || fresh >= a.n_pages) {
                flag(a.status, kBadPage);
                ok = false;
            }
        }
        if (i < a.n) a.ws[i] = ok ? fresh : -2;
        if (valid) a.kv_len[d] = ok ? n : 0;
    }
    if (tid == 0) *a.n_free_out = height - (int)min(before, (long long)height);
}
static __global__ void __launch_bounds__(256) k_page_fork_copy(const ForkArgs a) {
    pdl_wait();
    const int i = blockIdx.x, fresh = a.ws[i];
    if (fresh != -2) fork_copy(a, a.src[i], a.dst[i], a.kv_len[a.dst[i]], fresh, threadIdx.x, 256);
}

// ---- release ------------------------------------------------------------------------------------------

struct ReleaseArgs {
    const int32_t *t_len, *n_new, *table, *n_free;
    int32_t *free_pages, *kv_len, *n_free_out, *ws;       // ws[p]: the first place of the table that names page p, -1 if a running request does
    int B, W, n_pages, page_shift;
    unsigned int *status;
};

// One cluster, the grid.  A row is cut into `parts` runs of pages, one a warp's: one where there are rows enough for the warps.
//
// Short: every warp has K runs of up to 256 pages at most and keeps them in registers from the first load to the last store, and the pages that running
// requests name are bits in shared memory, each CTA's own first, then all of them.  What bounds it is the chain: lengths, entries, three meetings of the
// cluster, the stack.  (512 requests of up to 256 pages: 34 us with each row read in every phase and eight CTAs; 25 with the entries in registers and the
// running requests' pages as atomics to global memory, 22 as bits, 18 with sixteen CTAs.  32 rows: 8.6 us with sixteen CTAs, 6.5
// with one.)
constexpr int kReleaseShort = 65536;                      // pages
__device__ __forceinline__ uint32_t load_of_cta(const uint32_t *p, int cta) {        // what p is in another CTA of the cluster
    uint32_t at, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(cta));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
template <int K>
static __global__ void __launch_bounds__(kPlanThreads) k_page_release_short(const ReleaseArgs a, const int parts) {
    __shared__ int32_t count[32 * K + 1];
    __shared__ uint32_t own[kReleaseShort / 32], live[kReleaseShort / 32];
    const int words = (a.n_pages + 31) / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = (int)cluster_rank(), ctas = K > 1 ? kCluster : (int)gridDim.x;
    const long long cap = (long long)a.W << a.page_shift;
    const int page = 1 << a.page_shift;
    const int height = height_of(a.n_free, a.n_pages, a.status, tid == 0 && rank == 0);
    int32_t *totals = a.ws + a.n_pages;
    for (int w = tid; w < words; w += kPlanThreads) own[w] = 0u;
    int id[K][8], e[K], row[K];
    bool gone[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int item = (rank * 32 + warp) * K + k;
        row[k] = item / parts < a.B ? item / parts : -1;
        const int b = max(row[k], 0), part = item - item / parts * parts;
        gone[k] = row[k] >= 0 && a.n_new[b] < 0;
        const int held = row[k] < 0 ? 0 : (int)(((long long)length_of(a.t_len, b, cap, a.status) + page - 1) >> a.page_shift);
        const int run = (held + parts - 1) / parts, end = min(held, (part + 1) * run);
        e[k] = b * a.W + part * run + lane;
#pragma unroll
        for (int j = 0; j < 8; ++j) id[k][j] = part * run + 32 * j + lane < end ? max(a.table[e[k] + 32 * j], -1) : -2;   // -2: no entry
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (id[k][j] == -1 || id[k][j] >= a.n_pages) {
                flag(a.status, kBadPage);
                id[k][j] = -2;
            }
            if (id[k][j] < 0) continue;
            if (gone[k]) a.ws[id[k][j]] = 0x7fffffff;
            else atomicOr(own + (id[k][j] >> 5), 1u << (id[k][j] & 31));
        }
    cluster_sync();
    for (int w = tid; w < words; w += kPlanThreads) {
        uint32_t m = 0;
#pragma unroll(K > 1 ? kCluster : 4)
        for (int r = 0; r < ctas; ++r) m |= load_of_cta(own + w, r);
        live[w] = m;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (row[k] >= 0 && lane == 0) a.kv_len[row[k]] = gone[k] ? 0 : a.t_len[row[k]];   // (kv_len may be t_len: the same warps have read it)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (gone[k] && id[k][j] >= 0) atomicMin(a.ws + id[k][j], e[k] + 32 * j);
    }
    cluster_sync();                                        // (and no CTA ends while another reads its bits)
    uint32_t mine[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        int first[8];
        mine[k] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) first[j] = gone[k] && id[k][j] >= 0 && !((live[id[k][j] >> 5] >> (id[k][j] & 31)) & 1u) ? __ldcg(a.ws + id[k][j]) : -1;
#pragma unroll
        for (int j = 0; j < 8; ++j) mine[k] |= (uint32_t)(first[j] == e[k] + 32 * j) << j;
        const int n = __reduce_add_sync(0xffffffffu, __popc(mine[k]));
        if (lane == 0) count[warp * K + k] = n;
    }
    __syncthreads();
    if (warp == 0) {                                       // exclusive sums, the CTA's behind the last
        int n[K], sum = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) { n[k] = count[lane * K + k]; sum += n[k]; }
        int upto = sum;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, upto, s);
            if (lane >= s) upto += o;
        }
        int at = upto - sum;
#pragma unroll
        for (int k = 0; k < K; ++k) { count[lane * K + k] = at; at += n[k]; }
        if (lane == 31) { count[32 * K] = upto; totals[rank] = upto; }
    }
    cluster_sync();
    long long at0 = height, all = height;
#pragma unroll(K > 1 ? kCluster : 1)
    for (int r = 0; r < ctas; ++r) {
        const int n = __ldcg(totals + r);
        if (r < rank) at0 += n;
        all += n;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        long long at = at0 + count[warp * K + k];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool push = (mine[k] >> j) & 1u;
            const uint32_t m = __ballot_sync(0xffffffffu, push);
            const long long to = at + __popc(m & ((1u << lane) - 1u));
            if (push) {
                if (to < a.n_pages) a.free_pages[to] = id[k][j];
                else flag(a.status, kBadFreeList);
            }
            at += __popc(m);
        }
    }
    if (tid == 0 && rank == 0) *a.n_free_out = (int)min(all, (long long)a.n_pages);   // (n_free_out may be n_free: all have read it)
}

// Any number of rows and pages, by a cluster of CTAS: the runs are read again in every phase.
template <int CTAS>
static __global__ void __launch_bounds__(kPlanThreads) k_page_release(const ReleaseArgs a, const int parts) {
    __shared__ long long warp_sums[32];
    __shared__ int32_t count[65536 / CTAS];                // items of a CTA: one warp's part of a row
    constexpr int kWarps = kPlanThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = (int)cluster_rank();
    const long long cap = (long long)a.W << a.page_shift;
    const int page = 1 << a.page_shift;
    const int height = height_of(a.n_free, a.n_pages, a.status, tid == 0 && rank == 0);
    int32_t *totals = a.ws + a.n_pages;
    // items of this CTA: consecutive, so that the pages it pushes are too
    const int n_items = a.B * parts, each = (n_items + CTAS - 1) / CTAS;
    const int item0 = min(n_items, rank * each), item1 = min(n_items, item0 + each);
    // f(entry, page) for the pages of an item
    auto entries = [&](int item, auto f) {
        const int b = item / parts, part = item - b * parts;
        const int held = (int)(((long long)length_of(a.t_len, b, cap, a.status) + page - 1) >> a.page_shift);
        const int run = (held + parts - 1) / parts, end = min(held, (part + 1) * run);
        const int32_t *row = a.table + (size_t)b * a.W;
        for (int p0 = part * run; p0 < end; p0 += 256) {   // eight entries a lane in flight
            int id[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) id[k] = p0 + 32 * k + lane < end ? row[p0 + 32 * k + lane] : -1;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (p0 + 32 * k + lane < end && (id[k] < 0 || id[k] >= a.n_pages)) {
                    flag(a.status, kBadPage);
                    id[k] = -1;
                }
            f(b * a.W + p0 + lane, id);
        }
    };
    // the entries that are the first to name their page, and no running request names it: a bit each
    auto pushed = [&](int e, const int(&id)[8]) {
        int first[8];
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) first[k] = id[k] >= 0 ? __ldcg(a.ws + id[k]) : -1;
#pragma unroll
        for (int k = 0; k < 8; ++k) m |= (uint32_t)(id[k] >= 0 && first[k] == e + 32 * k) << k;
        return m;
    };
    for (int i = item0 + warp; i < item1; i += kWarps)
        if (a.n_new[i / parts] < 0)
            entries(i, [&](int, const int(&id)[8]) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (id[k] >= 0) a.ws[id[k]] = 0x7fffffff;
            });
    cluster_sync();
    for (int i = item0 + warp; i < item1; i += kWarps) {
        const bool gone = a.n_new[i / parts] < 0;
        entries(i, [&](int e, const int(&id)[8]) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (id[k] >= 0) atomicMin(a.ws + id[k], gone ? e + 32 * k : -1);
        });
    }
    cluster_sync();
    for (int i = item0 + warp; i < item1; i += kWarps) {
        int n = 0;
        if (a.n_new[i / parts] < 0)
            entries(i, [&](int e, const int(&id)[8]) { n += __popc(pushed(e, id)); });
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) count[i - item0] = n;
    }
    __syncthreads();
    int base = 0;
    for (int i0 = 0; i0 < item1 - item0; i0 += kPlanThreads) {
        const int i = i0 + tid, n = i < item1 - item0 ? count[i] : 0;
        long long total;
        const int upto = (int)block_scan(n, warp_sums, &total);
        if (i < item1 - item0) count[i] = base + upto - n;
        base += (int)total;
    }
    if (tid == 0) totals[rank] = base;
    cluster_sync();
    long long at0 = height, all = height;
    for (int r = 0; r < CTAS; ++r) {
        const int n = __ldcg(totals + r);
        if (r < rank) at0 += n;
        all += n;
    }
    for (int i = item0 + warp; i < item1; i += kWarps) {
        const int b = i / parts;
        if (a.n_new[b] >= 0) continue;
        long long at = at0 + count[i - item0];
        entries(i, [&](int e, const int(&id)[8]) {
            const uint32_t mine = pushed(e, id);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bool push = (mine >> k) & 1u;
                const uint32_t m = __ballot_sync(0xffffffffu, push);
                const long long to = at + __popc(m & ((1u << lane) - 1u));
                if (push) {
                    if (to < a.n_pages) a.free_pages[to] = id[k];
                    else flag(a.status, kBadFreeList);
                }
                at += __popc(m);
            }
        });
    }
    cluster_sync();                                       // kv_len may be t_len, n_free_out may be n_free
    for (int b = rank * kPlanThreads + tid; b < a.B; b += CTAS * kPlanThreads) a.kv_len[b] = a.n_new[b] < 0 ? 0 : a.t_len[b];
    if (tid == 0 && rank == 0) *a.n_free_out = (int)min(all, (long long)a.n_pages);
}

// ---- compact ------------------------------------------------------------------------------------------

struct CompactArgs {
    const int32_t *kv_len, *table;
    int32_t *table_out, *free_pages, *n_free, *new_id, *ws;   // ws: [kCompactHead] counts, [n_pages / 2] holes, [n_pages / 2] pages that move
    uint8_t *codes[2];
    float *scale[2];
    int B, W, H, n_pages, page_shift;
    unsigned int *status;
};
constexpr int kCompactHead = 64;                          // counts: live pages of each CTA's range, then holes, then pages that move; the last: all of those

// One cluster: which pages are in use, and where each goes.  With n of them, the pages in use from n on go to the pages below n
// that are not, both in ascending order: the fewest moves, and no page is read and written.
template <int CTAS>
static __global__ void __launch_bounds__(kPlanThreads) k_page_compact_plan(const CompactArgs a) {
    __shared__ long long warp_sums[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = (int)cluster_rank();
    const long long cap = (long long)a.W << a.page_shift;
    const int page = 1 << a.page_shift, all = CTAS * kPlanThreads, me = rank * kPlanThreads + tid;
    int32_t *holes = a.ws + kCompactHead, *moves = holes + a.n_pages / 2;
    for (int p = me; p < a.n_pages; p += all) a.new_id[p] = -1;
    cluster_sync();
    const int warps = all / 32, parts = max(1, warps / a.B);
    for (int i = rank * (kPlanThreads / 32) + warp; i < a.B * parts; i += warps) {
        const int b = i / parts, part = i - b * parts;
        const int held = (int)(((long long)length_of(a.kv_len, b, cap, a.status) + page - 1) >> a.page_shift);
        for (int p0 = part * 256 + lane; p0 < held; p0 += parts * 256) {   // eight entries a lane in flight
            int id[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) id[k] = p0 + 32 * k < held ? a.table[(size_t)b * a.W + p0 + 32 * k] : -1;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (p0 + 32 * k >= held) continue;
                if (id[k] < 0 || id[k] >= a.n_pages) flag(a.status, kBadPage);
                else a.new_id[id[k]] = 0;
            }
        }
    }
    cluster_sync();
    // consecutive pages of a CTA, of a thread
    const int each = ((a.n_pages + CTAS - 1) / CTAS + kPlanThreads - 1) / kPlanThreads;
    const long long lo = (long long)me * each;
    const int p0 = (int)min(lo, (long long)a.n_pages), p1 = (int)min(lo + each, (long long)a.n_pages);
    int live = 0;
    for (int p = p0; p < p1; ++p) live += __ldcg(a.new_id + p) == 0;
    long long total;
    block_scan(live, warp_sums, &total);
    if (tid == 0) a.ws[rank] = (int)total;
    cluster_sync();
    int n = 0;
    for (int r = 0; r < CTAS; ++r) n += __ldcg(a.ws + r);
    long long mine = 0;                                   // holes, and pages that move in the upper half
    for (int p = p0; p < p1; ++p) {
        const bool used = __ldcg(a.new_id + p) == 0;
        if (p < n && !used) mine += 1;
        if (p >= n && used) mine += 1LL << 32;
    }
    const long long upto = block_scan(mine, warp_sums, &total);
    if (tid == 0) {
        a.ws[CTAS + rank] = (int)(total & 0xffffffffLL);
        a.ws[2 * CTAS + rank] = (int)(total >> 32);
    }
    cluster_sync();
    long long at = upto - mine;
    int n_moves = 0;
    for (int r = 0; r < CTAS; ++r) {
        const int m = __ldcg(a.ws + 2 * CTAS + r);
        if (r < rank) at += (long long)__ldcg(a.ws + CTAS + r) + ((long long)m << 32);
        n_moves += m;
    }
    for (int p = p0; p < p1; ++p) {
        const bool used = __ldcg(a.new_id + p) == 0;
        if (p < n && used) a.new_id[p] = p;
        if (p < n && !used) {
            holes[(int)(at & 0xffffffffLL)] = p;
            at += 1;
        }
        if (p >= n && used) {
            moves[(int)(at >> 32)] = p;
            at += 1LL << 32;
        }
    }
    for (int i = me; i < a.n_pages - n; i += all) a.free_pages[i] = a.n_pages - 1 - i;
    if (me == 0) {
        *a.n_free = a.n_pages - n;
        a.ws[kCompactHead - 1] = n_moves;
    }
    cluster_sync();
    for (int k = me; k < n_moves; k += all) a.new_id[__ldcg(moves + k)] = __ldcg(holes + k);
}

// The same by one CTA with a bit for each page in shared memory, for pools of up to kCompactShort pages: a page's rank among those in use gives its place
// in either list.
constexpr int kCompactShort = 65536;
static __global__ void __launch_bounds__(kPlanThreads) k_page_compact_short(const CompactArgs a) {
    __shared__ uint32_t used[kCompactShort / 32];
    __shared__ int32_t before[kCompactShort / 32];        // pages in use before a word's
    __shared__ long long warp_sums[32];
    constexpr int kWords = kCompactShort / 32 / kPlanThreads;                // of a thread
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, page = 1 << a.page_shift;
    const long long cap = (long long)a.W << a.page_shift;
    int32_t *holes = a.ws + kCompactHead, *moves = holes + a.n_pages / 2;
#pragma unroll
    for (int i = 0; i < kWords; ++i) used[tid + i * kPlanThreads] = 0u;
    __syncthreads();
    const int parts = max(1, 32 / a.B);                    // warps of a row
    for (int i = warp; i < a.B * parts; i += 32) {
        const int b = i / parts, part = i - b * parts;
        const int held = (int)(((long long)length_of(a.kv_len, b, cap, a.status) + page - 1) >> a.page_shift);
        for (int p0 = part * 256 + lane; p0 < held; p0 += parts * 256) {     // eight entries a lane in flight
            int id[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) id[k] = p0 + 32 * k < held ? a.table[(size_t)b * a.W + p0 + 32 * k] : -1;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (p0 + 32 * k >= held) continue;
                if (id[k] < 0 || id[k] >= a.n_pages) flag(a.status, kBadPage);
                else atomicOr(used + (id[k] >> 5), 1u << (id[k] & 31));
            }
        }
    }
    __syncthreads();
    uint32_t word[kWords];
    int live = 0;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        word[i] = used[tid * kWords + i];
        live += __popc(word[i]);
    }
    long long total;
    int rank = (int)block_scan(live, warp_sums, &total) - live;
    const int n = (int)total;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        before[tid * kWords + i] = rank;
        rank += __popc(word[i]);
    }
    __syncthreads();
    auto rank_of = [&](int p) { return before[p >> 5] + __popc(used[p >> 5] & ((1u << (p & 31)) - 1u)); };
    const int n_low = n < a.n_pages ? rank_of(n) : n;      // in use below n
    for (int p = tid; p < a.n_pages; p += kPlanThreads) {
        const bool in_use = (used[p >> 5] >> (p & 31)) & 1u;
        const int r = rank_of(p);
        if (p < n && !in_use) holes[p - r] = p;
        if (p >= n && in_use) moves[r - n_low] = p;
        if (p < n || !in_use) a.new_id[p] = in_use ? p : -1;
    }
    for (int i = tid; i < a.n_pages - n; i += kPlanThreads) a.free_pages[i] = a.n_pages - 1 - i;
    if (tid == 0) {
        *a.n_free = a.n_pages - n;
        a.ws[kCompactHead - 1] = n - n_low;
    }
    __syncthreads();
    for (int k = tid; k < n - n_low; k += kPlanThreads) a.new_id[__ldcg(moves + k)] = __ldcg(holes + k);
}

// The pages that move, 16 KB of a tensor at a time, and the tables.  Bound by memory: 2048 of 8192 pages (8 heads of 64 tokens, 268 MB read and as many
// written) 97 us with the plan before it, 82 at the rate of a plain copy.
constexpr int kMoveUnits = 1024;                          // of 16 bytes
static __global__ void __launch_bounds__(256) k_page_move(const CompactArgs a) {
    pdl_wait();
    const int tid = threadIdx.x, page = 1 << a.page_shift;
    const long long cap = (long long)a.W << a.page_shift, n_entries = (long long)a.B * a.W;
    for (long long e = (long long)blockIdx.x * 256 + tid; e < n_entries; e += (long long)gridDim.x * 256) {
        const int b = (int)(e / a.W), p = (int)(e - (long long)b * a.W);
        const int t = (int)min(max((long long)a.kv_len[b], 0LL), cap), id = a.table[e];
        const bool named = p < ((t + (long long)page - 1) >> a.page_shift) && id >= 0 && id < a.n_pages;
        a.table_out[e] = named ? a.new_id[id] : id;
    }
    const int32_t *holes = a.ws + kCompactHead, *moves = holes + a.n_pages / 2;
    const int n_moves = a.ws[kCompactHead - 1];
    const long long units = (long long)a.H * page * (kHeadDim / 16);          // of a page of one tensor
    const int chunks = (int)((units + kMoveUnits - 1) / kMoveUnits);
    const long long jobs = (long long)n_moves * 2 * chunks;
    for (long long j = blockIdx.x; j < jobs; j += gridDim.x) {
        const long long k = j / chunks;
        const int chunk = (int)(j - k * chunks), which = (int)(k & 1), m = (int)(k >> 1);
        const int from = moves[m], to = holes[m];
        if (!FAEDKV_IN_BOUNDS(kTagPageShare, from >= 0 && from < a.n_pages && to >= 0 && to < from)) continue;
        const uint4 *x = reinterpret_cast<const uint4 *>(which == 0 ? a.codes[0] : a.codes[1]) + from * units;
        uint4 *y = reinterpret_cast<uint4 *>(which == 0 ? a.codes[0] : a.codes[1]) + to * units;
        uint4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long u = (long long)chunk * kMoveUnits + i * 256 + tid;
            if (u < units) v[i] = __ldcs(x + u);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long u = (long long)chunk * kMoveUnits + i * 256 + tid;
            if (u < units) __stcs(y + u, v[i]);
        }
        float *scale = which == 0 ? a.scale[0] : a.scale[1];
        if (chunk == 0)
            for (int h = tid; h < a.H; h += 256) scale[(size_t)to * a.H + h] = scale[(size_t)from * a.H + h];
    }
}

}  // namespace pages
}  // namespace faedkv
