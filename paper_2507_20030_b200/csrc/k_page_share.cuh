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
constexpr int kCluster = 8;                               // CTAs that meet in one launch: as many as every part can be asked for

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

// One CTA: which forks are done, their fresh pages, lengths.  A row that is both taken from and written, and all but the first
// fork into a row, are refused: a mark for each row finds them (the smallest fork that writes it, -1 if one takes from it).
__global__ void __launch_bounds__(kPlanThreads) k_page_fork_plan(const ForkArgs a) {
    __shared__ long long warp_sums[32];
    const int tid = threadIdx.x, page = 1 << a.page_shift;
    const long long cap = (long long)a.W << a.page_shift;
    const int height = height_of(a.n_free, a.n_pages, a.status, tid == 0);
    int32_t *mark = a.ws + a.n;
    auto rows = [&](int i, int &s, int &d) {
        s = a.src[i];
        d = a.dst[i];
        return s >= 0 && s < a.B && d >= 0 && d < a.B;
    };
    int s, d;
    for (int i = tid; i < a.n; i += kPlanThreads)
        if (rows(i, s, d)) mark[s] = mark[d] = 0x7fffffff;
        else if (s >= 0) flag(a.status, kBadRow);
    __syncthreads();
    for (int i = tid; i < a.n; i += kPlanThreads)
        if (rows(i, s, d)) {
            atomicMin(mark + d, i);
            atomicMin(mark + s, -1);
        }
    __syncthreads();
    int taken = 0;
    long long before = 0;
    for (int i0 = 0; i0 < a.n; i0 += kPlanThreads) {
        const int i = i0 + tid;
        bool valid = i < a.n && rows(i, s, d);
        if (valid && __ldcg(mark + d) != i) {
            flag(a.status, kBadRow);
            valid = false;
        }
        int n = 0;
        if (valid) {
            n = length_of(a.kv_len, s, cap, a.status);
            if (a.len != nullptr) {
                const int most = a.len[i];
                if (most < 0) flag(a.status, kBadLength);
                n = min(n, max(most, 0));
            }
        }
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
    taken = (int)min(before, (long long)height);
    if (tid == 0) *a.n_free_out = height - taken;
}

// Grid (forks, 2 H): one (tensor, head) of the open page, and a share of the table row.
__global__ void __launch_bounds__(256) k_page_fork_copy(const ForkArgs a) {
    pdl_wait();
    const int i = blockIdx.x, tid = threadIdx.x, fresh = a.ws[i];
    if (fresh == -2) return;
    const int s = a.src[i], d = a.dst[i], n = a.kv_len[d], whole = n >> a.page_shift, rest = n & ((1 << a.page_shift) - 1);
    const int32_t *from = a.table + (size_t)s * a.W;
    int32_t *to = a.table + (size_t)d * a.W;
    for (int p = blockIdx.y * 256 + tid; p < whole; p += gridDim.y * 256) to[p] = from[p];
    if (rest == 0 || !FAEDKV_IN_BOUNDS(kTagPageShare, whole < a.W && fresh >= 0 && fresh < a.n_pages)) return;
    if (blockIdx.y == 0 && tid == 0) to[whole] = fresh;
    const int open = from[whole];
    if (open < 0 || open >= a.n_pages) {
        if (tid == 0) flag(a.status, kBadPage);
        return;
    }
    const int which = blockIdx.y & 1, h = blockIdx.y >> 1;
    uint8_t *codes = which == 0 ? a.codes[0] : a.codes[1];
    float *scale = which == 0 ? a.scale[0] : a.scale[1];
    const size_t row = (size_t)kHeadDim << a.page_shift, ph = (size_t)open * a.H + h, ph_new = (size_t)fresh * a.H + h;
    const uint4 *x = reinterpret_cast<const uint4 *>(codes + ph * row);
    uint4 *y = reinterpret_cast<uint4 *>(codes + ph_new * row);
    uint4 v[4];                                           // a page of a head is 128 rows of 8 at most
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (tid + 256 * k < rest * 8) v[k] = x[tid + 256 * k];
    const float sc = scale[ph];
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (tid + 256 * k < rest * 8) y[tid + 256 * k] = v[k];
    if (tid == 0) scale[ph_new] = sc;
}

// ---- release ------------------------------------------------------------------------------------------

struct ReleaseArgs {
    const int32_t *t_len, *n_new, *table, *n_free;
    int32_t *free_pages, *kv_len, *n_free_out, *ws;       // ws[p]: the first place of the table that names page p, -1 if a running request does
    int B, W, n_pages, page_shift;
    unsigned int *status;
};

constexpr int kReleaseItems = 65536 / kCluster;           // items of a CTA: one warp's part of a row

// One cluster.  A row is cut into `parts` runs of pages, one a warp's: one where there are rows enough for the warps.
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kPlanThreads) k_page_release(const ReleaseArgs a, const int parts) {
    __shared__ long long warp_sums[32];
    __shared__ int32_t count[kReleaseItems];
    constexpr int kWarps = kPlanThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = (int)cluster_rank();
    const long long cap = (long long)a.W << a.page_shift;
    const int page = 1 << a.page_shift;
    const int height = height_of(a.n_free, a.n_pages, a.status, tid == 0 && rank == 0);
    int32_t *totals = a.ws + a.n_pages;
    // items of this CTA: consecutive, so that the pages it pushes are too
    const int n_items = a.B * parts, each = (n_items + kCluster - 1) / kCluster;
    const int item0 = min(n_items, rank * each), item1 = min(n_items, item0 + each);
    // f(entry, page) for the pages of an item
    auto entries = [&](int item, auto f) {
        const int b = item / parts, part = item - b * parts;
        const int held = (int)(((long long)length_of(a.t_len, b, cap, a.status) + page - 1) >> a.page_shift);
        const int run = (held + parts - 1) / parts, end = min(held, (part + 1) * run);
        const int32_t *row = a.table + (size_t)b * a.W;
        for (int p0 = part * run; p0 < end; p0 += 32) {
            const int p = p0 + lane;
            int id = p < end ? row[p] : -1;
            if (p < end && (id < 0 || id >= a.n_pages)) {
                flag(a.status, kBadPage);
                id = -1;
            }
            f(b * a.W + p, id);
        }
    };
    for (int i = item0 + warp; i < item1; i += kWarps)
        if (a.n_new[i / parts] < 0)
            entries(i, [&](int, int id) { if (id >= 0) a.ws[id] = 0x7fffffff; });
    cluster_sync();
    for (int i = item0 + warp; i < item1; i += kWarps) {
        const bool gone = a.n_new[i / parts] < 0;
        entries(i, [&](int e, int id) { if (id >= 0) atomicMin(a.ws + id, gone ? e : -1); });
    }
    cluster_sync();
    for (int i = item0 + warp; i < item1; i += kWarps) {
        int n = 0;
        if (a.n_new[i / parts] < 0)
            entries(i, [&](int e, int id) { n += __popc(__ballot_sync(0xffffffffu, id >= 0 && __ldcg(a.ws + id) == e)); });
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
    for (int r = 0; r < kCluster; ++r) {
        const int n = __ldcg(totals + r);
        if (r < rank) at0 += n;
        all += n;
    }
    for (int i = item0 + warp; i < item1; i += kWarps) {
        const int b = i / parts;
        if (a.n_new[b] >= 0) continue;
        long long at = at0 + count[i - item0];
        entries(i, [&](int e, int id) {
            const bool push = id >= 0 && __ldcg(a.ws + id) == e;
            const uint32_t m = __ballot_sync(0xffffffffu, push);
            const long long to = at + __popc(m & ((1u << lane) - 1u));
            if (push) {
                if (to < a.n_pages) a.free_pages[to] = id;
                else flag(a.status, kBadFreeList);
            }
            at += __popc(m);
        });
    }
    cluster_sync();                                       // kv_len may be t_len, n_free_out may be n_free
    for (int b = rank * kPlanThreads + tid; b < a.B; b += kCluster * kPlanThreads) a.kv_len[b] = a.n_new[b] < 0 ? 0 : a.t_len[b];
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
constexpr int kCompactHead = 32;                          // counts: live pages of each CTA's range, then holes, then pages that move; at 31 all of those

// One cluster: which pages are in use, and where each goes.  With n of them, the pages in use from n on go to the pages below n
// that are not, both in ascending order: the fewest moves, and no page is read and written.
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kPlanThreads) k_page_compact_plan(const CompactArgs a) {
    __shared__ long long warp_sums[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = (int)cluster_rank();
    const long long cap = (long long)a.W << a.page_shift;
    const int page = 1 << a.page_shift, all = kCluster * kPlanThreads, me = rank * kPlanThreads + tid;
    int32_t *holes = a.ws + kCompactHead, *moves = holes + a.n_pages / 2;
    for (int p = me; p < a.n_pages; p += all) a.new_id[p] = -1;
    cluster_sync();
    const int warps = all / 32, parts = max(1, warps / a.B);
    for (int i = rank * (kPlanThreads / 32) + warp; i < a.B * parts; i += warps) {
        const int b = i / parts, part = i - b * parts;
        const int held = (int)(((long long)length_of(a.kv_len, b, cap, a.status) + page - 1) >> a.page_shift);
        for (int p = part * 32 + lane; p < held; p += parts * 32) {
            const int id = a.table[(size_t)b * a.W + p];
            if (id < 0 || id >= a.n_pages) flag(a.status, kBadPage);
            else a.new_id[id] = 0;
        }
    }
    cluster_sync();
    // consecutive pages of a CTA, of a thread
    const int each = ((a.n_pages + kCluster - 1) / kCluster + kPlanThreads - 1) / kPlanThreads;
    const long long lo = (long long)me * each;
    const int p0 = (int)min(lo, (long long)a.n_pages), p1 = (int)min(lo + each, (long long)a.n_pages);
    int live = 0;
    for (int p = p0; p < p1; ++p) live += __ldcg(a.new_id + p) == 0;
    long long total;
    block_scan(live, warp_sums, &total);
    if (tid == 0) a.ws[rank] = (int)total;
    cluster_sync();
    int n = 0;
    for (int r = 0; r < kCluster; ++r) n += __ldcg(a.ws + r);
    long long mine = 0;                                   // holes, and pages that move in the upper half
    for (int p = p0; p < p1; ++p) {
        const bool used = __ldcg(a.new_id + p) == 0;
        if (p < n && !used) mine += 1;
        if (p >= n && used) mine += 1LL << 32;
    }
    const long long upto = block_scan(mine, warp_sums, &total);
    if (tid == 0) {
        a.ws[kCluster + rank] = (int)(total & 0xffffffffLL);
        a.ws[2 * kCluster + rank] = (int)(total >> 32);
    }
    cluster_sync();
    long long at = upto - mine;
    int n_moves = 0;
    for (int r = 0; r < kCluster; ++r) {
        const int m = __ldcg(a.ws + 2 * kCluster + r);
        if (r < rank) at += (long long)__ldcg(a.ws + kCluster + r) + ((long long)m << 32);
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

// The pages that move, 16 KB of a tensor at a time, and the tables.
constexpr int kMoveUnits = 1024;                          // of 16 bytes
__global__ void __launch_bounds__(256) k_page_move(const CompactArgs a) {
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
