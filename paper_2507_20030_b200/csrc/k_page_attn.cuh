// Attention over the paged 8-bit cache on the tensor cores.
//
//     out[i, g] = sum_n softmax_n( scale * q[i, g] . K[n] ) V[n],   n < kv_len - n_new + i + 1
//
// for the i-th of a sequence's n_new newest tokens; K and V are code * scale of the pages in the sequence's table row.
//
// The codes go from memory to the tensor cores as they lie in the pages: TMA brings tiles of 128 tokens x 128 channels
// into shared memory, and both products take them as their 128-row A operand,
//     S[token, col]   = sum_d  K[token, d] * q[col, d]        (A = the K tile, K-major)
//     O[d, col]      += sum_n  V[n, d]     * w[n, col]        (A = the V tile, MN-major)
// with the query columns (new tokens x query heads of one kv head) as N.  The other operand has to be e4m3 too, so a
// query element and a softmax weight are written as sums of e4m3 terms of four significant bits each, the i-th scaled by
// 16^i: their products are exact and accumulate in float32, so nothing of the cache is converted anywhere and what is
// lost is only what the last term rounds off (bf16 q: two terms, exact; bf16 weights: three terms, 2^-13 of a weight, or
// two, 2^-9, where many columns share a tile; float32: six terms, 2^-25).
//
// Softmax runs in base 2 with the page scales inside: x = s * (k_scale * scale * log2 e) + log2(v_scale), weights
// w = 2^(x - Mu), sum l += w / v_scale.  Mu follows the column maximum lazily: it is raised (and O, l rescaled) only when
// some x exceeds it by 8, and then to 6 below the maximum, so weights stay in e4m3's range and most tiles exchange one
// vote instead of a maximum per column.  O stays in TMEM over all tiles of a segment.
//
// A CTA: warps 0-3 softmax (thread = token row of S, channel row of O), warp 4 TMA, warp 5 MMA.
#pragma once
#include "common.cuh"
#include "k_pages.cuh"
#include "umma_common.cuh"

namespace faedkv {
namespace pages {

constexpr int kTile = 128;                                // tokens of a tile
constexpr uint32_t kTileBytes = kTile * kHeadDim;         // 16 KB: K or V codes of a tile
constexpr int kAttnThreads = 192;
constexpr float kLagMax = 8.0f, kLagTo = 6.0f;            // weights stay <= 2^8; after a raise the largest is 2^6
constexpr float kMuNone = -3e38f;
constexpr unsigned int kErrAttnTma = 0x41, kErrAttnMma = 0x42, kErrAttnSoftmax = 0x43;

// Instances: QC query columns, QT / PT terms of q / of the weights, the terms side by side as further columns of one
// product (CHAIN = false: few columns, one pass over the tile) or added up in the same accumulator (CHAIN = true).
template <typename T_, int QC_, int QT_, int PT_, bool CHAIN_, int STAGES_, int PBUFS_, int CTAS_> struct AttnCfg {
    using T = T_;
    static constexpr int QC = QC_, QT = QT_, PT = PT_, STAGES = STAGES_, PBUFS = PBUFS_, CTAS = CTAS_;
    static constexpr bool CHAIN = CHAIN_;
    static constexpr int NS = CHAIN ? QC : (QC * QT + 15) / 16 * 16;          // columns of S, of O
    static constexpr int NO = CHAIN ? QC : (QC * PT + 15) / 16 * 16;
    static constexpr int kTmemUsed = 2 * NS + NO;
    static constexpr uint32_t kTmemCols = kTmemUsed <= 32 ? 32 : kTmemUsed <= 64 ? 64 : kTmemUsed <= 128 ? 128 : kTmemUsed <= 256 ? 256 : 512;
    static constexpr uint32_t kQBytes = (CHAIN ? QT * QC : NS) * 128;
    static constexpr uint32_t kOffQ = STAGES * 2 * kTileBytes;
    static constexpr uint32_t kOffP = kOffQ + (kQBytes + 1023) / 1024 * 1024;
    static constexpr uint32_t kOffMisc = kOffP + PBUFS * kTileBytes;
    static constexpr uint32_t kSmemBytes = kOffMisc + sizeof(float) * (4 * QC + 4 * QC + STAGES * 32 + 64) + 1024 + 1024;
};

struct AttnArgs {
    const void *q;
    void *out;
    const int32_t *q_start, *kv_len, *table;              // q_start may be NULL: one token per sequence
    const float *ks, *vs;
    long long ld_q;
    int n_tokens, B, H, G, W, n_pages, page_shift, splits;
    float scale_log2;                                     // scale * log2(e)
    unsigned char *ws;
    unsigned int *status;
};

// Workspace of a decode step (MODE 0): header, one record per (sequence, kv head), two partial results per CTA.
struct UnitMeta { long long first; int tiles, pad; };
__host__ __device__ constexpr size_t attn_slot_floats(int qc) { return (size_t)qc * (kHeadDim + 2); }

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float warp_max(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ bool softmax_any(bool v) {     // over the four softmax warps; a barrier
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\t"
                 "setp.ne.u32 q, %1, 0;\n\t"
                 "barrier.cta.red.or.pred p, 1, 128, q;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(r) : "r"((uint32_t)v) : "memory");
    return r != 0;
}
__device__ __forceinline__ void softmax_bar() { asm volatile("barrier.cta.sync 1, 128;" ::: "memory"); }

__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&r)[16]) {
    uint32_t u[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]),
          "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
        : "r"(taddr) : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = __uint_as_float(u[i]);
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float (&r)[16]) {
    uint32_t u[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) u[i] = __float_as_uint(r[i]);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]),
          "r"(u[8]), "r"(u[9]), "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}

// The leading four significant bits of w as an e4m3 value (0 below e4m3's normal range), and what they leave.
__device__ __forceinline__ float lead4(float w) {
    const float h = __uint_as_float(__float_as_uint(w) & 0xfff00000u);
    return fabsf(w) >= 0.015625f ? h : 0.f;
}

// One unit of work is the columns of one (sequence, kv head, block of new tokens); a segment is a run of its tiles.
struct Segment {
    int b, h, tok0, n_tok;       // first query row (of q, out) and number of query tokens
    int see0;                    // tokens that the first query token sees (its column limit); the i-th sees see0 + i
    int live;                    // tokens that the last one sees, >= 0
    int t0, t1, tiles;           // tiles of the segment, of the unit
    long long slot;              // where a partial result goes
};

__device__ __forceinline__ long long clamp_len(const AttnArgs &a, int b, bool report) {
    long long n = a.kv_len[b];
    const long long cap = (long long)a.W << a.page_shift;
    if (n < 0 || n > cap) {
        if (report) flag(a.status, kBadLength);
        n = n < 0 ? 0 : cap;
    }
    return n;
}
__device__ __forceinline__ int tiles_of(long long live) { return live <= 0 ? 1 : (int)((live + kTile - 1) / kTile); }

// MODE 0, a decode step: the tiles of all (sequence, head) units in a row are cut into equal shares, one per CTA; a share
// begins and ends anywhere inside a unit.  MODE 1, blocks of new tokens: CTA (v, h, s) is split s of one unit.
template <int MODE> struct Work;

template <> struct Work<0> {
    int b, h, t, tiles;
    long long pos, end;
    bool at_start;
    __device__ __forceinline__ bool next(const AttnArgs &a, int, Segment &s) {
        if (pos >= end) return false;
        s.b = b; s.h = h; s.tok0 = b; s.n_tok = 1;
        s.live = (int)clamp_len(a, b, false);
        s.see0 = s.live;
        tiles = tiles_of(s.live);
        s.tiles = tiles; s.t0 = t;
        const long long left = end - pos;
        s.t1 = left < tiles - t ? t + (int)left : tiles;
        s.slot = (long long)blockIdx.x * 2 + (at_start ? 0 : 1);
        at_start = false;
        pos += s.t1 - s.t0;
        t = 0;
        if (++h == a.H) { h = 0; ++b; }
        return true;
    }
};

template <> struct Work<1> {
    bool done;
    __device__ __forceinline__ bool next(const AttnArgs &a, int qc, Segment &s) {
        if (done) return false;
        done = true;
        const int tq = qc / a.G;
        const int v = (int)(gridDim.x - 1 - blockIdx.x);   // the blocks that see most first
        // block v of the call is block v - (q_start[b] / tq + b) of sequence b: sequences begin at distinct numbers
        int lo = 0, hi = a.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.q_start[mid] / tq + mid <= v) lo = mid; else hi = mid - 1;
        }
        const int first = a.q_start[lo];
        int n = a.q_start[lo + 1] - first;
        if (first < 0 || n < 0 || first > a.n_tokens - n) {
            if (threadIdx.x == 0) flag(a.status, kBadStart);
            return false;
        }
        const int j = v - (first / tq + lo);
        if (j < 0 || (long long)j * tq >= n) return false;
        s.b = lo; s.h = blockIdx.y; s.tok0 = first + j * tq;
        s.n_tok = min(tq, n - j * tq);
        const int kv = (int)clamp_len(a, lo, threadIdx.x == 0);
        s.see0 = kv - n + j * tq + 1;
        s.live = max(0, s.see0 + s.n_tok - 1);
        s.tiles = tiles_of(s.live);
        s.t0 = (int)((long long)s.tiles * blockIdx.z / a.splits);
        s.t1 = (int)((long long)s.tiles * (blockIdx.z + 1) / a.splits);
        s.slot = ((long long)v * a.H + s.h) * a.splits + blockIdx.z;
        return true;
    }
};

template <typename C, int MODE>
__global__ void __launch_bounds__(kAttnThreads, C::CTAS)
k_page_attn(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const AttnArgs a) {
    using namespace umma;
    using T = typename C::T;
    constexpr int QC = C::QC, QT = C::QT, PT = C::PT, NS = C::NS, NO = C::NO, STAGES = C::STAGES, PB = C::PBUFS;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *gbase = smem_raw + (base - smem_u32(smem_raw));
    auto k_tile = [&](int s) { return base + (uint32_t)s * 2 * kTileBytes; };
    auto v_tile = [&](int s) { return base + (uint32_t)s * 2 * kTileBytes + kTileBytes; };
    const uint32_t q_base = base + C::kOffQ;
    auto p_tile = [&](int p) { return base + C::kOffP + (uint32_t)p * kTileBytes; };
    float *col_cs = reinterpret_cast<float *>(gbase + C::kOffMisc);          // [QC] factor of a column's raw score
    float *col_mu = col_cs + QC;                                             // [QC] Mu
    float *col_f = col_mu + QC;                                              // [QC] rescale factor / 1 / l
    int *col_lim = reinterpret_cast<int *>(col_f + QC);                      // [QC] tokens that the column sees
    float *red = reinterpret_cast<float *>(col_lim + QC);                    // [4][QC]
    float *stage_ks = red + 4 * QC;                                          // [STAGES][32]: 8 k_scale, 8 log2 v_scale, 8 1 / v_scale, pages mask
    uint64_t *bars = reinterpret_cast<uint64_t *>(stage_ks + STAGES * 32);
    const uint32_t bar0 = smem_u32(bars);
    auto kfull = [&](int s) { return bar0 + 8 * s; };
    auto vfull = [&](int s) { return bar0 + 8 * (STAGES + s); };
    auto empty = [&](int s) { return bar0 + 8 * (2 * STAGES + s); };
    auto sfull = [&](int i) { return bar0 + 8 * (3 * STAGES + i); };
    auto pfull = [&](int i) { return bar0 + 8 * (3 * STAGES + 2 + i); };
    auto pdone = [&](int i) { return bar0 + 8 * (3 * STAGES + 2 + PB + i); };
    const uint32_t qfull = bar0 + 8 * (3 * STAGES + 2 + 2 * PB);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 3 * STAGES + 3 + 2 * PB);
    volatile uint32_t *abort_flag = tmem_slot + 1;
    static_assert(8 * (3 * STAGES + 4 + 2 * PB) <= 256, "barriers fit the room behind the stages");

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int page = 1 << a.page_shift;

    // ---- this CTA's work
    Work<MODE> w0;
    if constexpr (MODE == 0) {
        // prefix sums of the sequences' tiles: 128 runs of consecutive sequences, one per thread
        __shared__ long long run_sum[128];
        __shared__ long long found[4];
        const int run = (a.B + 127) / 128;
        if (tid < 128) {
            long long n = 0;
            for (int b = tid * run; b < min(a.B, (tid + 1) * run); ++b) n += tiles_of(clamp_len(a, b, blockIdx.x == 0));
            const long long own = n;
#pragma unroll
            for (int s = 1; s < 32; s <<= 1) {
                const long long o = __shfl_up_sync(0xffffffffu, n, s);
                if (lane >= s) n += o;
            }
            run_sum[tid] = n - own;                       // within the warp, exclusive
            if (lane == 31) found[warp] = n;
        }
        __syncthreads();
        const long long w_sum[4] = {found[0], found[1], found[2], found[3]};
        const long long total = (w_sum[0] + w_sum[1] + w_sum[2] + w_sum[3]) * a.H;
        const long long share = (total + gridDim.x - 1) / gridDim.x;
        w0.pos = share * blockIdx.x;
        w0.end = min(total, w0.pos + share);
        if (w0.pos >= w0.end) return;                     // the whole CTA
        w0.at_start = true;
        if (tid == 0 && blockIdx.x == 0) *reinterpret_cast<long long *>(a.ws) = share;
        // the run that holds sequence tile pos / H ... then the sequence, one after the other
        int lo = 0, hi = 127;
        auto before = [&](int i) { return run_sum[i] + (i >= 32 ? w_sum[0] : 0) + (i >= 64 ? w_sum[1] : 0) + (i >= 96 ? w_sum[2] : 0); };
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (mid * run < a.B && before(mid) * a.H <= w0.pos) lo = mid; else hi = mid - 1;
        }
        long long at = before(lo) * a.H;
        int b = lo * run, n = tiles_of(clamp_len(a, b, false));
        while (at + (long long)n * a.H <= w0.pos) {
            at += (long long)n * a.H;
            n = tiles_of(clamp_len(a, ++b, false));
        }
        w0.b = b;
        w0.h = (int)((w0.pos - at) / n);
        w0.t = (int)((w0.pos - at) % n);
        w0.tiles = n;
    } else {
        w0.done = false;
        Work<MODE> probe = w0;
        Segment s;
        if (!probe.next(a, QC, s)) return;                // no such block (the whole CTA)
    }

    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(kfull(s), 1); mbar_init(vfull(s), 1); mbar_init(empty(s), 1); }
        for (int i = 0; i < 2; ++i) mbar_init(sfull(i), 1);
        for (int i = 0; i < PB; ++i) { mbar_init(pfull(i), 4); mbar_init(pdone(i), 1); }
        mbar_init(qfull, 4);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 5) tmem_alloc(smem_u32(tmem_slot), C::kTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(tmem_slot);
    const uint32_t tmem_s = tmem, tmem_o = tmem + 2 * NS;

    bool dead = false;                                    // a bounded wait gave up: no further waits, run out
    auto wait = [&](uint32_t bar, uint32_t parity, unsigned int code) {
        if (dead) return;
        if (*abort_flag || !mbar_wait(bar, parity)) {
            if (!*abort_flag) atomicExch(a.status, code);
            *abort_flag = 1;
            dead = true;
        }
    };

    if (warp == 4) {
        // ------------------------------------------------------------------------ producer: pages by TMA, scales
        const int lg_ppt = 7 - a.page_shift, ppt = 1 << lg_ppt;               // pages of a tile
        const int tiles_batch = 32 >> lg_ppt;                                 // a lane looks after one page of the next 32
        Work<MODE> w = w0;
        Segment s;
        int it = 0, issued = 0;
        while (w.next(a, QC, s)) {
            const int32_t *row = a.table + (size_t)s.b * a.W;
            auto fetch = [&](int t_first, int &id, float &ks, float &vs) {
                const long long p = ((long long)t_first << lg_ppt) + lane;
                id = -1; ks = 0.f; vs = 1.f;
                if ((p << a.page_shift) < s.live && t_first + (lane >> lg_ppt) < s.t1) {
                    id = row[p];
                    if (id < 0 || id >= a.n_pages) {
                        flag(a.status, kBadPage);
                        id = -1;
                    } else {
                        const size_t ph = (size_t)id * a.H + s.h;
                        ks = a.ks[ph];
                        vs = fmaxf(a.vs[ph], 1.17549435e-38f);
                    }
                }
            };
            int id, id_next;
            float ks, vs, ks_next, vs_next;
            fetch(s.t0, id, ks, vs);
            for (int tb = s.t0; tb < s.t1; tb += tiles_batch) {
                fetch(tb + tiles_batch, id_next, ks_next, vs_next);
                const int tn = min(tiles_batch, s.t1 - tb);
                for (int i = 0; i < tn; ++i, ++it) {
                    const int st = it % STAGES;
                    wait(empty(st), ((uint32_t)(it / STAGES) & 1u) ^ 1u, kErrAttnTma);
                    const bool mine = (lane >> lg_ppt) == i;
                    const int k = lane & (ppt - 1);
                    const uint32_t have = __ballot_sync(0xffffffffu, mine && id >= 0) >> (i << lg_ppt);
                    const uint32_t bytes = (uint32_t)__popc(have) * (uint32_t)(page * kHeadDim);
                    dead = __any_sync(0xffffffffu, dead);
                    if (dead) continue;
                    if (lane == 0) mbar_expect_tx(kfull(st), bytes);
                    __syncwarp();
                    if (mine && id >= 0) {
                        const int y = (id * a.H + s.h) << a.page_shift;
                        const uint32_t off = (uint32_t)(k << a.page_shift) * kHeadDim;
                        tma_load_2d(k_tile(st) + off, &map_k, kfull(st), 0, y);
                        tma_load_2d(v_tile(st) + off, &map_v, vfull(st), 0, y);
                    }
                    float *sc = stage_ks + st * 32;
                    if (mine) {
                        sc[k] = ks;
                        sc[8 + k] = __log2f(vs);
                        sc[16 + k] = __frcp_rn(vs);
                    }
                    if (lane == 0) reinterpret_cast<uint32_t *>(sc)[24] = have;
                    __syncwarp();
                    if (lane == 0) mbar_expect_tx(vfull(st), bytes);
                    issued = it + 1;
                }
                id = id_next; ks = ks_next; vs = vs_next;
            }
        }
        if (dead)                                          // leave no copy in flight behind
            for (int i = max(0, issued - STAGES); i < issued; ++i) {
                mbar_wait(kfull(i % STAGES), (uint32_t)(i / STAGES) & 1u);
                mbar_wait(vfull(i % STAGES), (uint32_t)(i / STAGES) & 1u);
            }
    } else if (warp == 5) {
        // ------------------------------------------------------------------------ MMA issuer
        if (lane == 0) {
            constexpr uint32_t kIdescS = make_idesc(0u, 0u, 0u, NS), kIdescO = make_idesc(0u, 1u, 1u, NO);
            Work<MODE> w = w0;
            Segment s;
            int it = 0;                                    // tiles whose S has been issued
            uint32_t seg = 0;
            auto scores = [&]() {
                const int st = it % STAGES;
                wait(kfull(st), (uint32_t)(it / STAGES) & 1u, kErrAttnMma);
                if (!dead) {
                    tc_fence_after();
#pragma unroll
                    for (int term = 0; term < (C::CHAIN ? QT : 1); ++term)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            mma_f8(tmem_s + (it & 1) * NS, desc_kmajor_sw128(k_tile(st) + k * 32),
                                   desc_kmajor_sw128(q_base + term * QC * 128 + k * 32), kIdescS, (term | k) ? 1u : 0u);
                    mma_commit(sfull(it & 1));
                }
                ++it;
            };
            auto output = [&](int i, bool first) {
                const int st = i % STAGES, pb = i % PB;
                wait(pfull(pb), (uint32_t)(i / PB) & 1u, kErrAttnMma);
                wait(vfull(st), (uint32_t)(i / STAGES) & 1u, kErrAttnMma);
                if (!dead) {
                    tc_fence_after();
#pragma unroll
                    for (int term = 0; term < (C::CHAIN ? PT : 1); ++term)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            mma_f8(tmem_o, desc_mnmajor_sw128(v_tile(st) + k * 4096, kTileBytes),
                                   desc_mnmajor_sw128(p_tile(pb) + term * QC + k * 4096, kTileBytes), kIdescO,
                                   (!first || term || k) ? 1u : 0u);
                    mma_commit(empty(st));
                    mma_commit(pdone(pb));
                }
            };
            while (w.next(a, QC, s)) {
                wait(qfull, seg & 1u, kErrAttnMma);
                ++seg;
                if (s.t1 > s.t0) scores();
                for (int t = s.t0; t < s.t1; ++t) {
                    const int i = it - 1;
                    if (t + 1 < s.t1) scores();            // the next tile's scores before this one's output
                    output(i, t == s.t0);
                }
            }
        }
    } else {
        // ------------------------------------------------------------------------ softmax
        const uint32_t lane_addr = (uint32_t)(warp * 32) << 16;
        const uint32_t sw = (uint32_t)(tid & 7);
        constexpr float kTerm = 1.0f / 16.0f;
        Work<MODE> w = w0;
        Segment s;
        int it = 0;
        while (w.next(a, QC, s)) {
            const int n_cols = s.n_tok * a.G;
            // -- the query columns as e4m3 terms, each column with a power of two of its own
            for (int c = warp; c < QC; c += 4) {
                float x[4] = {0.f, 0.f, 0.f, 0.f};
                float qs = 1.f;
                if (c < n_cols) {
                    const int tok = s.tok0 + c / a.G, hq = s.h * a.G + c % a.G;
                    const float4 v = load4(static_cast<const T *>(a.q) + (size_t)tok * a.ld_q + (size_t)hq * kHeadDim + lane * 4);
                    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
                    uint32_t m = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) m = max(m, finite_bits(x[e]));
                    qs = 2.0f * scale_for(__uint_as_float(__reduce_max_sync(0xffffffffu, m)));
                    const float inv = __uint_as_float((254u << 23) - __float_as_uint(qs));
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = fabsf(x[e]) < INFINITY ? x[e] * inv : __uint_as_float(0x7fffffffu);
                }
                if (lane == 0) {
                    col_cs[c] = qs * a.scale_log2;
                    col_mu[c] = kMuNone;
                    col_lim[c] = s.see0 + c / a.G;
                }
#pragma unroll
                for (int i = 0; i < QT; ++i) {
                    float t[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (i < QT - 1) {
                            t[e] = lead4(x[e]);
                            x[e] -= t[e];
                            if (!C::CHAIN) x[e] *= 16.0f;
                        } else {
                            t[e] = x[e];
                        }
                    }
                    const uint32_t codes = to_e4m3x2(t[0], t[1]) | to_e4m3x2(t[2], t[3]) << 16;
                    const uint32_t row = (uint32_t)(i * QC + c);
                    *reinterpret_cast<uint32_t *>(gbase + C::kOffQ + row * 128 + ((((uint32_t)lane >> 2) ^ (row & 7)) << 4) + (lane & 3) * 4) = codes;
                }
            }
            if constexpr (!C::CHAIN && NS > QC * QT)
                for (int r = QC * QT + warp; r < NS; r += 4)
                    *reinterpret_cast<uint32_t *>(gbase + C::kOffQ + r * 128 + lane * 4) = 0u;
            fence_proxy_async();
            softmax_bar();                                 // col_* are read by all four warps
            if (lane == 0) mbar_arrive(qfull);

            float l[QC];
#pragma unroll
            for (int c = 0; c < QC; ++c) l[c] = 0.f;
            unsigned long long poison = 0;                 // columns whose channel `tid` met a NaN value

            for (int t = s.t0; t < s.t1; ++t, ++it) {
                const int st = it % STAGES, pb = it % PB;
                wait(vfull(st), (uint32_t)(it / STAGES) & 1u, kErrAttnSoftmax);
                const float *sc = stage_ks + st * 32;
                const int pg = tid >> a.page_shift;
                const float ks = sc[pg], lvs = sc[8 + pg];
                float ivs = sc[16 + pg];
                const uint32_t have = reinterpret_cast<const uint32_t *>(sc)[24];
                const int tok = t * kTile + tid;
                // columns may see a different number of this tile's tokens, or pages may be missing
                const bool masked = (t + 1) * kTile > s.see0 || have != (1u << (kTile >> a.page_shift)) - 1u;
                const bool valid = tok < s.live && ((have >> pg) & 1u);
                wait(sfull(it & 1), (uint32_t)(it >> 1) & 1u, kErrAttnSoftmax);
                tc_fence_after();
                float x[QC];
                {
                    const uint32_t ts = tmem_s + (it & 1) * NS + lane_addr;
                    float raw[NS];
#pragma unroll
                    for (int c0 = 0; c0 < NS; c0 += 16) tmem_ld16(ts + c0, *reinterpret_cast<float(*)[16]>(raw + c0));
                    tmem_ld_wait();
#pragma unroll
                    for (int c = 0; c < QC; ++c) {
                        if (C::CHAIN) {
                            x[c] = raw[c];
                        } else {
                            float v = raw[(QT - 1) * QC + c];
#pragma unroll
                            for (int i = QT - 2; i >= 0; --i) v = fmaf(v, kTerm, raw[i * QC + c]);
                            x[c] = v;
                        }
                    }
                }
                float excess = -INFINITY;
#pragma unroll
                for (int c = 0; c < QC; ++c) {
                    x[c] = fmaf(x[c], ks * col_cs[c], lvs);
                    if (masked) x[c] = valid && tok < col_lim[c] && c < n_cols ? x[c] : -INFINITY;
                    excess = fmaxf(excess, x[c] - col_mu[c]);
                }
                if (masked && !valid) ivs = 0.f;
                if (softmax_any(excess > kLagMax)) {
                    // raise Mu to 6 below the column maxima, rescale what has been summed
                    if (t > s.t0) wait(pdone((it - 1) % PB), (uint32_t)((it - 1) / PB) & 1u, kErrAttnSoftmax);
#pragma unroll
                    for (int c = 0; c < QC; ++c) {
                        const float m = warp_max(x[c]);
                        if (lane == 0) red[warp * QC + c] = m;
                    }
                    softmax_bar();
                    for (int c = tid; c < QC; c += 128) {
                        const float m = fmaxf(fmaxf(red[c], red[QC + c]), fmaxf(red[2 * QC + c], red[3 * QC + c])) - kLagTo;
                        const float old = col_mu[c], mu = m > old ? m : old;
                        col_mu[c] = mu;
                        col_f[c] = ex2(old - mu);
                    }
                    softmax_bar();
#pragma unroll
                    for (int c = 0; c < QC; ++c) l[c] *= col_f[c];
                    if (t > s.t0) {
                        tc_fence_after();
#pragma unroll 1
                        for (int c0 = 0; c0 < NO; c0 += 16) {
                            float o[16];
                            tmem_ld16(tmem_o + lane_addr + c0, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] *= col_f[(c0 + e) % QC];
                            tmem_st16(tmem_o + lane_addr + c0, o);
                        }
                        tmem_st_wait();
                    }
                }
                // weights, their sum, their e4m3 terms
#pragma unroll
                for (int c = 0; c < QC; ++c) {
                    x[c] = ex2(x[c] - col_mu[c]);
                    l[c] = fmaf(x[c], ivs, l[c]);
                }
                // PV(it - PB) has read this weight buffer
                if (it >= PB) wait(pdone(pb), (uint32_t)((it - PB) / PB) & 1u, kErrAttnSoftmax);
                uint8_t *prow = gbase + C::kOffP + pb * kTileBytes + tid * 128;
                if constexpr (C::CHAIN) {
#pragma unroll
                    for (int i = 0; i < PT; ++i)
#pragma unroll
                        for (int c0 = 0; c0 < QC; c0 += 16) {
                            uint32_t u[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                float y[4];
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const int c = c0 + 4 * k + e;
                                    y[e] = i < PT - 1 ? lead4(x[c]) : x[c];
                                    x[c] -= y[e];
                                }
                                u[k] = to_e4m3x2(y[0], y[1]) | to_e4m3x2(y[2], y[3]) << 16;
                            }
                            *reinterpret_cast<uint4 *>(prow + ((((uint32_t)(i * QC + c0) >> 4) ^ sw) << 4)) = make_uint4(u[0], u[1], u[2], u[3]);
                        }
                } else {
                    uint32_t u[NO / 4];
#pragma unroll
                    for (int i = 0; i < NO / 4; ++i) u[i] = 0u;
#pragma unroll
                    for (int i = 0; i < PT; ++i)
#pragma unroll
                        for (int c0 = 0; c0 < QC; c0 += 4) {
                            float y[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int c = c0 + e;
                                y[e] = i < PT - 1 ? lead4(x[c]) : x[c];
                                x[c] = (x[c] - y[e]) * 16.0f;
                            }
                            u[(i * QC + c0) / 4] = to_e4m3x2(y[0], y[1]) | to_e4m3x2(y[2], y[3]) << 16;
                        }
#pragma unroll
                    for (int k = 0; k < NO / 16; ++k)
                        *reinterpret_cast<uint4 *>(prow + (((uint32_t)k ^ sw) << 4)) = make_uint4(u[4 * k], u[4 * k + 1], u[4 * k + 2], u[4 * k + 3]);
                }
                if (masked) {
                    uint8_t *vrow = gbase + (uint32_t)st * 2 * kTileBytes + kTileBytes + tid * 128;
                    if (!valid) {                          // 0 * NaN is not 0: values behind the end must not reach the product
#pragma unroll
                        for (int k = 0; k < 8; ++k) reinterpret_cast<uint4 *>(vrow)[k] = make_uint4(0u, 0u, 0u, 0u);
                    }
                }
                if (MODE == 1 && s.n_tok > 1 && (t + 1) * kTile > s.see0) {
                    // a NaN value of a token that some columns see and others do not: taken out of the product, and noted
                    // for the columns that see it
                    uint8_t *vtile = gbase + (uint32_t)st * 2 * kTileBytes + kTileBytes;
                    bool nan = false;
                    if (valid) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const uint4 v = reinterpret_cast<const uint4 *>(vtile + tid * 128)[k];
                            const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) nan |= __vcmpeq4(u[e] & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0u;
                        }
                    }
                    if (softmax_any(nan)) {
                        for (int r = 0; r < kTile; ++r) {
                            const int pos = t * kTile + r;
                            if (pos >= s.live) break;
                            uint8_t *cell = vtile + r * 128 + ((((uint32_t)tid >> 4) ^ (r & 7)) << 4) + (tid & 15);
                            if ((*cell & 0x7f) == 0x7f) {
                                const int c = max(0, pos + 1 - s.see0) * a.G;          // first column that sees it
                                if (c < 64) poison |= ~0ull << c;
                                *cell = 0;
                            }
                        }
                    }
                }
                fence_proxy_async();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pfull(pb));
            }

            // -- the segment's end: sums over the 128 token rows, then this thread's channel of every column
#pragma unroll
            for (int c = 0; c < QC; ++c) {
                float v = l[c];
#pragma unroll
                for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
                if (lane == 0) red[warp * QC + c] = v;
            }
            if (s.t1 > s.t0) wait(pdone((it - 1) % PB), (uint32_t)((it - 1) / PB) & 1u, kErrAttnSoftmax);
            tc_fence_after();
            softmax_bar();
            const bool whole = MODE == 0 ? s.t0 == 0 && s.t1 == s.tiles : a.splits == 1;
            float *slot = nullptr;
            if (!whole) {
                const size_t head = MODE == 0 ? 16 + sizeof(UnitMeta) * (size_t)a.B * a.H : 0;
                slot = reinterpret_cast<float *>(a.ws + head) + (size_t)s.slot * attn_slot_floats(QC);
                for (int c = tid; c < n_cols; c += 128) {
                    slot[c] = col_mu[c];
                    slot[QC + c] = red[c] + red[QC + c] + red[2 * QC + c] + red[3 * QC + c];
                }
            }
            if constexpr (MODE == 0)
                if (s.t0 == 0 && tid == 0) {               // first tile of the unit: where the join finds its parts
                    UnitMeta *m = reinterpret_cast<UnitMeta *>(a.ws + 16) + (size_t)s.b * a.H + s.h;
                    m->first = w.pos - (s.t1 - s.t0);
                    m->tiles = s.tiles;
                }
            float raw[NO];
#pragma unroll
            for (int c0 = 0; c0 < NO; c0 += 16) tmem_ld16(tmem_o + lane_addr + c0, *reinterpret_cast<float(*)[16]>(raw + c0));
            tmem_ld_wait();
#pragma unroll
            for (int c = 0; c < QC; ++c) {
                if (c < n_cols) {
                    float v;
                    if (C::CHAIN) {
                        v = raw[c];
                    } else {
                        v = raw[(PT - 1) * QC + c];
#pragma unroll
                        for (int i = PT - 2; i >= 0; --i) v = fmaf(v, kTerm, raw[i * QC + c]);
                    }
                    if (s.t1 == s.t0) v = 0.f;             // an empty split
                    if (MODE == 1 && c < 64 && ((poison >> c) & 1ull)) v = __uint_as_float(0x7fffffffu);
                    if (whole) {
                        const float sum = red[c] + red[QC + c] + red[2 * QC + c] + red[3 * QC + c];
                        const float y = sum == 0.f ? 0.f : __fdiv_rn(v, sum);
                        store1(static_cast<T *>(a.out) + ((size_t)(s.tok0 + c / a.G) * a.H * a.G + (size_t)s.h * a.G + c % a.G) * kHeadDim + tid, y);
                    } else {
                        slot[2 * QC + (size_t)c * kHeadDim + tid] = v;
                    }
                }
            }
            tc_fence_before();
            softmax_bar();                                 // red and col_* are free for the next segment
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        tmem_dealloc(tmem, C::kTmemCols);
    }
}

// Joins the partial results of a unit: rescaled to the largest Mu, summed in order, divided.  Grid (units, columns of a
// unit), a thread per channel.  MODE 0: a unit's parts lie in the slots of the consecutive CTAs that shared it.  MODE 1:
// one slot per split.
template <typename T, int MODE>
__global__ void __launch_bounds__(kHeadDim) k_page_attn_join(const AttnArgs a, const int qc) {
    pdl_wait();
    const int c = blockIdx.y, d = threadIdx.x;
    long long first_slot = 0;
    int n = 0, first_odd = 0;
    size_t out_row = 0;
    const float *slots;
    if constexpr (MODE == 0) {
        const int b = blockIdx.x / a.H, h = blockIdx.x % a.H;
        const UnitMeta m = reinterpret_cast<const UnitMeta *>(a.ws + 16)[blockIdx.x];
        const long long share = *reinterpret_cast<const long long *>(a.ws);
        const long long cta0 = m.first / share, cta1 = (m.first + m.tiles - 1) / share;
        if (cta0 == cta1) return;                          // one CTA had it all and wrote the result
        n = (int)(cta1 - cta0) + 1;
        first_slot = cta0 * 2;
        first_odd = m.first % share != 0 ? 1 : 0;
        out_row = (size_t)b * a.H * a.G + (size_t)h * a.G + c;
        slots = reinterpret_cast<const float *>(a.ws + 16 + sizeof(UnitMeta) * (size_t)a.B * a.H);
    } else {
        const int tq = qc / a.G, v = blockIdx.x / a.H, h = blockIdx.x % a.H;
        int lo = 0, hi = a.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.q_start[mid] / tq + mid <= v) lo = mid; else hi = mid - 1;
        }
        const int first = a.q_start[lo], nn = a.q_start[lo + 1] - first, j = v - (first / tq + lo);
        if (first < 0 || nn < 0 || first > a.n_tokens - nn || j < 0 || (long long)j * tq + c / a.G >= nn) return;
        n = a.splits;
        first_slot = (long long)blockIdx.x * a.splits;
        out_row = (size_t)(first + j * tq + c / a.G) * a.H * a.G + (size_t)h * a.G + c % a.G;
        slots = reinterpret_cast<const float *>(a.ws);
    }
    auto slot = [&](int i) {
        const long long at = MODE == 0 ? (i == 0 ? first_slot + first_odd : first_slot + 2LL * i) : first_slot + i;
        return slots + (size_t)at * attn_slot_floats(qc);
    };
    float mu = kMuNone;
    for (int i = 0; i < n; ++i) mu = fmaxf(mu, slot(i)[c]);
    float sum = 0.f, o = 0.f;
    for (int i = 0; i < n; ++i) {
        const float *p = slot(i);
        const float f = ex2(p[c] - mu);
        sum = fmaf(p[qc + c], f, sum);
        o = fmaf(p[2 * qc + (size_t)c * kHeadDim + d], f, o);
    }
    store1(static_cast<T *>(a.out) + out_row * kHeadDim + d, sum == 0.f ? 0.f : __fdiv_rn(o, sum));
}

}  // namespace pages
}  // namespace faedkv
