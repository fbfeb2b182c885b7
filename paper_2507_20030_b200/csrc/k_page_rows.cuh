// Attention over the paged 8-bit cache with the query columns as the rows of both products, for units of many of them.
//
//     S[row, token]  = sum_d q[row, d] * K[token, d]      (A = q as e4m3 + e5m2 terms, B = the K tile as it lies in the pages)
//     O[row, d]     += sum_n w[row, n] * V[n, d]          (A = weights in f16, in tensor memory; B = the V tile, converted to f16, exact)
//
// A row is a query token and head (and map) of one kv head.  Its thread has all the scores of a tile of 128 tokens, so that the maximum, the sum and the
// weights need no exchange between threads, and a scale of its own costs a row nothing: a third of the instructions that the form with tokens as
// rows (k_page_attn.cuh) takes for 128 columns.  That one stays for few columns, where 128 rows would mostly be empty.
//
// Softmax in base 2: y = s * (k_scale * q_scale * scale * log2 e) - Mu, p = 2^y, l += p, w = p * (v_scale / Vref).  Mu follows the row's largest weight
// lazily: when the weights of half a tile sum up to more than 2^15.5 it is raised by a whole number that puts the largest at 2^6 .. 2^7, what was summed (l and O) is
// multiplied by a power of two, and they are taken once more.  No maximum is formed otherwise.  Weights w therefore keep 2^-11 of themselves and 2^-31 of the
// row's largest.  Vref is the power of two above the first tile's largest v_scale (2^-46 at least).  It stays, so that a page of other values changes nothing for those
// that follow: y has the logarithm of v_scale / Vref in it, from 2^-80 to 2^60, and p is 2^y times the inverse, which float32 holds with a sum of a
// billion tokens (with Vref raised for pages beyond 2^20 and lower ones held to 2^-20, ordinary pages behind one 2^26 times as loud lost their weights'
// bits, behind one 2^31 times all of them).  Only a v_scale beyond 2^60 of it moves Vref, and O with it.
//
// Two softmax warpgroups work on half tiles, 64 tokens.  Each has room for one half's scores and for two halves' weights in tensor memory: once it has the
// scores in registers the next ones are computed, and no product waits for another one's end.  A unit of more than 128 rows is
// two row tiles over the same tokens (K, V and the conversion shared); one of up to 128 rows gives every other tile of tokens to each
// warpgroup, and the two results meet as parts of a softmax do.  Four warps convert V; a TMA warp; one warp issues the first product and one
// the second, since what an issuer waits for between products would leave the tensor cores idle.
//
// What bounds it is the two softmax warps of a scheduler: a half tile of both takes them some 2200 cycles, of which the exponentials are 1024 and the
// tensor cores' products as many; the rest is what a warp waits for between its steps (loads from tensor memory, its turn, stores), and registers leave
// no room for a third.  1024 + 1 + 333 new tokens over 9216 + 4001 + 333, 8 kv x 16 differential heads: 190 to 195 us, 0.35 of the tensor cores' measured rate
// (303 in k_page_attn's form with 128 columns).
#pragma once
#include "k_page_attn.cuh"

namespace faedkv {
namespace pages {

constexpr int kRowsQC = 256, kRowsK = 3, kRowsV = 2, kRowsH = 2, kRowsRing = 8, kRowsSegs = 4;
constexpr int kRowsConvert = 128, kRowsThreads = 256 + kRowsConvert + 128;  // 128 registers a thread at launch (the last warp only hands some on)
constexpr int kRowsRegsSoftmax = 160, kRowsRegsConvert = 96, kRowsRegsIssue = 80;
constexpr int kRowsRegsLaunch = 124;
static_assert(2 * kRowsRegsSoftmax + kRowsRegsConvert + kRowsRegsIssue <= 4 * kRowsRegsLaunch, "a launch has these to share out");
constexpr float kRowsScaleUp = 0x1p60f, kRowsScaleDown = -80.f;   // of v_scale about Vref; the logarithm
constexpr int kRowsCost = 13;                             // what a unit's start and end take, in tiles of one row tile (1024 new tokens over 9216: 228 us at 6, 193 at 10, 190 at 13, 192 at 16, 196 at 20)
constexpr uint32_t kRowsOffV = kRowsK * kTileBytes, kRowsOffH = kRowsOffV + kRowsV * kTileBytes;
constexpr uint32_t kRowsOffQ = kRowsOffH + kRowsH * 2 * kTileBytes, kRowsOffMisc = kRowsOffQ + 4 * kTileBytes;
constexpr uint32_t kRowsFloats = kRowsQC + 2 * 128 * 4 + kRowsRing * 40 + 4 * 128;
constexpr uint32_t kRowsSmem = kRowsOffMisc + 4 * kRowsFloats + 384 + 64 * kRowsSegs + 4 * (kMaxBlocks + 1) + 1024;
static_assert(kRowsSmem <= 232448, "shared memory of a CTA");
static_assert(kRowsRing >= kRowsK + 3, "scales outlive their tile's K");

// Two f16 as e4m3 or e5m2 codes (the lower 16 bits), nearest even.
__device__ __forceinline__ uint32_t f16x2_to_e4m3x2(uint32_t h) {
    uint32_t r;
    asm("{\n\t.reg .b16 c;\n\tcvt.rn.satfinite.e4m3x2.f16x2 c, %1;\n\tcvt.u32.u16 %0, c;\n\t}" : "=r"(r) : "r"(h));
    return r;
}
__device__ __forceinline__ uint32_t f16x2_to_e5m2x2(uint32_t h) {
    uint32_t r;
    asm("{\n\t.reg .b16 c;\n\tcvt.rn.satfinite.e5m2x2.f16x2 c, %1;\n\tcvt.u32.u16 %0, c;\n\t}" : "=r"(r) : "r"(h));
    return r;
}
// An MMA warp goes through its code with all lanes and issues by one, so that descriptors stay in uniform registers: an instruction issued by a
// lane in a branch of its own takes some 95 cycles, more than its product.
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r;
}
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ void mma_f8_by(uint32_t who, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(who) : "memory");
}
// D = A B with A in tensor memory.
__device__ __forceinline__ void mma_f16_ts_by(uint32_t who, uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(who) : "memory");
}
__device__ __forceinline__ void mma_commit_by(uint32_t who, uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(who) : "memory");
}
__device__ __forceinline__ void tmem_st16u(uint32_t taddr, const uint32_t (&u)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]),
          "r"(u[8]), "r"(u[9]), "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]) : "memory");
}

__device__ __forceinline__ uint64_t desc_of(uint32_t lo, uint32_t hi) { return (uint64_t)hi << 32 | lo; }

struct Phase { uint32_t bar, parity; };

struct RowsSegment : Segment {
    int n_cols, weight;                                   // rows (0: there are no more segments); 2 where they are two row tiles
};
__device__ __forceinline__ int rows_weight(int n_cols) { return n_cols > 128 ? 2 : 1; }

// MODE as in k_page_attn: 1 and 3 share the tiles of all units out evenly (a tile of two row tiles counts twice; it belongs to the share in
// which it begins), 2 and 4 give each unit a CTA.
template <int MODE> struct RowsWork {
    int v, h, per_head;
    long long pos, end;
    const int32_t *before;
    __device__ __forceinline__ void set(const AttnArgs &a, const Block &k, RowsSegment &s) const {
        s.b = k.b; s.tok0 = k.tok0; s.n_tok = k.n_tok; s.see0 = k.see0; s.live = k.live; s.page0 = k.page0; s.own = k.own;
        s.n_cols = k.n_tok * a.G;
        s.weight = rows_weight(s.n_cols);
    }
    __device__ __forceinline__ bool next(const AttnArgs &a, RowsSegment &s) {
        if constexpr (MODE == 2 || MODE == 4) {
            if (pos >= end) return false;
            pos = end;
            Block k;
            if (!find_unit<MODE>(a, kRowsQC / a.G, (int)(gridDim.x - 1 - blockIdx.x), threadIdx.x == 0, k)) return false;   // those that see most first
            set(a, k, s);
            s.h = blockIdx.y;
            s.tiles = tiles_of(s.live);
            s.t0 = 0; s.t1 = s.tiles; s.first = 0;
            return true;
        } else {
            while (pos < end) {
                while (before[v + 1] == before[v])        // not a block
                    if (++v == a.blocks) { v = 0; ++h; }
                const long long u0 = (long long)h * per_head + before[v];
                const int size = before[v + 1] - before[v], to = (int)min((long long)size, end - u0);
                const int from = max(0, (int)(pos - u0) - kRowsCost), upto = max(0, to - kRowsCost), block = v;
                s.h = h;
                pos = u0 + to;
                if (++v == a.blocks) { v = 0; ++h; }
                if (upto <= from) continue;               // the share ended before the unit's first tile
                Block k;
                if (!find_unit<MODE>(a, kRowsQC / a.G, block, false, k)) return false;
                set(a, k, s);
                s.t0 = (from + s.weight - 1) / s.weight;
                s.t1 = (upto + s.weight - 1) / s.weight;
                if (s.t1 <= s.t0) continue;
                s.tiles = (size - kRowsCost) / s.weight;
                s.first = u0 + kRowsCost;
                return true;
            }
            return false;
        }
    }
};

// ---- parts of split units

// Which CTA has a position, where each has `share` of them.  (A 32-bit division where that will do.)
__device__ __forceinline__ int cta_of(long long pos, long long share) {
    return pos < (1LL << 31) && share < (1LL << 31) ? (int)((uint32_t)pos / (uint32_t)share) : (int)(pos / share);
}
// A column's partial result: Mu, the sum, 128 channels divided by it.
struct PartColumn { const float *mu, *sum, *o; };
__device__ __forceinline__ PartColumn SlotColumn(const float *slot, int qc, int c) { return {slot + c, slot + qc + c, slot + 2 * qc + (size_t)c * kHeadDim}; }

// N columns' results from their n parts, four channels a lane: sum_i l_i 2^(m_i - m) o_i / sum_i l_i 2^(m_i - m).  32 parts at a time: a lane has the
// statistics of one, all have every one's output; eight parts' outputs are on their way together.
template <int N, typename Part>
__device__ __forceinline__ void gather_parts(Part part, int n, int lane, float4 (&o)[N]) {
    float mu[N], sum[N];
#pragma unroll
    for (int k = 0; k < N; ++k) { mu[k] = kMuNone; sum[k] = 0.f; o[k] = make_float4(0.f, 0.f, 0.f, 0.f); }
    for (int i0 = 0; i0 < n; i0 += 32) {
        const int here = min(32, n - i0);
        float w[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float m = kMuNone, l = 0.f;
            if (lane < here) {
                const PartColumn p = part(i0 + lane, k);
                m = *p.mu;
                l = *p.sum;
            }
            const float top = fmaxf(mu[k], warp_max(m)), back = mu[k] - top;
            w[k] = fade(l, m - top);
            float all = w[k];
#pragma unroll
            for (int s = 16; s; s >>= 1) all += __shfl_xor_sync(0xffffffffu, all, s);
            sum[k] = fade(sum[k], back) + all;
            o[k] = make_float4(fade(o[k].x, back), fade(o[k].y, back), fade(o[k].z, back), fade(o[k].w, back));
            mu[k] = top;
        }
        for (int i = 0; i < here; i += 8) {
            float4 x[N][8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int k = 0; k < N; ++k) x[k][j] = i + j < here ? load4(part(i0 + i + j, k).o + 4 * lane) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float f = __shfl_sync(0xffffffffu, w[k], (i + j) & 31);
                    if (i + j < here) o[k] = make_float4(fmaf(x[k][j].x, f, o[k].x), fmaf(x[k][j].y, f, o[k].y), fmaf(x[k][j].z, f, o[k].z), fmaf(x[k][j].w, f, o[k].w));
                }
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float inv = sum[k] == 0.f ? 0.f : __frcp_rn(sum[k]);
        o[k] = sum[k] == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o[k].x * inv, o[k].y * inv, o[k].z * inv, o[k].w * inv);
    }
}

// What FORM 1 does with the maps of a head (k_page_diff.cuh).
struct DiffArgs {
    const float *maps;                                    // [n_tokens][n_q_heads][2][128]
    const float *lam, *gain;                              // [n_q_heads]; [128] or NULL
    void *out;
    const int32_t *q_start;                               // may be NULL: every row is a token
    int n_tokens, B, HQ;
    float eps;
};
// What a row is multiplied by before it is squared once more, where its mean square m is beyond 2^-100 .. 2^120: there squares leave float32's range, o and
// the result do not.  (2^-70 and 2^75 put every float32 where 128 squares add up; eps goes with the square of it.)
__device__ __forceinline__ bool diff_in_range(float m) { return m >= 0x1p-100f && m <= 0x1p120f; }
__device__ __forceinline__ float diff_unit(float m) { return m > 1.f ? 0x1p-70f : 0x1p75f; }
// 1 / sqrt(mean(o^2) + eps) from the sum of squares: a row of zeros stays one without eps, NaN stays NaN.
__device__ __forceinline__ float diff_norm(float squares, float eps) {
    const float m = squares * (1.0f / kHeadDim) + eps;
    return m > 0.f ? rsqrtf(m) : m;
}

template <int MODE, int FORM>
__global__ void __launch_bounds__(kRowsThreads, 1)
k_page_rows(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const AttnArgs a, const DiffArgs diff) {
    using namespace umma;
    using T = __nv_bfloat16;
    static_assert((MODE >= 3) == (FORM == 0), "rows of new tokens are differential attention's, rows that share pages softmax attention's");
    constexpr int kSoftmax = 256, kWarpTma = 12, kWarpScores = 13, kWarpOutput = 14;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *gbase = smem_raw + (base - smem_u32(smem_raw));
    auto k_tile = [&](int s) { return base + (uint32_t)s * kTileBytes; };
    auto v_tile = [&](int s) { return base + kRowsOffV + (uint32_t)s * kTileBytes; };
    auto h_tile = [&](int s) { return base + kRowsOffH + (uint32_t)s * 2 * kTileBytes; };
    auto q_off = [](int t) { return kRowsOffQ + (t == 0 ? 2u * kTileBytes : 0u); };                  // row tile t, two terms: the second lies behind the buffers of V in f16, and is a third one where there is one row tile
    float *row_cs = reinterpret_cast<float *>(gbase + kRowsOffMisc);         // [256] a row's factor of the raw scores
    float4 *exch = reinterpret_cast<float4 *>(row_cs + kRowsQC);             // [2][128] Mu, l, Vref
    float *ring = reinterpret_cast<float *>(exch + 2 * 128);                 // [kRowsRing][40] of a tile: for its 8 pages k_scale, lr, 2^-lr, c; then Vref, the pages that are there, whether every c is 1
    int *nan_first = reinterpret_cast<int *>(ring + kRowsRing * 40);         // [4][128] first token with a NaN value, by channel
    uint64_t *bars = reinterpret_cast<uint64_t *>(nan_first + 4 * 128);
    int *seg_ring = reinterpret_cast<int *>(bars + 48);                      // [kRowsSegs][16] segments, from the TMA warp to the others
    int32_t *before = seg_ring + 16 * kRowsSegs;
    const uint32_t bar0 = smem_u32(bars);
    auto kfull = [&](int s) { return bar0 + 8 * s; };
    auto kempty = [&](int s) { return bar0 + 8 * (3 + s); };
    auto vfull = [&](int s) { return bar0 + 8 * (6 + s); };
    auto vempty = [&](int s) { return bar0 + 8 * (8 + s); };
    auto hfull = [&](int s) { return bar0 + 8 * (10 + s); };
    auto hempty = [&](int s) { return bar0 + 8 * (13 + s); };
    auto sfull = [&](int g) { return bar0 + 8 * (16 + g); };
    auto sread = [&](int g) { return bar0 + 8 * (18 + g); };
    auto pfull = [&](int g, int half) { return bar0 + 8 * (20 + 2 * g + half); };
    auto pdone = [&](int g, int half) { return bar0 + 8 * (24 + 2 * g + half); };
    const uint32_t qfull = bar0 + 8 * 28;
    auto gfull = [&](int s) { return bar0 + 8 * (29 + s); };
    auto gempty = [&](int s) { return bar0 + 8 * (33 + s); };
    auto drain = [&](int i) { return bar0 + 8 * (37 + i); };
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 39);
    volatile uint32_t *abort_flag = tmem_slot + 1;
    static_assert(kRowsK == 3 && kRowsV == 2 && kRowsH == 2 && kRowsSegs == 4, "the barriers' places");

    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    const int page = 1 << a.page_shift;

    // ---- what needs nothing of the call's inputs, while the stream's previous kernel drains
    if (tid == 0) {
        for (int s = 0; s < kRowsK; ++s) { mbar_init(kfull(s), 1); mbar_init(kempty(s), 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(vfull(s), 1); mbar_init(vempty(s), kRowsConvert / 32); mbar_init(sfull(s), 1); mbar_init(sread(s), 4); }
        for (int s = 0; s < 3; ++s) { mbar_init(hfull(s), kRowsConvert / 32); mbar_init(hempty(s), 1); }
        for (int s = 0; s < 4; ++s) { mbar_init(pfull(s >> 1, s & 1), 4); mbar_init(pdone(s >> 1, s & 1), 1); }
        for (int s = 0; s < kRowsSegs; ++s) { mbar_init(gfull(s), 1); mbar_init(gempty(s), 8 + kRowsConvert / 32 + 2); }
        mbar_init(qfull, 8);
        mbar_init(drain(0), 1);
        mbar_init(drain(1), 1);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == kWarpScores) tmem_alloc(smem_u32(tmem_slot), 512);
    pdl_wait();
    // the rows' own tokens: their CTAs begin where these have ended (64 rows behind 32768 tokens 92.5 us without, 88.8 so; a join released like this, which
    // can only wait, costs 2 us)
    if (MODE >= 3) pdl_release();

    // ---- this CTA's work
    RowsWork<MODE> w0;
    if constexpr (MODE == 1 || MODE == 3) {
        for (int v = tid; v < a.blocks; v += kRowsThreads) {
            Block k;
            before[v + 1] = find_unit<MODE>(a, kRowsQC / a.G, v, blockIdx.x == 0, k) ? kRowsCost + rows_weight(k.n_tok * a.G) * tiles_of(k.live) : 0;
        }
        if (tid == 0) before[0] = 0;
        __syncthreads();
        if (warp == 0)
            for (int v0 = 0, carry = 0; v0 < a.blocks; v0 += 32) {
                int n = v0 + lane < a.blocks ? before[v0 + lane + 1] : 0;
#pragma unroll
                for (int s = 1; s < 32; s <<= 1) {
                    const int o = __shfl_up_sync(0xffffffffu, n, s);
                    if (lane >= s) n += o;
                }
                n += carry;
                if (v0 + lane < a.blocks) before[v0 + lane + 1] = n;
                carry = __shfl_sync(0xffffffffu, n, 31);
            }
        __syncthreads();
        const int per_head = before[a.blocks];
        const long long total = (long long)per_head * a.H;
        const long long share = max(2LL, (total + gridDim.x - 1) / gridDim.x);   // (a share of one could lie inside a tile)
        w0.before = before;
        w0.pos = share * blockIdx.x;
        w0.end = min(total, w0.pos + share);
        w0.per_head = per_head;
        if (tid == 0 && blockIdx.x == 0) *reinterpret_cast<long long *>(a.ws) = share;
        if (MODE == 1 && tid == 0) reinterpret_cast<CtaMeta *>(a.ws + 16)[blockIdx.x].tiles = 0;
        if (MODE == 3 && blockIdx.x == 0)                  // the join finds the units' parts by these
            for (int v = tid; v <= a.blocks; v += kRowsThreads) reinterpret_cast<int32_t *>(a.ws + 16)[v] = before[v];
        if (w0.pos < w0.end) {
            w0.h = (int)(w0.pos / per_head);
            const int in = (int)(w0.pos - (long long)w0.h * per_head);
            int lo = 0, hi = a.blocks - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (before[mid] <= in) lo = mid; else hi = mid - 1;
            }
            w0.v = lo;
        }
    } else {
        w0.pos = 0;
        w0.end = 1;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(tmem_slot);
    auto tmem_s = [&](int g) { return tmem + 64 * g; };                             // scores of 64 tokens
    auto tmem_p = [&](int g, int half) { return tmem + 128 + 64 * g + 32 * half; }; // their weights, two f16 a column
    auto tmem_o = [&](int g) { return tmem + 256 + 128 * g; };

    bool dead = false;                                    // a bounded wait gave up: no further waits, run out
    auto wait = [&](uint32_t bar, uint32_t parity, unsigned int code) {
        if (dead || mbar_try_wait(bar, parity)) return;
        if (*abort_flag || !mbar_wait(bar, parity, a.wait_limit)) {
            if (!*abort_flag) atomicExch(a.status, code);
            *abort_flag = 1;
            dead = true;
        }
    };
    // two of them, asked for together, since an answer takes some hundred cycles
    auto wait_for = [&](Phase x, Phase y) {
        const bool there_x = mbar_try_wait(x.bar, x.parity), there_y = mbar_try_wait(y.bar, y.parity);
        if (!there_x) wait(x.bar, x.parity, kErrAttnMma);
        if (!there_y) wait(y.bar, y.parity, kErrAttnMma);
    };
    // The next segment, from the ring (the other warps): finding it is a chain of loads that the TMA warp has gone through ahead of them.  Warps that gave up
    // go through the segments as the others do, since those meet them at barriers; the TMA warp marks the end in any case.
    auto next_segment = [&](uint32_t seg, RowsSegment &s) {
        const int at = seg % kRowsSegs;
        if (!__all_sync(0xffffffffu, mbar_wait(gfull(at), (seg / kRowsSegs) & 1u, 8 * a.wait_limit))) return false;
        const int *r = seg_ring + 16 * at;
        s.b = 0; s.page0 = 0;
        s.h = r[0]; s.tok0 = r[1]; s.n_tok = r[2]; s.see0 = r[3]; s.live = r[4]; s.own = r[5]; s.t0 = r[6]; s.t1 = r[7]; s.tiles = r[8];
        s.n_cols = r[9]; s.weight = r[10];
        s.first = (long long)(uint32_t)r[11] | (long long)r[12] << 32;
        __syncwarp();
        if (lane == 0) mbar_arrive(gempty(at));
        return s.n_cols > 0;
    };
    // Items of a segment: half tiles of a warpgroup.  Warpgroup g has tiles_of_group() tiles, its own row tile's all or every other one; the q-th of its
    // items is half q & 1 of its tile q >> 1.  The tensor cores see them as 0, 1, 2, ..: item i is the (i >> 1)-th of warpgroup i & 1.
    auto tiles_of_group = [](const RowsSegment &s, int g) { return s.weight == 2 ? s.t1 - s.t0 : (s.t1 - s.t0 + 1 - g) >> 1; };
    auto tile_of = [](const RowsSegment &s, int g, int q) { return s.weight == 2 ? q >> 1 : (q >> 1) * 2 + g; };   // counted from the segment's first
    auto buffers = [](const RowsSegment &s) { return s.weight == 2 ? 2 : 3; };                       // of V in f16; each segment starts with the first
    auto whole_tile = [&](const RowsSegment &s, int t, uint32_t have) {      // every row sees all of it
        return (t + 1) * kTile <= s.see0 && have == (1u << (kTile >> a.page_shift)) - 1u;
    };

    if (warp >= kWarpTma) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRowsRegsIssue));
    if (warp == kWarpTma) {
        // ------------------------------------------------------------------------ producer: pages by TMA, scales
        const int lg_ppt = 7 - a.page_shift, ppt = 1 << lg_ppt;               // pages of a tile
        const int tiles_batch = 32 >> lg_ppt;                                 // a lane looks after one page of the next 32
        RowsWork<MODE> w = w0;
        RowsSegment s;
        int it = 0, issued_k = 0, issued_v = 0;
        uint32_t seg = 0;
        for (;; ++seg) {
            const bool more = w.next(a, s);
            const int at = seg % kRowsSegs;
            wait(gempty(at), ((seg / kRowsSegs) & 1u) ^ 1u, kErrAttnTma);
            dead = __any_sync(0xffffffffu, dead);
            if (dead) break;
            if (lane == 0) {
                int *r = seg_ring + 16 * at;
                r[0] = s.h; r[1] = s.tok0; r[2] = s.n_tok; r[3] = s.see0; r[4] = s.live; r[5] = s.own; r[6] = s.t0; r[7] = s.t1; r[8] = s.tiles;
                r[9] = more ? s.n_cols : 0;
                r[10] = s.weight;
                r[11] = (int)(uint32_t)s.first;
                r[12] = (int)(s.first >> 32);
                mbar_arrive(gfull(at));
            }
            __syncwarp();
            if (!more) break;
            const int32_t *row = a.table + (size_t)s.b * a.W;
            auto fetch = [&](int t_first, int &id, float &ks, float &vs) {
                const long long p_live = ((long long)t_first << lg_ppt) + lane, p = s.page0 + p_live;
                id = -1; ks = 0.f; vs = 0.f;
                if ((p_live << a.page_shift) < s.live && t_first + (lane >> lg_ppt) < s.t1 && FAEDKV_IN_BOUNDS(kTagPageAttn, p >= 0 && p < a.W && s.b >= 0 && s.b < a.B && s.h < a.H)) {
                    id = row[p];
                    if (id < 0 || id >= a.n_pages) {
                        flag(a.status, kBadPage);
                        id = -1;
                    } else {
                        const size_t ph = (size_t)id * a.H + s.h;
                        ks = a.ks[ph];
                        vs = a.vs[ph];
                    }
                }
            };
            int id, id_next;
            float ks, vs, ks_next, vs_next, v_ref = 0.f, v_inv = 0.f, v_lg = -126.f;
            fetch(s.t0, id, ks, vs);
            for (int tb = s.t0; tb < s.t1; tb += tiles_batch) {
                fetch(tb + tiles_batch, id_next, ks_next, vs_next);
                const int tn = min(tiles_batch, s.t1 - tb);
                for (int i = 0; i < tn; ++i, ++it) {
                    const int st = it % kRowsK, sv = it % kRowsV;
                    wait(kempty(st), ((uint32_t)(it / kRowsK) & 1u) ^ 1u, kErrAttnTma);
                    const bool mine = (lane >> lg_ppt) == i;
                    const int k = lane & (ppt - 1);
                    const uint32_t have = __ballot_sync(0xffffffffu, mine && id >= 0) >> (i << lg_ppt);
                    const uint32_t bytes = (uint32_t)__popc(have) * (uint32_t)(page * kHeadDim);
                    dead = __any_sync(0xffffffffu, dead);
                    if (dead) continue;
                    const int y = (id * a.H + s.h) << a.page_shift;
                    const uint32_t off = (uint32_t)(k << a.page_shift) * kHeadDim;
                    if (mine && id >= 0) tma_load_2d(k_tile(st) + off, &map_k, kfull(st), 0, y);
                    // the scales before the barrier's own arrival.  Their room is free: the scores that had this K's room are complete, so the
                    // tiles two before them are done with
                    float *sc = ring + (it & (kRowsRing - 1)) * 40;
                    const float v_max = warp_max(mine ? fabsf(vs) : 0.f);
                    if (v_ref == 0.f || v_max > v_ref * kRowsScaleUp) {
                        v_ref = scale_ref(v_max, 0x1p-46f);
                        v_inv = __fdiv_rn(1.f, v_ref);
                        v_lg = __log2f(v_ref);
                    }
                    // a page's weights are 2^(y + lr) * c: lr is the logarithm of v_scale / Vref, at least -80 (p of a page of zeros stays in
                    // reach), and c what that leaves, 1 for all but such pages and negative scales; p is the weight times 2^-lr
                    const float lr = id >= 0 ? fmaxf(__log2f(fmaxf(fabsf(vs), 1.17549435e-38f)) - v_lg, kRowsScaleDown) : 0.f, inv_r = ex2(-lr), c = id >= 0 ? vs * v_inv * inv_r : 1.f;
                    const uint32_t odd = __ballot_sync(0xffffffffu, mine && !(c > 0.9999f));
                    if (mine) {
                        sc[k] = ks;
                        sc[8 + k] = lr;
                        sc[16 + k] = inv_r;
                        sc[24 + k] = c;
                    }
                    if (lane == 0) {
                        sc[32] = v_ref;
                        reinterpret_cast<uint32_t *>(sc)[33] = have;
                        reinterpret_cast<uint32_t *>(sc)[34] = odd == 0u;
                    }
                    __syncwarp();
                    if (lane == 0) mbar_expect_tx(kfull(st), bytes);
                    issued_k = it + 1;
                    wait(vempty(sv), ((uint32_t)(it / kRowsV) & 1u) ^ 1u, kErrAttnTma);
                    dead = __any_sync(0xffffffffu, dead);
                    if (dead) continue;
                    if (mine && id >= 0) tma_load_2d(v_tile(sv) + off, &map_v, vfull(sv), 0, y);
                    __syncwarp();
                    if (lane == 0) mbar_expect_tx(vfull(sv), bytes);
                    issued_v = it + 1;
                }
                id = id_next; ks = ks_next; vs = vs_next;
            }
        }
        if (dead && lane == 0) {                           // the end, for those who did not give up
            if (mbar_wait(gempty(seg % kRowsSegs), ((seg / kRowsSegs) & 1u) ^ 1u, 4 * a.wait_limit)) {
                seg_ring[16 * (seg % kRowsSegs) + 9] = 0;
                mbar_arrive(gfull(seg % kRowsSegs));
            }
        }
        {                                                  // leave no copy in flight behind, whoever gave up
            for (int i = max(0, issued_k - kRowsK); i < issued_k; ++i) mbar_wait(kfull(i % kRowsK), (uint32_t)(i / kRowsK) & 1u, a.wait_limit);
            for (int i = max(0, issued_v - kRowsV); i < issued_v; ++i) mbar_wait(vfull(i % kRowsV), (uint32_t)(i / kRowsV) & 1u, a.wait_limit);
        }
    } else if (warp == kWarpScores || warp == kWarpOutput) {
        // ------------------------------------------------------------------------ MMA issuers: all lanes go along, one issues
        // formats: scores e4m3 x e4m3, the second term of q (A) e5m2; output f16, V MN-major
        constexpr uint32_t kIdescS = make_idesc(0u, 0u, 0u, 64), kIdescS1 = kIdescS | 1u << 7, kIdescO = make_idesc(0u, 0u, 1u, 128);
        // descriptors: the lower words of the first tiles; a tile further 1024 more, in 16 bytes
        const uint64_t q_desc = desc_kmajor_sw128(base + q_off(0)), k_desc = desc_kmajor_sw128(k_tile(0)), h_desc = desc_mnmajor_sw128(h_tile(0), kTileBytes);
        const uint32_t q_lo = (uint32_t)q_desc, k_lo = (uint32_t)k_desc, h_lo = (uint32_t)h_desc;
        const uint32_t kmajor_hi = (uint32_t)(q_desc >> 32), h_hi = (uint32_t)(h_desc >> 32);
        RowsSegment s;
        const uint32_t who = elect_one();
        const bool first = warp == kWarpScores;
        int st_base = 0, base0 = 0, base1 = 0;             // tiles of the segments before: their number modulo kRowsK, and each warpgroup's
        uint32_t uses = 0;                                 // a bit a buffer of K, or of V in f16: the lowest of the number of its uses
        for (uint32_t seg = 0; next_segment(seg, s); ++seg) {
            // (where a wait gives up, the products go on over what lies there: nothing is read or written elsewhere, and the call's result is void)
            const int weight = uniform(s.weight), n_tiles = uniform(s.t1 - s.t0), n_buf = first ? kRowsK : weight == 2 ? 2 : 3;
            const int n0 = weight == 2 ? 2 * n_tiles : n_tiles + (n_tiles & 1), n1 = weight == 2 ? n0 : n_tiles & ~1;
            if (first) wait(qfull, seg & 1u, kErrAttnMma);
#pragma unroll 1
            for (int i = 0; i < 2 * n0; ++i) {
                const int g = i & 1, q = i >> 1, half = q & 1, t = weight == 2 ? i >> 2 : (i >> 2) * 2 + g;
                if (q >= (g ? n1 : n0)) continue;
                if (first) {
                    // scores, once their warpgroup has those of its item before in registers
                    const int st = (st_base + t) % kRowsK;
                    wait_for({kfull(st), (uses >> st ^ (uint32_t)(t / kRowsK)) & 1u}, {sread(g), (uint32_t)(q - 1) & 1u});
                    tc_fence_after();
                    const uint32_t qa = q_lo - (weight == 2 && g == 1 ? 2048 : 0), kb = k_lo + st * 1024 + half * 512, d = tmem_s(g);
#pragma unroll
                    for (int term = 0; term < 2; ++term)
#pragma unroll
                        for (int k = 0; k < 4; ++k)        // 32 channels each
                            mma_f8_by(who, d, desc_of(qa + term * 1024 + k * 2, kmajor_hi), desc_of(kb + k * 2, kmajor_hi), term ? kIdescS1 : kIdescS, (term | k) ? 1u : 0u);
                    mma_commit_by(who, sfull(g));
                    if (half == 1 && (weight == 1 || g == 1)) mma_commit_by(who, kempty(st));
                } else {
                    const int hb = t % n_buf;
                    wait_for({hfull(hb), (uses >> hb ^ (uint32_t)(t / n_buf)) & 1u}, {pfull(g, half), (uint32_t)((g ? base1 : base0) + (q >> 1)) & 1u});
                    tc_fence_after();
                    const uint32_t p = tmem_p(g, half), o = tmem_o(g), hd = h_lo + hb * 2048 + half * 512;
#pragma unroll
                    for (int k = 0; k < 4; ++k)            // 16 tokens each
                        mma_f16_ts_by(who, o, p + k * 8, desc_of(hd + k * 128, h_hi), kIdescO, (q > 0 || k) ? 1u : 0u);
                    mma_commit_by(who, pdone(g, half));
                    if (half == 1 && (weight == 1 || g == 1)) mma_commit_by(who, hempty(hb));
                }
            }
            const int b0 = first ? st_base : 0;
            for (int t = 0; t < min(n_buf, n_tiles); ++t) uses ^= (uint32_t)((n_tiles - t + n_buf - 1) / n_buf & 1) << (b0 + t) % n_buf;
            st_base = (st_base + n_tiles) % kRowsK;
            base0 += n0 / 2;
            base1 += n1 / 2;
        }
        // no product may be on its way when the tensor memory is given back
        mma_commit_by(who, drain(first ? 0 : 1));
        mbar_wait(drain(first ? 0 : 1), 0u, a.wait_limit);
    } else if (warp >= kWarpTma) {
    } else if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRowsRegsConvert));
        // ------------------------------------------------------------------------ V tiles to f16, a token a thread
        RowsSegment s;
        const int row = tid - kSoftmax;
        int it = 0;
        uint32_t h_uses = 0;
        for (uint32_t seg = 0; next_segment(seg, s); ++seg) {
            int *first = nan_first + (seg & 3u) * 128;
            const int n_buf = buffers(s), n = s.t1 - s.t0;
            for (int i = 0, hb = 0, round = 0; i < n; ++i, ++it) {
                const int t = s.t0 + i, sv = it % kRowsV;
                wait(vfull(sv), (uint32_t)(it / kRowsV) & 1u, kErrAttnSoftmax);
                const uint32_t have = reinterpret_cast<const uint32_t *>(ring + (it & (kRowsRing - 1)) * 40)[33];
                const bool all = whole_tile(s, t, have), ragged = (MODE == 1 || MODE == 2) && s.n_tok > 1 && (t + 1) * kTile > s.see0;
                const uint8_t *from = gbase + kRowsOffV + (uint32_t)sv * kTileBytes;
                uint8_t *to = gbase + kRowsOffH + (uint32_t)hb * 2 * kTileBytes;
                uint4 v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const uint4 *>(from + mn_chunk<128>(row, j));
                wait(hempty(hb), ((h_uses >> hb ^ (uint32_t)round) & 1u) ^ 1u, kErrAttnSoftmax);
                // the third buffer is also the second row tile's q, and the room its results go out through: those of the segment before are done with
                // it once this segment's q is there
                if (hb == 2 && round == 0) wait(qfull, seg & 1u, kErrAttnSoftmax);
                // (the segment four before has been written out: its place is free)
                if ((MODE == 1 || MODE == 2) && i == 0) {
                    first[row] = 0x7fffffff;
                    softmax_bar(3, kRowsConvert);
                }
                if (!all) {
                    // 0 * NaN is not 0: values behind the end must not reach the product, nor a NaN value of a token that some rows see and
                    // others do not: it is noted by its channel, for the rows that see it
                    const int tok = t * kTile + row;
                    const bool valid = tok < s.live && ((have >> (row >> a.page_shift)) & 1u);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (!valid) v[j] = make_uint4(0u, 0u, 0u, 0u);
                        uint32_t *u = reinterpret_cast<uint32_t *>(&v[j]);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t is_nan = ragged ? ((u[k] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u : 0u;   // the top bit of each NaN code
                            if (is_nan != 0u) {
#pragma unroll 1
                                for (int e = 0; e < 4; ++e)
                                    if ((is_nan >> (8 * e + 7)) & 1u) atomicMin(first + 16 * j + 4 * k + e, tok);
                                u[k] &= ~((is_nan >> 7) * 255u);
                            }
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {                            // 16 channels
                    const uint4 lo = make_uint4(e4m3x2_to_f16x2(v[j].x), e4m3x2_to_f16x2(v[j].x >> 16), e4m3x2_to_f16x2(v[j].y), e4m3x2_to_f16x2(v[j].y >> 16));
                    const uint4 hi = make_uint4(e4m3x2_to_f16x2(v[j].z), e4m3x2_to_f16x2(v[j].z >> 16), e4m3x2_to_f16x2(v[j].w), e4m3x2_to_f16x2(v[j].w >> 16));
                    *reinterpret_cast<uint4 *>(to + (j >> 2) * kTileBytes + mn_chunk<128>(row, (2 * j) & 7)) = lo;
                    *reinterpret_cast<uint4 *>(to + (j >> 2) * kTileBytes + mn_chunk<128>(row, (2 * j + 1) & 7)) = hi;
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(hfull(hb));
                    mbar_arrive(vempty(sv));
                }
                if (++hb == n_buf) { hb = 0; ++round; }
            }
            for (int t = 0; t < min(n_buf, n); ++t) h_uses ^= (uint32_t)((n - t + n_buf - 1) / n_buf & 1) << t;
        }
    } else {
        // ------------------------------------------------------------------------ softmax: a row a thread
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRowsRegsSoftmax));
        const int g = warp >> 2, row = tid & 127;
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t to = tmem_o(g) + lane_addr;
        constexpr float kMostSum = 46336.f, kLag = 7.f;        // 2^15.5: no weight of a sum up to that is beyond f16
        RowsSegment s;
        int count = 0, it = 0;                            // this warpgroup's tiles, and all, of the segments before
        for (uint32_t seg = 0; next_segment(seg, s); ++seg) {
            const bool two = s.weight == 2;
            const int c = (two ? g * 128 : 0) + row, tok = c * a.inv_g >> 16;              // this thread's row, and its token
            const bool warp_on = (c & ~31) < s.n_cols;
            // -- the rows of q as two terms, each row with a power of two of its own.  Half a warp has a row of q (and, differential, the rows of its two
            // maps), 16 bytes a lane, the next one on its way.  (A row a thread took 17 000 cycles, a line for each lane of a load; eight rows at a time
            // 21 000: instructions that are run once come from afar.)
            {
                constexpr int kMaps = FORM == 1 ? 2 : 1;
                const int l16 = lane & 15, map = FORM == 1 ? l16 >> 3 : 0;
                const int first = (two ? g * (128 / kMaps) + (warp & 3) * 2 : warp * 2) + (lane >> 4), step = two ? 8 : 16;
                const int end = min(two ? (g + 1) * 128 : 128, (s.n_cols + 31) / 32 * 32) / kMaps;   // rows up to whole warps' are zero
                auto load = [&](int r) {
                    const int col = r * kMaps, k = col * a.inv_g >> 16;
                    const bool there = r < end && col < s.n_cols && FAEDKV_IN_BOUNDS(kTagPageAttn, s.tok0 >= 0 && s.tok0 + k < a.n_tokens);
                    const T *from = static_cast<const T *>(a.q) + (size_t)(s.tok0 + k) * a.ld_q + ((size_t)s.h * (a.G / kMaps) + (col - k * a.G) / kMaps) * kHeadDim + l16 * 8;
                    return there ? *reinterpret_cast<const uint4 *>(from) : make_uint4(0u, 0u, 0u, 0u);
                };
                constexpr int kTogether = FORM == 1 ? 1 : 2;               // rows of a half warp at a time (two make the other form slower)
                uint4 next[kTogether];
#pragma unroll
                for (int j = 0; j < kTogether; ++j) next[j] = load(first + j * step);
#pragma unroll 1
                for (int r0 = first; r0 - (lane >> 4) < end; r0 += kTogether * step) {
                    uint32_t u[kTogether][4], top[kTogether];
                    bool odd = false;
#pragma unroll
                    for (int j = 0; j < kTogether; ++j) {
                        u[j][0] = next[j].x; u[j][1] = next[j].y; u[j][2] = next[j].z; u[j][3] = next[j].w;
                        next[j] = load(r0 + (kTogether + j) * step);
                        // the largest magnitude of the row (of the map), as bf16 bits; where an infinity or NaN is among them, of the others
                        top[j] = __vmaxu2(__vmaxu2(u[j][0] & 0x7fff7fffu, u[j][1] & 0x7fff7fffu), __vmaxu2(u[j][2] & 0x7fff7fffu, u[j][3] & 0x7fff7fffu));
                        odd |= max(top[j] & 0xffffu, top[j] >> 16) >= 0x7f80u;
                    }
                    odd = __any_sync(0xffffffffu, odd);
                    if (odd) {
#pragma unroll
                        for (int j = 0; j < kTogether; ++j) {
                            top[j] = 0;
#pragma unroll 1
                            for (int e = 0; e < 8; ++e) {
                                const uint32_t m = (e < 2 ? u[j][0] : e < 4 ? u[j][1] : e < 6 ? u[j][2] : u[j][3]) >> (16 * (e & 1)) & 0x7fffu;
                                if (m < 0x7f80u) top[j] = max(top[j], m);
                            }
                        }
                    }
#pragma unroll
                    for (int o = 1; o < 16 / kMaps; o <<= 1)
#pragma unroll
                        for (int j = 0; j < kTogether; ++j) top[j] = __vmaxu2(top[j], __shfl_xor_sync(0xffffffffu, top[j], o));
#pragma unroll
                    for (int j = 0; j < kTogether; ++j) {
                        const int r = r0 + j * step;
                        const float qs = 2.0f * scale_for(__uint_as_float(max(top[j] & 0xffffu, top[j] >> 16) << 16));    // the largest element to 112 .. 224
                        const float inv = __uint_as_float((254u << 23) - __float_as_uint(qs));
                        // what the first term leaves of an element above 2^-6 has three significant bits (bf16's eight less its four, and a sign),
                        // which e5m2 holds; of smaller ones e5m2's rounding is at most 2^-14
                        uint32_t c1[4], c2[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float lo = __uint_as_float(u[j][e] << 16) * inv, hi = __uint_as_float(u[j][e] & 0xffff0000u) * inv;
                            if (odd) {                     // infinities and NaN make their row's scores NaN
                                if (!(fabsf(lo) < INFINITY)) lo = __uint_as_float(0x7fffffffu);
                                if (!(fabsf(hi) < INFINITY)) hi = __uint_as_float(0x7fffffffu);
                            }
                            const uint32_t h = pack_f16(lo, hi);                                 // exact (or, of elements far below the row's largest, to 2^-25)
                            c1[e] = f16x2_to_e4m3x2(h);
                            const uint32_t back = e4m3x2_to_f16x2(c1[e]);
                            const __half2 left = __hsub2(*reinterpret_cast<const __half2 *>(&h), *reinterpret_cast<const __half2 *>(&back));
                            c2[e] = f16x2_to_e5m2x2(*reinterpret_cast<const uint32_t *>(&left));
                        }
                        if (r < end) {
                            const int col = r * kMaps + map;
                            uint8_t *at = gbase + q_off(col >> 7) + (l16 & 1) * 8;
                            const uint32_t here = mn_chunk<128>((uint32_t)(col & 127), (uint32_t)l16 >> 1);
                            *reinterpret_cast<uint2 *>(at + here) = make_uint2(c1[0] | c1[1] << 16, c1[2] | c1[3] << 16);
                            *reinterpret_cast<uint2 *>(at + kTileBytes + here) = make_uint2(c2[0] | c2[1] << 16, c2[2] | c2[3] << 16);
                            if (FORM == 1) {               // the map's other half
                                const uint32_t zero = mn_chunk<128>((uint32_t)(col & 127), (uint32_t)(l16 ^ 8) >> 1);
                                *reinterpret_cast<uint2 *>(at + zero) = make_uint2(0u, 0u);
                                *reinterpret_cast<uint2 *>(at + kTileBytes + zero) = make_uint2(0u, 0u);
                            }
                            if ((l16 & (16 / kMaps - 1)) == 0) row_cs[col] = qs * a.scale_log2;
                        }
                    }
                }
            }
            fence_proxy_async();
            softmax_bar(1, kSoftmax);
            if (lane == 0) mbar_arrive(qfull);

            const int n = 2 * tiles_of_group(s, g);
            const int lim = MODE >= 3 || c >= s.n_cols ? s.see0 : s.see0 + tok;
            const float cs = warp_on ? row_cs[c] : 0.f;
            float mu = 0.f, v_ref = 0.f;
            bool set = false;                              // Mu stands for a weight
            float2 l = make_float2(0.f, 0.f);
#pragma unroll 1
            for (int q = 0; q < n; ++q) {
                const int half = q & 1, i_tile = tile_of(s, g, q), t = s.t0 + i_tile;
                const uint32_t ts = tmem_s(g) + lane_addr, tp = tmem_p(g, half) + lane_addr;
                const float *sc = ring + ((it + i_tile) & (kRowsRing - 1)) * 40;
                // the scores; and the product that read these weights' room two items ago has ended
                wait_for({sfull(g), (uint32_t)q & 1u}, {pdone(g, half), (uint32_t)(count + (q >> 1) - 1) & 1u});
                tc_fence_after();
                auto scores_read = [&]() {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(sread(g));
                };
                // The two warps of a scheduler take turns with the exponentials: side by side they would both wait for the unit, and then both for the
                // tensor cores.  Item q of the second warpgroup follows item q of the first.  A turn ends with the third quarter of them, since a warp
                // alone does not fill the unit (1024 new tokens over 9216: 193.5 us after a quarter or half, 189.5 so, 193 at their end)
                const int other = 2 * tiles_of_group(s, g ^ 1);
                auto turn_begin = [&]() {
                    if (g == 1 || (q > 0 && q - 1 < other)) softmax_bar(4 + 2 * (warp & 3) + g, 64);
                };
                auto turn_end = [&]() {
                    if (g == 0 ? q < other : q + 1 < other) asm volatile("barrier.cta.arrive %0, %1;" ::"r"(5 + 2 * (warp & 3) - g), "r"(64) : "memory");
                };
                if (!warp_on) {
                    scores_read();
                    turn_begin();
                    turn_end();
                } else {
                    float raw[2][32];
                    tmem_ld<32>(ts, raw[0]);
                    tmem_ld<32>(ts + 32, raw[1]);
                    // O times f, once the product before has been added to it
                    auto rescale = [&](float f) {
                        wait(pdone(g, half ^ 1), (uint32_t)(count + ((q - 1) >> 1)) & 1u, kErrAttnSoftmax);
                        tc_fence_after();
#pragma unroll 1
                        for (int d = 0; d < kHeadDim; d += 16) {
                            float o[16];
                            tmem_ld<16>(to + d, o);
                            tmem_ld_done<16>(o);
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] *= f;
                            tmem_st16(to + d, o);
                        }
                        tmem_st_wait();
                    };
                    // 16 tokens lie in one page
                    const uint32_t have = reinterpret_cast<const uint32_t *>(sc)[33], plain = reinterpret_cast<const uint32_t *>(sc)[34];
                    const float v_now = sc[32];
                    float kf[4], add[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int pg = (64 * half + 16 * k) >> a.page_shift;
                        kf[k] = sc[pg] * cs;
                        add[k] = sc[8 + pg] - mu;
                    }
                    tmem_ld_done<32>(raw[0]);
                    tmem_ld_done<32>(raw[1]);
                    scores_read();
                    if (v_now != v_ref) {
                        if (v_ref > 0.f && q > 0) rescale(v_ref / v_now);
                        v_ref = v_now;
                    }
                    if (!whole_tile(s, t, have)) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int at = 64 * half + 16 * k, left = (have >> (at >> a.page_shift)) & 1u ? lim - (t * kTile + at) : 0;
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                float &x = raw[k >> 1][(k & 1) * 16 + e];
                                x = e < left ? x * kf[k] : -INFINITY;
                            }
                            kf[k] = 1.f;
                        }
                    }
                    float2 l_half;                         // this half tile's part of the sum: a few dozen additions, however long the row
                    float2 y[4][8];                        // in the scores' registers
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int p = 0; p < 8; ++p)
                            y[k][p] = fma2(make_float2(raw[k >> 1][(k & 1) * 16 + 2 * p], raw[k >> 1][(k & 1) * 16 + 2 * p + 1]), make_float2(kf[k], kf[k]), make_float2(add[k], add[k]));
                    // the weights, into their place; returns their sum
                    auto weights = [&](auto general, bool again) {
                        float sum = 0.f;
                        l_half = make_float2(0.f, 0.f);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            uint32_t packed[16];
#pragma unroll
                            for (int k = 2 * i; k < 2 * i + 2; ++k) {
                                const int pg = (64 * half + 16 * k) >> a.page_shift;
                                const float c = decltype(general)::value ? sc[24 + pg] : 1.f, inv_r = sc[16 + pg];
                                float2 part = make_float2(0.f, 0.f);
#pragma unroll
                                for (int p = 0; p < 8; ++p) {
                                    float2 e = make_float2(ex2(y[k][p].x), ex2(y[k][p].y));
                                    part = add2(part, e);
                                    if (decltype(general)::value) e = mul2(e, make_float2(c, c));
                                    packed[8 * (k & 1) + p] = pack_f16(e.x, e.y);
                                }
                                l_half = fma2(part, make_float2(inv_r, inv_r), l_half);
                                sum += part.x + part.y;
                                if (k == 2 && !again) turn_end();
                            }
                            tmem_st16u(tp + 16 * i, packed);
                        }
                        return sum;
                    };
                    for (bool again = false;; again = true) {
                        if (!again) turn_begin();
                        const float sum = plain ? weights(std::false_type{}, again) : weights(std::true_type{}, again);
                        // beyond what f16 holds, or no reference yet: Mu is raised, and the weights once more
                        const bool need = !set || !(sum <= kMostSum);
                        if (again || !__any_sync(0xffffffffu, need)) break;
                        float top = -INFINITY;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
#pragma unroll
                            for (int p = 0; p < 8; ++p) top = max3(top, y[k][p].x, y[k][p].y);
                        const bool seen = need && top > -INFINITY;
                        const float d = !seen ? 0.f : set ? fmaxf(ceilf(top) - kLag, 0.f) : ceilf(top) - kLag;
                        const float f = seen && set ? (d > 120.f ? 0.f : ex2(-d)) : 1.f;
                        l = make_float2(set && seen ? fade(l.x, -d) : l.x, set && seen ? fade(l.y, -d) : l.y);
                        mu += d;
                        set |= seen;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
#pragma unroll
                            for (int p = 0; p < 8; ++p) y[k][p] = make_float2(y[k][p].x - d, y[k][p].y - d);
                        if (q > 0 && __any_sync(0xffffffffu, f != 1.f)) rescale(f);
                    }
                    l = add2(l, l_half);
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && (warp != 0 || half != 0 || count + (q >> 1) + 1 != a.withhold)) mbar_arrive(pfull(g, half));
            }
            it += s.t1 - s.t0;
            count += n / 2;

            // -- the segment's end: this row's sum, then its channels (one row tile: half of them each warpgroup, of both's results)
            if (n > 0) wait(pdone(g, 1), (uint32_t)(count - 1) & 1u, kErrAttnSoftmax);
            tc_fence_after();
            float sum = l.x + l.y, f[2] = {0.f, 0.f};
            if (!two) {
                exch[g * 128 + row] = make_float4(mu, sum, v_ref, 0.f);
                tc_fence_before();
                softmax_bar(1, kSoftmax);
                tc_fence_after();
                const float4 x0 = exch[row], x1 = exch[128 + row];
                mu = fmaxf(x0.y == 0.f ? kMuNone : x0.x, x1.y == 0.f ? kMuNone : x1.x);
                const float l0 = x0.y == 0.f ? 0.f : fade(x0.y, x0.x - mu), l1 = x1.y == 0.f ? 0.f : fade(x1.y, x1.x - mu);
                sum = l0 + l1;
                const float inv = sum == 0.f ? 0.f : __frcp_rn(sum);
                f[0] = x0.y == 0.f ? 0.f : ex2(x0.x - mu) * inv * x0.z;
                f[1] = x1.y == 0.f ? 0.f : ex2(x1.x - mu) * inv * x1.z;
            } else {
                f[0] = sum == 0.f ? 0.f : __frcp_rn(sum) * v_ref;
            }
            const bool whole = MODE == 2 || MODE == 4 || (s.t0 == 0 && s.t1 == s.tiles);
            const bool on = c < s.n_cols && FAEDKV_IN_BOUNDS(kTagPageAttn, s.tok0 + tok < a.n_tokens && s.h < a.H);
            const SharedParts parts(a.whole, (size_t)a.B * a.H * a.G, s.own);
            auto row_of = [&](int col) {                   // of [n_tokens][H][G]
                const int k = col * a.inv_g >> 16;
                return ((size_t)(s.tok0 + k) * a.H + s.h) * a.G + (col - k * a.G);
            };
            float *slot = nullptr;
            if (!whole) {
                float *slots = MODE == 3 ? a.slots : reinterpret_cast<float *>(a.ws + attn_meta_bytes(MODE, (size_t)a.B * a.H, gridDim.x));
                slot = slots + ((size_t)blockIdx.x * 2 + (s.t0 > 0 ? 0 : 1)) * attn_slot_floats(kRowsQC);
            }
            if (on && (two || g == 0)) {
                const float m = sum == 0.f ? kMuNone : mu;
                if (!whole) { slot[c] = m; slot[kRowsQC + c] = sum; }
                else if (MODE >= 3) parts.stat[row_of(c)] = make_float2(m, sum);
            }
            // (MODE 1: where the join finds the unit's parts: as many positions as lie between its first tile's and its last one's)
            if (MODE == 1 && s.t0 > 0 && tid == 0) reinterpret_cast<CtaMeta *>(a.ws + 16)[blockIdx.x] = CtaMeta{s.first, (s.tiles - 1) * s.weight + 1, s.tok0, s.n_cols, s.h};
            const int *first = nan_first + (seg & 3u) * 128;
            // 16 channels of this row
            auto result = [&](int d, float(&o)[16]) {
                tmem_ld<16>((two ? to : tmem_o(0) + lane_addr) + d, o);
                tmem_ld_done<16>(o);
                if (!two && s.t1 - s.t0 > 1) {
                    float o1[16];
                    tmem_ld<16>(tmem_o(1) + lane_addr + d, o1);
                    tmem_ld_done<16>(o1);
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = (f[0] == 0.f ? 0.f : o[e] * f[0]) + (f[1] == 0.f ? 0.f : o1[e] * f[1]);
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = f[0] == 0.f ? 0.f : o[e] * f[0];             // no token: zero
                }
                if (MODE == 1 || MODE == 2) {
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const int4 at = *reinterpret_cast<const int4 *>(first + d + e);
                        if (lim > at.x) o[e] = __uint_as_float(0x7fffffffu);
                        if (lim > at.y) o[e + 1] = __uint_as_float(0x7fffffffu);
                        if (lim > at.z) o[e + 2] = __uint_as_float(0x7fffffffu);
                        if (lim > at.w) o[e + 3] = __uint_as_float(0x7fffffffu);
                    }
                }
            };
            const int d0 = two ? 0 : g * 64, d1 = two ? kHeadDim : d0 + 64;
            if (FORM == 1 && whole) {
                // the two maps of a head are rows of neighbouring threads: their difference, its norm (over two warpgroups' channels, where they have
                // half each), and the head's output
                const bool second = lane & 1;
                const float lam = on ? diff.lam[s.h * (a.G >> 1) + ((c - tok * a.G) >> 1)] : 0.f;
                auto difference = [&](int d, float(&o)[16]) {
                    result(d, o);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float x = __shfl_xor_sync(0xffffffffu, o[e], 1);
                        o[e] = second ? fmaf(-lam, o[e], x) : fmaf(-lam, x, o[e]);
                    }
                };
                float squares = 0.f, unit = 1.f;
                for (bool again = false; diff.gain != nullptr; again = true) {
                    squares = 0.f;
                    if (warp_on)
#pragma unroll 1
                        for (int d = d0; d < d1; d += 16) {
                            float o[16];
                            difference(d, o);
#pragma unroll
                            for (int e = 0; e < 16; ++e) squares = fmaf(o[e] * unit, o[e] * unit, squares);
                        }
                    if (!two) {
                        softmax_bar(1, kSoftmax);          // (row_cs has been read)
                        row_cs[g * 128 + row] = squares;
                        softmax_bar(1, kSoftmax);
                        squares = row_cs[row] + row_cs[128 + row];
                    }
                    if (again) break;
                    // once more, in another unit, where some row's squares are out of range (both threads of a row find the same)
                    const float m = squares * (1.0f / kHeadDim) + diff.eps;
                    const bool odd = on && !diff_in_range(m);
                    if (!(two ? (bool)__any_sync(0xffffffffu, odd) : softmax_any(odd, 1, kSoftmax))) break;
                    if (odd) unit = diff_unit(m);
                }
                const float r = diff_norm(squares, diff.eps * unit * unit);
                T *out = static_cast<T *>(diff.out) + (row_of(c) >> 1) * kHeadDim;
                if (warp_on)
#pragma unroll 1
                    for (int d = d0; d < d1; d += 16) {
                        float o[16];
                        difference(d, o);
                        if (!on) continue;
                        if (diff.gain != nullptr) {
#pragma unroll
                            for (int e = 0; e < 16; e += 4) {
                                const float4 w = load4(diff.gain + d + e);
                                o[e] *= unit; o[e + 1] *= unit; o[e + 2] *= unit; o[e + 3] *= unit;
                                o[e] *= r * w.x; o[e + 1] *= r * w.y; o[e + 2] *= r * w.z; o[e + 3] *= r * w.w;
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 8; e += 4)     // half of them each
                            store4(out + d + (second ? 8 : 0) + e, second ? make_float4(o[8 + e], o[9 + e], o[10 + e], o[11 + e]) : make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]));
                    }
            } else if (two) {
                // 64 channels at a time through this warpgroup's rows of q, so that what is written together lies together
                uint8_t *stage = gbase + q_off(g);
                float *dst = whole ? parts.o : slot + 2 * kRowsQC;
#pragma unroll 1
                for (int part = 0; part < 2; ++part) {
                    if (warp_on)
#pragma unroll 1
                        for (int d = 0; d < 64; d += 16) {
                            float o[16];
                            result(64 * part + d, o);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                *reinterpret_cast<float4 *>(stage + row * 256 + (((d >> 2) + e) ^ (row & 15)) * 16) = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                        }
                    softmax_bar(12 + g, 128);
#pragma unroll 4
                    for (int i = 0; i < 16; ++i) {
                        const int r = i * 8 + (row >> 4), k = row & 15, col = g * 128 + r;
                        const float4 x = *reinterpret_cast<const float4 *>(stage + r * 256 + (k ^ (r & 15)) * 16);
                        if (col < s.n_cols) *reinterpret_cast<float4 *>(dst + (whole ? row_of(col) : (size_t)col) * kHeadDim + 64 * part + 4 * k) = x;
                    }
                    softmax_bar(12 + g, 128);
                }
            } else if (warp_on) {
                float *dst = (whole ? parts.o + row_of(c) * kHeadDim : slot + 2 * kRowsQC + (size_t)c * kHeadDim);
#pragma unroll 1
                for (int d = d0; d < d1; d += 16) {
                    float o[16];
                    result(d, o);
                    if (on)
#pragma unroll
                        for (int e = 0; e < 16; e += 4) store4(dst + d + e, make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]));
                }
            }
            tc_fence_before();
            softmax_bar(1, kSoftmax);                      // q, exch and O are free for the next segment
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == kWarpScores) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

}  // namespace pages
}  // namespace faedkv
