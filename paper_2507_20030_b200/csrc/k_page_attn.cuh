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
// with the query columns (new tokens x query heads of one kv head) as N.  The other operand has to be of eight bits too, so a
// query element is written as a sum of e4m3 terms of four significant bits each, the i-th scaled by 16^i, and a softmax
// weight as a sum of e5m2 terms of three, scaled by 8^i: their products are exact and accumulate in float32, so nothing of
// the cache is converted anywhere and what is lost is only what the last term rounds off (bf16 q: two terms, 2^-17 of its
// row's largest element at most; weights: four terms for bf16, 2^-12 of a weight and 2^-34 of the column's largest, eight for
// float32, 2^-24 and 2^-46).  e5m2 for the
// weights because of its range: with e4m3 terms a weight had fewer bits the smaller it was, and below 2^-20 of the largest
// none.  Where 128 columns share a tile, the weights are f16 and the V tile is converted to f16 (exact) before the second
// product, which costs as much as two e4m3 terms and keeps small weights.
//
// Softmax runs in base 2: y = s * (k_scale * scale * log2 e) - Mu, p = 2^y, l += p, weights w = p * (v_scale / Vref).  Mu
// follows the column's largest weight lazily: it is raised (and O, l rescaled) only when some weight exceeds 2^15 or so, and then
// to 2^-6 or 2^-8 of the largest, so weights stay in their format's range and most tiles exchange one vote instead of a maximum per
// column.  It follows the weights and not p, so a page of large values that hardly counts takes no bits from the others.  Vref is
// the power of two above the first tile's largest v_scale (2^-66 at least), and stays: p is the weight over v_scale / Vref, from 2^-60 to 2^40, and float32 holds it
// and l (pages of zeros have the smallest scale, and their tokens count in l all the same).  Only a scale beyond 2^40 of Vref moves it, and rescales
// O.  From the first page on that lies beyond 2^20 of it (a segment `far`), Mu is settled before every tile's weights are taken, since p of a tile taken
// again would pass float32.  O stays in TMEM over all tiles of a segment.
//
// Measured: a decode step over 16 x 16384 tokens of 8 kv heads 89 us (6.0 TB/s of codes), over 131072 tokens 54 us (39 us of
// it in the tiles); 2048 new tokens over 18432 962 us (608 TFLOP/s), bound by the softmax warps (an instruction issued in 53 %
// of the cycles, tensor pipe 29 %); float32, six ragged sequences up to 4096 tokens 17.3 us.  128 columns over four warpgroups
// were faster than over two or 96 over three (879, 992 and 961 us with e4m3 weights), eight columns at a time than sixteen
// (931, 952 with f16 weights and one scale for q).
//
// A CTA: one to four softmax warpgroups (thread = token row of S, channel row of O; a warpgroup has its share of the
// columns), a TMA warp, an MMA warp.
#pragma once
#include <type_traits>

#include "common.cuh"
#include "k_pages.cuh"
#include "umma_common.cuh"

namespace faedkv {
namespace pages {

constexpr int kTile = 128;                                // tokens of a tile
constexpr uint32_t kTileBytes = kTile * kHeadDim;         // 16 KB: K or V codes of a tile
// of v_scale about Vref: within `near` weights are taken before Mu is known to hold them; beyond `up` Vref moves; below `down` (a logarithm) p is cut off
constexpr float kScaleNear = 0x1p20f, kScaleUp = 0x1p40f, kScaleDown = -60.f;
// Vref for a largest v_scale of v_max: the power of two above it, no less than `least`, 2^-126 of pages of zeros over the factor `down`: their p then stand so
// far above their weights that what follows finds Mu low.
__device__ __forceinline__ float scale_ref(float v_max, float least) { return __uint_as_float((__float_as_uint(fmaxf(v_max, least)) + 0x7fffffu) & 0xff800000u); }
constexpr float kMuNone = -3e38f;                         // a part that saw no token
constexpr int kMaxBlocks = 1024;                          // blocks of new tokens that MODE 1 takes
constexpr unsigned int kErrAttnTma = 0x41, kErrAttnMma = 0x42, kErrAttnSoftmax = 0x43;

// Instances: QC query columns over WGS softmax warpgroups.  Few columns (WIDE = false): QT e4m3 terms of q, PT e5m2 terms of the
// weights side by side as further columns of one product, V as it lies.  Many (WIDE = true): QT terms of q added up in the same accumulator;
// weights in f16, which holds them to 2^-11 down to 2^-20 of the largest and to 2^-31 of it below, and V converted to f16 (exact)
// by the softmax warps, a tile at a time into one buffer (two more warps that convert it were slower, 1016 us for 931 at 2048 new
// tokens over 18432: with one buffer their work lies between two products).  (Two e4m3 terms on one grid lost every weight below
// 2^-14 of the largest: beside a loud token thousands of those are half of the output.)  KST / VST: tiles of K and of V on their way.
template <typename T_, int QC_, int WGS_, int QT_, int PT_, bool WIDE_, int PART_, int KST_, int VST_, int CTAS_> struct AttnCfg {
    using T = T_;
    static constexpr int QC = QC_, WGS = WGS_, QT = QT_, PT = PT_, PART = PART_, KST = KST_, VST = VST_, CTAS = CTAS_;
    static constexpr bool WIDE = WIDE_;
    static constexpr int QW = QC / WGS;                                       // columns of a warpgroup
    static constexpr int kThreads = 128 * WGS + 64;
    // the largest weight: f16 ends at 2^16, e5m2 at 1.75 2^15, which the terms that follow must not be rounded beyond
    static constexpr float kMostWeight = WIDE ? 46336.f : 32768.f;
    // and after a raise of Mu: room to grow before the next one, against the bits of the small weights (2048 new tokens over
    // 18432: 985 us at 10, 931 at 6, 930 at 4)
    static constexpr float kLagTo = WIDE ? 6.0f : 8.0f;
    static constexpr int NS = WIDE ? QC : (QC * QT + 15) / 16 * 16;           // columns of S, of O
    static constexpr int NO = WIDE ? QC : (QC * PT + 15) / 16 * 16;
    static constexpr int kTmemUsed = 2 * NS + NO;
    static constexpr uint32_t kTmemCols = kTmemUsed <= 32 ? 32 : kTmemUsed <= 64 ? 64 : kTmemUsed <= 128 ? 128 : kTmemUsed <= 256 ? 256 : 512;
    static constexpr uint32_t PW = NO <= 32 ? 32 : NO <= 64 ? 64 : 128;       // bytes of a token's e5m2 weights
    static constexpr uint32_t kPBytes = WIDE ? 2 * kTile * QC : kTile * PW;
    static constexpr uint32_t kHBytes = WIDE ? 2 * kTileBytes : 0;            // a V tile in f16
    static constexpr uint32_t kQBytes = (WIDE ? QT * QC : NS) * 128;
    static constexpr uint32_t kOffV = KST * kTileBytes;
    static constexpr uint32_t kOffQ = kOffV + VST * kTileBytes;
    static constexpr uint32_t kOffP = kOffQ + (kQBytes + 1023) / 1024 * 1024;
    static constexpr uint32_t kOffH = kOffP + 2 * kPBytes;
    static constexpr uint32_t kOffMisc = kOffH + kHBytes;
    static constexpr uint32_t kSmemBytes = kOffMisc + sizeof(float) * (9 * QC + KST * 32) + 256 + 1024;
    static constexpr uint32_t kSmemBlocks = 4 * (kMaxBlocks + 1);             // MODE 1 appends its prefix sums
    static_assert(!WIDE || (QC == 128 && WGS == 4 && QT == 2 && PT == 1 && KST <= VST + 1), "the layouts of the wide form");
    static_assert(!WIDE || (PART % 8 == 0 && QW % PART == 0), "whole parts");
    static_assert(WIDE || (WGS == 1 && KST == VST), "a tile's K and V leave together");
};

struct AttnArgs {
    const void *q;
    void *out;
    const int32_t *q_start, *kv_len, *table;              // q_start may be NULL: one token per sequence
    const float *ks, *vs;
    long long ld_q;
    int n_tokens, B, H, G, W, n_pages, page_shift, blocks;
    uint32_t inv_g;                                       // c * inv_g >> 16 = c / G for the columns c < 256, G <= 8
    float scale_log2;                                     // scale * log2(e)
    unsigned char *ws;
    unsigned int *status;
    unsigned long long wait_limit;                        // ns, of a bounded wait
    int withhold;                                         // test hook: the tile (from 1) whose weights are not announced; 0: none
    // MODE 3 and 4: groups of rows, and the tokens that the rows of each share; which blocks the launch has (1 those of groups, 2 the rows' own);
    // results of whole units by query row, partial ones by CTA
    const int32_t *group_start, *shared_len;
    int n_groups, which;
    float *whole, *slots;
};

constexpr uint32_t inverse_g(int g) { return 65536u / (unsigned)g + 1u; }
constexpr bool divides_columns() {
    for (int g = 1; g <= 8; ++g)
        for (uint32_t c = 0; c < 256; ++c)
            if ((c * inverse_g(g) >> 16) != c / (unsigned)g) return false;
    return true;
}
static_assert(divides_columns(), "inv_g");

// Workspace of MODE 0 and 1: header, records, two partial results per CTA (of the unit it goes on with, of the one it leaves).
struct UnitMeta { long long first; int tiles, pad; };                             // MODE 0, by unit
struct CtaMeta { long long first; int tiles, tok0, n_cols, h; };                  // MODE 1, by CTA: the unit that a CTA goes on with (tiles = 0: none)
__host__ __device__ constexpr size_t attn_meta_bytes(int mode, size_t units, size_t ctas) {
    return 16 + (mode == 0 ? sizeof(UnitMeta) * units : (sizeof(CtaMeta) * ctas + 15) / 16 * 16);
}
__host__ __device__ constexpr size_t attn_slot_floats(int qc) { return (size_t)qc * (kHeadDim + 2); }
// Workspace of MODE 3 and 4: for each launch a header with the prefix sums of its blocks' sizes, and (MODE 3) two partial results per CTA; for the call
// the results of whole units by query row (cols of them: rows x heads), first those of the groups' blocks, then those of the rows' own.
__host__ __device__ constexpr size_t shared_before_bytes(int blocks) { return 16 + ((size_t)blocks + 4) / 4 * 16; }
__host__ __device__ constexpr size_t shared_whole_bytes(size_t cols) { return 2 * cols * (sizeof(float2) + sizeof(float) * kHeadDim); }
struct SharedParts {
    float2 *stat;                                         // Mu and the sum
    float *o;
    __device__ __forceinline__ SharedParts(float *whole, size_t cols, int own) {
        float2 *s = reinterpret_cast<float2 *>(whole);
        stat = s + own * cols;
        o = whole + 4 * cols + own * cols * kHeadDim;
    }
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// x * 2^e for e <= 0, also where 2^e alone is no float32: sums hold pages of zeros, whose p are up to 2^80 times the weights'.
__device__ __forceinline__ float fade(float x, float e) { return x * ex2(fmaxf(e, -100.f)) * ex2(fminf(e + 100.f, 0.f)); }
__device__ __forceinline__ float warp_max(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
// Barriers over `threads` softmax threads, the first with a vote.
__device__ __forceinline__ bool softmax_any(bool v, int id, int threads) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\t"
                 "setp.ne.u32 q, %1, 0;\n\t"
                 "barrier.cta.red.or.pred p, %2, %3, q;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(r) : "r"((uint32_t)v), "r"(id), "r"(threads) : "memory");
    return r != 0;
}
__device__ __forceinline__ void softmax_bar(int id, int threads) {
    asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
// Two float32 operations an instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(reinterpret_cast<unsigned long long &>(d))
        : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)), "l"(reinterpret_cast<unsigned long long &>(c)));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long &>(d))
        : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long &>(d))
        : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)));
    return d;
}
__device__ __forceinline__ float2 sub2(float2 a, float2 b) {
    float2 d;
    asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long &>(d))
        : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// MN-major operand: rows of `row` bytes (32, 64 or 128) along MN, one row per K index, swizzled over their own width;
// eight rows to a group, groups back to back.
template <uint32_t row>
__device__ __forceinline__ uint64_t desc_mn_rows(uint32_t saddr) {
    constexpr uint64_t layout = row == 128 ? 2 : row == 64 ? 4 : 6;
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)((8 * row) >> 4) << 16) | ((uint64_t)((8 * row) >> 4) << 32) |
           ((uint64_t)1 << 46) | (layout << 61);
}
// Where 16-byte chunk k of row r of such an operand lies.
template <uint32_t row>
__device__ __forceinline__ uint32_t mn_chunk(uint32_t r, uint32_t k) {
    return r * row + ((k ^ (row == 128 ? r & 7u : row == 64 ? (r >> 1) & 3u : (r >> 2) & 1u)) << 4);
}

__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]),
          "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float *r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]) : "r"(taddr));
}
// N columns (a multiple of 8) of this warp's lanes; completed by tmem_ld_done(), which names the registers, so that other
// work may be scheduled between the two.
template <int N>
__device__ __forceinline__ void tmem_ld(uint32_t taddr, float (&r)[N]) {
#pragma unroll
    for (int c = 0; c + 16 <= N; c += 16) tmem_ld16(taddr + c, *reinterpret_cast<float(*)[16]>(r + c));
    if (N % 16 != 0) tmem_ld8(taddr + N - 8, r + N - 8);
}
template <int N>
__device__ __forceinline__ void tmem_ld_done(float (&r)[N]) {
#pragma unroll
    for (int c = 0; c < N; c += 8) {
        float *f = r + c;
        if (c == 0)
            asm volatile("tcgen05.wait::ld.sync.aligned;"
                         : "+f"(f[0]), "+f"(f[1]), "+f"(f[2]), "+f"(f[3]), "+f"(f[4]), "+f"(f[5]), "+f"(f[6]), "+f"(f[7]));
        else
            asm volatile("" : "+f"(f[0]), "+f"(f[1]), "+f"(f[2]), "+f"(f[3]), "+f"(f[4]), "+f"(f[5]), "+f"(f[6]), "+f"(f[7]));
    }
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
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const float *r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]) : "memory");
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

// Two e4m3 codes (the lower 16 bits) as f16: exact, NaN stays NaN.
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t codes) {
    uint32_t h;
    asm("{\n\t.reg .b16 c;\n\tcvt.u16.u32 c, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, c;\n\t}" : "=r"(h) : "r"(codes));
    return h;
}

// The leading three significant bits of w as an e5m2 value (0 below e5m2's normal range).
__device__ __forceinline__ float lead3(float w) {
    const float h = __uint_as_float(__float_as_uint(w) & 0xffe00000u);
    return fabsf(w) >= 6.103515625e-05f ? h : 0.f;
}
// e5m2 codes, round to nearest even; the first in the lowest byte.
__device__ __forceinline__ uint32_t to_e5m2x4(float a, float b, float c, float d) {
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "cvt.rn.satfinite.e5m2x2.f32 lo, %2, %1;\n\t"
        "cvt.rn.satfinite.e5m2x2.f32 hi, %4, %3;\n\t"
        "mov.b32 %0, {lo, hi};\n\t}" : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}

// One unit of work is the columns of one (sequence, kv head, block of new tokens); a segment is a run of its tiles.
struct Segment {
    int b, h, tok0, n_tok;       // first query row (of q, out) and number of query tokens
    int see0;                    // tokens that the first query token sees (its column limit); the i-th sees see0 + i
    int live;                    // tokens that the last one sees, >= 0
    int page0, own;              // place in the table row of the unit's first page, from where the tokens above are counted; Block's own
    int t0, t1, tiles;           // tiles of the segment, of the unit
    long long first;             // position of the unit's first tile among all
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

// Which new tokens block v of a call with blocks of tq holds: block v - (q_start[b] / tq + b) of sequence b, since sequences
// begin at distinct numbers of that form.  Not every v is a block.
struct Block { int b, tok0, n_tok, see0, live, page0, own; };   // own: 1 a row's own block of MODE 3 and 4
__device__ __forceinline__ bool find_block(const AttnArgs &a, int tq, int v, bool report, Block &k) {
    int lo = 0, hi = a.B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.q_start[mid] / tq <= v - mid) lo = mid; else hi = mid - 1;   // (any int32 may stand there: no sum with it)
    }
    const int first = a.q_start[lo], n = a.q_start[lo + 1] - first;
    if (first < 0 || n < 0 || first > a.n_tokens - n) {
        if (report) flag(a.status, kBadStart);
        return false;
    }
    const int j = v - (first / tq + lo);
    if (j < 0 || (long long)j * tq >= n) return false;
    k.b = lo;
    k.tok0 = first + j * tq;
    k.n_tok = min(tq, n - j * tq);
    k.see0 = (int)clamp_len(a, lo, report) - n + j * tq + 1;
    k.live = max(0, k.see0 + k.n_tok - 1);
    k.page0 = k.own = 0;
    return true;
}

// MODE 3 and 4, a decode step of rows that share pages: first blocks of a group's rows over the tokens that it shares, then for each row
// a block of its own over those behind, or only the ones or the others.  The blocks of rows are numbered as above; row b's own is the b-th behind them.
// The whole pages that row b shares with its group, in tokens: none for the only row of a group, for one that is shorter than what its
// group shares, and for one that stands in no group.  g, first: the group, its first row.
__device__ __forceinline__ int shared_of(const AttnArgs &a, int b, int live, bool report, int &g, int &first) {
    int lo = 0, hi = a.n_groups - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.group_start[mid] <= b) lo = mid; else hi = mid - 1;
    }
    g = lo;
    first = a.group_start[lo];
    const int end = a.group_start[lo + 1];
    if (first < 0 || end > a.B || b < first || b >= end) {
        if (report) flag(a.status, kBadStart);
        return 0;
    }
    const int n = a.shared_len[lo] >> a.page_shift << a.page_shift;
    if (n < 0 || n > a.W << a.page_shift) {
        if (report) flag(a.status, kBadLength);
        return 0;
    }
    return end - first > 1 && live >= n ? n : 0;
}
__host__ __device__ __forceinline__ int shared_blocks(int B, int n_groups, int tq) { return B / tq + n_groups; }
__device__ __forceinline__ bool find_shared(const AttnArgs &a, int tq, int v, bool report, Block &k) {
    const int n_shared = a.which & 1 ? shared_blocks(a.B, a.n_groups, tq) : 0;
    int g, first;
    if (v >= n_shared) {
        const int b = v - n_shared, live = (int)clamp_len(a, b, report), n = shared_of(a, b, live, report, g, first);
        k.b = k.tok0 = b;
        k.n_tok = k.own = 1;
        k.page0 = n >> a.page_shift;
        k.see0 = k.live = live - n;
        return live > n;
    }
    int lo = 0, hi = a.n_groups - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.group_start[mid] / tq <= v - mid) lo = mid; else hi = mid - 1;   // (any int32 may stand there: no sum with it)
    }
    first = a.group_start[lo];
    const int n = a.group_start[lo + 1] - first;
    if (first < 0 || n < 0 || first > a.B - n) return false;   // (reported with its rows)
    const int j = v - (first / tq + lo);
    if (j < 0 || (long long)j * tq >= n) return false;
    k.tok0 = first + j * tq;
    k.n_tok = min(tq, n - j * tq);
    // read through the first row that has them all; a row that has not, or none, is left to its own block
    for (int b = k.tok0; b < k.tok0 + k.n_tok; ++b) {
        const int share = shared_of(a, b, (int)clamp_len(a, b, false), false, g, first);
        if (share > 0) {
            k.b = b;
            k.see0 = k.live = share;
            k.page0 = k.own = 0;
            return true;
        }
    }
    return false;
}
template <int MODE>
__device__ __forceinline__ bool find_unit(const AttnArgs &a, int tq, int v, bool report, Block &k) {
    if constexpr (MODE >= 3) return find_shared(a, tq, v, report, k);
    else return find_block(a, tq, v, report, k);
}

// MODE 0, a decode step: the tiles of all (sequence, head) units in a row are cut into equal shares, one per CTA; a share
// begins and ends anywhere inside a unit.  MODE 1, blocks of new tokens: the same over (head, block) units, whose sizes stand
// as prefix sums in shared memory; a unit counts for kUnitCost positions more than it has tiles, which is what its queries,
// its first maxima and its output take.  MODE 2, more blocks than MODE 1 takes: a CTA per unit.
constexpr int kUnitCost = 8;
// In a decode step over shared pages (MODE 3) fewer, since no unit has more than eight columns or a mask of its own: eight rows behind 2048 tokens 17.4 us
// at 8, 16.5 at 6, 16.3 at 4, 16.0 at 2, behind 8192 22.9, 22.7, 21.9 and 25.2, five float32 rows of seven heads behind 4000 23.1, 23.1, 22.6 and 24.1.
constexpr int kSharedCost = 4;
__host__ __device__ constexpr int unit_cost(int mode) { return mode == 3 ? kSharedCost : kUnitCost; }
template <int MODE> struct Work;

template <> struct Work<0> {
    int b, h, t;
    long long pos, end;
    __device__ __forceinline__ bool next(const AttnArgs &a, int, Segment &s) {
        if (pos >= end) return false;
        s.b = b; s.h = h; s.tok0 = b; s.n_tok = 1; s.page0 = s.own = 0;
        s.live = (int)clamp_len(a, b, false);
        s.see0 = s.live;
        const int tiles = tiles_of(s.live);
        s.tiles = tiles; s.t0 = t;
        s.first = pos - t;
        const long long left = end - pos;
        s.t1 = left < tiles - t ? t + (int)left : tiles;
        pos += s.t1 - s.t0;
        t = 0;
        if (++h == a.H) { h = 0; ++b; }
        return true;
    }
};

template <int MODE> struct WorkShares {
    int v, h, per_head;
    long long pos, end;
    const int32_t *before;                                // [blocks + 1]: positions of one head's blocks before block v
    __device__ __forceinline__ bool next(const AttnArgs &a, int qc, Segment &s) {
        while (pos < end) {
            while (before[v + 1] == before[v])            // not a block
                if (++v == a.blocks) { v = 0; ++h; }
            const long long u0 = (long long)h * per_head + before[v];
            const int size = before[v + 1] - before[v], to = (int)min((long long)size, end - u0);
            s.t0 = max(0, (int)(pos - u0) - unit_cost(MODE));
            s.t1 = max(0, to - unit_cost(MODE));
            s.h = h;
            const int block = v;
            pos = u0 + to;
            if (++v == a.blocks) { v = 0; ++h; }
            if (s.t1 <= s.t0) continue;                   // the share ended before the unit's first tile
            Block k;
            if (!find_unit<MODE>(a, qc / a.G, block, false, k)) return false;
            s.b = k.b; s.tok0 = k.tok0; s.n_tok = k.n_tok; s.see0 = k.see0; s.live = k.live; s.page0 = k.page0; s.own = k.own;
            s.tiles = size - unit_cost(MODE);
            s.first = u0 + unit_cost(MODE);
            return true;
        }
        return false;
    }
};
template <> struct Work<1> : WorkShares<1> {};
template <> struct Work<3> : WorkShares<3> {};

template <int MODE> struct WorkOne {
    bool done;
    __device__ __forceinline__ bool next(const AttnArgs &a, int qc, Segment &s) {
        if (done) return false;
        done = true;
        Block k;
        // the blocks that see most first
        if (!find_unit<MODE>(a, qc / a.G, (int)(gridDim.x - 1 - blockIdx.x), threadIdx.x == 0, k)) return false;
        s.b = k.b; s.h = blockIdx.y; s.tok0 = k.tok0; s.n_tok = k.n_tok; s.see0 = k.see0; s.live = k.live; s.page0 = k.page0; s.own = k.own;
        s.tiles = tiles_of(s.live);
        s.t0 = 0; s.t1 = s.tiles; s.first = 0;
        return true;
    }
};
template <> struct Work<2> : WorkOne<2> {};
template <> struct Work<4> : WorkOne<4> {};

// FORM 0: softmax attention.  FORM 1, differential attention: a head's query row and the cached keys are two halves of 64 channels, and
// each half has a softmax of its own over the same values; a column is (head, half), G counts both, and its query is zero in the other half,
// so one product over 128 channels gives either score.  The results of the columns are float32 and meet in k_page_diff.
template <typename C, int FORM> struct AttnOut { using T = typename C::T; };
template <typename C> struct AttnOut<C, 1> { using T = float; };

template <typename C, int MODE, int FORM>
__global__ void __launch_bounds__(C::kThreads, C::CTAS)
k_page_attn(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const AttnArgs a) {
    using namespace umma;
    using T = typename C::T;
    constexpr int QC = C::QC, QW = C::QW, WGS = C::WGS, QT = C::QT, PT = C::PT, NS = C::NS, NO = C::NO, KST = C::KST, VST = C::VST;
    constexpr int kSoftmax = 128 * WGS, kWarpTma = 4 * WGS, kWarpMma = 4 * WGS + 1;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *gbase = smem_raw + (base - smem_u32(smem_raw));
    auto k_tile = [&](int s) { return base + (uint32_t)s * kTileBytes; };
    auto v_tile = [&](int s) { return base + C::kOffV + (uint32_t)s * kTileBytes; };
    const uint32_t q_base = base + C::kOffQ;
    auto p_tile = [&](int p) { return base + C::kOffP + (uint32_t)p * C::kPBytes; };
    float *col = reinterpret_cast<float *>(gbase + C::kOffMisc);             // per pair of columns: factors of the raw scores, -Mu (wide: [QC] -Mu, [QC] factors)
    float *col_f = col + 2 * QC;                                             // [QC] 2^-raise
    int *col_lim = reinterpret_cast<int *>(col_f + QC);                      // [QC] tokens that the column sees
    int *col_set = col_lim + QC;                                             // [QC] Mu stands for a maximum
    float *red = reinterpret_cast<float *>(col_set + QC);                    // [4][QC]
    float *stage_ks = red + 4 * QC;                                          // [KST][32]: 8 k_scale, 8 v_scale, Vref, at 24 the pages that are there and, as the sign, whether the segment is far
    uint64_t *bars = reinterpret_cast<uint64_t *>(stage_ks + KST * 32);
    const uint32_t bar0 = smem_u32(bars);
    constexpr int kBars = 2 * (KST + VST);
    auto kfull = [&](int s) { return bar0 + 8 * s; };
    auto kempty = [&](int s) { return bar0 + 8 * (KST + s); };                // (narrow: of the tile's K and V)
    auto vfull = [&](int s) { return bar0 + 8 * (2 * KST + s); };
    auto vempty = [&](int s) { return bar0 + 8 * (2 * KST + VST + s); };      // wide only
    auto sfull = [&](int i) { return bar0 + 8 * (kBars + i); };
    auto pfull = [&](int i) { return bar0 + 8 * (kBars + 2 + i); };
    auto pdone = [&](int i) { return bar0 + 8 * (kBars + 4 + i); };
    const uint32_t qfull = bar0 + 8 * (kBars + 6);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + kBars + 7);
    volatile uint32_t *abort_flag = tmem_slot + 1;
    static_assert(8 * (kBars + 8) <= 256, "barriers fit the room behind the stages");

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int page = 1 << a.page_shift;

    // ---- what needs nothing of the call's inputs, while the stream's previous kernel drains
    if (tid == 0) {
        for (int s = 0; s < KST; ++s) { mbar_init(kfull(s), 1); mbar_init(kempty(s), 1); }
        for (int s = 0; s < VST; ++s) { mbar_init(vfull(s), 1); mbar_init(vempty(s), 4 * WGS); }
        for (int i = 0; i < 2; ++i) mbar_init(sfull(i), 1);
        for (int i = 0; i < 2; ++i) { mbar_init(pfull(i), 4 * WGS); mbar_init(pdone(i), 1); }
        mbar_init(qfull, 4 * WGS);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == kWarpMma) tmem_alloc(smem_u32(tmem_slot), C::kTmemCols);
    // (releasing the join from here on was slower: 17.5 us, not 16.5, at six ragged sequences)
    // The launch of the rows' own tokens needs nothing of the one of the groups' before it, which has waited for all that came earlier.
    if (MODE < 3 || a.which != 2) pdl_wait();

    // ---- this CTA's work
    Work<MODE> w0;
    if constexpr (MODE == 0) {
        // prefix sums of the sequences' tiles: 128 runs of consecutive sequences, one per thread.  The thread whose run holds
        // the CTA's first position finds the place in it for all.
        __shared__ long long warp_sum[4];
        __shared__ Work<MODE> place;
        const int run = (a.B + 127) / 128;
        long long n = 0, upto = 0;
        if (tid < 128) {
            for (int b = tid * run; b < min(a.B, (tid + 1) * run); ++b) n += tiles_of(clamp_len(a, b, blockIdx.x == 0));
            upto = n;
#pragma unroll
            for (int s = 1; s < 32; s <<= 1) {
                const long long o = __shfl_up_sync(0xffffffffu, upto, s);
                if (lane >= s) upto += o;
            }
            if (lane == 31) warp_sum[warp] = upto;
        }
        __syncthreads();
        const long long w_sum[4] = {warp_sum[0], warp_sum[1], warp_sum[2], warp_sum[3]};
        const long long total = (w_sum[0] + w_sum[1] + w_sum[2] + w_sum[3]) * a.H;
        // (a 32-bit division where that will do: a 64-bit one is a long way for every CTA to go)
        const long long share = total < (1LL << 31) ? (long long)(((uint32_t)total + gridDim.x - 1) / gridDim.x) : (total + gridDim.x - 1) / gridDim.x;
        const long long pos = share * blockIdx.x, end = min(total, pos + share);
        if (tid == 0) {
            if (blockIdx.x == 0) *reinterpret_cast<long long *>(a.ws) = share;
            if (pos >= end) place.pos = place.end = 0;
        }
        if (tid < 128) {
            upto += (warp > 0 ? w_sum[0] : 0) + (warp > 1 ? w_sum[1] : 0) + (warp > 2 ? w_sum[2] : 0);
            if (pos < end && (upto - n) * a.H <= pos && pos < upto * a.H) {
                long long at = (upto - n) * a.H;
                int b = tid * run, tiles = tiles_of(clamp_len(a, b, false));
                while (at + (long long)tiles * a.H <= pos) {
                    at += (long long)tiles * a.H;
                    tiles = tiles_of(clamp_len(a, ++b, false));
                }
                const long long in = pos - at;             // < tiles * H
                place.b = b;
                place.h = in < (1LL << 31) ? (int)((uint32_t)in / (uint32_t)tiles) : (int)(in / tiles);
                place.t = (int)(in - (long long)place.h * tiles);
                place.pos = pos;
                place.end = end;
            }
        }
        tc_fence_before();
        __syncthreads();
        w0 = place;
    } else if constexpr (MODE == 1 || MODE == 3) {
        int32_t *before = reinterpret_cast<int32_t *>(gbase + C::kOffMisc + (C::kSmemBytes - 1024 - C::kOffMisc));
        for (int v = tid; v < a.blocks; v += C::kThreads) {
            Block k;
            before[v + 1] = find_unit<MODE>(a, QC / a.G, v, blockIdx.x == 0, k) ? unit_cost(MODE) + tiles_of(k.live) : 0;
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
        const long long total = (long long)per_head * a.H, share = (total + gridDim.x - 1) / gridDim.x;
        w0.before = before;
        w0.pos = share * blockIdx.x;
        w0.end = min(total, w0.pos + share);
        w0.per_head = per_head;
        if (tid == 0 && blockIdx.x == 0) *reinterpret_cast<long long *>(a.ws) = share;
        if (MODE == 1 && tid == 0) reinterpret_cast<CtaMeta *>(a.ws + 16)[blockIdx.x].tiles = 0;
        if (MODE == 3 && blockIdx.x == 0)                  // the join finds the units' parts by these
            for (int v = tid; v <= a.blocks; v += C::kThreads) reinterpret_cast<int32_t *>(a.ws + 16)[v] = before[v];
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
        w0.done = false;
    }
    if constexpr (MODE != 0) {                             // (MODE 0 has just met)
        tc_fence_before();
        __syncthreads();
    }
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(tmem_slot);
    const uint32_t tmem_s = tmem, tmem_o = tmem + 2 * NS;

    bool dead = false;                                    // a bounded wait gave up: no further waits, run out
    auto wait = [&](uint32_t bar, uint32_t parity, unsigned int code) {
        if (dead || mbar_try_wait(bar, parity)) return;
        if (*abort_flag || !mbar_wait(bar, parity, a.wait_limit)) {
            if (!*abort_flag) atomicExch(a.status, code);
            *abort_flag = 1;
            dead = true;
        }
    };

    if (warp == kWarpTma) {
        // ------------------------------------------------------------------------ producer: pages by TMA, scales
        const int lg_ppt = 7 - a.page_shift, ppt = 1 << lg_ppt;               // pages of a tile
        const int tiles_batch = 32 >> lg_ppt;                                 // a lane looks after one page of the next 32
        Work<MODE> w = w0;
        Segment s;
        int it = 0, issued_k = 0, issued_v = 0;
        while (w.next(a, QC, s)) {
            const int32_t *row = a.table + (size_t)s.b * a.W;
            auto fetch = [&](int t_first, int &id, float &ks, float &vs) {
                const long long p_live = ((long long)t_first << lg_ppt) + lane, p = MODE >= 3 ? s.page0 + p_live : p_live;
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
            float ks, vs, ks_next, vs_next, v_ref = 0.f;
            bool far = false;
            fetch(s.t0, id, ks, vs);
            for (int tb = s.t0; tb < s.t1; tb += tiles_batch) {
                fetch(tb + tiles_batch, id_next, ks_next, vs_next);
                const int tn = min(tiles_batch, s.t1 - tb);
                for (int i = 0; i < tn; ++i, ++it) {
                    const int st = it % KST, sv = it % VST;
                    wait(kempty(st), ((uint32_t)(it / KST) & 1u) ^ 1u, kErrAttnTma);
                    const bool mine = (lane >> lg_ppt) == i;
                    const int k = lane & (ppt - 1);
                    const uint32_t have = __ballot_sync(0xffffffffu, mine && id >= 0) >> (i << lg_ppt);
                    const uint32_t bytes = (uint32_t)__popc(have) * (uint32_t)(page * kHeadDim);
                    dead = __any_sync(0xffffffffu, dead);
                    if (dead) continue;
                    const int y = (id * a.H + s.h) << a.page_shift;
                    const uint32_t off = (uint32_t)(k << a.page_shift) * kHeadDim;
                    if (mine && id >= 0) {
                        tma_load_2d(k_tile(st) + off, &map_k, kfull(st), 0, y);
                        if (!C::WIDE) tma_load_2d(v_tile(sv) + off, &map_v, vfull(sv), 0, y);
                    }
                    // the scales (their loads may still be on their way) before the barrier's own arrival.  Their room is free: the
                    // softmax warps are done with the tile that had it (wide: they gave its V's room, which the tile before this
                    // one has taken, so KST is at most VST + 1)
                    float *sc = stage_ks + st * 32;
                    const float v_abs = fabsf(vs), v_max = warp_max(mine ? v_abs : 0.f);
                    if (v_ref == 0.f || v_max > v_ref * kScaleUp) {
                        far |= v_ref > 0.f;
                        v_ref = scale_ref(v_max, 0x1p-66f);
                    }
                    far |= __any_sync(0xffffffffu, mine && id >= 0 && !(v_abs >= v_ref * (1.f / kScaleNear) && v_abs <= v_ref * kScaleNear));
                    if (mine) {
                        sc[k] = ks;
                        sc[8 + k] = vs;
                    }
                    if (lane == 0) {
                        sc[16] = v_ref;
                        reinterpret_cast<uint32_t *>(sc)[24] = have | (far ? 0x80000000u : 0u);
                    }
                    __syncwarp();
                    if (lane == 0) {
                        mbar_expect_tx(kfull(st), bytes);
                        if (!C::WIDE) mbar_expect_tx(vfull(sv), bytes);
                    }
                    issued_k = it + 1;
                    if constexpr (C::WIDE) {
                        wait(vempty(sv), ((uint32_t)(it / VST) & 1u) ^ 1u, kErrAttnTma);
                        dead = __any_sync(0xffffffffu, dead);
                        if (dead) continue;
                        if (mine && id >= 0) tma_load_2d(v_tile(sv) + off, &map_v, vfull(sv), 0, y);
                        __syncwarp();
                        if (lane == 0) mbar_expect_tx(vfull(sv), bytes);
                    }
                    issued_v = it + 1;
                }
                id = id_next; ks = ks_next; vs = vs_next;
            }
        }
        if (dead) {                                        // leave no copy in flight behind
            for (int i = max(0, issued_k - KST); i < issued_k; ++i) mbar_wait(kfull(i % KST), (uint32_t)(i / KST) & 1u, a.wait_limit);
            for (int i = max(0, issued_v - VST); i < issued_v; ++i) mbar_wait(vfull(i % VST), (uint32_t)(i / VST) & 1u, a.wait_limit);
        }
    } else if (warp == kWarpMma) {
        // ------------------------------------------------------------------------ MMA issuer
        if (lane == 0) {
            // formats: 0 is e4m3, or f16 in the wide form's second product; 1 e5m2 (operand B: the wide form's second term of q, the
            // narrow form's weights)
            constexpr uint32_t kIdescS = make_idesc(0u, 0u, 0u, NS), kIdescS1 = kIdescS | 1u << 10, kIdescO = make_idesc(0u, 1u, 1u, NO) | (C::WIDE ? 0u : 1u << 10);
            Work<MODE> w = w0;
            Segment s;
            int it = 0;                                    // tiles whose S has been issued
            int last_s = -1, last_o = -1;                  // the last products that were
            uint32_t seg = 0;
            auto scores = [&]() {
                const int st = it % KST;
                wait(kfull(st), (uint32_t)(it / KST) & 1u, kErrAttnMma);
                if (!dead) {
                    tc_fence_after();
#pragma unroll
                    for (int term = 0; term < (C::WIDE ? QT : 1); ++term)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            mma_f8(tmem_s + (it & 1) * NS, desc_kmajor_sw128(k_tile(st) + k * 32),
                                   desc_kmajor_sw128(q_base + term * QC * 128 + k * 32), term ? kIdescS1 : kIdescS, (term | k) ? 1u : 0u);
                    mma_commit(sfull(it & 1));
                    if (C::WIDE) mma_commit(kempty(st));
                    last_s = it;
                }
                ++it;
            };
            auto output = [&](int i, bool first) {
                const int sv = i % VST, pb = i & 1;
                wait(pfull(pb), (uint32_t)(i >> 1) & 1u, kErrAttnMma);
                if (!C::WIDE) wait(vfull(sv), (uint32_t)(i / VST) & 1u, kErrAttnMma);
                if (!dead) {
                    tc_fence_after();
                    if constexpr (C::WIDE) {
#pragma unroll
                        for (int k = 0; k < 8; ++k)        // 16 tokens each
                            mma_bf16(tmem_o, desc_mnmajor_sw128(base + C::kOffH + k * 2048, kTileBytes),
                                     desc_mnmajor_sw128(p_tile(pb) + k * 2048, kTileBytes), kIdescO, (!first || k) ? 1u : 0u);
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            mma_f8(tmem_o, desc_mnmajor_sw128(v_tile(sv) + k * 4096, kTileBytes),
                                   desc_mn_rows<C::PW>(p_tile(pb) + k * 32 * C::PW), kIdescO, (!first || k) ? 1u : 0u);
                        mma_commit(kempty(i % KST));
                    }
                    mma_commit(pdone(pb));
                    last_o = i;
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
            // no product may be on its way when the tensor memory is given back (it never is, unless the softmax warps gave up)
            if (last_s >= 0) mbar_wait(sfull(last_s & 1), (uint32_t)(last_s >> 1) & 1u, a.wait_limit);
            if (last_o >= 0) mbar_wait(pdone(last_o & 1), (uint32_t)(last_o >> 1) & 1u, a.wait_limit);
        }
    } else {
        // ------------------------------------------------------------------------ softmax
        const int wg = warp >> 2, row = tid & 127, c_wg = wg * QW;            // this thread's token / channel, its first column
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        constexpr float kTerm = 1.0f / 16.0f, kWeightTerm = 1.0f / 8.0f;
        auto mu_at = [&](int c) -> float & { return C::WIDE ? col[c] : col[(c >> 1) * 4 + 2 + (c & 1)]; };   // -Mu of column c
        const float2 *col_mu = reinterpret_cast<const float2 *>(col);
        const float4 *col4 = reinterpret_cast<const float4 *>(col);           // factors and -Mu of columns 2 p, 2 p + 1
        constexpr int kPart = C::WIDE ? C::PART : QW, kLoad = C::WIDE ? C::PART : NS;  // columns at a time, raw scores of them
        Work<MODE> w = w0;
        Segment s;
        int it = 0;
        while (w.next(a, QC, s)) {
            const int n_cols = s.n_tok * a.G;
            // -- the query columns as e4m3 terms, each column with a power of two of its own
            constexpr int kEach = QC / (4 * WGS);          // columns of a warp: their loads first, then the work
            constexpr int kMaps = FORM == 1 ? 2 : 1;       // columns of a query row
            const T *q_row = static_cast<const T *>(a.q) + (size_t)s.tok0 * a.ld_q + (size_t)s.h * (a.G / kMaps) * kHeadDim + lane * 4;
            float4 q_in[kEach];
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const int c = warp + 4 * WGS * j, tok = c * a.inv_g >> 16;
                q_in[j] = c < n_cols && FAEDKV_IN_BOUNDS(kTagPageAttn, s.tok0 >= 0 && s.tok0 + tok < a.n_tokens) ? load4(q_row + (size_t)tok * a.ld_q + (c - tok * a.G) / kMaps * kHeadDim) : make_float4(0.f, 0.f, 0.f, 0.f);
                if (FORM == 1 && ((c - tok * a.G) & 1) != lane >> 4) q_in[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            }
            uint32_t top[kEach];                           // the columns' largest finite magnitudes
#pragma unroll
            for (int j = 0; j < kEach; ++j)
                top[j] = __reduce_max_sync(0xffffffffu, max(max(finite_bits(q_in[j].x), finite_bits(q_in[j].y)), max(finite_bits(q_in[j].z), finite_bits(q_in[j].w))));
            // Many columns, all within 2^3 of one another (but for zeros): one power of two for all, which stays out of the softmax's
            // inner loop (2048 new tokens over 18432: 969 us; with a factor for each column always 1008).  Else each has its own
            // (1000 us; in a pass over the scores as masks take, 942 and 1331)
            bool common = false;
            float unit_cs = 0.f;
            uint32_t unit_top = 0;
            if constexpr (C::WIDE) {
                uint32_t hi = 0, lo = 0x7fffffffu;
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    hi = max(hi, top[j]);
                    if (top[j] != 0u) lo = min(lo, top[j]);
                }
                if (lane == 0) *reinterpret_cast<uint2 *>(red + 2 * warp) = make_uint2(hi, lo);
                softmax_bar(1, kSoftmax);
#pragma unroll 4
                for (int i = 0; i < 4 * WGS; ++i) {
                    const uint2 r = *reinterpret_cast<const uint2 *>(red + 2 * i);
                    hi = max(hi, r.x);
                    lo = min(lo, r.y);
                }
                softmax_bar(1, kSoftmax);
                common = hi == 0u || scale_for(__uint_as_float(hi)) <= 8.0f * scale_for(__uint_as_float(lo));
                unit_top = hi;
                unit_cs = 2.0f * scale_for(__uint_as_float(hi)) * a.scale_log2;
            }
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const int c = warp + 4 * WGS * j;
                float x[4] = {q_in[j].x, q_in[j].y, q_in[j].z, q_in[j].w};
                const float qs = 2.0f * scale_for(__uint_as_float(common ? unit_top : top[j]));       // the largest element to 112 .. 224
                const float inv = __uint_as_float((254u << 23) - __float_as_uint(qs));
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = fabsf(x[e]) < INFINITY ? x[e] * inv : __uint_as_float(0x7fffffffu);
                if (lane == 0) {
                    col[C::WIDE ? QC + c : (c >> 1) * 4 + (c & 1)] = qs * a.scale_log2;
                    mu_at(c) = 0.f;
                    col_lim[c] = c >= n_cols ? 0 : MODE >= 3 ? s.see0 : s.see0 + (int)(c * a.inv_g >> 16);
                    col_set[c] = c < n_cols ? 0 : 1;
                }
                auto put_codes = [&](int term, uint32_t codes) {
                    const uint32_t r = (uint32_t)(term * QC + c);
                    *reinterpret_cast<uint32_t *>(gbase + C::kOffQ + mn_chunk<128>(r, (uint32_t)lane >> 2) + (lane & 3) * 4) = codes;
                };
                if constexpr (C::WIDE) {
                    // both terms on one grid: what the first leaves of an element above 2^-6 has three significant bits (bf16's eight
                    // less its four, and a sign), which e5m2 holds; of smaller ones e5m2's rounding is at most 2^-14
                    float hi[4];
                    const uint32_t codes = to_e4m3x4(x[0], x[1], x[2], x[3]);
                    from_e4m3x4(codes, hi);
                    put_codes(0, codes);
                    put_codes(1, to_e5m2x4(x[0] - hi[0], x[1] - hi[1], x[2] - hi[2], x[3] - hi[3]));
                } else {
#pragma unroll
                    for (int i = 0; i < QT; ++i) {
                        float t[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (i < QT - 1) {
                                t[e] = lead4(x[e]);
                                x[e] = (x[e] - t[e]) * 16.0f;
                            } else {
                                t[e] = x[e];
                            }
                        }
                        put_codes(i, to_e4m3x4(t[0], t[1], t[2], t[3]));
                    }
                }
            }
            if constexpr (!C::WIDE && NS > QC * QT)
                for (int r = QC * QT + warp; r < NS; r += 4)
                    *reinterpret_cast<uint32_t *>(gbase + C::kOffQ + r * 128 + lane * 4) = 0u;
            fence_proxy_async();
            softmax_bar(1, kSoftmax);                      // the col arrays are read by all warps
            if (lane == 0) mbar_arrive(qfull);

            float2 l[QW / 2];
#pragma unroll
            for (int p = 0; p < QW / 2; ++p) l[p] = make_float2(0.f, 0.f);
            unsigned long long poison = 0;                 // columns (of the warpgroup) whose channel `row` met a NaN value
            static_assert(!C::WIDE || QW == 32, "four chunks of eight columns a warpgroup");
            // wide: where this row's first chunk of eight weights lies (64 columns a block of 128-byte rows); k further: bits 4, 5
            const uint32_t p_off = (c_wg >> 6) * kTileBytes + mn_chunk<128>(row, (uint32_t)(c_wg & 63) >> 3);
            bool unset_any = true;                         // some column's Mu does not stand for a maximum yet
            float v_ref = 0.f, v_inv = 0.f;

            for (int t = s.t0; t < s.t1; ++t, ++it) {
                const int st = it % KST, sv = it % VST, pb = it & 1;
                bool done_max = false;                     // Mu has been set by this tile's maxima
                // the scores of this tile are complete: so are its K copy, behind which the scales were written, and the
                // output product of two tiles ago, issued before these scores, which read this tile's weight buffer
                wait(sfull(it & 1), (uint32_t)(it >> 1) & 1u, kErrAttnSoftmax);
                tc_fence_after();
                const float *sc = stage_ks + st * 32;
                const int pg = row >> a.page_shift;
                const float ks = sc[pg], vs = sc[8 + pg], v_now = sc[16];
                const uint32_t have = reinterpret_cast<const uint32_t *>(sc)[24];
                const int tok = t * kTile + row;
                // columns may see a different number of this tile's tokens, pages may be missing, or the segment is far
                const bool masked = (t + 1) * kTile > s.see0 || have != (1u << (kTile >> a.page_shift)) - 1u;
                const bool valid = tok < s.live && ((have >> pg) & 1u);
                const uint32_t ts = tmem_s + (it & 1) * NS + lane_addr + c_wg;
                float kf = C::WIDE ? ks * unit_cs : ks;
                if (masked) {
                    // a pass of its own over the scores, which leaves them multiplied by their factor, or minus infinity: the loop
                    // below need not know of masks
#pragma unroll 1
                    for (int c0 = 0; c0 < QW; c0 += 8) {
                        constexpr int kTerms = C::WIDE ? 1 : QT;
                        float v[8 * kTerms];
#pragma unroll
                        for (int i = 0; i < kTerms; ++i) tmem_ld8(ts + i * QC + c0, v + 8 * i);
                        tmem_ld_done<8 * kTerms>(v);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
#pragma unroll
                            for (int i = kTerms - 2; i >= 0; --i) v[8 * i + e] = fmaf(v[8 * (i + 1) + e], kTerm, v[8 * i + e]);
                            const float f = C::WIDE ? ks * col[QC + c_wg + c0 + e] : ks;
                            v[e] = valid && tok < col_lim[c_wg + c0 + e] ? v[e] * f : -INFINITY;
#pragma unroll
                            for (int i = 1; i < kTerms; ++i) v[8 * i + e] = 0.f;
                        }
#pragma unroll
                        for (int i = 0; i < kTerms; ++i) tmem_st8(ts + i * QC + c0, v + 8 * i);
                    }
                    tmem_st_wait();
                    kf = 1.f;
                }
                const bool own = C::WIDE && !masked && !common;            // each column's factor is still to come
                if (own) kf = ks;
                const float2 ks2 = make_float2(kf, kf);
                // a column without a maximum, v_scales far apart: Mu is settled before the weights are taken
                bool raise = unset_any || (int32_t)have < 0;
                float o_factor = 1.f;
                if (v_now != v_ref) {
                    if (v_ref > 0.f) o_factor = v_ref / v_now;
                    v_ref = v_now;
                    v_inv = __fdiv_rn(1.f, v_now);
                }
                const float2 r2 = make_float2(vs * v_inv, vs * v_inv);
                // y of the columns c_wg + c0 .. from their raw scores
                auto exponents = [&](const float(&raw)[kLoad], int c0, float2(&y)[kPart / 2]) {
                    if (C::WIDE && own) {
#pragma unroll
                        for (int p = 0; p < kPart / 2; ++p)
                            y[p] = fma2(make_float2(raw[2 * p], raw[2 * p + 1]), mul2(ks2, col_mu[(QC + c_wg + c0) / 2 + p]), col_mu[(c_wg + c0) / 2 + p]);
                        return;
                    }
#pragma unroll
                    for (int p = 0; p < kPart / 2; ++p) {
                        float2 v;
                        if constexpr (C::WIDE) {
                            v = make_float2(raw[2 * p], raw[2 * p + 1]);
                        } else {
                            v = make_float2(raw[(QT - 1) * QC + 2 * p], raw[(QT - 1) * QC + 2 * p + 1]);
#pragma unroll
                            for (int i = QT - 2; i >= 0; --i)
                                v = fma2(v, make_float2(kTerm, kTerm), make_float2(raw[i * QC + 2 * p], raw[i * QC + 2 * p + 1]));
                        }
                        if constexpr (C::WIDE) {
                            y[p] = fma2(v, ks2, col_mu[(c_wg + c0) / 2 + p]);
                        } else {
                            const float4 fm = col4[(c_wg + c0) / 2 + p];
                            y[p] = fma2(v, mul2(ks2, make_float2(fm.x, fm.y)), make_float2(fm.z, fm.w));
                        }
                    }
                };
                uint8_t *prow = gbase + C::kOffP + pb * C::kPBytes;
                // weights, their sum, what the product takes of them; returns the largest exponent
                auto weights = [&](auto repeat) {
                    float excess = -INFINITY;
                    float raw[2][kLoad];
                    tmem_ld<kLoad>(ts, raw[0]);
                    tmem_ld_done<kLoad>(raw[0]);
#pragma unroll
                    for (int c0 = 0; c0 < QW; c0 += kPart) {
                        float2 y[kPart / 2];
                        float(&now)[kLoad] = raw[c0 / kPart & 1], (&next)[kLoad] = raw[(c0 / kPart + 1) & 1];
                        if (c0 + kPart < QW) tmem_ld<kLoad>(ts + c0 + kPart, next);   // the next columns' scores on their way
                        exponents(now, c0, y);
#pragma unroll
                        for (int p = 0; p < kPart / 2; ++p) {
                            excess = max3(excess, y[p].x, y[p].y);
                            y[p] = make_float2(ex2(y[p].x), ex2(y[p].y));
                            float2 &sum = l[c0 / 2 + p];
                            if (!decltype(repeat)::value) {
                                sum = add2(sum, y[p]);
                            } else {                       // this tile is in the sum already, unless that was dropped
                                const float2 f = *reinterpret_cast<const float2 *>(col_f + c_wg + c0 + 2 * p);
                                if (f.x == 0.f) sum.x = y[p].x;
                                if (f.y == 0.f) sum.y = y[p].y;
                            }
                            y[p] = mul2(y[p], r2);
                        }
                        if constexpr (C::WIDE) {
#pragma unroll
                            for (int j = 0; j < kPart; j += 8) {
                                uint32_t u[4];
#pragma unroll
                                for (int k = 0; k < 4; ++k) u[k] = pack_f16(y[j / 2 + k].x, y[j / 2 + k].y);
                                *reinterpret_cast<uint4 *>(prow + (p_off ^ (uint32_t)((c0 + j) >> 3 << 4))) = make_uint4(u[0], u[1], u[2], u[3]);
                            }
                        } else {
                            const float2 eight = make_float2(8.f, 8.f);
                            uint32_t u[NO / 4];
#pragma unroll
                            for (int i = 0; i < NO / 4; ++i) u[i] = 0u;
#pragma unroll
                            for (int i = 0; i < PT; ++i)
#pragma unroll
                                for (int j = 0; j < QC; j += 4) {
                                    float2 h[2];
#pragma unroll
                                    for (int e = 0; e < 2; ++e) {
                                        float2 &v = y[j / 2 + e];
                                        h[e] = v;
                                        if (i < PT - 1) {
                                            h[e] = make_float2(lead3(v.x), lead3(v.y));
                                            v = mul2(sub2(v, h[e]), eight);
                                        }
                                    }
                                    u[(i * QC + j) / 4] = to_e5m2x4(h[0].x, h[0].y, h[1].x, h[1].y);
                                }
#pragma unroll
                            for (int k = 0; k < NO / 16; ++k)
                                *reinterpret_cast<uint4 *>(prow + mn_chunk<C::PW>(row, k)) = make_uint4(u[4 * k], u[4 * k + 1], u[4 * k + 2], u[4 * k + 3]);
                        }
                        if (c0 + kPart < QW) tmem_ld_done<kLoad>(next);
                    }
                    return excess;
                };
                bool again = false;
                for (;;) {
                    if (raise) {
                        const bool far = (int32_t)have < 0;
                        // Mu to kLagTo below the column maxima, and what has been summed rescaled
                        if (t > s.t0) wait(pdone((it - 1) & 1), (uint32_t)((it - 1) >> 1) & 1u, kErrAttnSoftmax);
                        const float lift = fmaxf(__log2f(fabsf(r2.x)), kScaleDown);
#pragma unroll 1
                        for (int c0 = 0; c0 < QW; c0 += kPart) {
                            float raw[kLoad];
                            float2 y[kPart / 2];
                            tmem_ld<kLoad>(ts + c0, raw);
                            tmem_ld_done<kLoad>(raw);
                            exponents(raw, c0, y);
#pragma unroll
                            for (int p = 0; p < kPart / 2; ++p) {
                                const float m0 = warp_max(y[p].x + lift), m1 = warp_max(y[p].y + lift);
                                if (lane == 0) *reinterpret_cast<float2 *>(red + (warp & 3) * QC + c_wg + c0 + 2 * p) = make_float2(m0, m1);
                            }
                        }
                        softmax_bar(2 + wg, 128);
                        bool unset = false;
                        if (row < QW) {
                            const int c = c_wg + row;
                            const float m = fmaxf(fmaxf(red[c], red[QC + c]), fmaxf(red[2 * QC + c], red[3 * QC + c])) - C::kLagTo;
                            const bool first = col_set[c] == 0, seen = m > -INFINITY;
                            const float d = !seen || !(first || m > 0.f) ? 0.f : far ? 2.f * ceilf(0.5f * m) : m;
                            mu_at(c) -= d;
                            // 1: nothing has been summed yet; 0: what has been is beyond float32's reach, or was summed as infinity
                            // (p of a tile that is taken again reaches 2^(d + kLagTo + 20)).  Far: no tile is, but sums reach 2^75 and more, which
                            // factors down to float32's least subnormal, powers of two, bring to where new weights leave them nothing
                            const float root = ex2(-0.5f * d);
                            col_f[c] = first ? 1.f : far ? __fmul_rn(root, root) : d > 96.f ? 0.f : ex2(-d);
                            if (seen) col_set[c] = 1;
                            unset = first && !seen;
                        }
                        unset_any = softmax_any(unset, 2 + wg, 128);
#pragma unroll
                        for (int p = 0; p < QW / 2; ++p) l[p] = mul2(l[p], *reinterpret_cast<const float2 *>(col_f + c_wg + 2 * p));
                    }
                    if (t > s.t0 && (raise || o_factor != 1.f)) {
                        if (!raise) wait(pdone((it - 1) & 1), (uint32_t)((it - 1) >> 1) & 1u, kErrAttnSoftmax);
                        tc_fence_after();
                        constexpr int kCols = C::WIDE ? QW : NO;
#pragma unroll 1
                        for (int c0 = 0; c0 < kCols; c0 += 16) {
                            float o[16];
                            tmem_ld<16>(tmem_o + lane_addr + c_wg + c0, o);
                            tmem_ld_done<16>(o);
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] *= (raise ? col_f[(c_wg + c0 + e) % QC] : 1.f) * o_factor;
                            tmem_st16(tmem_o + lane_addr + c_wg + c0, o);
                        }
                        tmem_st_wait();
                    }
                    o_factor = 1.f;
                    if (raise) {
                        done_max = true;
                        raise = false;
                    }
                    const float excess = again ? weights(std::true_type{}) : weights(std::false_type{});
                    // a weight beyond its format's range: raise Mu, and the weights once more
                    if (done_max || !softmax_any(ex2(excess) * fabsf(r2.x) > C::kMostWeight, 2 + wg, 128)) break;
                    raise = again = true;
                }
                uint8_t *vtile = gbase + C::kOffV + (uint32_t)sv * kTileBytes;
                // some columns see a token of this tile that others do not
                const bool ragged = (MODE == 1 || MODE == 2) && s.n_tok > 1 && (t + 1) * kTile > s.see0;
                const int n_live = min(kTile, s.live - t * kTile);
                auto cell = [&](int r) { return vtile + mn_chunk<128>(r, (uint32_t)row >> 4) + (row & 15); };
                auto note_nan = [&](int r) {               // the columns that see token r
                    const int c = max(0, max(0, t * kTile + r + 1 - s.see0) * a.G - c_wg);   // the first of them
                    if (c < 64) poison |= ~0ull << c;
                };
                if constexpr (C::WIDE) {
                    // this thread's share of the V tile in f16: WGS threads a token.  The product of the tile before read the buffer
                    wait(vfull(sv), (uint32_t)(it / VST) & 1u, kErrAttnSoftmax);
                    if (t > s.t0) wait(pdone((it - 1) & 1), (uint32_t)((it - 1) >> 1) & 1u, kErrAttnSoftmax);
                    bool nan = false;
                    uint8_t *to = gbase + C::kOffH + (wg >> 1) * kTileBytes;     // 64 channels a block
                    if (!masked) {
#pragma unroll
                        for (int j = 2 * wg; j < 2 * wg + 2; ++j) {              // 16 channels
                            const uint4 v = *reinterpret_cast<const uint4 *>(vtile + mn_chunk<128>(row, j));
                            const uint4 lo = make_uint4(e4m3x2_to_f16x2(v.x), e4m3x2_to_f16x2(v.x >> 16), e4m3x2_to_f16x2(v.y), e4m3x2_to_f16x2(v.y >> 16));
                            const uint4 hi = make_uint4(e4m3x2_to_f16x2(v.z), e4m3x2_to_f16x2(v.z >> 16), e4m3x2_to_f16x2(v.w), e4m3x2_to_f16x2(v.w >> 16));
                            *reinterpret_cast<uint4 *>(to + mn_chunk<128>(row, (2 * j) & 7)) = lo;
                            *reinterpret_cast<uint4 *>(to + mn_chunk<128>(row, (2 * j + 1) & 7)) = hi;
                        }
                    } else {
                        // 0 * NaN is not 0: values behind the end must not reach the product, nor a NaN value of a token that some
                        // columns see and others do not: that one is noted for the columns that see it
#pragma unroll 1
                        for (int i = 0; i < 8; ++i) {                            // four channels
                            const int j = 2 * wg + (i >> 2);
                            const uint32_t u = *reinterpret_cast<const uint32_t *>(vtile + mn_chunk<128>(row, j) + (i & 3) * 4);
                            const uint32_t is_nan = __vcmpeq4(u & 0x7f7f7f7fu, 0x7f7f7f7fu), drop = !valid ? 0xffffffffu : ragged ? is_nan : 0u;
                            nan |= valid && is_nan != 0u;
                            *reinterpret_cast<uint2 *>(to + mn_chunk<128>(row, (2 * j + (i >> 1 & 1)) & 7) + (i & 1) * 8) =
                                make_uint2(e4m3x2_to_f16x2(u) & ~__byte_perm(drop, 0u, 0x1100), e4m3x2_to_f16x2(u >> 16) & ~__byte_perm(drop, 0u, 0x3322));
                        }
                    }
                    if (ragged && softmax_any(nan, 1, kSoftmax))
                        for (int r = 0; r < n_live; ++r)
                            if (((have >> (r >> a.page_shift)) & 1u) && (*cell(r) & 0x7f) == 0x7f) note_nan(r);
                } else {
                    if (masked) wait(vfull(sv), (uint32_t)(it / VST) & 1u, kErrAttnSoftmax);   // it is read and written below
                    if (masked && !valid) {                // 0 * NaN is not 0
#pragma unroll
                        for (int k = 0; k < 8; ++k) reinterpret_cast<uint4 *>(vtile + row * 128)[k] = make_uint4(0u, 0u, 0u, 0u);
                    }
                    if (ragged) {
                        bool nan = false;
                        if (valid) {
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const uint4 v = reinterpret_cast<const uint4 *>(vtile + row * 128)[k];
                                const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                for (int e = 0; e < 4; ++e) nan |= __vcmpeq4(u[e] & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0u;
                            }
                        }
                        if (softmax_any(nan, 1, kSoftmax)) {
                            for (int r = 0; r < n_live; ++r)
                                if ((*cell(r) & 0x7f) == 0x7f) {
                                    note_nan(r);
                                    *cell(r) = 0;
                                }
                        }
                    }
                }
                fence_proxy_async();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (warp != 0 || it + 1 != a.withhold) mbar_arrive(pfull(pb));
                    if (C::WIDE) mbar_arrive(vempty(sv));
                }
            }

            // -- the segment's end: sums over the 128 token rows, then this thread's channel of every column
#pragma unroll
            for (int p = 0; p < QW / 2; ++p) {
                float2 v = l[p];
#pragma unroll
                for (int o = 16; o; o >>= 1) {
                    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
                    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
                }
                if (lane == 0) *reinterpret_cast<float2 *>(red + (warp & 3) * QC + c_wg + 2 * p) = v;
            }
            if (s.t1 > s.t0) wait(pdone((it - 1) & 1), (uint32_t)((it - 1) >> 1) & 1u, kErrAttnSoftmax);
            tc_fence_after();
            softmax_bar(1, kSoftmax);
            const bool whole = MODE == 2 || MODE == 4 || (s.t0 == 0 && s.t1 == s.tiles);
            float *slot = nullptr;
            // MODE 3 and 4: a whole unit's columns beside the rows that they belong to, for the join
            const SharedParts parts(a.whole, (size_t)a.B * a.H * a.G, s.own);
            if (MODE >= 3 && whole) {
                for (int c = tid; c < n_cols; c += kSoftmax) {
                    const float sum = red[c] + red[QC + c] + red[2 * QC + c] + red[3 * QC + c];
                    const int k = c * a.inv_g >> 16;
                    if (!FAEDKV_IN_BOUNDS(kTagPageAttn, s.tok0 + k < a.B && s.h < a.H)) continue;
                    parts.stat[((size_t)(s.tok0 + k) * a.H + s.h) * a.G + (c - k * a.G)] = make_float2(sum == 0.f ? kMuNone : -mu_at(c), sum);
                }
            }
            if (!whole) {
                float *slots = MODE == 3 ? a.slots : reinterpret_cast<float *>(a.ws + attn_meta_bytes(MODE, (size_t)a.B * a.H, gridDim.x));
                slot = slots + ((size_t)blockIdx.x * 2 + (s.t0 > 0 ? 0 : 1)) * attn_slot_floats(QC);
                for (int c = tid; c < n_cols; c += kSoftmax) {
                    const float sum = red[c] + red[QC + c] + red[2 * QC + c] + red[3 * QC + c];
                    slot[c] = sum == 0.f ? kMuNone : -mu_at(c);
                    slot[QC + c] = sum;
                }
            }
            if (MODE == 0 && s.t0 == 0 && tid == 0) {      // where the join finds the unit's parts
                UnitMeta *m = reinterpret_cast<UnitMeta *>(a.ws + 16) + (size_t)s.b * a.H + s.h;
                m->first = s.first;
                m->tiles = s.tiles;
            }
            if (MODE == 1 && s.t0 > 0 && tid == 0) reinterpret_cast<CtaMeta *>(a.ws + 16)[blockIdx.x] = CtaMeta{s.first, s.tiles, s.tok0, n_cols, s.h};
            // where a column's results go: the token's row of the output, or the column of the slot
            for (int c = tid; c < QC; c += kSoftmax) {
                const int k = c * a.inv_g >> 16;
                col_lim[c] = whole ? (k * a.H * a.G + (c - k * a.G)) * kHeadDim : c * kHeadDim;
            }
            for (int c = tid; c < QC; c += kSoftmax) {
                const float sum = red[c] + red[QC + c] + red[2 * QC + c] + red[3 * QC + c];
                col_f[c] = sum == 0.f ? 0.f : __frcp_rn(sum);
            }
            softmax_bar(1, kSoftmax);
            using Out = std::conditional_t<MODE >= 3, float, typename AttnOut<C, FORM>::T>;
            Out *out_row = static_cast<Out *>(MODE >= 3 ? parts.o : a.out) + ((size_t)s.tok0 * a.H + s.h) * a.G * kHeadDim + row;
            float *part_row = whole ? nullptr : slot + 2 * QC + row;
            auto put = [&](int c, float v) {
                if (c >= n_cols || !FAEDKV_IN_BOUNDS(kTagPageAttn, !whole || s.tok0 + (int)(c * a.inv_g >> 16) < a.n_tokens)) return;
                const float f = col_f[c];
                v = f == 0.f ? 0.f : v * f * v_ref;        // no token: zero
                if (MODE != 0 && poison != 0 && ((poison >> (c - c_wg)) & 1ull)) v = __uint_as_float(0x7fffffffu);
                if (whole) store1(out_row + col_lim[c], v);
                else part_row[col_lim[c]] = v;
            };
            if constexpr (C::WIDE) {
#pragma unroll 1
                for (int c0 = 0; c0 < QW; c0 += 16) {
                    float o[16];
                    tmem_ld<16>(tmem_o + lane_addr + c_wg + c0, o);
                    tmem_ld_done<16>(o);
#pragma unroll
                    for (int e = 0; e < 16; ++e) put(c_wg + c0 + e, o[e]);
                }
            } else {
                float o[NO];
                tmem_ld<NO>(tmem_o + lane_addr, o);
                tmem_ld_done<NO>(o);
#pragma unroll
                for (int c = 0; c < QC; ++c) {
                    float v = o[(PT - 1) * QC + c];
#pragma unroll
                    for (int i = PT - 2; i >= 0; --i) v = fmaf(v, kWeightTerm, o[i * QC + c]);
                    put(c, v);
                }
            }
            tc_fence_before();
            softmax_bar(1, kSoftmax);                      // red and the col arrays are free for the next segment
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == kWarpMma) {
        tc_fence_after();
        tmem_dealloc(tmem, C::kTmemCols);
    }
    if (MODE >= 3 && a.which == 2) pdl_wait();             // the join waits for this launch, and by it for the other
}

// Joins the partial results of a unit: rescaled to the largest Mu, summed in order, divided.  They lie in the slots of the
// consecutive CTAs that shared the unit, the first one in its second slot (a part that begins a unit), the others in their
// first.  Grid: MODE 0 (units, columns); MODE 1 (CTAs, groups of `each` columns), where the second CTA of a shared unit is the
// one that looks after it.  Four threads per channel share the parts or the columns.
constexpr int kJoinGroups = 4;
template <typename T, int MODE>
__global__ void __launch_bounds__(kHeadDim *kJoinGroups) k_page_attn_join(const AttnArgs a, const int qc, const int each, const int ctas) {
    pdl_wait();
    const int d = threadIdx.x, grp = threadIdx.y;
    const long long share = *reinterpret_cast<const long long *>(a.ws);
    long long first;
    int tiles, tok0, n_cols, h;
    if constexpr (MODE == 0) {
        const UnitMeta m = reinterpret_cast<const UnitMeta *>(a.ws + 16)[blockIdx.x];
        first = m.first; tiles = m.tiles;
        h = blockIdx.x % a.H; tok0 = blockIdx.x / a.H; n_cols = a.G;
    } else {
        const CtaMeta m = reinterpret_cast<const CtaMeta *>(a.ws + 16)[blockIdx.x];
        first = m.first; tiles = m.tiles;
        h = m.h; tok0 = m.tok0; n_cols = m.n_cols;
        if (tiles == 0) return;                            // this CTA began with a unit of its own
    }
    auto cta_of = [&](long long pos) { return pos < (1LL << 31) && share < (1LL << 31) ? (int)((uint32_t)pos / (uint32_t)share) : (int)(pos / share); };
    const int cta0 = cta_of(first), cta1 = cta_of(first + tiles - 1);
    if (MODE == 0 ? cta0 == cta1 : cta0 + 1 != (int)blockIdx.x) return;       // one CTA had it all; another one's join
    const int n = cta1 - cta0 + 1;
    if (!FAEDKV_IN_BOUNDS(kTagPageAttn, cta0 >= 0 && cta1 < ctas)) return;
    const float *slots = reinterpret_cast<const float *>(a.ws + attn_meta_bytes(MODE, (size_t)a.B * a.H, ctas));
    auto slot = [&](int i) { return slots + (size_t)(2 * (cta0 + i) + (i == 0 ? 1 : 0)) * attn_slot_floats(qc); };
    auto store = [&](int c, float o) {
        const int tok = c / a.G;
        if (!FAEDKV_IN_BOUNDS(kTagPageAttn, tok0 >= 0 && tok0 + tok < a.n_tokens && h >= 0 && h < a.H)) return;
        store1(static_cast<T *>(a.out) + (((size_t)(tok0 + tok) * a.H + h) * a.G + (c - tok * a.G)) * kHeadDim + d, o);
    };
    const int c_end = min((int)(blockIdx.y + 1) * each, n_cols);
    if constexpr (MODE == 1) {
        // four columns a thread (c, c + 4, ...: `each` is 16), so that their loads are on the way together
        const int c0 = blockIdx.y * each + grp;
        float mu[4], sum[4], o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) { mu[k] = kMuNone; sum[k] = 0.f; o[k] = 0.f; }
#pragma unroll 2
        for (int i = 0; i < n; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int c = c0 + kJoinGroups * k;
                if (c < c_end) mu[k] = fmaxf(mu[k], slot(i)[c]);
            }
#pragma unroll 2
        for (int i = 0; i < n; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int c = c0 + kJoinGroups * k;
                if (c < c_end) {
                    const float *p = slot(i);
                    const float l = fade(p[qc + c], p[c] - mu[k]);             // a part's output is divided by its sum already
                    sum[k] += l;
                    o[k] = fmaf(p[2 * qc + (size_t)c * kHeadDim + d], l, o[k]);
                }
            }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int c = c0 + kJoinGroups * k;
            if (c < c_end) store(c, sum[k] == 0.f ? 0.f : __fdiv_rn(o[k], sum[k]));
        }
    } else {
        // 128 parts at a time: their Mu and sums by one thread each, then a thread adds up its channel of every fourth part
        __shared__ float f_s[kHeadDim], red_s[2][4], o_s[kJoinGroups][kHeadDim];
        for (int c = blockIdx.y * each; c < c_end; ++c) {
            float mu = kMuNone, sum = 0.f, o = 0.f;
            for (int i0 = 0; i0 < n; i0 += kHeadDim) {
                const int k = min(kHeadDim, n - i0);
                float m = kMuNone, l = 0.f;
                if (grp == 0) {
                    if (d < k) {
                        const float *p = slot(i0 + d);
                        m = p[c];
                        l = p[qc + c];
                    }
                    const float wm = warp_max(m);
                    if ((d & 31) == 0) red_s[0][d >> 5] = wm;
                }
                __syncthreads();
                const float top = fmaxf(mu, fmaxf(fmaxf(red_s[0][0], red_s[0][1]), fmaxf(red_s[0][2], red_s[0][3])));
                const float back = mu - top;
                if (grp == 0) {
                    l = fade(l, m - top);
                    f_s[d] = l;
#pragma unroll
                    for (int s = 16; s; s >>= 1) l += __shfl_xor_sync(0xffffffffu, l, s);
                    if ((d & 31) == 0) red_s[1][d >> 5] = l;
                }
                __syncthreads();
                sum = fade(sum, back) + (red_s[1][0] + red_s[1][1]) + (red_s[1][2] + red_s[1][3]);
                o = fade(o, back);
                mu = top;
#pragma unroll 8
                for (int i = grp; i < k; i += kJoinGroups) o = fmaf(slot(i0 + i)[2 * qc + (size_t)c * kHeadDim + d], f_s[i], o);
                __syncthreads();
            }
            o_s[grp][d] = o;
            __syncthreads();
            if (grp == 0) store(c, sum == 0.f ? 0.f : __fdiv_rn((o_s[0][d] + o_s[1][d]) + (o_s[2][d] + o_s[3][d]), sum));
            __syncthreads();
        }
    }
}

}  // namespace pages
}  // namespace faedkv
