// Instances and launches of the attention kernel, for the calls that are attention over the paged 8-bit cache.
#pragma once
#include "pages_host.cuh"
#include "k_page_attn.cuh"
#include "k_page_rows.cuh"

namespace {

//                                  type           columns, warpgroups, terms of q and w, wide, columns at a time, tiles of K and V, CTAs per SM
using DecodeBf16 = pages::AttnCfg<__nv_bfloat16, 8, 1, 2, 4, false, 8, 3, 3, 2>;
using DecodeF32 = pages::AttnCfg<float, 8, 1, 6, 8, false, 8, 2, 2, 2>;
using ChunkBf16 = pages::AttnCfg<__nv_bfloat16, 128, 4, 2, 1, true, 8, 3, 2, 1>;
constexpr int kDecodeCtas = DecodeBf16::CTAS;
static_assert(kDecodeCtas == DecodeF32::CTAS && DecodeF32::QC == 8 && DecodeBf16::QC == 8, "one plan for both types");

// How a call is cut up.
struct AttnPlan {
    bool wide;               // 128 columns a unit instead of 8
    int qc, blocks;          // columns of a unit; blocks of new tokens, at most
    bool shared;             // blocks few enough for their tiles to be shared out evenly (MODE 1); else a CTA each (MODE 2)
    long long max_tiles;     // of a table row
    int ctas0, ctas1;        // MODE 0 and 1
    size_t bytes0, bytes1;   // workspace of MODE 0, of the others
};

// gq: query columns of a token and kv head.  wide: whether blocks of many columns may be taken.
[[maybe_unused]] AttnPlan plan_attn(const faedkv_pages *pg, int gq, int batch, int n_tokens, bool wide = true) {
    const faedkv_pages_config &c = pg->cfg;
    AttnPlan p{};
    p.max_tiles = ((long long)c.max_pages * c.page_size + pages::kTile - 1) / pages::kTile;
    // more than 8 query columns a sequence on average: blocks of 128 columns, which read the cache once for all of theirs.  The host
    // does not know how the tokens lie: where every sequence has as many, blocks of 8 stay ahead to 16 columns or 24 (16 x 16384
    // tokens, 8 kv heads: 115 us in 8s and 244 in 128s at 8 columns, 185 and 246 at 16, 266 and 247 at 24), but one long chunk
    // among decoding requests would go over its cache once for every 8 of them (120 tokens over 65536 beside 63 requests of 1000, 11
    // columns on average: 803 and 343 us; 320 tokens, 24 on average: 1973 and 650), so the rule leans to the side that loses less
    p.wide = wide && c.kv_dtype == FAEDKV_BF16 && (long long)n_tokens * gq > 8LL * batch;
    p.qc = p.wide ? ChunkBf16::QC : 8;
    p.blocks = n_tokens / (p.qc / gq) + batch;
    p.shared = p.blocks <= pages::kMaxBlocks && p.blocks * (p.max_tiles + pages::kUnitCost) < (1LL << 31);   // (32-bit positions)
    auto ctas = [&](long long units, int per_sm) {
        const long long most = (long long)pg->n_sm * per_sm, tiles = p.max_tiles * units;
        return (int)(tiles < most ? tiles : most);
    };
    auto slots = [&](int n_ctas, int qc) { return (size_t)n_ctas * 2 * pages::attn_slot_floats(qc) * sizeof(float); };
    const long long units0 = (long long)batch * c.n_kv_heads, units1 = (long long)p.blocks * c.n_kv_heads;
    p.ctas0 = ctas(units0, kDecodeCtas);
    p.ctas1 = ctas(units1, p.wide ? ChunkBf16::CTAS : kDecodeCtas);
    p.bytes0 = pages::attn_meta_bytes(0, (size_t)units0, 0) + slots(p.ctas0, 8);
    p.bytes1 = p.shared ? pages::attn_meta_bytes(1, 0, (size_t)p.ctas1) + slots(p.ctas1, p.qc) : 16;
    return p;
}

template <typename C, int MODE, int FORM>
int launch_attn(faedkv_pages *pg, const CUtensorMap &mk, const CUtensorMap &mv, const pages::AttnArgs &a, const AttnPlan &p, int attr_bit,
                cudaStream_t st) {
    auto kernel = pages::k_page_attn<C, MODE, FORM>;
    using Out = typename pages::AttnOut<C, FORM>::T;
    constexpr uint32_t smem = C::kSmemBytes + (MODE == 1 ? C::kSmemBlocks : 0);
    if (!(pg->attr_set & (1u << attr_bit))) {
        CUDA_TRY(pg, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        pg->attr_set |= 1u << attr_bit;
    }
    const dim3 grid = MODE == 0 ? dim3(p.ctas0) : MODE == 1 ? dim3(p.ctas1) : dim3(p.blocks, a.H);
    CUDA_TRY(pg, launch_pdl(kernel, grid, dim3(C::kThreads), smem, st, mk, mv, a));
    if (int r = launch_check(pg, "k_page_attn")) return r;
    if (MODE == 2 || p.max_tiles == 1) return FAEDKV_OK;                     // no unit is ever in parts
    if constexpr (MODE == 0 && FORM == 1) return FAEDKV_OK;                   // the caller puts the parts together
    else if constexpr (MODE != 2) {
        const int cols = MODE == 0 ? a.G : C::QC / a.G * a.G, each = MODE == 0 ? 1 : 16;
        const dim3 jgrid((unsigned)(MODE == 0 ? a.B * a.H : p.ctas1), (cols + each - 1) / each);
        CUDA_TRY(pg, launch_pdl(pages::k_page_attn_join<Out, MODE>, jgrid, dim3(kHeadDim, pages::kJoinGroups), 0, st, a, (int)C::QC,
                                each, MODE == 0 ? p.ctas0 : p.ctas1));
        return launch_check(pg, "k_page_attn_join");
    }
    return FAEDKV_OK;
}

// The form with query columns as rows, for new tokens of bf16 calls: plan and launch.
[[maybe_unused]] AttnPlan plan_rows(const faedkv_pages *pg, int gq, int batch, int n_tokens) {
    AttnPlan p{};
    p.max_tiles = ((long long)pg->cfg.max_pages * pg->cfg.page_size + pages::kTile - 1) / pages::kTile;
    p.wide = true;
    p.qc = pages::kRowsQC;
    p.blocks = n_tokens / (p.qc / gq) + batch;
    p.shared = p.blocks <= pages::kMaxBlocks && p.blocks * (2 * p.max_tiles + pages::kRowsCost) < (1LL << 31);
    const long long tiles = p.max_tiles * p.blocks * pg->cfg.n_kv_heads;
    p.ctas1 = (int)(tiles < pg->n_sm ? tiles : pg->n_sm);
    p.bytes1 = p.shared ? pages::attn_meta_bytes(1, 0, (size_t)p.ctas1) + (size_t)p.ctas1 * 2 * pages::attn_slot_floats(p.qc) * sizeof(float) : 16;
    return p;
}

template <int MODE, int FORM>
int launch_rows(faedkv_pages *pg, const CUtensorMap &mk, const CUtensorMap &mv, const pages::AttnArgs &a, const pages::DiffArgs &diff, dim3 grid,
                int attr_bit, cudaStream_t st) {
    auto kernel = pages::k_page_rows<MODE, FORM>;
    if (!(pg->attr_set & (1u << attr_bit))) {
        cudaFuncAttributes f;                              // the kernel shares its registers out anew: it would wait for ones that the launch has not
        CUDA_TRY(pg, cudaFuncGetAttributes(&f, kernel));
        if (f.numRegs < pages::kRowsRegsLaunch) return fail(pg, FAEDKV_ERR_CUDA, "k_page_rows was built with %d registers", f.numRegs);
        CUDA_TRY(pg, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)pages::kRowsSmem));
        pg->attr_set |= 1u << attr_bit;
    }
    CUDA_TRY(pg, launch_pdl(kernel, grid, dim3(pages::kRowsThreads), pages::kRowsSmem, st, mk, mv, a, diff));
    return launch_check(pg, "k_page_rows");
}

// The instance for a call: by type, new tokens, and how many blocks they make.  bit: the first of eight in attr_set.
template <int FORM>
int dispatch_attn(faedkv_pages *pg, const CUtensorMap &mk, const CUtensorMap &mv, const pages::AttnArgs &a, const AttnPlan &p, int bit, cudaStream_t st) {
    if (pg->cfg.kv_dtype == FAEDKV_F32)
        return a.q_start == nullptr ? launch_attn<DecodeF32, 0, FORM>(pg, mk, mv, a, p, bit, st)
               : p.shared           ? launch_attn<DecodeF32, 1, FORM>(pg, mk, mv, a, p, bit + 1, st)
                                    : launch_attn<DecodeF32, 2, FORM>(pg, mk, mv, a, p, bit + 2, st);
    if (a.q_start == nullptr) return launch_attn<DecodeBf16, 0, FORM>(pg, mk, mv, a, p, bit + 3, st);
    if constexpr (FORM == 0)
        if (p.wide)
            return p.shared ? launch_attn<ChunkBf16, 1, FORM>(pg, mk, mv, a, p, bit + 4, st) : launch_attn<ChunkBf16, 2, FORM>(pg, mk, mv, a, p, bit + 5, st);
    return p.shared ? launch_attn<DecodeBf16, 1, FORM>(pg, mk, mv, a, p, bit + 6, st) : launch_attn<DecodeBf16, 2, FORM>(pg, mk, mv, a, p, bit + 7, st);
}

}  // namespace
