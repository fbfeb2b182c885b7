// Host side of a decode step over pages that rows share.  See include/faedkv.h for the contract of the call.
#include "pages_attn_host.cuh"
#include "k_page_shared.cuh"

namespace {

struct SharedPlan {
    int tq, blocks, ctas;    // rows of a shared block; blocks of rows, at most; CTAs
    bool spread;             // blocks few enough for their tiles to be shared out evenly (MODE 3); else a CTA each (MODE 4)
    size_t bytes;
};

template <typename C>
SharedPlan plan_shared(const faedkv_pages *pg, int batch, int n_groups) {
    const faedkv_pages_config &c = pg->cfg;
    SharedPlan p{};
    p.tq = C::QC / pg->gq;
    p.blocks = pages::shared_blocks(batch, n_groups, p.tq) + batch;
    const long long max_tiles = ((long long)c.max_pages * c.page_size + pages::kTile - 1) / pages::kTile;
    p.spread = p.blocks <= pages::kMaxBlocks && p.blocks * (max_tiles + pages::kUnitCost) < (1LL << 31);
    const long long most = (long long)pg->n_sm * C::CTAS, tiles = max_tiles * p.blocks * c.n_kv_heads;
    p.ctas = (int)(tiles < most ? tiles : most);
    p.bytes = pages::shared_meta_bytes(p.blocks, (size_t)batch * c.n_q_heads) +
              (p.spread ? (size_t)p.ctas * 2 * pages::attn_slot_floats(C::QC) * sizeof(float) : 0);
    return p;
}

template <typename C>
int launch_shared(faedkv_pages *pg, const CUtensorMap &mk, const CUtensorMap &mv, pages::AttnArgs a, int bit, cudaStream_t st) {
    const SharedPlan p = plan_shared<C>(pg, a.B, a.n_groups);
    a.blocks = p.blocks;
    auto kernel = p.spread ? pages::k_page_attn<C, 3, 0> : pages::k_page_attn<C, 4, 0>;
    const uint32_t smem = C::kSmemBytes + (p.spread ? C::kSmemBlocks : 0);
    if (!p.spread) ++bit;
    if (!(pg->attr_set & (1u << bit))) {
        CUDA_TRY(pg, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        pg->attr_set |= 1u << bit;
    }
    CUDA_TRY(pg, launch_pdl(kernel, p.spread ? dim3(p.ctas) : dim3(p.blocks, a.H), dim3(C::kThreads), smem, st, mk, mv, a));
    if (int r = launch_check(pg, "k_page_attn")) return r;
    auto join = p.spread ? pages::k_page_join_shared<typename C::T, 3> : pages::k_page_join_shared<typename C::T, 4>;
    CUDA_TRY(pg, launch_pdl(join, dim3((unsigned)(a.B * a.H)), dim3(kHeadDim, pages::kJoinGroups), 0, st, a, (int)C::QC, p.ctas));
    return launch_check(pg, "k_page_join_shared");
}

}  // namespace

extern "C" {

size_t faedkv_pages_attn_shared_bytes(const faedkv_pages *pg, int batch, int n_groups) {
    if (pg == nullptr || batch < 1 || batch > pg->cfg.max_batch || n_groups < 1 || n_groups > batch) return 0;
    return pg->cfg.kv_dtype == FAEDKV_F32 ? plan_shared<DecodeF32>(pg, batch, n_groups).bytes : plan_shared<DecodeBf16>(pg, batch, n_groups).bytes;
}

int faedkv_pages_attn_shared(faedkv_pages *pg, const void *q, long long ld_q, const int32_t *group_start, const int32_t *shared_len,
                             int n_groups, int batch, const int32_t *kv_len, const int32_t *table, const void *k_pages,
                             const void *v_pages, const float *k_scale, const float *v_scale, float scale, void *out, void *ws,
                             size_t ws_bytes, void *stream) {
    const CallRange nvtx_range("faedkv_pages_attn_shared");
    if (pg == nullptr) return FAEDKV_ERR_INVALID_ARG;
    if (int r = check_batch(pg, batch)) return r;
    if (n_groups < 1 || n_groups > batch) return fail(pg, FAEDKV_ERR_SHAPE, "n_groups = %d outside [1, batch=%d]", n_groups, batch);
    if (!(scale >= 0.0f) || std::isinf(scale)) return fail(pg, FAEDKV_ERR_INVALID_ARG, "scale must be >= 0 and finite");
    if (q == nullptr || group_start == nullptr || shared_len == nullptr || kv_len == nullptr || table == nullptr || k_pages == nullptr ||
        v_pages == nullptr || k_scale == nullptr || v_scale == nullptr || out == nullptr || ws == nullptr)
        return fail(pg, FAEDKV_ERR_INVALID_ARG, "NULL tensor passed to faedkv_pages_attn_shared");
    if (int r = check_align(pg, {q, k_pages, v_pages, k_scale, v_scale, out, ws}, {group_start, shared_len, kv_len, table})) return r;
    const faedkv_pages_config &c = pg->cfg;
    if (int r = check_ld(pg, "ld_q", ld_q, c.n_q_heads)) return r;
    const size_t need = faedkv_pages_attn_shared_bytes(pg, batch, n_groups);
    if (ws_bytes < need) return fail(pg, FAEDKV_ERR_SHAPE, "workspace of %zu bytes, %zu needed", ws_bytes, need);
    if (scale == 0.0f) scale = 1.0f / sqrtf((float)c.head_dim);
    const DeviceGuard guard(pg);
    if (!guard.ok) return fail(pg, FAEDKV_ERR_CUDA, "cannot select device %d", pg->device);
    CUtensorMap mk, mv;
    if (int r = make_map(pg, &mk, k_pages)) return r;
    if (int r = make_map(pg, &mv, v_pages)) return r;
    const pages::AttnArgs a{q, out, nullptr, kv_len, table, k_scale, v_scale, ld_q, batch, batch, c.n_kv_heads, pg->gq, c.max_pages,
                            c.n_pages, pg->page_shift, 0, 65536u / (unsigned)pg->gq + 1u, scale * 1.44269504088896341f,
                            static_cast<unsigned char *>(ws), pg->dev_status, pg->wait_limit_ns, pg->withhold_tile, group_start, shared_len,
                            n_groups};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return c.kv_dtype == FAEDKV_F32 ? launch_shared<DecodeF32>(pg, mk, mv, a, 16, st) : launch_shared<DecodeBf16>(pg, mk, mv, a, 18, st);
}

}  // extern "C"

long long pages_shared_debug_word(faedkv_pages *pg) { return debug_word_here(pg); }
