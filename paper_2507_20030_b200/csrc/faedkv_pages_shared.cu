// Host side of a decode step over pages that rows share.  See include/faedkv.h for the contract of the call.
#include "pages_attn_host.cuh"
#include "k_page_shared.cuh"

namespace {

struct SharedPlan {
    int tq, blocks, ctas;    // rows of a shared block; blocks of rows, at most; CTAs
    bool spread;             // blocks few enough for their tiles to be shared out evenly (MODE 3); else a CTA each (MODE 4)
    size_t bytes;
};

// bf16: query columns as rows, 256 of them; float32: 8 columns.
SharedPlan plan_shared(const faedkv_pages *pg, int batch, int n_groups) {
    const faedkv_pages_config &c = pg->cfg;
    const bool rows = c.kv_dtype == FAEDKV_BF16;
    const int qc = rows ? pages::kRowsQC : DecodeF32::QC;
    SharedPlan p{};
    p.tq = qc / pg->gq;
    p.blocks = pages::shared_blocks(batch, n_groups, p.tq) + batch;
    const long long max_tiles = ((long long)c.max_pages * c.page_size + pages::kTile - 1) / pages::kTile;
    p.spread = p.blocks <= pages::kMaxBlocks && p.blocks * (2 * max_tiles + pages::kUnitCost) < (1LL << 31);
    const long long most = (long long)pg->n_sm * (rows ? 1 : DecodeF32::CTAS), tiles = max_tiles * p.blocks * c.n_kv_heads;
    p.ctas = (int)(tiles < most ? tiles : most);
    p.bytes = pages::shared_meta_bytes(p.blocks, (size_t)batch * c.n_q_heads) +
              (p.spread ? (size_t)p.ctas * 2 * pages::attn_slot_floats(qc) * sizeof(float) : 0);
    return p;
}

template <typename T, int MODE>
int launch_join(faedkv_pages *pg, const pages::AttnArgs &a, int qc, int ctas, cudaStream_t st) {
    CUDA_TRY(pg, launch_pdl(pages::k_page_join_shared<T, MODE>, dim3((unsigned)(((long long)a.B * a.H * a.G + 7) / 8)), dim3(256), 0, st, a, qc,
                            qc == pages::kRowsQC, ctas));
    return launch_check(pg, "k_page_join_shared");
}

template <int MODE>
int launch_shared(faedkv_pages *pg, const CUtensorMap &mk, const CUtensorMap &mv, const pages::AttnArgs &a, const SharedPlan &p, cudaStream_t st) {
    const dim3 grid = MODE == 3 ? dim3(p.ctas) : dim3(p.blocks, a.H);
    if (pg->cfg.kv_dtype == FAEDKV_BF16) {
        if (int r = launch_rows<MODE, 0>(pg, mk, mv, a, pages::DiffArgs{}, grid, 16 + MODE, st)) return r;
        return launch_join<__nv_bfloat16, MODE>(pg, a, pages::kRowsQC, p.ctas, st);
    }
    using C = DecodeF32;
    auto kernel = pages::k_page_attn<C, MODE, 0>;
    constexpr uint32_t smem = C::kSmemBytes + (MODE == 3 ? C::kSmemBlocks : 0);
    if (!(pg->attr_set & (1u << (18 + MODE)))) {
        CUDA_TRY(pg, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        pg->attr_set |= 1u << (18 + MODE);
    }
    CUDA_TRY(pg, launch_pdl(kernel, grid, dim3(C::kThreads), smem, st, mk, mv, a));
    if (int r = launch_check(pg, "k_page_attn")) return r;
    return launch_join<float, MODE>(pg, a, C::QC, p.ctas, st);
}

}  // namespace

extern "C" {

size_t faedkv_pages_attn_shared_bytes(const faedkv_pages *pg, int batch, int n_groups) {
    if (pg == nullptr || batch < 1 || batch > pg->cfg.max_batch || n_groups < 1 || n_groups > batch) return 0;
    return plan_shared(pg, batch, n_groups).bytes;
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
    const SharedPlan p = plan_shared(pg, batch, n_groups);
    const pages::AttnArgs a{q, out, nullptr, kv_len, table, k_scale, v_scale, ld_q, batch, batch, c.n_kv_heads, pg->gq, c.max_pages,
                            c.n_pages, pg->page_shift, p.blocks, 65536u / (unsigned)pg->gq + 1u, scale * 1.44269504088896341f,
                            static_cast<unsigned char *>(ws), pg->dev_status, pg->wait_limit_ns, pg->withhold_tile, group_start, shared_len,
                            n_groups};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return p.spread ? launch_shared<3>(pg, mk, mv, a, p, st) : launch_shared<4>(pg, mk, mv, a, p, st);
}

}  // extern "C"

long long pages_shared_debug_word(faedkv_pages *pg) { return debug_word_here(pg); }
