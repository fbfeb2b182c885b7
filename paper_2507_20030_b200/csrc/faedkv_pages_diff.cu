// Host side of differential attention over the paged 8-bit cache.  See include/faedkv.h for the contract of the call.
#include "pages_attn_host.cuh"
#include "k_page_diff.cuh"

namespace {

// Blocks of many columns take the form with rows: more than eight a sequence on average, as in plan_attn(), unless all of them in eights over the longest
// sequence that the tables hold would take less than the 20 us that the other form needs at least (3.1 ns a tile of eight columns).
AttnPlan plan_diff(const faedkv_pages *pg, int batch, int n_tokens) {
    const int gq = 2 * pg->gq;
    const AttnPlan p = plan_attn(pg, gq, batch, n_tokens);
    if (!p.wide) return p;
    const double tiles = ((double)n_tokens * gq / 8 + batch) * (double)p.max_tiles * pg->cfg.n_kv_heads;
    return tiles * 3.1 > 20000.0 ? plan_rows(pg, gq, batch, n_tokens) : plan_attn(pg, gq, batch, n_tokens, false);
}
// The workspace: parts of split units, then the maps' results of whole ones, float32 by token and head.  The form with rows (more tokens than sequences, so
// never a decode step) has none of those: it finishes whole units where they are attended.
struct DiffBytes { size_t parts, maps; };
DiffBytes diff_bytes(const faedkv_pages *pg, int batch, int n_tokens) {
    const AttnPlan p = plan_diff(pg, batch, n_tokens), q = plan_attn(pg, 2 * pg->gq, batch, n_tokens);
    return {((n_tokens == batch && q.bytes0 > p.bytes1 ? q.bytes0 : p.bytes1) + 15) / 16 * 16,
            p.wide ? 0 : sizeof(float) * 2 * kHeadDim * (size_t)n_tokens * pg->cfg.n_q_heads};
}

}  // namespace

extern "C" {

size_t faedkv_pages_attn_diff_bytes(const faedkv_pages *pg, int batch, int n_tokens) {
    if (pg == nullptr || pg->gq > 4 || batch < 1 || batch > pg->cfg.max_batch || n_tokens < 0) return 0;
    if ((long long)n_tokens + batch > (1LL << 30)) return 0;
    const DiffBytes b = diff_bytes(pg, batch, n_tokens);
    return b.parts + b.maps;
}

int faedkv_pages_attn_diff(faedkv_pages *pg, const void *q, long long ld_q, const int32_t *q_start, int n_tokens, int batch,
                           const int32_t *kv_len, const int32_t *table, const void *k_pages, const void *v_pages,
                           const float *k_scale, const float *v_scale, float scale, const float *lam, const float *gain, float eps,
                           void *out, void *ws, size_t ws_bytes, void *stream) {
    const CallRange nvtx_range("faedkv_pages_attn_diff");
    if (pg == nullptr) return FAEDKV_ERR_INVALID_ARG;
    if (int r = check_batch(pg, batch)) return r;
    const faedkv_pages_config &c = pg->cfg;
    if (pg->gq > 4) return fail(pg, FAEDKV_ERR_UNSUPPORTED, "differential attention takes 1 to 4 query heads per kv head, not %d", pg->gq);
    if (n_tokens < 0 || (long long)n_tokens + batch > (1LL << 30))
        return fail(pg, FAEDKV_ERR_SHAPE, "n_tokens = %d outside [0, 2^30 - batch]", n_tokens);
    if (q_start == nullptr && n_tokens != batch)
        return fail(pg, FAEDKV_ERR_SHAPE, "without q_start there is one token per sequence: n_tokens = %d, batch = %d", n_tokens, batch);
    if (!(scale >= 0.0f) || std::isinf(scale)) return fail(pg, FAEDKV_ERR_INVALID_ARG, "scale must be >= 0 and finite");
    if (!(eps >= 0.0f) || std::isinf(eps)) return fail(pg, FAEDKV_ERR_INVALID_ARG, "eps must be >= 0 and finite");
    if (n_tokens == 0) return FAEDKV_OK;
    if (q == nullptr || kv_len == nullptr || table == nullptr || k_pages == nullptr || v_pages == nullptr || k_scale == nullptr ||
        v_scale == nullptr || lam == nullptr || out == nullptr || ws == nullptr)
        return fail(pg, FAEDKV_ERR_INVALID_ARG, "NULL tensor passed to faedkv_pages_attn_diff");
    if (int r = check_align(pg, {q, k_pages, v_pages, k_scale, v_scale, gain, out, ws}, {q_start, kv_len, table, lam})) return r;
    if (int r = check_ld(pg, "ld_q", ld_q, c.n_q_heads)) return r;
    const size_t need = faedkv_pages_attn_diff_bytes(pg, batch, n_tokens);
    if (ws_bytes < need) return fail(pg, FAEDKV_ERR_SHAPE, "workspace of %zu bytes, %zu needed", ws_bytes, need);
    if (scale == 0.0f) scale = 0.125f;
    const DeviceGuard guard(pg);
    if (!guard.ok) return fail(pg, FAEDKV_ERR_CUDA, "cannot select device %d", pg->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    CUtensorMap mk, mv;
    if (int r = make_map(pg, &mk, k_pages)) return r;
    if (int r = make_map(pg, &mv, v_pages)) return r;
    const int gq = 2 * pg->gq;
    const AttnPlan p = q_start == nullptr ? plan_attn(pg, gq, batch, n_tokens) : plan_diff(pg, batch, n_tokens);
    const DiffBytes b = diff_bytes(pg, batch, n_tokens);
    float *maps = b.maps == 0 ? nullptr : reinterpret_cast<float *>(static_cast<unsigned char *>(ws) + b.parts);
    const pages::AttnArgs a{q, maps, q_start, kv_len, table, k_scale, v_scale, ld_q, n_tokens, batch, c.n_kv_heads, gq, c.max_pages,
                            c.n_pages, pg->page_shift, p.blocks, pages::inverse_g(gq), scale * 1.44269504088896341f,
                            static_cast<unsigned char *>(ws), pg->dev_status, pg->wait_limit_ns, pg->withhold_tile};
    const pages::DiffArgs d{maps, lam, gain, out, q_start, n_tokens, batch, c.n_q_heads, eps};
    if (p.wide && q_start != nullptr) {                    // whole units are finished where they are attended
        if (!p.shared) return launch_rows<2, 1>(pg, mk, mv, a, d, dim3(p.blocks, a.H), 12, st);
        if (int r = launch_rows<1, 1>(pg, mk, mv, a, d, dim3(p.ctas1), 13, st)) return r;
        if (p.max_tiles == 1) return FAEDKV_OK;            // no unit is ever in parts
        const dim3 grid((unsigned)p.ctas1, (p.qc / 2 + 7) / 8);
        CUDA_TRY(pg, launch_pdl(pages::k_page_diff_join<__nv_bfloat16, 1>, grid, dim3(256), 0, st, a, d, p.qc, p.ctas1));
        return launch_check(pg, "k_page_diff_join");
    }
    if (int r = dispatch_attn<1>(pg, mk, mv, a, p, 8, st)) return r;
    const bool f32 = c.kv_dtype == FAEDKV_F32;
    const dim3 grid((unsigned)(((long long)n_tokens * c.n_q_heads + 7) / 8));
    if (q_start == nullptr) {
        if (f32) CUDA_TRY(pg, launch_pdl(pages::k_page_diff_join<float, 0>, grid, dim3(256), 0, st, a, d, p.qc, p.ctas0));
        else CUDA_TRY(pg, launch_pdl(pages::k_page_diff_join<__nv_bfloat16, 0>, grid, dim3(256), 0, st, a, d, p.qc, p.ctas0));
        return launch_check(pg, "k_page_diff_join");
    }
    if (f32) CUDA_TRY(pg, launch_pdl(pages::k_page_diff<float>, grid, dim3(256), 0, st, d));
    else CUDA_TRY(pg, launch_pdl(pages::k_page_diff<__nv_bfloat16>, grid, dim3(256), 0, st, d));
    return launch_check(pg, "k_page_diff");
}

}  // extern "C"

long long pages_diff_debug_word(faedkv_pages *pg) { return debug_word_here(pg); }
