// Host side of the paged 8-bit cache: argument checks and launches.  See include/faedkv.h for the contract of every call.
#include "pages_host.cuh"
#include "k_pages.cuh"
#include "pages_attn_host.cuh"

namespace {

template <typename T>
void launch_store(const pages::StoreArgs &a, int page, dim3 grid, cudaStream_t st) {
    switch (page) {
        case 16: pages::k_page_store<T, 16><<<grid, pages::kStoreThreads<T, 16>, 0, st>>>(a); break;
        case 32: pages::k_page_store<T, 32><<<grid, pages::kStoreThreads<T, 32>, 0, st>>>(a); break;
        case 64: pages::k_page_store<T, 64><<<grid, pages::kStoreThreads<T, 64>, 0, st>>>(a); break;
        default: pages::k_page_store<T, 128><<<grid, pages::kStoreThreads<T, 128>, 0, st>>>(a); break;
    }
}

}  // namespace

extern "C" {

int faedkv_pages_create(const faedkv_pages_config *cfg, faedkv_pages **out) {
    if (cfg == nullptr || out == nullptr) return FAEDKV_ERR_INVALID_ARG;
    *out = nullptr;
    const faedkv_pages_config &c = *cfg;
    if (c.n_kv_heads < 1 || c.n_q_heads < 1 || c.n_pages < 1 || c.max_pages < 1 || c.max_batch < 1) return FAEDKV_ERR_INVALID_ARG;
    if (c.kv_dtype != FAEDKV_F32 && c.kv_dtype != FAEDKV_BF16) return FAEDKV_ERR_INVALID_ARG;
    if (c.head_dim != kHeadDim) return FAEDKV_ERR_UNSUPPORTED;
    if (c.page_size != 16 && c.page_size != 32 && c.page_size != 64 && c.page_size != 128) return FAEDKV_ERR_UNSUPPORTED;
    if (c.n_q_heads % c.n_kv_heads != 0 || c.n_q_heads / c.n_kv_heads > 8) return FAEDKV_ERR_UNSUPPORTED;
    if (c.n_kv_heads > 4096 || c.max_batch > 65535) return FAEDKV_ERR_SHAPE;
    if ((long long)c.n_pages * c.page_size >= (1LL << 31) || (long long)c.n_pages * c.n_kv_heads >= (1LL << 31) ||
        (long long)c.n_pages * c.n_kv_heads * c.page_size >= (1LL << 31) || (long long)c.max_pages * c.page_size > (1LL << 30))
        return FAEDKV_ERR_SHAPE;
    faedkv_pages *pg = new (std::nothrow) faedkv_pages;
    if (pg == nullptr) return FAEDKV_ERR_CUDA;
    pg->cfg = c;
    pg->gq = c.n_q_heads / c.n_kv_heads;
    while ((1 << pg->page_shift) < c.page_size) ++pg->page_shift;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDevice(&pg->device) != cudaSuccess ||
        cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &pg->encode, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess || pg->encode == nullptr ||
        cudaDeviceGetAttribute(&pg->n_sm, cudaDevAttrMultiProcessorCount, pg->device) != cudaSuccess ||
        cudaMalloc(&pg->dev_status, sizeof(unsigned int)) != cudaSuccess ||
        cudaMemset(pg->dev_status, 0, sizeof(unsigned int)) != cudaSuccess) {
        cudaGetLastError();
        cudaFree(pg->dev_status);
        delete pg;
        return FAEDKV_ERR_CUDA;
    }
    *out = pg;
    return FAEDKV_OK;
}

void faedkv_pages_destroy(faedkv_pages *pg) {
    if (pg == nullptr) return;
    {
        const DeviceGuard guard(pg);
        cudaFree(pg->dev_status);
    }
    delete pg;
}

const char *faedkv_pages_last_error(const faedkv_pages *pg) { return pg ? pg->err : ""; }

size_t faedkv_pages_bytes(const faedkv_pages *pg) {
    return pg ? (size_t)pg->cfg.n_pages * pg->cfg.n_kv_heads * pg->cfg.page_size * kHeadDim : 0;
}

// Up to this many tokens and requests one CTA places the tokens itself; above, a second launch over all SMs is faster
// (32768 tokens: 40 us in one CTA) and the numbers between the two lie in the workspace.
static bool pages_in_one(int batch, int n_tokens) { return n_tokens <= 2048 && batch <= pages::kPlaceBatch; }

size_t faedkv_pages_tables_bytes(const faedkv_pages *pg, int batch, int n_tokens) {
    if (pg == nullptr || batch < 1 || batch > pg->cfg.max_batch || n_tokens < 0 || pages_in_one(batch, n_tokens)) return 0;
    return sizeof(int32_t) * ((size_t)batch + 1);
}

int faedkv_pages_tables(faedkv_pages *pg, const int32_t *t_len, const int32_t *n_new, int batch, int32_t *table,
                        int32_t *free_pages, const int32_t *n_free, int n_tokens, int32_t *q_start, int32_t *kv_len,
                        int32_t *slots, int32_t *n_free_out, int32_t *ws, void *stream) {
    const CallRange nvtx_range("faedkv_pages_tables");
    if (pg == nullptr) return FAEDKV_ERR_INVALID_ARG;
    if (int r = check_batch(pg, batch)) return r;
    if (n_tokens < 0) return fail(pg, FAEDKV_ERR_SHAPE, "n_tokens = %d is negative", n_tokens);
    if (t_len == nullptr || n_new == nullptr || table == nullptr || free_pages == nullptr || n_free == nullptr ||
        q_start == nullptr || kv_len == nullptr || (slots == nullptr && n_tokens > 0) || n_free_out == nullptr)
        return fail(pg, FAEDKV_ERR_INVALID_ARG, "NULL tensor passed to faedkv_pages_tables");
    if (int r = check_align(pg, {}, {t_len, n_new, table, free_pages, n_free, q_start, kv_len, slots, n_free_out, ws})) return r;
    const DeviceGuard guard(pg);
    if (!guard.ok) return fail(pg, FAEDKV_ERR_CUDA, "cannot select device %d", pg->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const pages::TablesArgs a{t_len, n_new, n_free, table, free_pages, q_start, kv_len, slots, n_free_out, ws, batch,
                              pg->cfg.max_pages, pg->page_shift, pg->cfg.n_pages, n_tokens, pg->dev_status};
    if (pages_in_one(batch, n_tokens)) {
        pages::k_page_plan<true><<<1, pages::kPlanThreads, 0, st>>>(a);
        return launch_check(pg, "k_page_plan");
    }
    if (ws == nullptr) return fail(pg, FAEDKV_ERR_INVALID_ARG, "NULL workspace passed to faedkv_pages_tables");
    pages::k_page_plan<false><<<1, pages::kPlanThreads, 0, st>>>(a);
    if (int r = launch_check(pg, "k_page_plan")) return r;
    if (n_tokens == 0) return FAEDKV_OK;                   // lengths and released pages only
    CUDA_TRY(pg, launch_pdl(pages::k_page_slots, dim3((unsigned)(((long long)n_tokens + 255) / 256)), dim3(256), 0, st, a));
    return launch_check(pg, "k_page_slots");
}

int faedkv_pages_store(faedkv_pages *pg, const void *k_new, const void *v_new, long long ld_new, const int32_t *slots,
                       int n_tokens, void *k_pages, void *v_pages, float *k_scale, float *v_scale, void *stream) {
    const CallRange nvtx_range("faedkv_pages_store");
    if (pg == nullptr) return FAEDKV_ERR_INVALID_ARG;
    if (n_tokens < 0) return fail(pg, FAEDKV_ERR_SHAPE, "n_tokens = %d is negative", n_tokens);
    if (n_tokens == 0) return FAEDKV_OK;
    if (k_new == nullptr || v_new == nullptr || slots == nullptr || k_pages == nullptr || v_pages == nullptr ||
        k_scale == nullptr || v_scale == nullptr)
        return fail(pg, FAEDKV_ERR_INVALID_ARG, "NULL tensor passed to faedkv_pages_store");
    if (int r = check_align(pg, {k_new, v_new, k_pages, v_pages, k_scale, v_scale}, {slots})) return r;
    const faedkv_pages_config &c = pg->cfg;
    if (int r = check_ld(pg, "ld_new", ld_new, c.n_kv_heads)) return r;
    const DeviceGuard guard(pg);
    if (!guard.ok) return fail(pg, FAEDKV_ERR_CUDA, "cannot select device %d", pg->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // tokens per CTA: one while that leaves every SM few CTAs (decode steps: a CTA's runs are done one after the other),
    // up to a page when there are many (prefill: a CTA per token would mostly find that its token starts no run)
    long long tile = ((long long)n_tokens * 2 * c.n_kv_heads + 8LL * pg->n_sm - 1) / (8LL * pg->n_sm);
    if (tile > c.page_size) tile = c.page_size;
    const pages::StoreArgs a{{k_new, v_new}, {static_cast<uint8_t *>(k_pages), static_cast<uint8_t *>(v_pages)}, {k_scale, v_scale},
                             slots, ld_new, n_tokens, (int)tile, c.n_kv_heads, c.n_pages, pg->dev_status};
    const long long ctas = (n_tokens + tile - 1) / tile * 2 * c.n_kv_heads;
    if (ctas >= (1LL << 31)) return fail(pg, FAEDKV_ERR_SHAPE, "n_tokens = %d is too many for one call", n_tokens);
    const dim3 grid((unsigned)ctas);
    if (c.kv_dtype == FAEDKV_BF16) launch_store<__nv_bfloat16>(a, c.page_size, grid, st);
    else launch_store<float>(a, c.page_size, grid, st);
    return launch_check(pg, "k_page_store");
}

size_t faedkv_pages_attn_bytes(const faedkv_pages *pg, int batch, int n_tokens) {
    if (pg == nullptr || batch < 1 || batch > pg->cfg.max_batch || n_tokens < 0) return 0;
    if ((long long)n_tokens + batch > (1LL << 30)) return 0;
    const AttnPlan p = plan_attn(pg, pg->gq, batch, n_tokens);
    return n_tokens == batch && p.bytes0 > p.bytes1 ? p.bytes0 : p.bytes1;
}

int faedkv_pages_attn(faedkv_pages *pg, const void *q, long long ld_q, const int32_t *q_start, int n_tokens, int batch,
                      const int32_t *kv_len, const int32_t *table, const void *k_pages, const void *v_pages,
                      const float *k_scale, const float *v_scale, float scale, void *out, void *ws, size_t ws_bytes,
                      void *stream) {
    const CallRange nvtx_range("faedkv_pages_attn");
    if (pg == nullptr) return FAEDKV_ERR_INVALID_ARG;
    if (int r = check_batch(pg, batch)) return r;
    if (n_tokens < 0 || (long long)n_tokens + batch > (1LL << 30))
        return fail(pg, FAEDKV_ERR_SHAPE, "n_tokens = %d outside [0, 2^30 - batch]", n_tokens);
    if (q_start == nullptr && n_tokens != batch)
        return fail(pg, FAEDKV_ERR_SHAPE, "without q_start there is one token per sequence: n_tokens = %d, batch = %d", n_tokens, batch);
    if (!(scale >= 0.0f) || std::isinf(scale)) return fail(pg, FAEDKV_ERR_INVALID_ARG, "scale must be >= 0 and finite");
    if (n_tokens == 0) return FAEDKV_OK;
    if (q == nullptr || kv_len == nullptr || table == nullptr || k_pages == nullptr || v_pages == nullptr || k_scale == nullptr ||
        v_scale == nullptr || out == nullptr || ws == nullptr)
        return fail(pg, FAEDKV_ERR_INVALID_ARG, "NULL tensor passed to faedkv_pages_attn");
    if (int r = check_align(pg, {q, k_pages, v_pages, k_scale, v_scale, out, ws}, {q_start, kv_len, table})) return r;
    const faedkv_pages_config &c = pg->cfg;
    if (int r = check_ld(pg, "ld_q", ld_q, c.n_q_heads)) return r;
    const size_t need = faedkv_pages_attn_bytes(pg, batch, n_tokens);
    if (ws_bytes < need) return fail(pg, FAEDKV_ERR_SHAPE, "workspace of %zu bytes, %zu needed", ws_bytes, need);
    if (scale == 0.0f) scale = 1.0f / sqrtf((float)c.head_dim);
    const DeviceGuard guard(pg);
    if (!guard.ok) return fail(pg, FAEDKV_ERR_CUDA, "cannot select device %d", pg->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    CUtensorMap mk, mv;
    if (int r = make_map(pg, &mk, k_pages)) return r;
    if (int r = make_map(pg, &mv, v_pages)) return r;
    const AttnPlan p = plan_attn(pg, pg->gq, batch, n_tokens);
    const pages::AttnArgs a{q, out, q_start, kv_len, table, k_scale, v_scale, ld_q, n_tokens, batch, c.n_kv_heads, pg->gq,
                            c.max_pages, c.n_pages, pg->page_shift, p.blocks,
                            pages::inverse_g(pg->gq), scale * 1.44269504088896341f,
                            static_cast<unsigned char *>(ws), pg->dev_status, pg->wait_limit_ns, pg->withhold_tile};
    return dispatch_attn<0>(pg, mk, mv, a, p, 0, st);
}

int faedkv_pages_load(faedkv_pages *pg, const int32_t *kv_len, const int32_t *table, int batch, int L, const void *k_pages,
                      const void *v_pages, const float *k_scale, const float *v_scale, void *K_out, void *V_out,
                      void *stream) {
    const CallRange nvtx_range("faedkv_pages_load");
    if (pg == nullptr) return FAEDKV_ERR_INVALID_ARG;
    if (int r = check_batch(pg, batch)) return r;
    const faedkv_pages_config &c = pg->cfg;
    if (L < 1 || L > (1 << 30)) return fail(pg, FAEDKV_ERR_SHAPE, "L = %d outside [1, 2^30]", L);
    const bool has_k = k_pages != nullptr || k_scale != nullptr || K_out != nullptr;
    const bool has_v = v_pages != nullptr || v_scale != nullptr || V_out != nullptr;
    if (kv_len == nullptr || table == nullptr || (!has_k && !has_v) ||
        (has_k && (k_pages == nullptr || k_scale == nullptr || K_out == nullptr)) ||
        (has_v && (v_pages == nullptr || v_scale == nullptr || V_out == nullptr)))
        return fail(pg, FAEDKV_ERR_INVALID_ARG, "NULL tensor passed to faedkv_pages_load");
    if (int r = check_align(pg, {k_pages, v_pages, k_scale, v_scale, K_out, V_out}, {kv_len, table})) return r;
    const DeviceGuard guard(pg);
    if (!guard.ok) return fail(pg, FAEDKV_ERR_CUDA, "cannot select device %d", pg->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const pages::LoadArgs a{{static_cast<const uint8_t *>(k_pages), static_cast<const uint8_t *>(v_pages)}, {k_scale, v_scale},
                            {K_out, V_out}, kv_len, table, c.n_kv_heads, L, c.max_pages, c.n_pages, pg->page_shift, pg->dev_status};
    const dim3 grid((L + c.page_size - 1) / c.page_size, c.n_kv_heads, batch);
    if (c.kv_dtype == FAEDKV_BF16) pages::k_page_load<__nv_bfloat16><<<grid, 256, 0, st>>>(a);
    else pages::k_page_load<float><<<grid, 256, 0, st>>>(a);
    return launch_check(pg, "k_page_load");
}

int faedkv_pages_device_status(faedkv_pages *pg, void *stream) {
    if (pg == nullptr) return FAEDKV_ERR_INVALID_ARG;
    const DeviceGuard guard(pg);
    if (!guard.ok) return fail(pg, FAEDKV_ERR_CUDA, "cannot select device %d", pg->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    unsigned int w = 0;
    CUDA_TRY(pg, cudaMemcpyAsync(&w, pg->dev_status, sizeof(w), cudaMemcpyDeviceToHost, st));
    CUDA_TRY(pg, cudaStreamSynchronize(st));
    return (int)w;
}

int faedkv_pages_reset_device_status(faedkv_pages *pg, void *stream) {
    if (pg == nullptr) return FAEDKV_ERR_INVALID_ARG;
    const DeviceGuard guard(pg);
    if (!guard.ok) return fail(pg, FAEDKV_ERR_CUDA, "cannot select device %d", pg->device);
    CUDA_TRY(pg, cudaMemsetAsync(pg->dev_status, 0, sizeof(unsigned int), static_cast<cudaStream_t>(stream)));
    return FAEDKV_OK;
}

int faedkv_pages_test_hooks(faedkv_pages *pg, unsigned long long wait_limit_ns, int withhold_tile) {
    if (pg == nullptr || withhold_tile < 0) return FAEDKV_ERR_INVALID_ARG;
    pg->wait_limit_ns = wait_limit_ns == 0 ? umma::kWaitLimitNs : wait_limit_ns;
    pg->withhold_tile = withhold_tile;
    return FAEDKV_OK;
}

long long faedkv_pages_debug_word(faedkv_pages *pg, void *stream) {
    if (pg == nullptr) return FAEDKV_ERR_INVALID_ARG;
#ifdef FAEDKV_DEBUG
    const DeviceGuard guard(pg);
    if (!guard.ok) return fail(pg, FAEDKV_ERR_CUDA, "cannot select device %d", pg->device);
    CUDA_TRY(pg, cudaStreamSynchronize(static_cast<cudaStream_t>(stream)));
    long long first = 0;
    for (long long (*word)(faedkv_pages *) : {debug_word_here, pages_share_debug_word, pages_diff_debug_word, pages_shared_debug_word}) {
        const long long w = word(pg);
        if (w < 0) return w;
        if (first == 0) first = w;
    }
    if (first != 0) fail(pg, FAEDKV_ERR_INVALID_ARG, "bounds check failed: file tag %lld, line %lld", first >> 16, first & 0xffff);
    return first;
#else
    (void)stream;
    return 0;
#endif
}

unsigned long long faedkv_pages_launch_count(const faedkv_pages *pg) { return pg ? pg->launches : 0ULL; }

}  // extern "C"
