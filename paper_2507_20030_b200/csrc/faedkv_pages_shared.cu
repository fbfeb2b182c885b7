// Host side of a decode step over pages that rows share.  See include/faedkv.h for the contract of the call.
#include "pages_attn_host.cuh"
#include "k_page_shared.cuh"

namespace {

struct SharedPlan {
    struct Launch {
        int which, qc, n_shared, blocks, ctas;
        bool rows;           // query columns as rows, 256 of them; else 8 columns
        size_t head, slots;  // bytes of the header, of the partial results
    } launch[2];
    int n;                   // launches: one for all blocks, or one for the groups' and one for the rows' own
    bool spread;             // blocks few enough for their tiles to be shared out evenly (MODE 3); else a CTA each (MODE 4)
    size_t whole, bytes;
};

SharedPlan plan_shared(const faedkv_pages *pg, int batch, int n_groups) {
    const faedkv_pages_config &c = pg->cfg;
    SharedPlan p{};
    // One launch, eight columns a block, or two: the form with rows for what groups share, eight columns for what each row has behind it.  In eights a
    // tile of a group costs 0.39 ns a column (3.1 ns a block: 148 SMs side by side), in the form with rows 10.7 ns up to 128 columns and 22 ns at 256, and
    // 10 us once.  (8 kv heads x 4 query heads, 60 tokens behind, us in eights and with rows: one group of 16 rows over 8192 tokens 31 and 35, over 16384 43
    // and 39; of 32 rows over 2048 28 and 33, over 4096 35.5 and 34.4; of 64 rows over 1024 36 and 40, over 2048 44 and 42, over 32768 218 and 81; four groups
    // of 8 rows over 8192 48 and 52, of 16 79 and 60.)  The host knows the tables' width, not the lengths: where they are far apart the second launch is
    // taken too early, which costs those 10 us at most (8 rows behind 2048 tokens, their table as wide or for 131072: 16.8 and 23.3 us).
    const long long max_tiles = ((long long)c.max_pages * c.page_size + pages::kTile - 1) / pages::kTile;
    const double cols = (double)batch * pg->gq / n_groups, group_tiles = (double)max_tiles * c.n_kv_heads * n_groups;
    const double saved = group_tiles * (0.39 * cols - (cols <= 128 ? 10.7 : 0.086 * cols));
    p.n = c.kv_dtype == FAEDKV_BF16 && saved > 10000.0 ? 2 : 1;
    p.spread = true;
    for (int i = 0; i < p.n; ++i) {
        SharedPlan::Launch &u = p.launch[i];
        u.which = p.n == 1 ? 3 : 1 + i;
        u.rows = p.n == 2 && i == 0;
        u.qc = u.rows ? pages::kRowsQC : 8;
        u.n_shared = u.which & 1 ? pages::shared_blocks(batch, n_groups, u.qc / pg->gq) : 0;
        u.blocks = u.n_shared + (u.which & 2 ? batch : 0);
        u.head = pages::shared_before_bytes(u.blocks);
        p.spread = p.spread && u.blocks <= pages::kMaxBlocks && u.blocks * (2 * max_tiles + pages::kRowsCost) < (1LL << 31);
        const long long most = (long long)pg->n_sm * (u.rows ? 1 : kDecodeCtas), tiles = max_tiles * u.blocks * c.n_kv_heads;
        u.ctas = (int)(tiles < most ? tiles : most);
        u.slots = (size_t)u.ctas * 2 * pages::attn_slot_floats(u.qc) * sizeof(float);
    }
    p.whole = pages::shared_whole_bytes((size_t)batch * c.n_q_heads);
    p.bytes = p.whole;
    for (int i = 0; i < p.n; ++i) p.bytes += p.launch[i].head + (p.spread ? p.launch[i].slots : 0);
    return p;
}

template <typename C, int MODE>
int launch_few(faedkv_pages *pg, const CUtensorMap &mk, const CUtensorMap &mv, const pages::AttnArgs &a, dim3 grid, int attr_bit, cudaStream_t st) {
    auto kernel = pages::k_page_attn<C, MODE, 0>;
    constexpr uint32_t smem = C::kSmemBytes + (MODE == 3 ? C::kSmemBlocks : 0);
    if (!(pg->attr_set & (1u << attr_bit))) {
        CUDA_TRY(pg, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        pg->attr_set |= 1u << attr_bit;
    }
    CUDA_TRY(pg, launch_pdl(kernel, grid, dim3(C::kThreads), smem, st, mk, mv, a));
    return launch_check(pg, "k_page_attn");
}

template <int MODE>
int launch_shared(faedkv_pages *pg, const CUtensorMap &mk, const CUtensorMap &mv, pages::AttnArgs a, const SharedPlan &p, cudaStream_t st) {
    unsigned char *at = a.ws + p.whole;
    a.whole = reinterpret_cast<float *>(a.ws);
    const bool f32 = pg->cfg.kv_dtype == FAEDKV_F32;
    pages::SharedLaunch done[2];
    for (int i = 0; i < p.n; ++i) {
        const SharedPlan::Launch &u = p.launch[i];
        a.which = u.which;
        a.blocks = u.blocks;
        a.ws = at;
        a.slots = reinterpret_cast<float *>(at + u.head);
        at += u.head + (p.spread ? u.slots : 0);
        const dim3 grid = MODE == 3 ? dim3(u.ctas) : dim3(u.blocks, a.H);
        if (int r = u.rows ? launch_rows<MODE, 0>(pg, mk, mv, a, pages::DiffArgs{}, grid, 13 + MODE, st)
                    : f32  ? launch_few<DecodeF32, MODE>(pg, mk, mv, a, grid, 15 + MODE, st)
                           : launch_few<DecodeBf16, MODE>(pg, mk, mv, a, grid, 17 + MODE, st)) return r;
        done[i] = {a.ws, a.slots, u.qc, u.rows ? pages::kRowsCost : pages::kSharedCost, u.rows, u.ctas, u.n_shared, u.blocks};
    }
    auto join = f32 ? pages::k_page_join_shared<float, MODE> : pages::k_page_join_shared<__nv_bfloat16, MODE>;
    CUDA_TRY(pg, launch_pdl(join, dim3((unsigned)(((long long)a.B * a.H * a.G + 7) / 8)), dim3(256), 0, st, a, done[0], done[p.n - 1]));
    return launch_check(pg, "k_page_join_shared");
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
                            c.n_pages, pg->page_shift, 0, pages::inverse_g(pg->gq), scale * 1.44269504088896341f,
                            static_cast<unsigned char *>(ws), pg->dev_status, pg->wait_limit_ns, pg->withhold_tile, group_start, shared_len,
                            n_groups, 0, nullptr, nullptr};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return p.spread ? launch_shared<3>(pg, mk, mv, a, p, st) : launch_shared<4>(pg, mk, mv, a, p, st);
}

}  // extern "C"

long long pages_shared_debug_word(faedkv_pages *pg) { return debug_word_here(pg); }
