// Host side of pages that several requests share: fork, release, compact.  See include/faedkv.h for the contract of every call.
#include "pages_host.cuh"
#include "k_page_share.cuh"

namespace {

// Rows and entries of a call's block table: places in it are counted in 32 bits.
int check_table(faedkv_pages *pg, int batch) {
    if (int r = check_batch(pg, batch)) return r;
    if ((long long)batch * pg->cfg.max_pages >= (1LL << 31))
        return fail(pg, FAEDKV_ERR_SHAPE, "batch %d * max_pages %d is 2^31 or more", batch, pg->cfg.max_pages);
    return FAEDKV_OK;
}

// A launch of one cluster; larger ones than the portable eight CTAs have to be asked for, once for each kernel.
template <typename... Args>
int launch_cluster(faedkv_pages *pg, const char *what, void (*kernel)(Args...), int attr_bit, int ctas, cudaStream_t st, Args... args) {
    if (!(pg->attr_set & (1u << attr_bit))) {
        CUDA_TRY(pg, cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        pg->attr_set |= 1u << attr_bit;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(pages::kPlanThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    CUDA_TRY(pg, cudaLaunchKernelEx(&cfg, kernel, args...));
    return launch_check(pg, what);
}

// CTAs of the largest cluster that the device can hold: a partition of one may have no sixteen SMs that reach one another.  Asked once a handle.
int cluster_most(faedkv_pages *pg) {
    if (pg->cluster_most == 0) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(pages::kCluster);
        cfg.blockDim = dim3(pages::kPlanThreads);
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = pages::kCluster;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        pg->cluster_most = pages::kCluster;
        auto room_for = [&](auto kernel) {
            int n = 0;
            return cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                   cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess && n > 0;
        };
        if (!room_for(pages::k_page_release<pages::kCluster>) || !room_for(pages::k_page_release_short<4>) ||
            !room_for(pages::k_page_compact_plan<pages::kCluster>)) {
            cudaGetLastError();                            // an answer, not an error of the call
            pg->cluster_most = pages::kClusterAnywhere;
        }
    }
    return pg->cluster_most;
}

// Up to this many forks and rows the CTAs that copy find out for themselves what comes before them: the marks fit shared memory.
bool forks_alone(int batch, int n_forks) { return n_forks <= pages::kForkSmall && batch <= pages::kForkRows; }

}  // namespace

extern "C" {

size_t faedkv_pages_fork_bytes(const faedkv_pages *pg, int batch, int n_forks) {
    if (pg == nullptr || batch < 1 || batch > pg->cfg.max_batch || n_forks < 0 || n_forks > batch) return 0;
    return forks_alone(batch, n_forks) ? 0 : sizeof(int32_t) * ((size_t)n_forks + batch);
}

int faedkv_pages_fork(faedkv_pages *pg, const int32_t *src, const int32_t *dst, const int32_t *len, int n_forks, int batch,
                      int32_t *kv_len, int32_t *table, const int32_t *free_pages, const int32_t *n_free, int32_t *n_free_out,
                      void *k_pages, void *v_pages, float *k_scale, float *v_scale, void *ws, void *stream) {
    const CallRange nvtx_range("faedkv_pages_fork");
    if (pg == nullptr) return FAEDKV_ERR_INVALID_ARG;
    if (int r = check_table(pg, batch)) return r;
    if (n_forks < 0 || n_forks > batch) return fail(pg, FAEDKV_ERR_SHAPE, "n_forks = %d outside [0, batch=%d]", n_forks, batch);
    if (((src == nullptr || dst == nullptr) && n_forks > 0) || kv_len == nullptr || table == nullptr || free_pages == nullptr ||
        n_free == nullptr || n_free_out == nullptr || k_pages == nullptr || v_pages == nullptr || k_scale == nullptr ||
        v_scale == nullptr || (ws == nullptr && !forks_alone(batch, n_forks)))
        return fail(pg, FAEDKV_ERR_INVALID_ARG, "NULL tensor passed to faedkv_pages_fork");
    if (int r = check_align(pg, {k_pages, v_pages, k_scale, v_scale}, {src, dst, len, kv_len, table, free_pages, n_free, n_free_out, ws})) return r;
    const DeviceGuard guard(pg);
    if (!guard.ok) return fail(pg, FAEDKV_ERR_CUDA, "cannot select device %d", pg->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const faedkv_pages_config &c = pg->cfg;
    const pages::ForkArgs a{src, dst, len, free_pages, n_free, kv_len, table, n_free_out, static_cast<int32_t *>(ws),
                            {static_cast<uint8_t *>(k_pages), static_cast<uint8_t *>(v_pages)}, {k_scale, v_scale},
                            n_forks, batch, c.max_pages, c.n_kv_heads, c.n_pages, pg->page_shift, pg->dev_status};
    if (forks_alone(batch, n_forks)) {
        const bool in_place = n_free_out == n_free;        // its height may be written once all have read it
        if (n_forks > 0) {
            int parts = 4 * pg->n_sm / n_forks;            // of a fork's copy: four CTAs a SM in all
            parts = parts < 1 ? 1 : parts > 2 * c.n_kv_heads ? 2 * c.n_kv_heads : parts;
            pages::k_page_fork<true><<<dim3(n_forks, parts), 256, 0, st>>>(a, !in_place);
            if (int r = launch_check(pg, "k_page_fork")) return r;
            if (!in_place) return FAEDKV_OK;
        }
        CUDA_TRY(pg, launch_pdl(pages::k_page_fork<false>, dim3(1), dim3(256), 0, st, a, true));
        return launch_check(pg, "k_page_fork");
    }
    pages::k_page_fork_plan<<<1, pages::kPlanThreads, 0, st>>>(a);
    if (int r = launch_check(pg, "k_page_fork_plan")) return r;
    if (n_forks == 0) return FAEDKV_OK;                    // the height of the stack only
    CUDA_TRY(pg, launch_pdl(pages::k_page_fork_copy, dim3(n_forks), dim3(256), 0, st, a));
    return launch_check(pg, "k_page_fork_copy");
}

size_t faedkv_pages_release_bytes(const faedkv_pages *pg) {
    return pg ? sizeof(int32_t) * ((size_t)pg->cfg.n_pages + pages::kCluster) : 0;
}

int faedkv_pages_release(faedkv_pages *pg, const int32_t *t_len, const int32_t *n_new, int batch, const int32_t *table,
                         int32_t *free_pages, const int32_t *n_free, int32_t *kv_len, int32_t *n_free_out, void *ws, void *stream) {
    const CallRange nvtx_range("faedkv_pages_release");
    if (pg == nullptr) return FAEDKV_ERR_INVALID_ARG;
    if (int r = check_table(pg, batch)) return r;
    if (t_len == nullptr || n_new == nullptr || table == nullptr || free_pages == nullptr || n_free == nullptr || kv_len == nullptr ||
        n_free_out == nullptr || ws == nullptr)
        return fail(pg, FAEDKV_ERR_INVALID_ARG, "NULL tensor passed to faedkv_pages_release");
    if (int r = check_align(pg, {}, {t_len, n_new, table, free_pages, n_free, kv_len, n_free_out, ws})) return r;
    const DeviceGuard guard(pg);
    if (!guard.ok) return fail(pg, FAEDKV_ERR_CUDA, "cannot select device %d", pg->device);
    const pages::ReleaseArgs a{t_len, n_new, table, n_free, free_pages, kv_len, n_free_out, static_cast<int32_t *>(ws), batch,
                               pg->cfg.max_pages, pg->cfg.n_pages, pg->page_shift, pg->dev_status};
    // parts of a row, a warp each: more than one where there are fewer rows than warps, or where that makes them short enough for registers
    const int warps = pages::kPlanThreads / 32, widest = cluster_most(pg), most = widest * warps;
    int parts = 1, ctas = widest;
    while (parts < 32 && pg->cfg.max_pages > 256 * parts) parts *= 2;
    // (two and four runs a warp by the full cluster only)
    const bool in_registers = pg->cfg.max_pages <= 256 * parts && parts * batch <= (widest == pages::kCluster ? 4 * most : most) &&
                              pg->cfg.n_pages <= pages::kReleaseShort;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (in_registers)                                      // as few CTAs as have the warps: a larger cluster takes longer to begin and to meet
        while (ctas > 1 && parts * batch <= ctas / 2 * warps) ctas /= 2;
    else
        parts = 1;
    while (parts < 32 && 2 * parts * batch <= ctas * warps) parts *= 2;
    const int each = !in_registers ? 0 : batch * parts <= most ? 1 : batch * parts <= 2 * most ? 2 : 4;
    return each == 1   ? launch_cluster(pg, "k_page_release_short", pages::k_page_release_short<1>, 22, ctas, st, a, parts)
           : each == 2 ? launch_cluster(pg, "k_page_release_short", pages::k_page_release_short<2>, 23, ctas, st, a, parts)
           : each == 4 ? launch_cluster(pg, "k_page_release_short", pages::k_page_release_short<4>, 24, ctas, st, a, parts)
           : widest == pages::kCluster ? launch_cluster(pg, "k_page_release", pages::k_page_release<pages::kCluster>, 25, ctas, st, a, parts)
                                       : launch_cluster(pg, "k_page_release", pages::k_page_release<pages::kClusterAnywhere>, 27, ctas, st, a, parts);
}

size_t faedkv_pages_compact_bytes(const faedkv_pages *pg) {
    return pg ? sizeof(int32_t) * (pages::kCompactHead + 2 * (size_t)(pg->cfg.n_pages / 2)) : 0;
}

int faedkv_pages_compact(faedkv_pages *pg, const int32_t *kv_len, int batch, const int32_t *table, int32_t *table_out,
                         int32_t *free_pages, int32_t *n_free, int32_t *new_id, void *k_pages, void *v_pages, float *k_scale,
                         float *v_scale, void *ws, void *stream) {
    const CallRange nvtx_range("faedkv_pages_compact");
    if (pg == nullptr) return FAEDKV_ERR_INVALID_ARG;
    if (int r = check_table(pg, batch)) return r;
    if (kv_len == nullptr || table == nullptr || table_out == nullptr || free_pages == nullptr || n_free == nullptr ||
        new_id == nullptr || k_pages == nullptr || v_pages == nullptr || k_scale == nullptr || v_scale == nullptr || ws == nullptr)
        return fail(pg, FAEDKV_ERR_INVALID_ARG, "NULL tensor passed to faedkv_pages_compact");
    if (int r = check_align(pg, {k_pages, v_pages, k_scale, v_scale}, {kv_len, table, table_out, free_pages, n_free, new_id, ws})) return r;
    const DeviceGuard guard(pg);
    if (!guard.ok) return fail(pg, FAEDKV_ERR_CUDA, "cannot select device %d", pg->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const faedkv_pages_config &c = pg->cfg;
    const pages::CompactArgs a{kv_len, table, table_out, free_pages, n_free, new_id, static_cast<int32_t *>(ws),
                               {static_cast<uint8_t *>(k_pages), static_cast<uint8_t *>(v_pages)}, {k_scale, v_scale},
                               batch, c.max_pages, c.n_kv_heads, c.n_pages, pg->page_shift, pg->dev_status};
    if (c.n_pages <= pages::kCompactShort && (long long)batch * c.max_pages <= 16 * pages::kCompactShort) {
        pages::k_page_compact_short<<<1, pages::kPlanThreads, 0, st>>>(a);
        if (int r = launch_check(pg, "k_page_compact_short")) return r;
    } else if (cluster_most(pg) == pages::kCluster) {
        if (int r = launch_cluster(pg, "k_page_compact_plan", pages::k_page_compact_plan<pages::kCluster>, 26, pages::kCluster, st, a)) return r;
    } else if (int r = launch_cluster(pg, "k_page_compact_plan", pages::k_page_compact_plan<pages::kClusterAnywhere>, 28, pages::kClusterAnywhere, st, a)) {
        return r;
    }
    CUDA_TRY(pg, launch_pdl(pages::k_page_move, dim3(pg->n_sm * 8), dim3(256), 0, st, a));
    return launch_check(pg, "k_page_move");
}

}  // extern "C"

extern "C" int faedkv_pages_test_cluster(faedkv_pages *pg, int most) {
    if (pg == nullptr || (most != 0 && most != pages::kClusterAnywhere)) return FAEDKV_ERR_INVALID_ARG;
    pg->cluster_most = most;
    return FAEDKV_OK;
}

// The checked build's word of this file's kernels (each translation unit has one).
long long pages_share_debug_word(faedkv_pages *pg) { return debug_word_here(pg); }
