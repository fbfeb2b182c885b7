// What the host sides of the paged 8-bit cache share: the handle, argument checks, launches.
#pragma once
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>
#include <new>

#include <nvtx3/nvToolsExt.h>

#include "../../include/faedkv.h"
#include "common.cuh"
#include "umma_common.cuh"

using namespace faedkv;

struct faedkv_pages {
    faedkv_pages_config cfg;
    int device = 0, n_sm = 1, page_shift = 0, gq = 1;
    unsigned int *dev_status = nullptr;
    unsigned int attr_set = 0;                 // attention instances already opted in to large shared memory
    void *encode = nullptr;                    // cuTensorMapEncodeTiled
    unsigned long long launches = 0;
    unsigned long long wait_limit_ns = umma::kWaitLimitNs;   // faedkv_pages_test_hooks
    int withhold_tile = 0;
    int cluster_most = 0;                      // CTAs of the largest cluster there is room for; 0: not asked yet
    char err[512] = {0};
};

namespace {

struct CallRange {
    explicit CallRange(const char *name) { nvtxRangePushA(name); }
    ~CallRange() { nvtxRangePop(); }
    CallRange(const CallRange &) = delete;
    CallRange &operator=(const CallRange &) = delete;
};

[[maybe_unused]] int fail(faedkv_pages *pg, int code, const char *fmt, ...) {
    if (pg != nullptr) {
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(pg->err, sizeof(pg->err), fmt, ap);
        va_end(ap);
    }
    return code;
}

#define CUDA_TRY(pg, expr)                                                                   \
    do {                                                                                     \
        cudaError_t e_ = (expr);                                                             \
        if (e_ != cudaSuccess) {                                                             \
            cudaGetLastError(); /* reported here: not by the next call's launch */           \
            return fail(pg, FAEDKV_ERR_CUDA, "%s failed: %s", #expr, cudaGetErrorString(e_));\
        }                                                                                    \
    } while (0)

// Makes the handle's device current for the length of a call.
struct DeviceGuard {
    int before = -1;
    bool ok = false;
    explicit DeviceGuard(const faedkv_pages *pg) {
        if (cudaGetDevice(&before) != cudaSuccess) { before = -1; cudaGetLastError(); return; }
        ok = before == pg->device || cudaSetDevice(pg->device) == cudaSuccess;
        if (!ok) cudaGetLastError();
        if (before == pg->device) before = -1;
    }
    ~DeviceGuard() { if (before >= 0) cudaSetDevice(before); }
    DeviceGuard(const DeviceGuard &) = delete;
    DeviceGuard &operator=(const DeviceGuard &) = delete;
};

[[maybe_unused]] int check_align(faedkv_pages *pg, std::initializer_list<const void *> p16, std::initializer_list<const void *> p4) {
    for (const void *p : p16)
        if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0) return fail(pg, FAEDKV_ERR_ALIGN, "device pointer %p is not 16-byte aligned", p);
    for (const void *p : p4)
        if ((reinterpret_cast<uintptr_t>(p) & 3u) != 0) return fail(pg, FAEDKV_ERR_ALIGN, "device pointer %p is not 4-byte aligned", p);
    return FAEDKV_OK;
}

[[maybe_unused]] int check_batch(faedkv_pages *pg, int batch) {
    if (batch < 1 || batch > pg->cfg.max_batch)
        return fail(pg, FAEDKV_ERR_SHAPE, "batch %d outside [1, max_batch=%d]", batch, pg->cfg.max_batch);
    return FAEDKV_OK;
}

[[maybe_unused]] int check_ld(faedkv_pages *pg, const char *name, long long ld, int heads) {
    const int elem = pg->cfg.kv_dtype == FAEDKV_BF16 ? 2 : 4;
    if (ld < (long long)heads * kHeadDim || ld > (1LL << 40))
        return fail(pg, FAEDKV_ERR_SHAPE, "%s = %lld is less than %d heads of %d elements", name, ld, heads, kHeadDim);
    if ((ld * elem) % 16 != 0) return fail(pg, FAEDKV_ERR_ALIGN, "%s = %lld elements is not a multiple of 16 bytes", name, ld);
    return FAEDKV_OK;
}

[[maybe_unused]] int launch_check(faedkv_pages *pg, const char *what) {
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(pg, FAEDKV_ERR_CUDA, "launch of %s failed: %s", what, cudaGetErrorString(e));
    pg->launches += 1;
    return FAEDKV_OK;
}

// Launch with programmatic stream serialisation: the kernel may start while the stream's previous kernel drains, and
// waits for it in pdl_wait().
template <typename... KArgs, typename... Args>
cudaError_t launch_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// All rows of a code tensor, [n_pages * H * page][128] bytes; a box is one head's page.
[[maybe_unused]] int make_map(faedkv_pages *pg, CUtensorMap *map, const void *codes) {
    const faedkv_pages_config &c = pg->cfg;
    const cuuint64_t dims[2] = {(cuuint64_t)kHeadDim, (cuuint64_t)c.n_pages * c.n_kv_heads * c.page_size};
    const cuuint64_t strides[1] = {(cuuint64_t)kHeadDim};
    const cuuint32_t box[2] = {(cuuint32_t)kHeadDim, (cuuint32_t)c.page_size}, step[2] = {1, 1};
    const CUresult r = reinterpret_cast<EncodeTiled>(pg->encode)(
        map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(codes), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(pg, FAEDKV_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
    return FAEDKV_OK;
}

// First failed bounds check of this translation unit's kernels, cleared (the checked build; else 0).
[[maybe_unused]] long long debug_word_here(faedkv_pages *pg) {
#ifdef FAEDKV_DEBUG
    unsigned int w = 0, zero = 0;
    CUDA_TRY(pg, cudaMemcpyFromSymbol(&w, g_faedkv_debug_word, sizeof(w)));
    CUDA_TRY(pg, cudaMemcpyToSymbol(g_faedkv_debug_word, &zero, sizeof(zero)));
    return (long long)w;
#else
    (void)pg;
    return 0;
#endif
}

}  // namespace

// The same of the other files.
long long pages_share_debug_word(faedkv_pages *pg);
long long pages_diff_debug_word(faedkv_pages *pg);
long long pages_shared_debug_word(faedkv_pages *pg);
