// Host side of the paged 8-bit cache: argument checks and launches.  See include/faedkv.h for the contract of every call.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>
#include <new>

#include <nvtx3/nvToolsExt.h>

#include "../../include/faedkv.h"
#include "common.cuh"
#include "k_pages.cuh"
#include "k_page_attn.cuh"

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
    char err[512] = {0};
};

namespace {

struct CallRange {
    explicit CallRange(const char *name) { nvtxRangePushA(name); }
    ~CallRange() { nvtxRangePop(); }
    CallRange(const CallRange &) = delete;
    CallRange &operator=(const CallRange &) = delete;
};

int fail(faedkv_pages *pg, int code, const char *fmt, ...) {
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

int check_align(faedkv_pages *pg, std::initializer_list<const void *> p16, std::initializer_list<const void *> p4) {
    for (const void *p : p16)
        if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0) return fail(pg, FAEDKV_ERR_ALIGN, "device pointer %p is not 16-byte aligned", p);
    for (const void *p : p4)
        if ((reinterpret_cast<uintptr_t>(p) & 3u) != 0) return fail(pg, FAEDKV_ERR_ALIGN, "device pointer %p is not 4-byte aligned", p);
    return FAEDKV_OK;
}

int check_batch(faedkv_pages *pg, int batch) {
    if (batch < 1 || batch > pg->cfg.max_batch)
        return fail(pg, FAEDKV_ERR_SHAPE, "batch %d outside [1, max_batch=%d]", batch, pg->cfg.max_batch);
    return FAEDKV_OK;
}

int check_ld(faedkv_pages *pg, const char *name, long long ld, int heads) {
    const int elem = pg->cfg.kv_dtype == FAEDKV_BF16 ? 2 : 4;
    if (ld < (long long)heads * kHeadDim || ld > (1LL << 40))
        return fail(pg, FAEDKV_ERR_SHAPE, "%s = %lld is less than %d heads of %d elements", name, ld, heads, kHeadDim);
    if ((ld * elem) % 16 != 0) return fail(pg, FAEDKV_ERR_ALIGN, "%s = %lld elements is not a multiple of 16 bytes", name, ld);
    return FAEDKV_OK;
}

int launch_check(faedkv_pages *pg, const char *what) {
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

template <typename T>
void launch_store(const pages::StoreArgs &a, int page, dim3 grid, cudaStream_t st) {
    switch (page) {
        case 16: pages::k_page_store<T, 16><<<grid, pages::kStoreThreads<T, 16>, 0, st>>>(a); break;
        case 32: pages::k_page_store<T, 32><<<grid, pages::kStoreThreads<T, 32>, 0, st>>>(a); break;
        case 64: pages::k_page_store<T, 64><<<grid, pages::kStoreThreads<T, 64>, 0, st>>>(a); break;
        default: pages::k_page_store<T, 128><<<grid, pages::kStoreThreads<T, 128>, 0, st>>>(a); break;
    }
}

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// All rows of a code tensor, [n_pages * H * page][128] bytes; a box is one head's page.
int make_map(faedkv_pages *pg, CUtensorMap *map, const void *codes) {
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

AttnPlan plan_attn(const faedkv_pages *pg, int batch, int n_tokens) {
    const faedkv_pages_config &c = pg->cfg;
    AttnPlan p{};
    p.max_tiles = ((long long)c.max_pages * c.page_size + pages::kTile - 1) / pages::kTile;
    // more than 8 query columns a sequence on average: blocks of 128 columns, which read the cache once for all of theirs.  The host
    // does not know how the tokens lie: where every sequence has as many, blocks of 8 stay ahead to 16 columns or 24 (16 x 16384
    // tokens, 8 kv heads: 115 us in 8s and 244 in 128s at 8 columns, 185 and 246 at 16, 266 and 247 at 24), but one long chunk
    // among decoding requests would go over its cache once for every 8 of them (120 tokens over 65536 beside 63 requests of 1000, 11
    // columns on average: 803 and 343 us; 320 tokens, 24 on average: 1973 and 650), so the rule leans to the side that loses less
    p.wide = c.kv_dtype == FAEDKV_BF16 && (long long)n_tokens * pg->gq > 8LL * batch;
    p.qc = p.wide ? ChunkBf16::QC : 8;
    p.blocks = n_tokens / (p.qc / pg->gq) + batch;
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

template <typename C, int MODE>
int launch_attn(faedkv_pages *pg, const CUtensorMap &mk, const CUtensorMap &mv, const pages::AttnArgs &a, const AttnPlan &p, int attr_bit,
                cudaStream_t st) {
    auto kernel = pages::k_page_attn<C, MODE>;
    constexpr uint32_t smem = C::kSmemBytes + (MODE == 1 ? C::kSmemBlocks : 0);
    if (!(pg->attr_set & (1u << attr_bit))) {
        CUDA_TRY(pg, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        pg->attr_set |= 1u << attr_bit;
    }
    const dim3 grid = MODE == 0 ? dim3(p.ctas0) : MODE == 1 ? dim3(p.ctas1) : dim3(p.blocks, a.H);
    CUDA_TRY(pg, launch_pdl(kernel, grid, dim3(C::kThreads), smem, st, mk, mv, a));
    if (int r = launch_check(pg, "k_page_attn")) return r;
    if (MODE == 2 || p.max_tiles == 1) return FAEDKV_OK;                     // no unit is ever in parts
    if constexpr (MODE != 2) {
        const int cols = MODE == 0 ? a.G : C::QC / a.G * a.G, each = MODE == 0 ? 1 : 16;
        const dim3 jgrid((unsigned)(MODE == 0 ? a.B * a.H : p.ctas1), (cols + each - 1) / each);
        CUDA_TRY(pg, launch_pdl(pages::k_page_attn_join<typename C::T, MODE>, jgrid, dim3(kHeadDim, pages::kJoinGroups), 0, st, a, (int)C::QC,
                                each, MODE == 0 ? p.ctas0 : p.ctas1));
        return launch_check(pg, "k_page_attn_join");
    }
    return FAEDKV_OK;
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
    const AttnPlan p = plan_attn(pg, batch, n_tokens);
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
    const AttnPlan p = plan_attn(pg, batch, n_tokens);
    const pages::AttnArgs a{q, out, q_start, kv_len, table, k_scale, v_scale, ld_q, n_tokens, batch, c.n_kv_heads, pg->gq,
                            c.max_pages, c.n_pages, pg->page_shift, p.blocks,
                            65536u / (unsigned)pg->gq + 1u, scale * 1.44269504088896341f,
                            static_cast<unsigned char *>(ws), pg->dev_status, pg->wait_limit_ns, pg->withhold_tile};
    if (c.kv_dtype == FAEDKV_F32)
        return q_start == nullptr ? launch_attn<DecodeF32, 0>(pg, mk, mv, a, p, 0, st)
               : p.shared         ? launch_attn<DecodeF32, 1>(pg, mk, mv, a, p, 1, st)
                                  : launch_attn<DecodeF32, 2>(pg, mk, mv, a, p, 2, st);
    if (q_start == nullptr) return launch_attn<DecodeBf16, 0>(pg, mk, mv, a, p, 3, st);
    if (p.wide)
        return p.shared ? launch_attn<ChunkBf16, 1>(pg, mk, mv, a, p, 4, st) : launch_attn<ChunkBf16, 2>(pg, mk, mv, a, p, 5, st);
    return p.shared ? launch_attn<DecodeBf16, 1>(pg, mk, mv, a, p, 6, st) : launch_attn<DecodeBf16, 2>(pg, mk, mv, a, p, 7, st);
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
    unsigned int w = 0, zero = 0;
    CUDA_TRY(pg, cudaStreamSynchronize(static_cast<cudaStream_t>(stream)));
    CUDA_TRY(pg, cudaMemcpyFromSymbol(&w, g_faedkv_debug_word, sizeof(w)));
    CUDA_TRY(pg, cudaMemcpyToSymbol(g_faedkv_debug_word, &zero, sizeof(zero)));
    if (w != 0) fail(pg, FAEDKV_ERR_INVALID_ARG, "bounds check failed: file tag %u, line %u", w >> 16, w & 0xffffu);
    return (long long)w;
#else
    (void)stream;
    return 0;
#endif
}

unsigned long long faedkv_pages_launch_count(const faedkv_pages *pg) { return pg ? pg->launches : 0ULL; }

}  // extern "C"
