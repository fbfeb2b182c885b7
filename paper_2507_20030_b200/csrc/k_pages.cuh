// The paged 8-bit cache: block tables and slots from request lengths, quantised writes, rows read back.
//
// A page holds `page` tokens of every kv head as e4m3 codes [n_pages][H][page][128]; one float32 scale per (page, head):
// value = code * scale.  The writes here choose scales that are powers of two: e4m3 is a floating-point format, so a
// power of two loses nothing of its relative precision (half a step is 2^-4 of the value), dividing by it is exact, and
// re-rounding older rows when a page's scale grows changes only codes that fall into e4m3's subnormal range.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace faedkv {
namespace pages {

// Device status word: codes of indices that came from device memory and lie outside what they index.  The access is
// skipped (the token is not stored / not attended to / reads as zero) and the kernel carries on.
constexpr unsigned int kBadPage = 0x101, kBadSlot = 0x102, kBadLength = 0x103, kBadFreeList = 0x104, kBadStart = 0x105;

__device__ __forceinline__ void flag(unsigned int *status, unsigned int code) { atomicCAS(status, 0u, code); }

// ---- tables -------------------------------------------------------------------------------------------

struct TablesArgs {
    const int32_t *t_len, *n_new, *n_free;
    int32_t *table, *free_pages, *q_start, *kv_len, *slots, *n_free_out, *ws;   // ws[b]: first new page in the running order, -1 denied; ws[B]: stack height before the grants
    int B, W, page_shift, n_pages, n_tokens;
    unsigned int *status;
};

constexpr int kPlanThreads = 1024;

// Inclusive sum over the block's threads; *total receives the block's sum.  Two barriers.
__device__ __forceinline__ long long block_scan(long long v, long long *warp_sums, long long *total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
        const long long o = __shfl_up_sync(0xffffffffu, v, s);
        if (lane >= s) v += o;
    }
    if (lane == 31) warp_sums[warp] = v;
    __syncthreads();
    long long w = warp_sums[lane];                       // 32 warps: one sum per lane
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
        const long long o = __shfl_up_sync(0xffffffffu, w, s);
        if (lane >= s) w += o;
    }
    *total = __shfl_sync(0xffffffffu, w, 31);
    const long long before = __shfl_sync(0xffffffffu, w, warp > 0 ? warp - 1 : 0);
    __syncthreads();
    return v + (warp > 0 ? before : 0);
}

// Last b with start[b] <= i, for i < start[B].
__device__ __forceinline__ int find_sequence(const int32_t *start, int B, int i) {
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (start[mid] <= i) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// Slot of new token i, and the table entry when the token opens a page.  start: q_start; base: ws.
__device__ __forceinline__ void place_token(const TablesArgs &a, int i, const int32_t *start, const int32_t *base) {
    int slot = -1;
    if (i < start[a.B]) {
        const int b = find_sequence(start, a.B, i);
        const int page0 = base[b];
        if (page0 >= 0) {
            const int first = start[b], n = start[b + 1] - first;
            const int t = a.kv_len[b] - n, pos = t + (i - first);
            const int p = pos >> a.page_shift, old = (t + (1 << a.page_shift) - 1) >> a.page_shift;
            int id = -1;
            if (!FAEDKV_IN_BOUNDS(kTagPages, b < a.B && p >= 0 && p < a.W)) {
            } else if (p < old) {
                id = a.table[(size_t)b * a.W + p];
            } else if (FAEDKV_IN_BOUNDS(kTagPages, page0 + p - old < base[a.B] && base[a.B] <= a.n_pages)) {
                id = a.free_pages[base[a.B] - 1 - (page0 + p - old)];
                if ((pos & ((1 << a.page_shift) - 1)) == 0) a.table[(size_t)b * a.W + p] = id;
            }
            if (id >= 0 && id < a.n_pages) slot = (id << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
            else flag(a.status, kBadPage);
        }
    }
    a.slots[i] = slot;
}

constexpr int kPlaceBatch = kPlanThreads;                 // requests that the one-launch form holds in shared memory

// One CTA: pushes the pages of finished requests, grants pages in request order (three block-wide sums per 1024
// requests), writes lengths and starts; with PLACE also the slots, from starts and page numbers kept in shared memory.
// Every input of a request is read before an output of the same request is written, and n_free before n_free_out, so
// outputs may be the inputs' own buffers.  Bound by latency, a chain of loads and three sums: 4.5 us at 16 requests of one
// token; 11 us with k_page_slots at 512 requests, 32768 tokens and 37 finished ones.
template <bool PLACE>
__global__ void __launch_bounds__(kPlanThreads) k_page_plan(const TablesArgs a) {
    __shared__ long long warp_sums[32];
    __shared__ int rel_base[kPlanThreads], rel_n[kPlanThreads];
    __shared__ int32_t start_s[PLACE ? kPlaceBatch + 1 : 1], base_s[PLACE ? kPlaceBatch + 1 : 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int page = 1 << a.page_shift;
    const long long cap = (long long)a.W * page;
    long long height = *a.n_free;
    if (height < 0 || height > a.n_pages) {
        if (tid == 0) flag(a.status, kBadFreeList);
        height = height < 0 ? 0 : a.n_pages;
    }
    // finished requests: pages onto the stack, in request order
    for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
        const int b = b0 + tid;
        long long held = 0;
        if (b < a.B && a.n_new[b] < 0) {
            const long long t = a.t_len[b];
            if (t < 0 || t > cap) flag(a.status, kBadLength);
            held = t <= 0 ? 0 : ((t < cap ? t : cap) + page - 1) >> a.page_shift;
        }
        if (!__syncthreads_or(held > 0)) continue;
        long long total;
        const long long upto = block_scan(held, warp_sums, &total);
        rel_base[tid] = (int)min(height + upto - held, (long long)a.n_pages);
        rel_n[tid] = (int)held;
        __syncthreads();
        for (int r = warp; r < min(kPlanThreads, a.B - b0); r += kPlanThreads / 32) {
            const int n = rel_n[r], base = rel_base[r];
            const int32_t *row = a.table + (size_t)(b0 + r) * a.W;
            for (int j0 = lane; j0 < n; j0 += 256) {       // eight entries a lane in flight
                int id[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) id[k] = j0 + 32 * k < n ? row[j0 + 32 * k] : 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int j = j0 + 32 * k;
                    if (j < n && base + j < a.n_pages) a.free_pages[base + j] = id[k];
                    else if (j < n) flag(a.status, kBadFreeList);
                }
            }
        }
        height = min(height + total, (long long)a.n_pages);
        __syncthreads();
    }
    // arriving tokens and the pages they need
    long long tok_before = 0, need_before = 0, taken = 0;
    for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
        const int b = b0 + tid;
        long long t = 0, n = 0;
        bool done = true, valid = false;
        if (b < a.B) {
            t = a.t_len[b];
            n = a.n_new[b];
            done = n < 0;
            if (done) n = 0;
        }
        long long tok_total, need_total;
        const long long tok_end = tok_before + block_scan(n, warp_sums, &tok_total);
        if (b < a.B && !done) {
            if (t < 0 || t > cap) flag(a.status, kBadLength);
            valid = t >= 0 && t + n <= cap && tok_end <= a.n_tokens;
        }
        const long long old = (t + page - 1) >> a.page_shift;
        const long long need = valid ? ((t + n + page - 1) >> a.page_shift) - old : 0;
        const long long need_end = need_before + block_scan(need, warp_sums, &need_total);
        const bool ok = valid && (need == 0 || need_end <= height);
        long long took_total;
        block_scan(ok ? need : 0, warp_sums, &took_total);
        if (b < a.B) {
            const int start = (int)min(tok_end - n, 0x7fffffffLL), end = (int)min(tok_end, 0x7fffffffLL);
            const int base = ok ? (int)min(need_end - need, (long long)a.n_pages) : -1;
            a.q_start[b] = start;
            if (b == a.B - 1) a.q_start[a.B] = end;
            a.kv_len[b] = done ? 0 : (ok ? (int)(t + n) : (int)t);
            if (PLACE) {
                start_s[b] = start;
                if (b == a.B - 1) start_s[a.B] = end;
                base_s[b] = base;
            } else {
                a.ws[b] = base;
            }
        }
        tok_before += tok_total;
        need_before += need_total;
        taken += took_total;
    }
    if (tid == 0) {
        (PLACE ? base_s : a.ws)[a.B] = (int)height;
        *a.n_free_out = (int)(height - taken);
    }
    if (PLACE) {
        __syncthreads();
        for (int i = tid; i < a.n_tokens; i += kPlanThreads) place_token(a, i, start_s, base_s);
    }
}

// The slots of many tokens.  The search for a token's request is a chain of loads: in shared memory while it fits.
constexpr int kSlotsBatch = 4096;
__global__ void __launch_bounds__(256) k_page_slots(const TablesArgs a) {
    __shared__ int32_t start_s[kSlotsBatch + 1];
    pdl_wait();
    const bool fits = a.B <= kSlotsBatch;
    if (fits) {
        for (int b = threadIdx.x; b <= a.B; b += 256) start_s[b] = a.q_start[b];
        __syncthreads();
    }
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < a.n_tokens) place_token(a, i, fits ? start_s : a.q_start, a.ws);
}

// ---- store --------------------------------------------------------------------------------------------

// The smallest power of two s >= 2^-126 with amax / s <= 448 (amax finite, >= 0): 448 = 1.75 * 2^8.
__device__ __forceinline__ float scale_for(float amax) {
    const uint32_t u = __float_as_uint(amax);
    int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    if (e < 1) e = 1;
    return __uint_as_float((uint32_t)e << 23);
}
// |x| of a finite x as bits (ordered like the values), 0 for infinities and NaN: they do not set a page's scale.
__device__ __forceinline__ uint32_t finite_bits(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}
// e4m3 codes, round to nearest even, |x| > 448 and infinities to 448, NaN to NaN; the first in the lowest byte.
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
        "mov.b32 %0, {lo, hi};\n\t}" : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}
__device__ __forceinline__ uint2 to_e4m3x8(const float (&x)[8], float mul) {
    return make_uint2(to_e4m3x4(x[0] * mul, x[1] * mul, x[2] * mul, x[3] * mul), to_e4m3x4(x[4] * mul, x[5] * mul, x[6] * mul, x[7] * mul));
}
// The values of two codes (exact: e4m3 is a subset of f16).
__device__ __forceinline__ float2 from_e4m3x2(uint32_t codes) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes & 0xffffu), __NV_E4M3);
    return __half22float2(__half2(h));
}
__device__ __forceinline__ void from_e4m3x4(uint32_t codes, float (&x)[4]) {
    const float2 a = from_e4m3x2(codes), b = from_e4m3x2(codes >> 16);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
}

template <typename T> struct Raw8;                        // 8 consecutive elements, as they lie in memory
template <> struct Raw8<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v = __ldcs(reinterpret_cast<const uint4 *>(p)); }
    __device__ __forceinline__ void zero() { v = make_uint4(0u, 0u, 0u, 0u); }
    // the largest magnitude so far, as bits: two bf16 maxima side by side until to_float_bits()  (NaN is passed over)
    __device__ __forceinline__ uint32_t max_bits(uint32_t m) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        __nv_bfloat162 h = *reinterpret_cast<const __nv_bfloat162 *>(&m);
#pragma unroll
        for (int i = 0; i < 4; ++i) h = __hmax2(h, __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&w[i])));
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    __device__ __forceinline__ uint32_t to_float_bits(uint32_t m) const { return max(m << 16, m & 0xffff0000u); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
};
template <> struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) {
        a = __ldcs(reinterpret_cast<const float4 *>(p));
        b = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
    }
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ uint32_t max_bits(uint32_t m) const {
        const float f[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(f[e]) & 0x7fffffffu);
        return m;
    }
    __device__ __forceinline__ uint32_t to_float_bits(uint32_t m) const { return m; }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
};

// Threads of a store CTA: few, since finding a run costs each warp about as much as 16 KB of its rows, but no more than 32
// registers of rows a thread (64 for pages of 128 float32 rows).
template <typename T, int PAGE> constexpr int kStoreThreads = PAGE * sizeof(T) <= 128 ? 128 : 256;

struct StoreArgs {
    const void *x[2];                                     // k_new, v_new: token rows `ld` elements apart, heads 128 apart
    uint8_t *codes[2];
    float *scale[2];
    const int32_t *slots;
    long long ld;
    int n_tokens, tile, H, n_pages;
    unsigned int *status;
};

// Grid: 2 H CTAs for each tile of consecutive tokens, one (tensor, head) each and next to one another, so that a token's
// row is read from memory while it is open.  The tokens of one page are a run of consecutive tokens with ascending slots;
// a CTA owns the runs that START in its tile: 16 threads per row of 128, 8 elements a thread.
// It reads a run once into registers, takes the largest finite magnitude, settles the page's scale, re-rounds the page's
// older rows if the scale grew, and writes the new codes: the data is read once and written once.  What it takes is a chain
// of dependent loads (slots, rows) and one barrier, so every warp finds the runs by itself and registers are kept few, for
// CTAs enough to cover it.  Measured: 32768 tokens x 8 heads, bf16, 34.1 us (5.9 TB/s; with half the rows a thread 40.3 us, bound
// by instructions), 2.5 us for 16 tokens.
template <typename T, int PAGE>
__global__ void __launch_bounds__(kStoreThreads<T, PAGE>, PAGE * sizeof(T) <= 128 ? 8 : PAGE * sizeof(T) <= 256 ? 4 : 2) k_page_store(const StoreArgs a) {
    constexpr int kRows = kStoreThreads<T, PAGE> / 16, kIter = (PAGE + kRows - 1) / kRows, kWords = (PAGE + 31) / 32;
    constexpr int kWarps = kStoreThreads<T, PAGE> / 32;
    __shared__ uint32_t max_s[2][kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned int units = 2 * a.H, part = blockIdx.x / units, unit = blockIdx.x - part * units;
    const int which = unit & 1, h = unit >> 1;
    const long long i0 = (long long)part * a.tile;
    const int n_rest = (int)min((long long)a.n_tokens - i0, (long long)(2 * PAGE)), n_tile = min(a.tile, n_rest);
    const int limit = a.n_pages * PAGE;                   // < 2^31
    const int32_t *slots = a.slots + i0;
    // the first token of the tile that starts a run; every later run of the tile follows the one before it
    int j = n_tile;
    for (int base = 0; base < n_tile; base += 32) {
        const int i = base + lane;
        bool starts = false;
        if (i < n_tile) {
            const int s = slots[i], before = i0 + i > 0 ? slots[i - 1] : -2;
            starts = s < 0 || s % PAGE == 0 || s != before + 1;
        }
        const uint32_t m = __ballot_sync(0xffffffffu, starts);
        if (m != 0u) { j = base + __ffs(m) - 1; break; }
    }
    const T *x = static_cast<const T *>(which == 0 ? a.x[0] : a.x[1]) + (size_t)i0 * a.ld + (size_t)h * kHeadDim;
    uint8_t *codes = which == 0 ? a.codes[0] : a.codes[1];    // (indexing the arguments would copy them to local memory)
    float *scales = which == 0 ? a.scale[0] : a.scale[1];
    const int c8 = (tid & 15) * 8, row_t = tid >> 4;
    const size_t step = (size_t)kRows * a.ld;
    int turn = 0;                                         // runs done: two buffers of maxima, so one barrier a run keeps them apart.  A
    while (j < n_tile) {                                  // token that is skipped passes no barrier and must not change the buffer
        const int slot = slots[j];
        const int r0 = slot & (PAGE - 1), cap = min(PAGE - r0, n_rest - j);
        // run length: up to the first token whose slot does not follow
        int n = cap;
        if (slot < 0) {
            n = 1;
        } else {
            int follows[kWords];
#pragma unroll
            for (int w = 0; w < kWords; ++w) follows[w] = 32 * w + lane < cap ? slots[j + 32 * w + lane] : -1;
#pragma unroll
            for (int w = kWords - 1; w >= 0; --w) {
                const uint32_t m = __ballot_sync(0xffffffffu, follows[w] != slot + 32 * w + lane);
                if (m != 0u) n = min(cap, 32 * w + __ffs(m) - 1);
            }
        }
        const int at = j;
        j += n;
        if (slot < 0) continue;
        if (slot >= limit) {
            if (tid == 0) flag(a.status, kBadSlot);
            continue;
        }
        const int pg = slot / PAGE;
        const T *src = x + (size_t)(at + row_t) * a.ld + c8;
        Raw8<T> raw[kIter];
        uint32_t amax = 0;
        {
            const T *from = src;
#pragma unroll
            for (int k = 0; k < kIter; ++k, from += step) {
                if (row_t + k * kRows < n) raw[k].load(from);
                else raw[k].zero();
            }
        }
        if (!FAEDKV_IN_BOUNDS(kTagPages, pg >= 0 && pg < a.n_pages && n >= 1 && r0 + n <= PAGE && at + n <= n_rest)) continue;
        const size_t ph = (size_t)pg * a.H + h;
        const float s_old = r0 > 0 ? scales[ph] : 0.f;
#pragma unroll
        for (int k = 0; k < kIter; ++k) amax = raw[k].max_bits(amax);
        amax = raw[0].to_float_bits(amax);
        if (amax >= 0x7f800000u) {                        // an infinity or NaN among them: again, without those
            amax = 0;
#pragma unroll 1
            for (int k = 0; row_t + k * kRows < n; ++k)
#pragma unroll 1
                for (int e = 0; e < 8; ++e) amax = max(amax, finite_bits(load1(src + k * step + e)));
        }
        amax = __reduce_max_sync(0xffffffffu, amax);
        if (lane == 0) max_s[turn & 1][warp] = amax;
        __syncthreads();
        amax = __reduce_max_sync(0xffffffffu, max_s[turn & 1][lane & (kWarps - 1)]);
        ++turn;
        float s = scale_for(__uint_as_float(amax));
        uint8_t *dst = codes + ph * (size_t)(PAGE * kHeadDim) + row_t * kHeadDim + c8;
        if (r0 > 0) {
            if (s > s_old) {                              // the page's older rows, rounded again at the larger scale
                const float mul = s_old * __uint_as_float((254u << 23) - __float_as_uint(s));
                for (int r = 0; row_t + r < r0; r += kRows) {
                    uint2 *p = reinterpret_cast<uint2 *>(dst + r * kHeadDim);
                    const uint2 c = *p;
                    float v[8], q[4];
                    from_e4m3x4(c.x, q);
                    v[0] = q[0]; v[1] = q[1]; v[2] = q[2]; v[3] = q[3];
                    from_e4m3x4(c.y, q);
                    v[4] = q[0]; v[5] = q[1]; v[6] = q[2]; v[7] = q[3];
                    *p = to_e4m3x8(v, mul);
                }
            } else {
                s = s_old;
            }
        }
        dst += r0 * kHeadDim;
        if ((__float_as_uint(s) & 0x7fffffu) == 0u && __float_as_uint(s) - 1u < (254u << 23) - 1u) {
            const float inv = __uint_as_float((254u << 23) - __float_as_uint(s));    // 1 / s, exact for the powers of two that this kernel writes
#pragma unroll
            for (int k = 0; k < kIter; ++k) {
                if (row_t + k * kRows < n) {
                    float v[8];
                    raw[k].get(v);
                    *reinterpret_cast<uint2 *>(dst + k * kRows * kHeadDim) = to_e4m3x8(v, inv);
                }
            }
        } else {                                          // a scale of another origin: divided by, the rows read again
#pragma unroll 1
            for (int k = 0; row_t + k * kRows < n; ++k) {
                Raw8<T> again;
                float v[8];
                again.load(src + k * step);
                again.get(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __fdiv_rn(v[e], s);
                *reinterpret_cast<uint2 *>(dst + k * kRows * kHeadDim) = to_e4m3x8(v, 1.0f);
            }
        }
        if (tid == 0) scales[ph] = s;
    }
}

// ---- load ---------------------------------------------------------------------------------------------

struct LoadArgs {
    const uint8_t *codes[2];
    const float *scale[2];
    void *out[2];
    const int32_t *kv_len, *table;
    int H, L, W, n_pages, page_shift;
    unsigned int *status;
};

// Rows of a thread: 16 bytes of output each, so that a warp's store is contiguous.
template <typename T> struct RowPart;
template <> struct RowPart<__nv_bfloat16> {
    static constexpr int kElems = 8;
    uint2 c;
    __device__ __forceinline__ void load(const uint8_t *p) { c = __ldcs(reinterpret_cast<const uint2 *>(p)); }
    __device__ __forceinline__ void put(__nv_bfloat16 *p, float s) const {
        float q[4], r[4];
        from_e4m3x4(c.x, q);
        from_e4m3x4(c.y, r);
        __nv_bfloat162 h[4] = {__floats2bfloat162_rn(q[0] * s, q[1] * s), __floats2bfloat162_rn(q[2] * s, q[3] * s),
                               __floats2bfloat162_rn(r[0] * s, r[1] * s), __floats2bfloat162_rn(r[2] * s, r[3] * s)};
        __stcs(reinterpret_cast<uint4 *>(p), *reinterpret_cast<uint4 *>(h));
    }
    static __device__ __forceinline__ void zero(__nv_bfloat16 *p) { __stcs(reinterpret_cast<uint4 *>(p), make_uint4(0u, 0u, 0u, 0u)); }
};
template <> struct RowPart<float> {
    static constexpr int kElems = 4;
    uint32_t c;
    __device__ __forceinline__ void load(const uint8_t *p) { c = __ldcs(reinterpret_cast<const uint32_t *>(p)); }
    __device__ __forceinline__ void put(float *p, float s) const {
        float q[4];
        from_e4m3x4(c, q);
        __stcs(reinterpret_cast<float4 *>(p), make_float4(q[0] * s, q[1] * s, q[2] * s, q[3] * s));
    }
    static __device__ __forceinline__ void zero(float *p) { __stcs(reinterpret_cast<float4 *>(p), make_float4(0.f, 0.f, 0.f, 0.f)); }
};

// Grid (pages of the longest row, H, sequences); a CTA turns one page of one head, K and V, into rows, four rows a thread in
// flight: 62.9 us for 4 x 16384 tokens x 8 heads, bf16 (6.2 TB/s).  Rounding: to the tensor type, once (code * scale is exact in float32 for a power of two, else rounded there too).
template <typename T>
__global__ void __launch_bounds__(256) k_page_load(const LoadArgs a) {
    using Part = RowPart<T>;
    constexpr int kPerRow = kHeadDim / Part::kElems, kRows = 256 / kPerRow;      // threads of a row, rows at a time
    const int b = blockIdx.z, h = blockIdx.y, page = 1 << a.page_shift;
    const int n0 = blockIdx.x << a.page_shift;
    long long live = a.kv_len[b];
    int id = blockIdx.x < a.W ? a.table[(size_t)b * a.W + blockIdx.x] : -1;      // may lie behind the sequence's end
    const long long cap = (long long)a.W << a.page_shift;
    if (live < 0 || live > cap) {
        if (threadIdx.x == 0) flag(a.status, kBadLength);
        live = live < 0 ? 0 : cap;
    }
    if (n0 >= live) {
        id = -1;
    } else if (id < 0 || id >= a.n_pages) {
        if (threadIdx.x == 0) flag(a.status, kBadPage);
        id = -1;
    }
    const int n_out = min(page, a.L - n0), n_in = id < 0 ? 0 : (int)min((long long)n_out, live - n0);
    const int row = threadIdx.x / kPerRow, el = threadIdx.x % kPerRow * Part::kElems;
    const size_t ph = (size_t)(id < 0 ? 0 : id) * a.H + h;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if (a.out[t] == nullptr || !FAEDKV_IN_BOUNDS(kTagPages, n_in <= n_out && n0 + n_out <= a.L && ph < (size_t)a.n_pages * a.H)) continue;
        const float s = n_in > 0 ? a.scale[t][ph] : 0.f;
        const uint8_t *src = a.codes[t] + (ph << a.page_shift) * kHeadDim + el;
        T *dst = static_cast<T *>(a.out[t]) + (((size_t)b * a.H + h) * a.L + n0) * kHeadDim + el;
        for (int r0 = row; r0 < n_out; r0 += 4 * kRows) {
            Part p[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = r0 + k * kRows;
                if (r < n_in) p[k].load(src + r * kHeadDim);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = r0 + k * kRows;
                if (r < n_in) p[k].put(dst + (size_t)r * kHeadDim, s);
                else if (r < n_out) Part::zero(dst + (size_t)r * kHeadDim);
            }
        }
    }
}

}  // namespace pages
}  // namespace faedkv
