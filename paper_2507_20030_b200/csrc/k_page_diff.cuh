// Differential attention over the paged 8-bit cache: the two maps of a head meet.
//
//     out[i, g] = norm(a1 - lam[g] * a2),   a_m = softmax(scale * q_m . K_m) V,   q = [q_1 | q_2], K = [K_1 | K_2], 64 channels each
//
// norm(o) = o * gain / sqrt(mean(o^2) + eps) over the head's 128 channels, or o itself without a gain.  k_page_attn computes the a_m as
// columns of one pass over the cache: the codes of K and V are read once for both maps of all heads.
#pragma once
#include "common.cuh"
#include "k_pages.cuh"

namespace faedkv {
namespace pages {

struct DiffArgs {
    const float *maps;                                    // [n_tokens][n_q_heads][2][128]
    const float *lam, *gain;                              // [n_q_heads]; [128] or NULL
    void *out;
    const int32_t *q_start;                               // may be NULL: every row is a token
    int n_tokens, B, HQ;
    float eps;
};

// o of one head, four channels a lane, normalised and stored.
template <typename T>
__device__ __forceinline__ void diff_finish(float4 a1, float4 a2, float lam, const float *gain, float eps, int lane, T *out) {
    float4 o = make_float4(fmaf(-lam, a2.x, a1.x), fmaf(-lam, a2.y, a1.y), fmaf(-lam, a2.z, a1.z), fmaf(-lam, a2.w, a1.w));
    if (gain != nullptr) {
        float ss = fmaf(o.x, o.x, o.y * o.y) + fmaf(o.z, o.z, o.w * o.w);
#pragma unroll
        for (int s = 16; s; s >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, s);
        const float m = ss * (1.0f / kHeadDim) + eps, r = m > 0.f ? rsqrtf(m) : m;   // a row of zeros stays one without eps; NaN stays NaN
        const float4 w = load4(gain + 4 * lane);
        o = make_float4(o.x * (r * w.x), o.y * (r * w.y), o.z * (r * w.z), o.w * (r * w.w));
    }
    store4(out + 4 * lane, o);
}

// A warp for each (token, head).
template <typename T>
__global__ void __launch_bounds__(256) k_page_diff(const DiffArgs a) {
    pdl_wait();
    const long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (i >= (long long)a.n_tokens * a.HQ) return;
    const int tok = (int)(i / a.HQ), g = (int)(i - (long long)tok * a.HQ);
    if (a.q_start != nullptr) {                            // rows of no sequence, or of one that passes n_tokens, are left as they were
        const int b = find_sequence(a.q_start, a.B, tok), first = a.q_start[b], end = a.q_start[b + 1];
        if (tok < first || tok >= end || first < 0 || end > a.n_tokens) return;
    }
    const float *x = a.maps + (size_t)i * 2 * kHeadDim + 4 * lane;
    diff_finish(load4(x), load4(x + kHeadDim), a.lam[g], a.gain, a.eps, lane, static_cast<T *>(a.out) + (size_t)i * kHeadDim);
}

}  // namespace pages
}  // namespace faedkv
