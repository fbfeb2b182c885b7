// Attention over the paged 8-bit cache.
//
//     out[i, g] = sum_n softmax_n( scale * q[i, g] . K[n] ) V[n],   n < kv_len - n_new + i + 1
//
// for the i-th of a sequence's n_new newest tokens; K and V are code * scale of the pages in the sequence's table row.
#pragma once
#include "common.cuh"
#include "k_pages.cuh"

namespace faedkv {
namespace pages {

struct AttnArgs {
    const void *q;
    void *out;
    const int32_t *q_start, *kv_len, *table;              // q_start may be NULL: one token per sequence
    const uint8_t *kc, *vc;
    const float *ks, *vs;
    long long ld_q;
    int n_tokens, B, H, G, W, n_pages, page_shift;
    float scale;
    unsigned int *status;
};

// One CTA per (query token, kv head): 8 warps stride over the cached tokens, a lane holds 4 channels of the G query
// heads; each warp keeps a running maximum, sum and output, joined at the end.
template <typename T, int G>
__global__ void __launch_bounds__(256) k_page_attn_simple(const AttnArgs a) {
    __shared__ float m_s[8][G], l_s[8][G], o_s[8][G][kHeadDim];
    const int i = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int b = i, n_new = 1, k = 0;
    if (a.q_start != nullptr) {
        if (i >= a.q_start[a.B]) return;
        b = find_sequence(a.q_start, a.B, i);
        n_new = a.q_start[b + 1] - a.q_start[b];
        k = i - a.q_start[b];
    }
    long long live = a.kv_len[b];
    if (live < 0 || live > ((long long)a.W << a.page_shift)) {
        if (threadIdx.x == 0) flag(a.status, kBadLength);
        live = live < 0 ? 0 : (long long)a.W << a.page_shift;
    }
    live = min(live, live - n_new + k + 1);
    float q[G][4], o[G][4], m[G], l[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const float4 v = load4(static_cast<const T *>(a.q) + (size_t)i * a.ld_q + (size_t)(h * G + g) * kHeadDim + lane * 4);
        q[g][0] = v.x; q[g][1] = v.y; q[g][2] = v.z; q[g][3] = v.w;
        o[g][0] = o[g][1] = o[g][2] = o[g][3] = 0.f;
        m[g] = -INFINITY; l[g] = 0.f;
    }
    for (int n = warp; n < live; n += 8) {
        const int id = a.table[(size_t)b * a.W + (n >> a.page_shift)];
        if (id < 0 || id >= a.n_pages) { if (lane == 0) flag(a.status, kBadPage); continue; }
        const size_t ph = (size_t)id * a.H + h;
        const size_t at = ((ph << a.page_shift) + (n & ((1 << a.page_shift) - 1))) * kHeadDim + lane * 4;
        float kx[4], vx[4];
        from_e4m3x4(*reinterpret_cast<const uint32_t *>(a.kc + at), kx);
        from_e4m3x4(*reinterpret_cast<const uint32_t *>(a.vc + at), vx);
        const float ks = a.ks[ph] * a.scale, vs = a.vs[ph];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float d = q[g][0] * kx[0] + q[g][1] * kx[1] + q[g][2] * kx[2] + q[g][3] * kx[3];
#pragma unroll
            for (int s = 16; s; s >>= 1) d += __shfl_xor_sync(0xffffffffu, d, s);
            d *= ks;
            const float mn = fmaxf(m[g], d), c = __expf(m[g] - mn), p = __expf(d - mn);
            m[g] = mn;
            l[g] = l[g] * c + p;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[g][e] = o[g][e] * c + p * vs * vx[e];
        }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
        if (lane == 0) { m_s[warp][g] = m[g]; l_s[warp][g] = l[g]; }
#pragma unroll
        for (int e = 0; e < 4; ++e) o_s[warp][g][lane * 4 + e] = o[g][e];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < G * kHeadDim; e += 256) {
        const int g = e / kHeadDim, c = e % kHeadDim;
        float mx = -INFINITY, ls = 0.f, acc = 0.f;
        for (int w = 0; w < 8; ++w) mx = fmaxf(mx, m_s[w][g]);
        if (mx > -INFINITY)
            for (int w = 0; w < 8; ++w) {
                const float f = __expf(m_s[w][g] - mx);
                ls += l_s[w][g] * f;
                acc += o_s[w][g][c] * f;
            }
        store1(static_cast<T *>(a.out) + ((size_t)i * a.H * G + h * G + g) * kHeadDim + c, ls > 0.f ? acc / ls : 0.f);
    }
}

}  // namespace pages
}  // namespace faedkv
