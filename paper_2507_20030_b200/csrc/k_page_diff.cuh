// Differential attention over the paged 8-bit cache: the two maps of a head meet.
//
//     out[i, g] = norm(a1 - lam[g] * a2),   a_m = softmax(scale * q_m . K_m) V,   q = [q_1 | q_2], K = [K_1 | K_2], 64 channels each
//
// norm(o) = o * gain / sqrt(mean(o^2) + eps) over the head's 128 channels, or o itself without a gain.  k_page_attn and k_page_rows compute the a_m as
// columns (rows) of one pass over the cache: the codes of K and V are read once for both maps of all heads, and a map's query is zero in the other's
// channels, so that one product over 128 channels gives either score; half of its multiplications are with zero, which costs a decode step nothing (16 x
// 16384 tokens, 8 kv heads: 89 to 93 us, the bytes alone 82) and a prompt a quarter of its products.
#pragma once
#include "k_page_rows.cuh"

namespace faedkv {
namespace pages {

// o of one head, four channels a lane, normalised and stored.
template <typename T>
__device__ __forceinline__ void diff_finish(float4 a1, float4 a2, float lam, const float *gain, float eps, int lane, T *out) {
    float4 o = make_float4(fmaf(-lam, a2.x, a1.x), fmaf(-lam, a2.y, a1.y), fmaf(-lam, a2.z, a1.z), fmaf(-lam, a2.w, a1.w));
    if (gain != nullptr) {
        auto squares = [&]() {
            float ss = fmaf(o.x, o.x, o.y * o.y) + fmaf(o.z, o.z, o.w * o.w);
#pragma unroll
            for (int s = 16; s; s >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, s);
            return ss;
        };
        float ss = squares();
        const float m = ss * (1.0f / kHeadDim) + eps;
        if (!diff_in_range(m)) {                           // (the same in all lanes)
            const float unit = diff_unit(m);
            o = make_float4(o.x * unit, o.y * unit, o.z * unit, o.w * unit);
            ss = squares();
            eps = eps * unit * unit;
        }
        const float r = diff_norm(ss, eps);
        const float4 w = load4(gain + 4 * lane);
        o = make_float4(o.x * (r * w.x), o.y * (r * w.y), o.z * (r * w.z), o.w * (r * w.w));
    }
    store4(out + 4 * lane, o);
}

// Split units and, of a decode step, all others.  A warp for each head.  MODE 0: grid (tokens x heads / 8); MODE 1 (the form with rows, which finishes its
// whole units itself): grid (CTAs, heads of a unit / 8), the second CTA of a shared unit looks after it.
template <typename T, int MODE>
__global__ void __launch_bounds__(256) k_page_diff_join(const AttnArgs a, const DiffArgs diff, const int qc, const int ctas) {
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float *slots = reinterpret_cast<const float *>(a.ws + attn_meta_bytes(MODE, (size_t)a.B * a.H, ctas));
    const size_t step = 2 * attn_slot_floats(qc);
    const int heads = a.G / 2;                             // of a kv head
    const long long share = *reinterpret_cast<const long long *>(a.ws);
    int tok, h, g, c;
    long long first;
    int tiles;
    if constexpr (MODE == 0) {
        const long long i = (long long)blockIdx.x * 8 + warp;
        if (i >= (long long)a.n_tokens * diff.HQ) return;
        tok = (int)(i / diff.HQ);
        const int head = (int)(i - (long long)tok * diff.HQ);
        h = head / heads;
        g = head - h * heads;
        c = 2 * g;
        const UnitMeta m = reinterpret_cast<const UnitMeta *>(a.ws + 16)[(size_t)tok * a.H + h];
        first = m.first; tiles = m.tiles;
    } else {
        const CtaMeta m = reinterpret_cast<const CtaMeta *>(a.ws + 16)[blockIdx.x];
        first = m.first; tiles = m.tiles;
        c = 2 * ((int)blockIdx.y * 8 + warp);
        if (tiles == 0 || c >= m.n_cols) return;           // this CTA began with a unit of its own
        const int k = c / a.G;
        tok = m.tok0 + k;
        h = m.h;
        g = (c - k * a.G) >> 1;
    }
    const int cta0 = cta_of(first, share), cta1 = cta_of(first + tiles - 1, share);
    if (MODE == 1 && cta0 + 1 != (int)blockIdx.x) return;  // another one's
    if (!FAEDKV_IN_BOUNDS(kTagPageAttn, cta0 >= 0 && cta1 < ctas && tok >= 0 && tok < a.n_tokens && h >= 0 && h < a.H)) return;
    const size_t row = ((size_t)tok * a.H + h) * heads + g;
    float4 a1, a2;
    if (MODE == 0 && cta0 == cta1) {                       // one CTA had it all
        const float *x = diff.maps + row * 2 * kHeadDim + 4 * lane;
        a1 = load4(x);
        a2 = load4(x + kHeadDim);
    } else {
        float4 maps[2];
        gather_parts<2>([&](int i, int k) { return SlotColumn(slots + (cta0 + i) * step + (i == 0 ? step / 2 : 0), qc, c + k); }, cta1 - cta0 + 1, lane, maps);
        a1 = maps[0];
        a2 = maps[1];
    }
    diff_finish(a1, a2, diff.lam[row % diff.HQ], diff.gain, diff.eps, lane, static_cast<T *>(diff.out) + row * kHeadDim);
}

// Heads whose maps are complete, a warp for each (token, head).
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
