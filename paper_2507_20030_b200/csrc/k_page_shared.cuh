// One new token of every row, where groups of rows share their first pages: the join.
//
// k_page_rows or k_page_attn (MODE 3, 4) attends the rows of a group together over the tokens that they share, as columns of one product that reads each
// shared page once, and each row alone over the tokens behind.  The two results of a query row, each in parts where it was split over
// CTAs, meet here as parts of any softmax do: out = sum_i l_i 2^(m_i - m) o_i / sum_i l_i 2^(m_i - m), m the largest m_i.
#pragma once
#include "k_page_rows.cuh"

namespace faedkv {
namespace pages {

// Where the parts of a unit lie: `n` of them, part i's statistics and output at strides.
struct UnitParts {
    const float *mu, *sum, *o;                            // of the first part
    long long step, skip;                                 // from part to part; from the first to the second besides
    int n;
    __device__ __forceinline__ long long at(int i) const { return i * step - (i > 0 ? skip : 0); }
};

// Grid: a CTA for each (row, kv head); 128 channels x kJoinGroups of its columns.
template <typename T, int MODE>
__global__ void __launch_bounds__(kHeadDim *kJoinGroups) k_page_join_shared(const AttnArgs a, const int qc, const bool rows, const int ctas) {
    pdl_wait();
    const int d = threadIdx.x, b = blockIdx.x / a.H, h = blockIdx.x - b * a.H, tq = qc / a.G;
    const int live = (int)clamp_len(a, b, false), n_shared = shared_blocks(a.B, a.n_groups, tq);
    int g, first;
    const int share = shared_of(a, b, live, false, g, first);
    const long long per_cta = MODE == 3 ? *reinterpret_cast<const long long *>(a.ws) : 1;
    const int32_t *before = reinterpret_cast<const int32_t *>(a.ws + 16);
    const float *slots = reinterpret_cast<const float *>(a.ws + shared_meta_bytes(a.blocks, (size_t)a.B * a.H * a.G));
    const long long step = 2 * (long long)attn_slot_floats(qc);
    for (int c = threadIdx.y; c < a.G; c += kJoinGroups) {
        const size_t i_row = ((size_t)b * a.H + h) * a.G + c;
        UnitParts parts[2];
#pragma unroll
        for (int own = 0; own < 2; ++own) {
            UnitParts &u = parts[own];
            u.n = 0;
            if (own ? live <= share : share == 0) continue;
            const SharedParts whole(a.ws, a.blocks, a.B, a.H * a.G, own);
            u.n = 1;
            u.mu = reinterpret_cast<const float *>(whole.stat + i_row);
            u.sum = u.mu + 1;
            u.o = whole.o + i_row * kHeadDim + d;
            u.step = u.skip = 0;
            if constexpr (MODE == 3) {
                const int j = own ? 0 : (b - first) / tq, v = own ? n_shared + b : first / tq + g + j;
                // positions of the unit's tiles, of one tile
                const int cost = rows ? kRowsCost : kUnitCost, n = before[v + 1] - before[v] - cost;
                const int each = rows && !own ? rows_weight(min(tq, a.group_start[g + 1] - first - j * tq) * a.G) : 1;
                const long long pos = (long long)h * before[a.blocks] + before[v] + cost;
                const int cta0 = (int)(pos / per_cta), cta1 = (int)((pos + n - each) / per_cta);
                if (!FAEDKV_IN_BOUNDS(kTagPageAttn, n > 0 && cta0 >= 0 && cta1 < ctas)) { u.n = 0; continue; }
                if (cta0 != cta1) {
                    const int col = own ? c : (b - first - j * tq) * a.G + c;
                    const float *slot = slots + cta0 * step + step / 2;      // a part that begins a unit: the CTA's second
                    u.n = cta1 - cta0 + 1;
                    u.mu = slot + col;
                    u.sum = slot + qc + col;
                    u.o = slot + 2 * qc + (size_t)col * kHeadDim + d;
                    u.step = step;
                    u.skip = step / 2;
                }
            }
        }
        float mu = kMuNone, sum = 0.f, o = 0.f;
#pragma unroll
        for (int own = 0; own < 2; ++own)
#pragma unroll 4
            for (int i = 0; i < parts[own].n; ++i) mu = fmaxf(mu, parts[own].mu[parts[own].at(i)]);
#pragma unroll
        for (int own = 0; own < 2; ++own)
#pragma unroll 4
            for (int i = 0; i < parts[own].n; ++i) {
                const long long at = parts[own].at(i);
                const float l = parts[own].sum[at] * ex2(parts[own].mu[at] - mu);      // a part's output is divided by its sum already
                sum += l;
                o = fmaf(parts[own].o[at], l, o);
            }
        store1(static_cast<T *>(a.out) + i_row * kHeadDim + d, sum == 0.f ? 0.f : __fdiv_rn(o, sum));
    }
}

}  // namespace pages
}  // namespace faedkv
