// One new token of every row, where groups of rows share their first pages: the join.
//
// k_page_rows or k_page_attn (MODE 3, 4) attends the rows of a group together over the tokens that they share, as columns of one product that reads each
// shared page once, and k_page_attn each row alone over the tokens behind.  The two results of a query row, each in parts where it was split over
// CTAs, meet here as parts of any softmax do: out = sum_i l_i 2^(m_i - m) o_i / sum_i l_i 2^(m_i - m), m the largest m_i.
//
// Measured, 8 kv x 32 query heads: 64 rows behind 32768 common tokens and up to 512 of their own 87 us (409 read by each row for itself; at full rate the
// shared pages take 10 us, the tails 5 and the products 20), 8 rows behind 2048 16.8 us (17.8), mostly start, join and its launch.
#pragma once
#include "k_page_rows.cuh"

namespace faedkv {
namespace pages {

// What the join has to know of a launch: where its header and its CTAs' partial results lie, columns of a block, positions that a unit costs besides its
// tiles, whether its form has rows (two row tiles count twice), CTAs, and the blocks of groups and all blocks that it numbers.
struct SharedLaunch {
    const unsigned char *ws;
    const float *slots;
    int qc, cost, rows, ctas, n_shared, blocks;
};

// A warp for each query row.  by_group, by_row: the launches of the groups' blocks and of the rows' own (the same, where one had both).
template <typename T, int MODE>
__global__ void __launch_bounds__(256) k_page_join_shared(const AttnArgs a, const SharedLaunch by_group, const SharedLaunch by_row) {
    pdl_wait();
    const int lane = threadIdx.x & 31, heads = a.H * a.G;
    const long long i_row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (i_row >= (long long)a.B * heads) return;
    const int b = (int)(i_row / heads), head = (int)(i_row - (long long)b * heads), h = head / a.G, c = head - h * a.G;
    const int live = (int)clamp_len(a, b, false);
    int g, first;
    const int share = shared_of(a, b, live, false, g, first);
    // the parts of the group's result (0) and of the row's own (1): how many, and where they are split the first one's CTA (else -1), the column
    int n[2] = {0, 0}, cta0[2] = {-1, -1}, col[2] = {0, c};
#pragma unroll
    for (int own = 0; own < 2; ++own) {
        const SharedLaunch &u = own ? by_row : by_group;
        if (own ? live <= share : share == 0) continue;
        n[own] = 1;
        if constexpr (MODE == 3) {
            const int32_t *before = reinterpret_cast<const int32_t *>(u.ws + 16);
            const long long per_cta = *reinterpret_cast<const long long *>(u.ws);
            const int tq = u.qc / a.G, j = own ? 0 : (b - first) / tq, v = own ? u.n_shared + b : first / tq + g + j;
            // positions of the unit's tiles, of one tile
            const int size = before[v + 1] - before[v] - u.cost;
            if (size <= 0) { n[own] = 0; continue; }       // (no such block)
            const int each = u.rows && !own ? rows_weight(min(tq, a.group_start[g + 1] - first - j * tq) * a.G) : 1;
            const long long pos = (long long)h * before[u.blocks] + before[v] + u.cost;
            const int from = cta_of(pos, per_cta), to = cta_of(pos + size - each, per_cta);
            if (!FAEDKV_IN_BOUNDS(kTagPageAttn, size > 0 && from >= 0 && to < u.ctas)) { n[own] = 0; continue; }
            if (from != to) {
                n[own] = to - from + 1;
                cta0[own] = from;
                if (!own) col[0] = (b - first - j * tq) * a.G + c;
            }
        }
    }
    float4 o[1];
    gather_parts<1>([&](int i, int) {
        const int own = i >= n[0], k = own ? i - n[0] : i, cta = own ? cta0[1] : cta0[0];
        if (cta < 0) {
            const SharedParts whole(a.whole, (size_t)a.B * heads, own);
            return PartColumn{&whole.stat[i_row].x, &whole.stat[i_row].y, whole.o + i_row * kHeadDim};
        }
        const int qc = own ? by_row.qc : by_group.qc;
        const size_t slot = attn_slot_floats(qc);          // a part that begins a unit: the CTA's second
        return SlotColumn((own ? by_row.slots : by_group.slots) + (2 * (size_t)(cta + k) + (k == 0 ? 1 : 0)) * slot, qc, own ? col[1] : col[0]);
    }, n[0] + n[1], lane, o);
    store4(static_cast<T *>(a.out) + i_row * kHeadDim + 4 * lane, o[0]);
}

}  // namespace pages
}  // namespace faedkv
