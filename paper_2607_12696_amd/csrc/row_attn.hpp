// One workgroup for one query row (token, head): each wavefront takes every
// fourth key, keeps its own running maximum, sum and output, and the four are
// joined at the end.
#pragma once

#include "attn.hpp"
#include "device.hpp"

namespace ecospec {

// Sequence of token t: the b with off[b] <= t < off[b+1].
__device__ __forceinline__ int sequence_of(const int32_t *off, int B, int t)
{
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (off[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ uint64_t bits_below(int n)
{
    return n >= 64 ? ~0ull : (1ull << n) - 1;
}

// K: key elements of the dot product, V: value elements, both split over the
// lanes; src.keys(): number of keys, src.seen(j), src.score(j, e): the products
// of the lane's elements, src.value(j, e).
template <int V, class Src>
__device__ void row_attention(const Src &src, float scale, uint16_t *o, float *lse)
{
    constexpr int kPer = V / kWave;
    __shared__ float sm[4], sl[4], so[4][V];
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    float m = -INFINITY, l = 0.f, acc[kPer] = {};
    for (int j = wave; j < src.keys(); j += 4) {
        if (!src.seen(j)) continue;
        const float s = wave_sum(src.dot(j, lane)) * scale;
        const float top = fmaxf(m, s), base = top == -INFINITY ? 0.f : top;
        const float down = expf(m - base), p = expf(s - base);
        l = l * down + p;
#pragma unroll
        for (int i = 0; i < kPer; ++i) acc[i] = acc[i] * down + p * src.value(j, lane * kPer + i);
        m = top;
    }
    sm[wave] = m;
    sl[wave] = l;
#pragma unroll
    for (int i = 0; i < kPer; ++i) so[wave][lane * kPer + i] = acc[i];
    __syncthreads();
    const float top = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3])), base = top == -INFINITY ? 0.f : top;
    float total = 0.f, f[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) total += sl[w] * (f[w] = expf(sm[w] - base));
    const float inv = total == 0.f ? 0.f : 1.f / total;
    for (int e = threadIdx.x; e < V; e += 256) {
        float r = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) r += so[w][e] * f[w];
        o[e] = f32_to_bf16_bits(r * inv);
    }
    if (lse && threadIdx.x == 0) *lse = total == 0.f ? -INFINITY : base + logf(total);
}

// What a draft token of a paged call sees: the cached tokens, then the drafts
// of its sequence by its mask.
struct PagedRow {
    int t, b, h, t0, len, drafts;
    uint64_t mask;
    const int32_t *table;
    int n_pages, page;

    __device__ PagedRow(const PagedArgs &a)
    {
        t = blockIdx.x / a.H;
        h = blockIdx.x % a.H;
        b = sequence_of(a.token_offsets, a.B, t);
        t0 = min(max(a.token_offsets[b], 0), t);
        drafts = min(min(max(a.token_offsets[b + 1], t), a.N) - t0, kMaxDrafts);
        len = min(max(a.cache_len[b], 0), a.max_blocks * a.page);
        mask = (a.mask ? a.mask[t] : bits_below(t - t0 + 1)) & bits_below(drafts);
        table = a.block_table + (long)b * a.max_blocks;
        n_pages = a.n_pages;
        page = a.page;
    }
    __device__ int keys() const { return len + drafts; }
    __device__ bool seen(int j) const { return j < len || (mask >> (j - len) & 1); }
    __device__ long page_of(int j) const { return min(max(table[j / page], 0), n_pages - 1); }
};

}  // namespace ecospec
