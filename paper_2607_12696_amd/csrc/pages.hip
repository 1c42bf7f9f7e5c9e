// Pages of sequences whose lengths change, and rows into the latent cache.
//
// pages_kernel: from the counts alone (old length, kept, new tokens) follow the
// pages that every sequence returns and takes; two prefix sums over the
// sequences give each its place in the list of free pages (the free ones, then
// the returned ones; taken from the end).  Every workgroup works the sums out
// for itself, up to 1024 sequences in LDS, and then does its share of the
// returned pages, the taken pages and the tokens: one search for the sequence,
// one read of the page.  A taken page that another sequence returns in the same
// call is read from that one's row of the table, which nothing changes, so no
// workgroup waits for another.
// What bounds it: latency (counts, prefix sums, search, page, store): 4
// sequences of 5 new tokens at most 3.6 us, 256 sequences of 28963 8.0.
#include "device.hpp"
#include "step.hpp"

namespace ecospec {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

// Sums past 2^30 cannot come from counts that keep their contract; they are cut there to stay in 32 bits.
constexpr long kMost = 1L << 30;

__device__ __forceinline__ long wave_inclusive_long(long v)
{
    const int lane = lane_id();
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
        const long x = __shfl_up(v, s, kWave);
        v += lane >= s ? x : 0;
    }
    return v;
}

struct Counts {
    int old, keep, from, fresh, have, want;  // want -1: past the table
};

struct Lds {
    Counts seq[kMaxSequences];
    int back[kMaxSequences], take[kMaxSequences];  // inclusive sums over the sequences
    long wave_back[kWaves], wave_take[kWaves];
    int refused[kWaves], taken[kWaves];
};

// First b of the sequences for which past(b) holds, B if none; past must not turn false again.
template <class F>
__device__ __forceinline__ int first_past(int B, F past)
{
    int lo = 0, hi = B;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (past(mid)) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

__global__ __launch_bounds__(kThreads) void pages_kernel(PagesArgs a)
{
    __shared__ Lds s;
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const long room = (long)a.max_blocks * a.page;
    long before_back = 0, before_take = 0;
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const int b = b0 + threadIdx.x;
        Counts c{};
        long back = 0, take = 0;
        if (b < a.B) {
            c.old = (int)min((long)max(a.cache_len[b], 0), room);
            c.keep = a.keep_len ? min(max(a.keep_len[b], 0), c.old) : c.old;
            c.from = min(max(a.token_offsets[b], 0), a.N);
            c.fresh = min(max(a.token_offsets[b + 1], c.from), a.N) - c.from;
            c.have = (c.old + a.page - 1) / a.page;
            c.want = (int)(((long)c.keep + c.fresh + a.page - 1) / a.page);
            if (c.want > a.max_blocks) c.want = -1;
            back = c.want >= 0 ? max(c.have - c.want, 0) : 0;
            take = max(c.want - c.have, 0);
            s.seq[b] = c;
        }
        back = wave_inclusive_long(back);
        take = wave_inclusive_long(take);
        if (lane == kWave - 1) {
            s.wave_back[wave] = back;
            s.wave_take[wave] = take;
        }
        __syncthreads();
        back += before_back;
        take += before_take;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            back += w < wave ? s.wave_back[w] : 0;
            take += w < wave ? s.wave_take[w] : 0;
            before_back += s.wave_back[w];
            before_take += s.wave_take[w];
        }
        if (b < a.B) {
            s.back[b] = (int)min(back, kMost);
            s.take[b] = (int)min(take, kMost);
        }
        __syncthreads();
    }
    const int n_free = min(max(*a.n_free, 0), a.n_pages);
    const int returned = (int)min(before_back, kMost), asked = (int)min(before_take, kMost);
    const long avail = (long)n_free + returned;

    auto fits = [&](int b) {
        const Counts &c = s.seq[b];
        return c.want >= 0 && (c.want <= c.have || s.take[b] <= avail);
    };
    // Page r of all that are returned, in order.
    auto returned_page = [&](int r) {
        const int b = min(first_past(a.B, [&](int i) { return s.back[i] > r; }), a.B - 1);
        const Counts &c = s.seq[b];
        const int last = max(c.have - 1, 0), blk = c.have - (s.back[b] - r);
        return a.block_table[(long)b * a.max_blocks + min(max(blk, 0), last)];
    };
    // Page t of all that are taken, in order.
    auto taken_page = [&](int t) {
        const long v = avail - 1 - t;
        return v < n_free ? a.free_pages[max(v, 0L)] : returned_page((int)(v - n_free));
    };

    const int at = blockIdx.x * kThreads + threadIdx.x, step = gridDim.x * kThreads;
    for (int r = at; r < returned && (long)n_free + r < a.n_pages; r += step) a.free_pages[n_free + r] = returned_page(r);
    for (int t = at; t < asked && t < avail; t += step) {
        const int b = min(first_past(a.B, [&](int i) { return s.take[i] > t; }), a.B - 1);
        if (s.take[b] > avail) break;  // refused, and so are all that come after
        const Counts &c = s.seq[b];
        const int blk = c.want - (s.take[b] - t);
        if (blk >= c.have) a.block_table[(long)b * a.max_blocks + blk] = taken_page(t);
    }
    for (int t = at; t < a.N && (a.slots || a.positions); t += step) {
        // The last sequence that begins at or before token t: the ones that begin there and end there come first.
        const int lo = max(first_past(a.B, [&](int i) { return s.seq[i].from > t; }) - 1, 0);
        const Counts &c = s.seq[lo];
        int pos = -1;
        long slot = -1;
        if (t >= c.from && t - c.from < c.fresh && fits(lo)) {
            pos = c.keep + (t - c.from);
            const int blk = pos / a.page;
            const int id = blk < c.have ? a.block_table[(long)lo * a.max_blocks + blk] : taken_page(s.take[lo] - (c.want - blk));
            slot = (long)id * a.page + pos % a.page;
        }
        if (a.slots) a.slots[t] = slot;
        if (a.positions) a.positions[t] = pos;
    }

    if (blockIdx.x) return;
    int refused = 0, taken = 0;
    for (int b = threadIdx.x; b < a.B; b += kThreads) {
        const Counts &c = s.seq[b];
        const bool ok = fits(b);
        a.new_len[b] = ok ? c.keep + c.fresh : c.old;
        refused += !ok;
        if (ok && c.want > c.have) taken = max(taken, s.take[b]);
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
        refused += __shfl_xor(refused, m, kWave);
        taken = max(taken, __shfl_xor(taken, m, kWave));
    }
    if (lane == 0) {
        s.refused[wave] = refused;
        s.taken[wave] = taken;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
            refused += s.refused[w];
            taken = max(taken, s.taken[w]);
        }
        *a.refused = refused;
        *a.n_free_out = (int)min(avail - taken, (long)a.n_pages);
    }
}

// A thread moves 16 bytes; a row of 576 elements has 72 such parts.  64 rows 2.2 us; 15001 rows, 34.6 MB read and written,
// 6.5 to 6.9 us: 5.1 TB/s, the rate of a large copy.
constexpr int kParts = kLatentRow / 8;

__global__ __launch_bounds__(kThreads) void latent_append_kernel(RowsArgs a)
{
    const uint32_t at = blockIdx.x * (uint32_t)kThreads + threadIdx.x, i = at / kParts, c = at % kParts;
    if (i >= (uint32_t)a.N) return;
    const long slot = a.slots[i];
    const int row = a.rows ? min(max(a.rows[i], 0), a.n_rows - 1) : (int)i;
    if (slot < 0 || slot >= a.slots_end) return;
    reinterpret_cast<u32x4 *>(a.pages)[slot * kParts + c] = reinterpret_cast<const u32x4 *>(a.kv_new)[(long)row * kParts + c];
}

}  // namespace

hipError_t launch_pages_update(const PagesArgs &a, hipStream_t stream)
{
    // A share of about 4 tokens or 16 table entries a thread, and no more workgroups than compute units.
    const long items = (long)a.N / 4 + (long)a.B * a.max_blocks / 16, want = items / kThreads + 1;
    pages_kernel<<<(unsigned)(want < 256 ? want : 256), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_latent_append(const RowsArgs &a, hipStream_t stream)
{
    const long threads = (long)a.N * kParts;
    latent_append_kernel<<<(unsigned)((threads + kThreads - 1) / kThreads), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace ecospec
