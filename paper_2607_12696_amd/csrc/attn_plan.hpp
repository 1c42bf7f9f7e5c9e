// How the attention kernels over a paged cache share out their work, and how the parts are joined.
//
// The query rows of a sequence that read the same keys (its tokens times the heads of one key/value head) are cut into
// row groups of ROWS; the keys of a row group (cached tokens, then drafts) are cut into tiles of KEYS, and its tiles into
// chunks of about equal length, one workgroup each.  Lengths are known on the device only, so every workgroup works the
// plan out for itself, from the two offsets and the length of each sequence: the chunk length is the smallest for which
// all chunks run at once, or in two rounds where those are shorter.  (Row groups of different lengths leave chunks of
// different lengths: 8 trees over 6000 to 20000 tokens have chunks of up to 188 tiles at once, of 143 on average, and of up
// to 79 in two rounds: 375 us instead of 405 where a pass stands among others, 359 instead of 357 back to back.)  A row
// group of several chunks leaves its parts (fp32 output sums with the reference maximum and the sum of the weights of each
// row) in the workspace, in the matrix cores' accumulator order, and join_kernel adds them up in chunk order.
#pragma once

#include "attn.hpp"
#include "device.hpp"

namespace ecospec {

typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr int kCus = 256;        // compute units of an MI355X
constexpr float kLog2e = 1.44269504088896341f;

struct Shape {
    int rows, keys;  // of a row group and of a key tile
    int min_tiles;   // shortest chunk
    int slots;       // workgroups that run at once
    int twice;       // length from which chunks are cut for two rounds if that is shorter (0: never)
};

struct GroupInfo {
    int b, group;         // sequence; key/value head and row tile: head * row tiles + tile
    int chunks, slot0, stride;  // parts at slots slot0, slot0 + stride, ..
};

struct Item {
    int b, group, row_tiles;
    int t0, n_tok, len;   // first token, tokens and cached tokens of the sequence
    int first, last;      // key tiles
    int chunks, slot;
};

// Workspace: the row groups' records, then each slot's (maximum, sum) of ROWS rows, then each slot's output sums.
struct Parts {
    int *groups;      // number of row groups
    GroupInfo *info;
    float2 *ml;
    float *o;
    int max_groups, max_slots;  // room for records and for parts
};

inline long group_bound(int N, int B, int per_token, int heads, int rows)
{
    return ((long)N * per_token / rows + (N < B ? N : B)) * heads;
}

// Beyond this many row groups a slot nothing is cut.
constexpr int kRounds = 4;

constexpr int kStart = 8;  // what a chunk costs besides its tiles, in tiles

inline long grid_bound(long groups, int slots, bool twice)
{
    const long rounds = groups / slots + 1, cut = slots * (twice && rounds < 2 ? 2 : rounds), most = (long)kRounds * slots;
    return (groups >= most ? groups : cut < most ? cut : most) + 7 & ~7L;  // whole rounds of the XCDs
}

// The workspace for at most `groups` row groups, and its size.
inline size_t parts_at(void *workspace, long groups, int slots, bool twice, int rows, int width, Parts *p)
{
    const long cut = grid_bound(groups, slots, twice), n = cut < (long)kRounds * slots ? cut : (long)kRounds * slots;
    char *w = static_cast<char *>(workspace);
    const size_t ml = 256 + ((size_t)groups * sizeof(GroupInfo) + 255) / 256 * 256;
    const size_t o = ml + (size_t)n * rows * sizeof(float2);
    if (p)
        *p = Parts{reinterpret_cast<int *>(w), reinterpret_cast<GroupInfo *>(w + 256), reinterpret_cast<float2 *>(w + ml),
                   reinterpret_cast<float *>(w + o), (int)groups, (int)n};
    return o + (size_t)n * rows * width * sizeof(float);
}

__device__ __forceinline__ int wave_sum_int(int v) { return __builtin_amdgcn_readlane(wave_inclusive_sum(v), 63); }

// Sum of values up to 2^40, in two halves for the lane moves.
__device__ __forceinline__ long wave_sum_long(long v)
{
    v = v < (1L << 40) ? v : 1L << 40;
    return ((long)wave_sum_int((int)(v >> 16)) << 16) + wave_sum_int((int)(v & 0xffff));
}

// A sequence of the batch: its tokens and cache, and the row groups and key tiles that they make.
struct Sequence {
    int t0, n, len, groups, tiles;
};

__device__ __forceinline__ Sequence sequence(const PagedArgs &a, int b, int per_token, int heads, const Shape &s)
{
    Sequence q{0, 0, 0, 0, 0};
    if (b >= a.B) return q;
    const int from = a.token_offsets[b], to = a.token_offsets[b + 1], len = a.cache_len[b];
    q.t0 = min(max(from, 0), a.N);
    q.n = min(max(to, q.t0), a.N) - q.t0;
    q.len = min(max(len, 0), a.max_blocks * a.page);
    q.groups = (int)(((long)q.n * per_token + s.rows - 1) / s.rows) * heads;
    q.tiles = q.n ? (q.len + s.keys - 1) / s.keys + (min(q.n, kMaxDrafts) + s.keys - 1) / s.keys : 0;
    return q;
}

// This workgroup's item; every wavefront works it out for itself, a lane a sequence.  per_token: query rows of a token for
// one key/value head; heads: key/value heads.
__device__ __forceinline__ bool plan_item(const PagedArgs &a, int per_token, int heads, const Shape &s, const Parts &parts,
                                          Item &it)
{
    const int lane = lane_id();
    const Sequence mine = sequence(a, lane, per_token, heads, s);  // the first 64; others are read where they are needed
    int groups = mine.groups;
    long total = (long)mine.groups * mine.tiles;
    for (int b = lane + kWave; b < a.B; b += kWave) {
        const Sequence q = sequence(a, b, per_token, heads, s);
        groups += q.groups;
        total += (long)q.groups * q.tiles;
    }
    groups = wave_sum_int(groups);
    total = wave_sum_long(total);
    int c = 1 << 30, items = groups;
    if (groups < kRounds * s.slots) {
        const int room = s.slots * ((groups + s.slots - 1) / s.slots);
        auto count = [&](int len) {
            int n = mine.groups * ((mine.tiles + len - 1) / len);
            for (int b = lane + kWave; b < a.B; b += kWave) {
                const Sequence q = sequence(a, b, per_token, heads, s);
                n += q.groups * ((q.tiles + len - 1) / len);
            }
            return wave_sum_int(n);
        };
        auto fit = [&](int room) {
            c = max(s.min_tiles, (int)((float)total / (float)max(room, 1)));
            items = count(c);
            // Ends: chunks as long as the longest row group make one item of each, and there is room for those.
            for (int i = 0; items > room; ++i) items = count(c += max(1, i < 12 ? c / 16 : c / 4));
        };
        fit(room);
        if (s.twice && c >= s.twice && groups <= s.slots) {
            const int once = c, once_items = items;
            fit(2 * s.slots);
            if (2 * (c + kStart) >= once + kStart) {
                c = once;
                items = once_items;
            }
        }
    }
    // Neighbouring items (the row groups of one chunk read the same keys) run on one XCD, whose L2 they share:
    // workgroups are dealt to the eight XCDs in turn.
    const int per = (items + 7) / 8, want = (int)(blockIdx.x % 8) * per + (int)(blockIdx.x / 8);
    // More row groups than the workspace was sized for means that the offsets break their contract: nothing is joined,
    // and nothing is written past it.
    if (blockIdx.x == 0 && threadIdx.x == 0) *parts.groups = groups <= parts.max_groups ? groups : 0;
    if ((int)(blockIdx.x / 8) >= per || want >= items) return false;
    int before = 0, groups_before = 0;
    for (int b0 = 0;; b0 += kWave) {
        const Sequence q = b0 ? sequence(a, b0 + lane, per_token, heads, s) : mine;
        const int n = (q.tiles + c - 1) / c;
        const int upto = wave_inclusive_sum(q.groups * n), gsum = wave_inclusive_sum(q.groups);
        const uint64_t past = __ballot(before + upto > want);
        if (!past) {
            if (b0 + kWave >= a.B) return false;  // cannot be: want < items
            before += __builtin_amdgcn_readlane(upto, 63);
            groups_before += __builtin_amdgcn_readlane(gsum, 63);
            continue;
        }
        const int at = __ffsll((unsigned long long)past) - 1;
        const int gb = __builtin_amdgcn_readlane(q.groups, at), tb = __builtin_amdgcn_readlane(q.tiles, at);
        const int nb = __builtin_amdgcn_readlane(n, at);
        const int rest = want - before - (__builtin_amdgcn_readlane(upto, at) - gb * nb);
        const int chunk = rest / gb;
        it.b = b0 + at;
        it.group = rest % gb;
        it.row_tiles = gb / heads;
        it.t0 = __builtin_amdgcn_readlane(q.t0, at);
        it.n_tok = __builtin_amdgcn_readlane(q.n, at);
        it.len = __builtin_amdgcn_readlane(q.len, at);
        it.first = chunk * (tb / nb) + min(chunk, tb % nb);
        it.last = it.first + tb / nb + (chunk < tb % nb);
        it.chunks = nb;
        it.slot = want;
        const int record = groups_before + __builtin_amdgcn_readlane(gsum, at) - gb + it.group;
        if (record >= parts.max_groups || (nb > 1 && want >= parts.max_slots)) return false;
        if (chunk == 0 && threadIdx.x == 0) parts.info[record] = GroupInfo{it.b, it.group, nb, want, gb};
        return true;
    }
}

// Adds up the parts of a row group, 32 rows x 32 elements at a time.  A wavefront has a quarter of such a block: lane l the
// four consecutive elements that registers 4 * quarter .. of lane l of the accumulators hold.  Of a SPLIT workgroup the four
// wavefronts have one quarter and take every fourth part, so that few row groups of many parts still fill the card;
// otherwise they have the four quarters and all parts.
// ROWS: rows of a group; W: width of an output row; blocks of a part: row tile * (W / 32) + element tile.
template <int ROWS, int W, bool SPLIT>
__global__ __launch_bounds__(256) void join_kernel(PagedArgs a, int per_token, Parts p)
{
    constexpr int kBlocks = ROWS / 32 * (W / 32);
    __shared__ float tops[4][32];
    __shared__ f32x4 sums[3][kWave];
    __shared__ float totals[3][kWave];
    const int block = SPLIT ? blockIdx.x / 4 : blockIdx.x, wave = threadIdx.x / kWave;
    const int g = block / kBlocks, blk = block % kBlocks, quarter = SPLIT ? blockIdx.x % 4 : wave;
    if (g >= *p.groups) return;
    const GroupInfo in = p.info[g];
    if (in.chunks <= 1) return;
    const int lane = lane_id(), col = lane % 32, row = blk / (W / 32) * 32 + col;
    const float2 *ml = p.ml + (long)in.slot0 * ROWS + row;
    const f32x4 *o = reinterpret_cast<const f32x4 *>(p.o) + ((long)in.slot0 * kBlocks + blk) * 256 + quarter * 64 + lane;
    const long ml_step = (long)in.stride * ROWS, o_step = (long)in.stride * kBlocks * 256;
    const int first = SPLIT ? wave : 0;
    constexpr int kStep = SPLIT ? 4 : 1;
    float top = -INFINITY;
#pragma unroll 8
    for (int c = first; c < in.chunks; c += kStep) top = fmaxf(top, ml[c * ml_step].x);
    if (SPLIT) {
        tops[wave][col] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, tops[w][col]);
    }
    const float base = top == -INFINITY ? 0.f : top;
    float total = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int c = first; c < in.chunks; c += kStep) {
        const f32x4 v = o[c * o_step];
        const float2 part = ml[c * ml_step];
        const float f = __builtin_amdgcn_exp2f(part.x - base);
        total = fmaf(part.y, f, total);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = fmaf(v[i], f, sum[i]);
    }
    if (SPLIT) {
        if (wave) {
            sums[wave - 1][lane] = sum;
            totals[wave - 1][lane] = total;
        }
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int w = 0; w < 3; ++w) {
            total += totals[w][lane];
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += sums[w][lane][i];
        }
    }
    const int t0 = min(max(a.token_offsets[in.b], 0), a.N), n = min(max(a.token_offsets[in.b + 1], t0), a.N) - t0;
    const int tiles = (int)(((long)n * per_token + ROWS - 1) / ROWS), r = in.group % tiles * ROWS + row;
    if (r >= n * per_token) return;
    const long at = (long)(t0 + r / per_token) * a.H + in.group / tiles * per_token + r % per_token;
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const int e = blk % (W / 32) * 32 + quarter * 8 + lane / 32 * 4;
    *reinterpret_cast<u32x2 *>(a.o + at * W + e) = u32x2{pack_bf16x2(sum[0] * inv, sum[1] * inv),
                                                         pack_bf16x2(sum[2] * inv, sum[3] * inv)};
    if (a.lse && blk % (W / 32) == 0 && quarter == 0 && lane < 32)
        a.lse[at] = total == 0.f ? -INFINITY : (base + __builtin_amdgcn_logf(total)) / kLog2e;
}

template <int ROWS, int W>
void launch_join(const PagedArgs &a, int per_token, const Parts &p, long groups, hipStream_t stream)
{
    // 512 blocks put two workgroups on a compute unit; with more, the four wavefronts need not share one.  (24000 blocks of
    // 4 or 5 parts: 17 us whole, 32 us split; 64 blocks of 103 parts: 13 us whole, 8 us split.)
    const long blocks = groups * (ROWS / 32) * (W / 32);
    if (blocks < 2 * kCus) join_kernel<ROWS, W, true><<<(unsigned)(blocks * 4), 256, 0, stream>>>(a, per_token, p);
    else join_kernel<ROWS, W, false><<<(unsigned)blocks, 256, 0, stream>>>(a, per_token, p);
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// Larger of the two halves' values of a row (lanes l and l ^ 32), and their sum.
__device__ __forceinline__ float halves_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float halves_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Arithmetic on an accumulator tile where it lies, in the accumulation registers: written out, because the compiler would
// move all sixteen tiles to vector registers, and those to scratch, for it.  The waits at either end cover the matrix
// instructions around it (19 wait states from a product's write to a read); the tile as an operand keeps them in place.
__device__ __forceinline__ void acc_wait(f32x16 &o) { asm volatile("s_nop 15\n\ts_nop 7" : "+a"(o)); }

__device__ __forceinline__ void acc_scale(f32x16 &o, float f)
{
    acc_wait(o);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float x = o[i], t;
        asm volatile("v_accvgpr_read_b32 %1, %0\n\tv_mul_f32 %1, %2, %1\n\tv_accvgpr_write_b32 %0, %1" : "+a"(x), "=&v"(t) : "v"(f));
        o[i] = x;
    }
    acc_wait(o);
}

__device__ __forceinline__ bf16x8 pack_bf16x8(const float *f)
{
    bf16x8 w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = static_cast<__bf16>(f[i]);
    return w;
}

__device__ __forceinline__ uint64_t bits_below(int n)
{
    return n >= 64 ? ~0ull : (1ull << n) - 1;
}

}  // namespace ecospec
