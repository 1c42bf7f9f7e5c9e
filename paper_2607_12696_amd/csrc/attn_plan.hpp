// How the attention kernels over a paged cache share out their work, and how the parts are joined.
//
// The query rows of a sequence that read the same keys (its tokens times the heads of one key/value head) are cut into
// row groups of ROWS; the keys of a row group (cached tokens, then drafts) are cut into tiles of KEYS, and its tiles into
// chunks of about equal length, one workgroup each.  Lengths are known on the device only, so every workgroup works the
// plan out for itself, from the two offsets and the length of each sequence: the chunk length is the smallest for which
// all chunks run at once.  A row group of several chunks leaves its parts (fp32 output sums with the reference maximum
// and the sum of the weights of each row) in the workspace, in the matrix cores' accumulator order, and join_kernel adds
// them up in chunk order.
#pragma once

#include "attn.hpp"
#include "device.hpp"

namespace ecospec {

typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr int kCus = 256;        // compute units of an MI355X
constexpr int kPlanB = 1024;     // most sequences of a call
constexpr float kLog2e = 1.44269504088896341f;

struct Shape {
    int rows, keys;  // of a row group and of a key tile
    int min_tiles;   // shortest chunk
    int slots;       // workgroups that run at once
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

inline long grid_bound(long groups, int slots)
{
    const long cut = (long)slots * (groups / slots + 1), most = (long)kRounds * slots;
    return (groups >= most ? groups : cut < most ? cut : most) + 7 & ~7L;  // whole rounds of the XCDs
}

// The workspace for at most `groups` row groups, and its size.
inline size_t parts_at(void *workspace, long groups, int slots, int rows, int width, Parts *p)
{
    const long cut = grid_bound(groups, slots), n = cut < (long)kRounds * slots ? cut : (long)kRounds * slots;
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

// This workgroup's item.  work: 2 * B ints of LDS, free again after the call's last barrier.  per_token: query rows of a
// token for one key/value head; heads: key/value heads.
__device__ __forceinline__ bool plan_item(const PagedArgs &a, int per_token, int heads, const Shape &s, const Parts &parts,
                                          int *work, Item &it)
{
    for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
        const int t0 = min(max(a.token_offsets[b], 0), a.N), n = min(max(a.token_offsets[b + 1], t0), a.N) - t0;
        const int len = min(max(a.cache_len[b], 0), a.max_blocks * a.page);
        work[2 * b] = (int)(((long)n * per_token + s.rows - 1) / s.rows) * heads;
        work[2 * b + 1] = n ? (len + s.keys - 1) / s.keys + (min(n, kMaxDrafts) + s.keys - 1) / s.keys : 0;
    }
    __syncthreads();
    const int lane = lane_id();
    int groups = 0;
    long total = 0;
    for (int b = lane; b < a.B; b += kWave) {
        groups += work[2 * b];
        total += (long)work[2 * b] * work[2 * b + 1];
    }
    groups = wave_sum_int(groups);
    total = wave_sum_long(total);
    int c = 1 << 30, items = groups;
    if (groups < kRounds * s.slots) {
        const int room = s.slots * ((groups + s.slots - 1) / s.slots);
        auto count = [&](int len) {
            int n = 0;
            for (int b = lane; b < a.B; b += kWave) n += work[2 * b] * ((work[2 * b + 1] + len - 1) / len);
            return wave_sum_int(n);
        };
        c = max(s.min_tiles, (int)((total + room - 1) / max(room, 1)));
        items = count(c);
        for (int i = 0; i < 12 && items > room; ++i) items = count(c += max(1, c / 16));
        if (items > room) {  // always fits: a row group has at most one chunk more than its share
            c = room > groups ? max(c, (int)((total + room - groups - 1) / (room - groups))) : 1 << 30;
            items = count(c);
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
        const int b = b0 + lane;
        const int g = b < a.B ? work[2 * b] : 0, tiles = b < a.B ? work[2 * b + 1] : 0, n = (tiles + c - 1) / c;
        const int upto = wave_inclusive_sum(g * n), gsum = wave_inclusive_sum(g);
        const uint64_t past = __ballot(before + upto > want);
        if (!past && b0 + kWave < a.B) {
            before += __builtin_amdgcn_readlane(upto, 63);
            groups_before += __builtin_amdgcn_readlane(gsum, 63);
            continue;
        }
        if (!past) return false;  // cannot be: want < items
        const int at = __ffsll((unsigned long long)past) - 1;
        const int gb = __builtin_amdgcn_readlane(g, at), tb = __builtin_amdgcn_readlane(tiles, at);
        const int nb = __builtin_amdgcn_readlane(n, at);
        const int rest = want - before - (__builtin_amdgcn_readlane(upto, at) - gb * nb);
        const int chunk = rest / gb;
        it.b = b0 + at;
        it.group = rest % gb;
        it.row_tiles = gb / heads;
        it.t0 = min(max(a.token_offsets[it.b], 0), a.N);
        it.n_tok = min(max(a.token_offsets[it.b + 1], it.t0), a.N) - it.t0;
        it.len = min(max(a.cache_len[it.b], 0), a.max_blocks * a.page);
        it.first = (int)((long)chunk * tb / nb);
        it.last = (int)((long)(chunk + 1) * tb / nb);
        it.chunks = nb;
        it.slot = want;
        const int record = groups_before + __builtin_amdgcn_readlane(gsum, at) - gb + it.group;
        if (record >= parts.max_groups || (nb > 1 && want >= parts.max_slots)) return false;
        if (chunk == 0 && threadIdx.x == 0) parts.info[record] = GroupInfo{it.b, it.group, nb, want, gb};
        return true;
    }
}

// Adds up the parts of a row group: one workgroup for each 32 x 32 block of its output (rows x elements), thread t having
// the four consecutive elements that lane t % 64 and registers 4 * (t / 64) .. of the accumulators hold.
// ROWS: rows of a group; W: width of an output row; blocks of a part: row tile * (W / 32) + element tile.
template <int ROWS, int W>
__global__ __launch_bounds__(256) void join_kernel(PagedArgs a, int per_token, Parts p)
{
    constexpr int kBlocks = ROWS / 32 * (W / 32), kJoin = 64;
    __shared__ float weight[kJoin * 32], sums[kJoin * 32];
    const int g = blockIdx.x / kBlocks, blk = blockIdx.x % kBlocks;
    if (g >= *p.groups) return;
    const GroupInfo in = p.info[g];
    if (in.chunks <= 1) return;
    const int lane = lane_id(), col = lane % 32, row = blk / (W / 32) * 32 + col;
    const float2 *ml = p.ml + (long)in.slot0 * ROWS + row;
    const long step = (long)in.stride * ROWS;
    // The largest reference maximum of each row; eight threads a row.
    float top = -INFINITY;
#pragma unroll 4
    for (int c = threadIdx.x / 32; c < in.chunks; c += 8) top = fmaxf(top, ml[c * step].x);
    weight[threadIdx.x] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, weight[i * 32 + col]);
    const float base = top == -INFINITY ? 0.f : top;
    float total = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int c0 = 0; c0 < in.chunks; c0 += kJoin) {
        const int n = min(in.chunks - c0, kJoin);
        __syncthreads();
        for (int c = threadIdx.x / 32; c < kJoin; c += 8) {
            float2 v = make_float2(-INFINITY, 0.f);
            if (c < n) v = ml[(c0 + c) * step];
            weight[c * 32 + col] = __builtin_amdgcn_exp2f(v.x - base);
            sums[c * 32 + col] = v.y;
        }
        __syncthreads();
        const f32x4 *o = reinterpret_cast<const f32x4 *>(p.o) + ((in.slot0 + (long)c0 * in.stride) * kBlocks + blk) * 256 + threadIdx.x;
#pragma unroll 16
        for (int c = 0; c < n; ++c) {
            const float f = weight[c * 32 + col];
            const f32x4 v = o[(long)c * in.stride * kBlocks * 256];
            total = fmaf(sums[c * 32 + col], f, total);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = fmaf(v[i], f, sum[i]);
        }
    }
    const int t0 = min(max(a.token_offsets[in.b], 0), a.N), n = min(max(a.token_offsets[in.b + 1], t0), a.N) - t0;
    const int tiles = (int)(((long)n * per_token + ROWS - 1) / ROWS), r = in.group % tiles * ROWS + row;
    if (r >= n * per_token) return;
    const long at = (long)(t0 + r / per_token) * a.H + in.group / tiles * per_token + r % per_token;
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const int e = blk % (W / 32) * 32 + threadIdx.x / 64 * 8 + lane / 32 * 4;
    *reinterpret_cast<u32x2 *>(a.o + at * W + e) = u32x2{pack_bf16x2(sum[0] * inv, sum[1] * inv),
                                                         pack_bf16x2(sum[2] * inv, sum[3] * inv)};
    if (a.lse && blk % (W / 32) == 0 && threadIdx.x < 32)
        a.lse[at] = total == 0.f ? -INFINITY : (base + __builtin_amdgcn_logf(total)) / kLog2e;
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

// The same over the two rows of 16 lanes of each half (lanes l and l ^ 16).
__device__ __forceinline__ float quads_max(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float quads_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
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
