// Log probabilities of given tokens, log-sum, entropy and the k best
// alternatives of rows of logits, read once.
//
// The sums: with a reference logit m and x = (l - m) * scale * log2 e,
//   S = sum 2^x,  A = sum 2^x x,
//   lse = m * scale + ln S,  entropy = ln S - ln 2 * A / S:
// both terms of the entropy are at least 0 where m is the largest logit, so
// nothing cancels.  Moving the reference by d = (m - m') * scale * log2 e takes A
// to (A + d S) 2^d and S to S 2^d, so every lane has a reference of its own, and
// they are joined at the end.
// The alternatives: a wavefront holds a bound below which nothing can be among
// its k best, and a list in LDS of what has passed it.  A tile of 32 elements a
// lane costs one maximum and one comparison (the maximum is needed anyway);
// where k lanes or more pass, the k-th largest of the lanes' maxima is a better
// bound, found bit by bit with ballots.  A full list is cut to its k best.
// Elements come in ascending order, so what only equals the bound of an earlier
// tile has k better ones before it.
// Parts of a row by different wavefronts (their sums, their lists) are joined
// by a second kernel, a wavefront a row.
// What bounds it: memory, for many rows; for few the two launches and the chain
// of load, bound, list, join.
#include "device.hpp"
#include "step.hpp"

namespace ecospec {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kTile = 32 * kWave;   // elements
constexpr int kGroup = 4;           // elements of a lane between looks at the list's room
constexpr int kList = (kGroup + 1) * kWave;  // entries of a wavefront's list
constexpr int kKept = 64;           // most entries that a wavefront leaves
constexpr int kMinParts = 4096;     // wavefronts that fill the card: 16 a compute unit
constexpr int kMaxParts = 256;      // of a row
constexpr float kFloor = -1e30f;    // stands for -inf where -inf * 0 must not arise
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;

struct Part {
    float m, s, a;
    int count;
    float value[kKept];
    int index[kKept];
};

// Wavefronts of a row.
__host__ __device__ inline int parts_of(int N, int V)
{
    const int tiles = (V + kTile - 1) / kTile, want = (kMinParts + N - 1) / N;
    const int most = want < kMaxParts ? want : kMaxParts;
    return tiles < most ? tiles : most;
}

// Order of a float as an unsigned number; -0 as +0; no NaN.
__device__ __forceinline__ uint32_t order_of(float v)
{
    const uint32_t b = __float_as_uint(v + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float float_of(uint32_t order)
{
    return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order);
}

// The smallest float above v.
__device__ __forceinline__ float above(float v)
{
    return v == INFINITY ? __uint_as_float(0x7fc00000u) : float_of(order_of(v) + 1);
}

__device__ __forceinline__ int lanes_before(uint64_t mask)
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

struct Sums {
    float m = kLowest, s = 0.f, a = 0.f;

    __device__ __forceinline__ void move(float to, float scale2)  // to >= m
    {
        const float d = fmaxf((m - to) * scale2, kFloor), f = __builtin_amdgcn_exp2f(d);
        a = fmaf(d, s, a) * f;
        s *= f;
        m = to;
    }
    __device__ __forceinline__ void add(float l, float scale2)
    {
        const float x = (l - m) * scale2, e = __builtin_amdgcn_exp2f(x);
        s += e;
        a = fmaf(e, fmaxf(x, kFloor), a);
    }
    __device__ __forceinline__ void join(Sums o, float scale2)
    {
        const float top = fmaxf(m, o.m);
        move(top, scale2);
        o.move(top, scale2);
        s += o.s;
        a += o.a;
    }
    __device__ __forceinline__ void join_lanes(float scale2)
    {
#pragma unroll
        for (int x = 32; x >= 1; x >>= 1) join(Sums{__shfl_xor(m, x, kWave), __shfl_xor(s, x, kWave), __shfl_xor(a, x, kWave)}, scale2);
    }
};

// What the wavefront's lanes have written to LDS is there for all of them.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The k best of what a wavefront has seen, in its list.  All members are uniform.
struct Best {
    float *value;  // kList entries
    int *index;
    int k, count = 0;
    float bound = -INFINITY;  // k entries of the list are at least this; -inf: perhaps fewer

    // The largest order that at least k of the lanes' n keys reach.
    template <int E>
    __device__ __forceinline__ static uint32_t kth(const uint32_t (&key)[E], int k)
    {
        uint32_t t = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t x = t | 1u << bit;
            int n = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) n += __builtin_popcountll(__ballot(key[e] >= x));
            if (n >= k) t = x;
        }
        return t;
    }

    // The list cut to its k best, equal ones by the lower index.
    __device__ __forceinline__ void cut()
    {
        if (count <= k) return;
        wave_fence();
        constexpr int E = kList / kWave;
        const int lane = lane_id();
        float v[E];
        int at[E];
        uint32_t key[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = e * kWave + lane;
            v[e] = i < count ? value[i] : 0.f;
            at[e] = i < count ? index[i] : 0;
            key[e] = i < count ? order_of(v[e]) : 0u;  // no number has order 0
        }
        const uint32_t t = kth(key, k);
        int more = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) more += __builtin_popcountll(__ballot(key[e] > t));
        // Of the equal ones the k - more of lowest index: their indices' complements as keys.
        uint32_t tie[E];
#pragma unroll
        for (int e = 0; e < E; ++e) tie[e] = key[e] == t ? ~(uint32_t)at[e] : 0u;
        const uint32_t last = kth(tie, k - more);
        wave_fence();
        count = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool stays = key[e] > t || (tie[e] && tie[e] >= last);
            const uint64_t mask = __ballot(stays);
            if (stays) {
                value[count + lanes_before(mask)] = v[e];
                index[count + lanes_before(mask)] = at[e];
            }
            count += __builtin_popcountll(mask);
        }
        bound = float_of(t);
    }

    // A tile of E elements a lane, of higher index than all before; top: the lane's largest.
    template <int E, class F>
    __device__ __forceinline__ void tile(const float (&v)[E], float top, F index_of)
    {
        const uint64_t pass = __ballot(top > bound);
        if (!pass) return;
        float from = above(bound);
        if (__builtin_popcountll(pass) >= k) {
            const uint32_t key[1] = {top > bound ? order_of(top) : 0u};
            bound = from = float_of(kth(key, k));
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (e % kGroup == 0 && count > kList - kGroup * kWave) {
                cut();
                from = fmaxf(from, bound);  // equal ones of this tile may have a lower index than what is listed
            }
            const bool in = v[e] >= from;
            const uint64_t mask = __ballot(in);
            if (!mask) continue;
            if (in) {
                value[count + lanes_before(mask)] = v[e];
                index[count + lanes_before(mask)] = index_of(e);
            }
            count += __builtin_popcountll(mask);
        }
    }
};

template <bool BF16>
__device__ __forceinline__ float logit(const void *p, long i)
{
    return BF16 ? bf16_bits_to_f32(static_cast<const uint16_t *>(p)[i]) : static_cast<const float *>(p)[i];
}

__device__ __forceinline__ float largest(const float (&v)[32])
{
    float t = fmaxf(fmaxf(v[0], v[1]), v[2]);
#pragma unroll
    for (int e = 3; e + 1 < 32; e += 2) t = fmaxf(fmaxf(v[e], v[e + 1]), t);
    return fmaxf(t, v[31]);
}

template <bool BF16, bool TOP>
__global__ __launch_bounds__(kThreads) void parts_kernel(LogprobArgs a, int parts, Part *out)
{
    constexpr int kVec = BF16 ? 8 : 4, kLoads = 32 / kVec, kBytes = BF16 ? 2 : 4;
    __shared__ float values[TOP ? kWaves : 1][TOP ? kList : 1];
    __shared__ int indices[TOP ? kWaves : 1][TOP ? kList : 1];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const long id = (long)blockIdx.x * kWaves + wave;
    if (id >= (long)a.N * parts) return;
    const int row = (int)(id / parts), part = (int)(id % parts);
    const char *p = static_cast<const char *>(a.logits) + row * a.stride * kBytes;
    // The row from its first whole 16 bytes on; what lies before and behind goes element by element.
    const int head = min((int)(-(uintptr_t)p % 16) / kBytes, a.V), vectors = (a.V - head) / kVec;
    const int tail = head + vectors * kVec, tiles = (vectors + kLoads * kWave - 1) / (kLoads * kWave);
    const int first = (int)((long)tiles * part / parts), last = (int)((long)tiles * (part + 1) / parts);
    const float scale2 = a.scale * kLog2e;

    Sums sums;
    Best best{values[TOP ? wave : 0], indices[TOP ? wave : 0], a.k};
    auto edge = [&](int from, int to) {  // up to 64 elements, one a lane
        const float v[1] = {from + lane < to ? logit<BF16>(p, from + lane) : -INFINITY};
        if (from + lane < to) {
            if (v[0] > sums.m) sums.move(v[0], scale2);
            sums.add(v[0], scale2);
        }
        if (TOP) best.tile(v, v[0], [&](int) { return from + lane; });
    };
    if (part == 0 && head) edge(0, head);
    const u32x4 *src = reinterpret_cast<const u32x4 *>(p + (long)head * kBytes);
#pragma unroll 1
    for (int t = first; t < last; ++t) {
        const int at = t * kLoads * kWave + lane;
        u32x4 w[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint32_t none = BF16 ? 0xff80ff80u : 0xff800000u;
            w[i] = u32x4{none, none, none, none};
            if (at + i * kWave < vectors) w[i] = src[at + i * kWave];
        }
        float v[32];
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (BF16) {
                    v[i * 8 + 2 * c] = __uint_as_float(w[i][c] << 16);
                    v[i * 8 + 2 * c + 1] = __uint_as_float(w[i][c] & 0xffff0000u);
                } else {
                    v[i * 4 + c] = __uint_as_float(w[i][c]);
                }
            }
        const float top = largest(v);
        if (top > sums.m) sums.move(top, scale2);
#pragma unroll
        for (int e = 0; e < 32; ++e) sums.add(v[e], scale2);
        if (TOP)
            best.tile(v, top, [&](int e) { return head + (at + e / kVec * kWave) * kVec + e % kVec; });
    }
    if (part == parts - 1 && tail < a.V) edge(tail, a.V);

    sums.join_lanes(scale2);
    Part *to = out + id;
    if (TOP) {
        if (best.count > kKept) best.cut();
        wave_fence();
        if (lane < best.count) {
            to->value[lane] = best.value[lane];
            to->index[lane] = best.index[lane];
        }
    }
    if (lane == 0) {
        to->m = sums.m;
        to->s = sums.s;
        to->a = sums.a;
        to->count = best.count;
    }
}

template <bool BF16>
__global__ __launch_bounds__(kWave) void join_kernel(LogprobArgs a, int parts, const Part *in)
{
    constexpr int kBytes = BF16 ? 2 : 4, kAtOnce = 8;
    __shared__ float values[kList];
    __shared__ int indices[kList];
    const int row = blockIdx.x, lane = lane_id();
    const char *p = static_cast<const char *>(a.logits) + row * a.stride * kBytes;
    const Part *mine = in + (long)row * parts;
    const float scale2 = a.scale * kLog2e;

    Sums sums;
    for (int i = lane; i < parts; i += kWave) sums.join(Sums{mine[i].m, mine[i].s, mine[i].a}, scale2);
    sums.join_lanes(scale2);
    const bool nothing = sums.s == 0.f;  // every logit is -inf
    const float log_s = logf(sums.s);
    if (lane == 0) {
        if (a.lse) a.lse[row] = nothing ? -INFINITY : fmaf(sums.m, a.scale, log_s);
        if (a.entropy) a.entropy[row] = nothing ? 0.f : fmaf(-kLn2, sums.a / sums.s, log_s);
    }
    auto logprob = [&](float l) { return nothing ? -INFINITY : fmaf(l - sums.m, a.scale, -log_s); };
    for (int i = lane; i < a.M; i += kWave) {
        const int t = a.tokens[(long)row * a.M + i];
        a.logprob[(long)row * a.M + i] = t >= 0 && t < a.V ? logprob(logit<BF16>(p, t)) : -INFINITY;
    }
    if (!a.k) return;

    Best best{values, indices, a.k};
    for (int i0 = 0; i0 < parts; i0 += kAtOnce) {
        float v[kAtOnce], top = -INFINITY;
        int at[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const bool has = i0 + i < parts && lane < mine[i0 + i].count;
            v[i] = has ? mine[i0 + i].value[lane] : -INFINITY;
            at[i] = has ? mine[i0 + i].index[lane] : 0;
            top = fmaxf(top, v[i]);
        }
        best.tile(v, top, [&](int e) { return at[e]; });
    }
    best.cut();
    // Fewer than k numbers above -inf: the first -inf, then the first NaN.
    for (int pass = 0; pass < 2 && best.count < a.k; ++pass) {
        for (int i0 = 0; i0 < a.V && best.count < a.k; i0 += kWave) {
            const float l = i0 + lane < a.V ? logit<BF16>(p, i0 + lane) : 0.f;
            const bool is = pass ? l != l : l == -INFINITY;
            const uint64_t mask = __ballot(is);
            const int place = best.count + lanes_before(mask);
            if (is && place < a.k) {
                values[place] = l;
                indices[place] = i0 + lane;
            }
            best.count = min(best.count + (int)__builtin_popcountll(mask), a.k);
        }
    }
    // Each lane's entry, and how many come before it.
    wave_fence();
    const bool has = lane < best.count;
    const float v = has ? values[lane] : 0.f;
    const int at = has ? indices[lane] : 0;
    const uint32_t key = v != v ? 0u : order_of(v);
    int rank = 0;
    for (int i = 0; i < best.count; ++i) {
        const uint32_t k = __builtin_amdgcn_readlane(key, i);
        const int x = __builtin_amdgcn_readlane(at, i);
        rank += k > key || (k == key && x < at);
    }
    if (!has) return;
    a.top_idx[(long)row * a.k + rank] = at;
    if (a.top_logprob) a.top_logprob[(long)row * a.k + rank] = logprob(v);
}

}  // namespace

size_t logprobs_workspace(int N)
{
    // parts_of(N, V) <= kMinParts / N + 1 for every V.
    return ((size_t)kMinParts + N) * sizeof(Part);
}

hipError_t launch_token_logprobs(const LogprobArgs &a, bool bf16, void *workspace, hipStream_t stream)
{
    const int parts = parts_of(a.N, a.V);
    Part *p = static_cast<Part *>(workspace);
    const unsigned grid = (unsigned)(((long)a.N * parts + kWaves - 1) / kWaves);
    if (bf16) {
        if (a.k) parts_kernel<true, true><<<grid, kThreads, 0, stream>>>(a, parts, p);
        else parts_kernel<true, false><<<grid, kThreads, 0, stream>>>(a, parts, p);
    } else {
        if (a.k) parts_kernel<false, true><<<grid, kThreads, 0, stream>>>(a, parts, p);
        else parts_kernel<false, false><<<grid, kThreads, 0, stream>>>(a, parts, p);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (bf16) join_kernel<true><<<(unsigned)a.N, kWave, 0, stream>>>(a, parts, p);
    else join_kernel<false><<<(unsigned)a.N, kWave, 0, stream>>>(a, parts, p);
    return hipGetLastError();
}

}  // namespace ecospec
