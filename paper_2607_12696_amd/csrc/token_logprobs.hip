// Log probabilities of given tokens, log-sum, entropy and the k best
// alternatives of rows of logits, read once.
//
// The sums: with a reference logit m, c = scale * log2 e and x = (l - m) c,
//   S = sum 2^x,  A = sum 2^x x,
//   lse = m * scale + ln S,  entropy = ln S - ln 2 * A / S:
// both terms of the entropy are at least 0 where m is the largest logit, so
// nothing cancels.  Moving the reference by d = (m - m') c takes A to
// (A + d S) 2^d and S to S 2^d, so every lane has a reference of its own, and
// they are joined at the end.
// The alternatives: a wavefront holds a bound below which nothing can be among
// its k best, and a list in LDS of what has passed it.  A tile of 32 elements a
// lane costs one maximum and one comparison (the maximum is needed anyway);
// where k lanes or more pass, the k-th largest of the lanes' maxima, for a large k
// of the maxima of eight elements, is a better bound, found bit by bit with
// ballots.  A full list is cut to its k best.
// Elements come in ascending order, so what only equals the bound of an earlier
// tile has k better ones before it.
// Parts of a row by different wavefronts leave their sums and their k best in
// order; they are joined in LDS, or by a second kernel: for a small k with a lane
// to a part, k times the largest head, the lowest lane among equal ones (its
// elements come first); for a larger one the lists in pairs.
// What bounds it: memory, for many rows (2048 of 200000 in bf16, k = 5: 157 us,
// 5.2 TB/s; k = 20 168, k = 64 234); for few the chain of load, bound, list, join
// and the launches (4 of 128000, k = 2: 5 us, and 3.1 the join; one of 32000, k =
// 5, 20 and 64: 8, 11.4 and 24).  Rising logits, of which every tile passes, take
// six times as long as others (512 of 200000, k = 5: 300 and 51 us).
#include "device.hpp"
#include "step.hpp"

namespace ecospec {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kTile = 32 * kWave;   // elements
constexpr int kGroup = 8;           // elements of a lane that are looked at together
constexpr int kRoom = 4 * kWave;    // entries that may come between looks at the list's length
constexpr int kList = 2 * kWave + kRoom;  // entries of a wavefront's list
constexpr int kKept = 64;           // most entries that a wavefront leaves
constexpr int kMinParts = 4096;     // wavefronts that fill the card: 16 a compute unit
constexpr int kMaxParts = kWave;    // of a row: a lane each when they are joined
constexpr int kCus = 256, kManyRows = 2 * kCus;
constexpr int kMostWaves = 16;      // of a workgroup that has a row to itself (waves_of)
constexpr float kFloor = -1e30f;    // stands for -inf where -inf * 0 must not arise
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;

// What the parts of a row leave, next to a list of k entries each, in order, zeros behind the last.
struct Head {
    double s;
    float m, a;
};

struct Work {
    Head *heads;        // [N][parts]
    uint64_t *entries;  // [N][parts][k]
};

// Wavefronts of a row of `tiles` tiles, at most `most`: all have the same number of tiles but the last.
inline int parts_of(int tiles, int most)
{
    const int each = (tiles + most - 1) / most;
    return (tiles + each - 1) / each;
}

// Wavefronts of a workgroup that has a row to itself: the most with which all rows' workgroups are there at once, of the 16
// wavefronts a compute unit that registers leave room for.  (2048 rows of 200000, k = 5: two, 157 us; one workgroup more than
// there is room for waits for all others: 2047 rows by three 185.  Five spread unevenly over four SIMDs: 700 rows 91, by four 73.)
inline int waves_of(int N)
{
    for (int w : {16, 8, 4, 3, 2})
        if (N <= kCus * (16 / w)) return w;
    // Twice what three have room for (2100 rows of 200000: 186 us, by one wavefront 221); then the least joining (3000 rows of
    // 50000, k = 20: 97, by two 113, by four 125; of 200000, k = 5, 236 to 248).
    return N <= 2 * kCus * (16 / 3) ? 3 : 1;
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

// An alternative as one number: what comes first is larger, and none is 0.
__device__ __forceinline__ uint64_t entry_of(float v, int at) { return (uint64_t)order_of(v) << 32 | ~(uint32_t)at; }

__device__ __forceinline__ int lanes_before(uint64_t mask)
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

// Lane moves within a register (row shifts, then row totals into the later rows), a few cycles each: lane 63 ends with f over
// all lanes.
template <int CTRL, int ROW_MASK, class T>
__device__ __forceinline__ T lane_move(T v, T none)
{
    if constexpr (sizeof(T) == 8) {
        const u32x2 x = __builtin_bit_cast(u32x2, v), n = __builtin_bit_cast(u32x2, none);
        return __builtin_bit_cast(T, u32x2{lane_move<CTRL, ROW_MASK>(x[0], n[0]), lane_move<CTRL, ROW_MASK>(x[1], n[1])});
    } else {
        const int to = __builtin_bit_cast(int, none), from = __builtin_bit_cast(int, v);
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(to, from, CTRL, ROW_MASK, 0xf, false));
    }
}

template <class T, class F>
__device__ __forceinline__ T along_lanes(T v, T none, F f)
{
    v = f(v, lane_move<0x111, 0xf>(v, none));  // row_shr:1
    v = f(v, lane_move<0x112, 0xf>(v, none));  // row_shr:2
    v = f(v, lane_move<0x114, 0xf>(v, none));  // row_shr:4
    v = f(v, lane_move<0x118, 0xf>(v, none));  // row_shr:8
    v = f(v, lane_move<0x142, 0xa>(v, none));  // row_bcast:15 into rows 1 and 3
    v = f(v, lane_move<0x143, 0xc>(v, none));  // row_bcast:31 into rows 2 and 3
    return v;
}

template <class T>
__device__ __forceinline__ T last_lane(T v)
{
    if constexpr (sizeof(T) == 8) {
        const u32x2 x = __builtin_bit_cast(u32x2, v);
        return __builtin_bit_cast(T, u32x2{last_lane(x[0]), last_lane(x[1])});
    } else {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), kWave - 1));
    }
}

// (l - m) c.  The difference may pass fp32's range where its product does not, so it is taken of the halves: one fma, and the
// factor of two is c's.  Halves are exact but for fp32's smallest numbers, whose last bit is 2^-22 of an exponent at most.  (Two
// forms by the size of m instead: 2048 rows of 200000 222 us, masked ones 208; so 163 and 172, as the plain difference.)
__device__ __forceinline__ float scaled_difference(float l, float m, float c) { return fmaf(l, 0.5f, -0.5f * m) * (2.f * c); }

// S is held in 64 bits: where one token has almost all of the probability, S is 1 and a little, and ln S, the token's log
// probability and most of the entropy are that little.
struct Sums {
    float m = kLowest, a = 0.f;
    double s = 0.;

    __device__ __forceinline__ void move(float to, float c)  // to >= m
    {
        const float d = fmaxf(scaled_difference(m, to, c), kFloor), f = __builtin_amdgcn_exp2f(d);
        a = fmaf(d, (float)s, a) * f;
        s *= f;
        m = to;
    }
    // Over the wavefront: the largest reference, then plain sums.
    __device__ __forceinline__ void join_lanes(float c)
    {
        move(last_lane(along_lanes(m, kLowest, [](float x, float y) { return fmaxf(x, y); })), c);
        a = last_lane(along_lanes(a, 0.f, [](float x, float y) { return x + y; }));
        s = last_lane(along_lanes(s, 0., [](double x, double y) { return x + y; }));
    }
    // E logits, none above m: two chains of additions.
    template <int E>
    __device__ __forceinline__ void add(const float (&l)[E], float c)
    {
        double t[2];
        float u[2];
        auto sum = [&](float floor) {
            t[0] = t[1] = 0.;
            u[0] = u[1] = 0.f;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float x = scaled_difference(l[i], m, c), e = __builtin_amdgcn_exp2f(x);
                t[i % 2] += e;
                u[i % 2] = fmaf(e, floor == 0.f ? x : fmaxf(x, floor), u[i % 2]);
            }
        };
        sum(0.f);
        // 0 * -inf where a logit is -inf: once more, with a finite number in its place.  (A maximum for each element instead
        // is a ninth of the instructions.)
        if (__any(u[0] + u[1] != u[0] + u[1])) sum(kFloor);
        s += t[0] + t[1];
        a += u[0] + u[1];
    }
};

// What the wavefront's lanes have written to LDS is there for all of them.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A number that at least k of the lanes' keys reach, the largest of the BITS upper bits or one that just k reach; `reach`: how
// many do.  0, and `reach` as it was, if there are fewer than k of 1 and more.
template <int BITS, int E>
__device__ __forceinline__ uint32_t kth(const uint32_t (&key)[E], int k, int &reach)
{
    uint32_t t = 0;
    for (int bit = 31; bit >= 32 - BITS; --bit) {
        const uint32_t x = t | 1u << bit;
        int n = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) n += __builtin_popcountll(__ballot(key[e] >= x));
        if (n < k) continue;
        t = x;
        reach = n;
        if (n == k) break;
    }
    return t;
}

// The k best of what a wavefront has seen, in its list.  All members are uniform.
struct Best {
    u32x2 *list;  // kList pairs of value and index
    // A list of more than `longest` is cut before it grows: twice k, and at least 64.  (A longer one is cut less often, but
    // the bound stays low until it is: 2048 rows of 200000, k = 5, up to 256 entries 171 us, 64 entries 164.)
    int k, longest, count = 0;
    float bound = -INFINITY;  // k entries of the list are at least this; -inf: perhaps fewer

    // The list, of at most E entries a lane, cut to its k best, equal ones by the lower index.
    template <int E>
    __device__ __forceinline__ void cut_of()
    {
        wave_fence();
        const int lane = lane_id();
        u32x2 entry[E];
        uint32_t key[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = e * kWave + lane;
            entry[e] = i < count ? list[i] : u32x2{0u, 0u};
            key[e] = i < count ? order_of(__uint_as_float(entry[e][0])) : 0u;  // no number has order 0
        }
        int reach = count;
        const uint32_t t = kth<32>(key, k, reach);
        uint32_t last = 0;
        if (reach > k) {
            // Some are equal to the k-th: those of lowest index stay, whose complements are the largest.
            int more = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) more += __builtin_popcountll(__ballot(key[e] > t));
            uint32_t tie[E];
#pragma unroll
            for (int e = 0; e < E; ++e) tie[e] = key[e] == t ? ~entry[e][1] : 0u;
            last = kth<32>(tie, k - more, reach);
        }
        wave_fence();
        count = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool stays = key[e] > t || (key[e] == t && ~entry[e][1] >= last);
            const uint64_t mask = __ballot(stays);
            if (stays) list[count + lanes_before(mask)] = entry[e];
            count += __builtin_popcountll(mask);
        }
        bound = float_of(t);
    }

    __device__ __forceinline__ void cut()
    {
        if (count <= k) return;
        if (count <= 2 * kWave) cut_of<2>();
        else cut_of<kList / kWave>();
    }

    // The lane's entry of at most 64, and how many come before it; a rank of at least 64 where it has none.
    __device__ __forceinline__ int ranked(uint64_t &mine) const
    {
        wave_fence();
        const bool has = lane_id() < count;
        const u32x2 entry = has ? list[lane_id()] : u32x2{0u, 0u};
        mine = has ? entry_of(__uint_as_float(entry[0]), (int)entry[1]) : 0;
        int rank = has ? 0 : kWave;
#pragma unroll 4
        for (int i = 0; i < count; ++i) {
            const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(mine >> 32), i);
            const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)mine, i);
            rank += ((uint64_t)hi << 32 | lo) > mine;
        }
        return rank;
    }

    // Its k best, in order, to k entries from `to` on, zeros behind the last.
    __device__ __forceinline__ void leave(uint64_t *to) const
    {
        uint64_t mine;
        const int rank = ranked(mine);
        if (rank < k) to[rank] = mine;
        if (lane_id() >= count && lane_id() < k) to[lane_id()] = 0;
    }

    // A tile of E elements a lane, of higher index than all before, by vectors of VEC of which all lanes' come before all lanes'
    // next; top: the lane's largest, group[g]: of the g-th kGroup.
    template <int VEC, int E, int G, class F>
    __device__ __forceinline__ void tile(const float (&v)[E], float top, const float (&group)[G], F index_of)
    {
        const uint64_t pass = __ballot(top > bound);
        if (!pass) return;
        float from = above(bound);
        // Sixteen bits, a bf16's, are near enough; fewer pass a whole number's.
        int reach;
        if (k <= kWave / 2 || G == 1) {
            if (__builtin_popcountll(pass) >= k) {
                const uint32_t key[1] = {top > bound ? order_of(top) : 0u};
                bound = from = fmaxf(from, float_of(kth<16>(key, k, reach)));
            }
        } else {
            // By the groups' maxima: of a first tile's 2048 elements 70 pass for k = 64, by the lanes' 250.
            uint32_t key[G];
            int n = 0;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                n += __builtin_popcountll(__ballot(group[g] > bound));
                key[g] = group[g] > bound ? order_of(group[g]) : 0u;
            }
            if (n >= k) bound = from = fmaxf(from, float_of(kth<16>(key, k, reach)));
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (!__any(group[g] >= from)) continue;
#pragma unroll
            for (int e = g * kGroup; e < min(E, (g + 1) * kGroup); ++e) {
                if (e % (kRoom / kWave) == 0 && count > longest) {
                    cut();
                    // What comes behind whole vectors of all lanes is of higher index than what is listed; within them an equal
                    // one's may be lower.  (512 rows of 200000 equal logits: 66 us, always taken as lower 150.)
                    from = fmaxf(from, e % VEC ? bound : above(bound));
                }
                const bool in = v[e] >= from;
                const uint64_t mask = __ballot(in);
                if (!mask) continue;
                if (in) list[count + lanes_before(mask)] = u32x2{__float_as_uint(v[e]), (uint32_t)index_of(e)};
                count += __builtin_popcountll(mask);
            }
        }
    }
};

template <bool BF16>
__device__ __forceinline__ float logit(const void *p, long i)
{
    return BF16 ? bf16_bits_to_f32(static_cast<const uint16_t *>(p)[i]) : static_cast<const float *>(p)[i];
}

__device__ __forceinline__ float largest(const float (&v)[32], float (&group)[32 / kGroup])
{
#pragma unroll
    for (int g = 0; g < 32 / kGroup; ++g) {
        float t = fmaxf(v[g * kGroup], v[g * kGroup + 1]);
#pragma unroll
        for (int e = 2; e + 1 < kGroup; e += 2) t = fmaxf(fmaxf(v[g * kGroup + e], v[g * kGroup + e + 1]), t);
        group[g] = t;
    }
    static_assert(kGroup % 2 == 0 && kGroup == 8, "four groups");
    return fmaxf(fmaxf(group[0], group[1]), fmaxf(group[2], group[3]));
}

// One wavefront's part of a row.
template <bool BF16, bool TOP>
__device__ __forceinline__ void scan(const LogprobArgs &a, int row, int part, int parts, Sums &sums, Best &best)
{
    constexpr int kVec = BF16 ? 8 : 4, kLoads = 32 / kVec, kBytes = BF16 ? 2 : 4;
    const int lane = lane_id();
    const char *p = static_cast<const char *>(a.logits) + row * a.stride * kBytes;
    // The row from its first whole 16 bytes on; what lies before and behind goes element by element.
    const int head = min((int)(-(uintptr_t)p % 16) / kBytes, a.V), vectors = (a.V - head) / kVec;
    const int tail = head + vectors * kVec, tiles = (vectors + kLoads * kWave - 1) / (kLoads * kWave);
    const int each = (tiles + parts - 1) / parts, first = min(part * each, tiles), last = min(first + each, tiles);
    const float c = a.scale * kLog2e;

    auto edge = [&](int from, int to) {  // up to 64 elements, one a lane
        const float v[1] = {from + lane < to ? logit<BF16>(p, from + lane) : -INFINITY};
        if (from + lane < to) {
            if (v[0] > sums.m) sums.move(v[0], c);
            sums.add(v, c);
        }
        if (TOP) best.tile<1>(v, v[0], v, [&](int) { return from + lane; });
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
        float group[32 / kGroup];
        const float top = largest(v, group);
        if (top > sums.m) sums.move(top, c);
        sums.add(v, c);
        if (TOP)
            best.tile<kVec>(v, top, group, [&](int e) { return head + (at + e / kVec * kWave) * kVec + e % kVec; });
    }
    if (part == parts - 1 && tail < a.V) edge(tail, a.V);

    sums.join_lanes(c);
    if (TOP && best.count > kKept) best.cut();
}

// Whether a row's alternatives are taken one after the other from its parts' heads, by one wavefront, or by joining the lists.
// (One row of 32000, 16 parts: k = 13 10.3 us either way, k = 20 12.2 and 11.4, k = 64 29.5 and 23.6.  One of 200000, 49 parts:
// k = 25 20.5 either way, k = 64 41.2 and 37.1.)
__host__ __device__ inline bool in_steps(int k, int parts) { return k <= (parts > kMostWaves ? 24 : 12); }

// Lists of k entries in order, `parts` of them one after the other at `from`, joined in pairs until one is left: an entry's place
// is its own in its list and that of the first smaller one in the other.  By a whole workgroup; `spare` has room for half of the
// lists, rounded up.  Where the list is, then.
__device__ __forceinline__ const uint64_t *join_lists(uint64_t *from, uint64_t *spare, int parts, int k)
{
    for (int n = parts; n > 1; n = (n + 1) / 2) {
        const int half = (n + 1) / 2;
        for (int i = threadIdx.x; i < n * k; i += blockDim.x) {
            const int p = i / k, other = p < half ? p + half : p - half;
            const uint64_t mine = from[i];
            int place = i - p * k;
            if (other < n) {
                // Equal are zeros only: those of the first list come first.
                const uint64_t *list = from + other * k;
                int lo = 0, hi = k;
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    const uint64_t x = list[mid];
                    if (x > mine || (p >= half && x == mine)) lo = mid + 1;
                    else hi = mid;
                }
                place += lo;
            }
            if (place < k) spare[min(p, other) * k + place] = mine;
        }
        __syncthreads();
        uint64_t *const x = from;
        from = spare;
        spare = x;
    }
    return from;
}

// A row's results from its parts (head: the lane's part's), by a whole workgroup.  Lists in LDS, one after the other, and room
// for half of them.
template <bool BF16>
__device__ __forceinline__ void finish(const LogprobArgs &a, int row, int parts, const Head &head, uint64_t *lists,
                                       uint64_t *spare)
{
    constexpr int kBytes = BF16 ? 2 : 4;
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const char *p = static_cast<const char *>(a.logits) + row * a.stride * kBytes;
    const float c = a.scale * kLog2e;
    Sums sums{head.m, head.a, head.s};
    sums.join_lanes(c);
    const bool nothing = sums.s == 0.;  // every logit is -inf
    // The sums know differences from the largest logit alone: where that one, scaled, is past fp32's range, it is said here.
    const float log_s = sums.m * a.scale == INFINITY ? __uint_as_float(0x7fc00000u) : (float)log(sums.s);
    if (threadIdx.x == 0) {
        if (a.lse) a.lse[row] = nothing ? -INFINITY : fmaf(sums.m, a.scale, log_s);
        if (a.entropy) a.entropy[row] = nothing ? 0.f : fmaf(-kLn2, sums.a / (float)sums.s, log_s);
    }
    auto logprob = [&](float l) { return nothing ? -INFINITY : fmaf(fmaf(l, 0.5f, -0.5f * sums.m), 2.f * a.scale, -log_s); };
    for (int i = threadIdx.x; i < a.M; i += blockDim.x) {
        const int t = a.tokens[(long)row * a.M + i];
        a.logprob[(long)row * a.M + i] = t >= 0 && t < a.V ? logprob(logit<BF16>(p, t)) : -INFINITY;
    }
    if (!a.k) return;

    // Lane r of the first wavefront keeps what comes r-th.
    uint64_t mine = 0;
    if (!in_steps(a.k, parts)) {
        const uint64_t *all = join_lists(lists, spare, parts, a.k);
        if (wave) return;
        if (lane < a.k) mine = all[lane];
    } else {
        if (wave) return;
        auto entry_at = [&](int r) { return lane < parts && r < a.k ? lists[lane * a.k + r] : 0; };
        uint64_t head_of = entry_at(0), second = entry_at(1);
        for (int n = 0, next = 0; n < a.k; ++n) {
            const uint32_t key = (uint32_t)(head_of >> 32);
            const uint32_t win = last_lane(along_lanes(key, 0u, [](uint32_t x, uint32_t y) { return x > y ? x : y; }));
            if (!win) break;
            // The lowest lane among equal ones: its elements come first.
            const int from = (int)__builtin_ctzll(__ballot(key == win));
            const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)head_of, from);
            if (lane == n) mine = (uint64_t)win << 32 | lo;
            if (lane == from) {
                head_of = second;
                second = entry_at(++next + 1);
            }
        }
    }
    float v = float_of((uint32_t)(mine >> 32));
    int at = (int)~(uint32_t)mine, count = __builtin_popcountll(__ballot(mine != 0));
    // Fewer than k numbers above -inf: the first -inf, then the first NaN.
    for (int pass = 0; pass < 2 && count < a.k; ++pass) {
        for (int i0 = 0; i0 < a.V && count < a.k; i0 += kWave) {
            const float l = i0 + lane < a.V ? logit<BF16>(p, i0 + lane) : 0.f;
            uint64_t mask = __ballot(pass ? l != l : l == -INFINITY);
            for (; mask && count < a.k; ++count, mask &= mask - 1) {
                const int from = (int)__builtin_ctzll(mask);
                const float w = __shfl(l, from, kWave);
                if (lane == count) {
                    v = w;
                    at = i0 + from;
                }
            }
        }
    }
    if (lane >= a.k) return;
    a.top_idx[(long)row * a.k + lane] = at;
    if (a.top_logprob) a.top_logprob[(long)row * a.k + lane] = logprob(v);
}

template <bool BF16, bool TOP>
__global__ __launch_bounds__(kThreads) void parts_kernel(LogprobArgs a, int parts, Work out)
{
    __shared__ u32x2 lists[TOP ? kWaves : 1][TOP ? kList : 1];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const long id = (long)blockIdx.x * kWaves + wave;
    if (id >= (long)a.N * parts) return;
    const int row = (int)(id / parts), part = (int)(id % parts);
    Sums sums;
    Best best{lists[TOP ? wave : 0], a.k, max(2 * a.k, kWave)};
    scan<BF16, TOP>(a, row, part, parts, sums, best);
    if (TOP) best.leave(out.entries + id * a.k);
    if (lane == 0) out.heads[id] = Head{sums.s, sums.m, sums.a};
}

template <bool BF16>
__global__ __launch_bounds__(kMostWaves *kWave) void join_kernel(LogprobArgs a, int parts, Work in)
{
    extern __shared__ uint64_t lists[];
    const int row = blockIdx.x, lane = lane_id(), entries = a.k * parts;
    const Head head = lane < parts ? in.heads[(long)row * parts + lane] : Head{0., kLowest, 0.f};
    for (int i = threadIdx.x; i < entries; i += blockDim.x) lists[i] = in.entries[(long)row * entries + i];
    __syncthreads();
    finish<BF16>(a, row, parts, head, lists, lists + entries);
}

// A row by one workgroup, a part by each of its wavefronts, joined in LDS.
template <bool BF16, bool TOP>
__global__ __launch_bounds__(kMostWaves *kWave) void row_kernel(LogprobArgs a, int parts)
{
    extern __shared__ double shared[];
    Head *heads = reinterpret_cast<Head *>(shared);
    uint64_t *lists = reinterpret_cast<uint64_t *>(heads + parts), *spare = lists + a.k * parts;
    const int row = blockIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    Sums sums;
    Best best{reinterpret_cast<u32x2 *>(spare) + wave * kList, a.k, max(2 * a.k, kWave)};
    scan<BF16, TOP>(a, row, wave, parts, sums, best);
    if (TOP) best.leave(lists + wave * a.k);
    if (lane == 0) heads[wave] = Head{sums.s, sums.m, sums.a};
    __syncthreads();
    finish<BF16>(a, row, parts, lane < parts ? heads[lane] : Head{0., kLowest, 0.f}, lists, spare);
}

template <bool BF16, bool TOP>
hipError_t launch(const LogprobArgs &a, void *workspace, hipStream_t stream)
{
    const int tiles = (a.V + kTile - 1) / kTile, most = waves_of(a.N);
    // A workgroup a row, in one launch, where each wavefront has a tile (60 rows of 20000, k = 20: 14.6 us, in two launches 18),
    // or where there are rows enough for them to fill the card (1000 of 200000, k = 5: 88 and 109 us; 512 of 50000, k = 20: 35 and
    // 38).  With fewer the parts of a row are more than a workgroup's wavefronts (300 of 50000, k = 20: 34 and 25).
    if (a.N >= kManyRows || tiles <= most) {
        const int waves = parts_of(tiles, most);
        const size_t lds = waves * (sizeof(Head) + (TOP ? 8 * a.k + 8 * kList : 0));
        row_kernel<BF16, TOP><<<(unsigned)a.N, waves * kWave, lds, stream>>>(a, waves);
        return hipGetLastError();
    }
    const int want = kMinParts / a.N, parts = parts_of(tiles, want < kMaxParts ? want : kMaxParts);
    const long n = (long)a.N * parts;
    Work w;
    w.heads = static_cast<Head *>(workspace);
    w.entries = reinterpret_cast<uint64_t *>(w.heads + n);
    parts_kernel<BF16, TOP><<<(unsigned)((n + kWaves - 1) / kWaves), kThreads, 0, stream>>>(a, parts, w);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // Long lists are brought, and joined, by more than one wavefront (one row of 200000, k = 64: a call with four 48 us, with
    // sixteen 36).
    const bool steps = in_steps(a.k, parts);
    const int entries = a.k * parts;
    const int waves = steps ? (entries > 4 * kWave ? 4 : 1) : min((entries + kWave - 1) / kWave, kMostWaves);
    const size_t lds = (entries + (steps ? 0 : a.k * ((parts + 1) / 2))) * sizeof(uint64_t);
    join_kernel<BF16><<<(unsigned)a.N, waves * kWave, lds, stream>>>(a, parts, w);
    return hipGetLastError();
}

}  // namespace

size_t logprobs_workspace()
{
    // At most kMinParts parts, whatever the rows: in one launch there are none.
    return (size_t)kMinParts * (sizeof(Head) + kKept * sizeof(uint64_t));
}

hipError_t launch_token_logprobs(const LogprobArgs &a, bool bf16, void *workspace, hipStream_t stream)
{
    if (bf16) return a.k ? launch<true, true>(a, workspace, stream) : launch<true, false>(a, workspace, stream);
    return a.k ? launch<false, true>(a, workspace, stream) : launch<false, false>(a, workspace, stream);
}

}  // namespace ecospec
