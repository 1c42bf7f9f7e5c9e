// Attention of whole prompts with grouped heads: causal, sequences of different lengths side by side.
//
// The query rows of a sequence that read the same keys are its tokens times the heads of one key/value head, token by
// token: a workgroup takes consecutive ones, 32 R of each of W wavefronts.  So short sequences fill its rows too, and
// long ones have few keys that only some of the rows see.
//   Scores are transposed (S^T = K Q^T): a lane holds one row, its scores are the value product's operand as they stand
//   (O^T = V^T P^T), and V^T is read with the transposing LDS load.
//   Three tiles of 32 keys are under way: while the matrix cores multiply the keys of tile t + 1 and the values of tile
//   t - 1, the vector unit works out the weights of tile t, a piece behind each product.
//   Keys and values go from memory straight to LDS, two steps (of KT tiles) before their products, in panels: of 64 elements
//   for keys (rows of 128 bytes, chunks of 16 XORed with row bits, so that 16 rows' chunks, a quarter of a read, lie in
//   different banks), of 32 for values (rows of 64 bytes: half a read is 256 in a row).  One barrier a step, and operands are
//   read seven products ahead, past it: keys land a tile earlier than that needs.
//   Where there are few row blocks, each one's keys are cut into chunks, a workgroup each, whose sums join_prompt_kernel
//   adds up in order.
#include "attn_plan.hpp"
#include "step.hpp"

namespace ecospec {
namespace {

constexpr int kKeys = 32, kSplitWaves = 4;
constexpr int kSplitRows = 32 * kSplitWaves;   // rows of a workgroup where keys are cut
constexpr int kSlots = 2 * kCus;               // workgroups of such a call
constexpr int kMinTiles = 4;                   // of a chunk
constexpr float kSlack = 8.f;  // powers of two that weights may pass 1 by before their reference maximum moves

typedef __attribute__((ext_vector_type(4))) short s16x4;

__device__ __forceinline__ u32x2 read_tr(const char *p)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
}

__device__ __forceinline__ bool not_finite(uint32_t bf16) { return (bf16 & 0x7f80u) == 0x7f80u; }

__device__ __forceinline__ float max2(float a, float b)  // without the copies that make signalling NaN quiet
{
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

// The score products, sums in vector registers, which the vector unit works on, queries in accumulation registers.  A sum is
// added to again two wait states later at the earliest: with one row tile (WAIT) they are written out.
__device__ __forceinline__ void mfma_first(f32x16 &s, const bf16x8 &k, const bf16x8 &q)
{
    asm("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "a"(q));
}

template <bool WAIT>
__device__ __forceinline__ void mfma_next(f32x16 &s, const bf16x8 &k, const bf16x8 &q)
{
    if (WAIT) asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "a"(q));
    else asm("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "a"(q));
}

// The chunks of a row block of `tiles` tiles.
__device__ __forceinline__ int chunks_of(int tiles, int most) { return min(most, max(tiles / kMinTiles, 1)); }

// A workgroup's row block: its sequence and key/value head, and what its rows see.
struct Block {
    int q0, nq, k0, nk, hk, rows, row0, tiles, G;

    __device__ __forceinline__ int limit(int row) const { return min(max(row / G + 1 + nk - nq, 0), nk); }  // keys of a query row

    __device__ __forceinline__ Block(const GroupedPromptArgs &a, int pair, int block, int block_rows)
    {
        const int b = pair / a.Hkv;
        hk = pair % a.Hkv;
        G = a.H / a.Hkv;
        q0 = __builtin_amdgcn_readfirstlane(min(max(a.q_offsets[b], 0), a.N));
        nq = __builtin_amdgcn_readfirstlane(min(max(a.q_offsets[b + 1], q0), a.N)) - q0;
        k0 = __builtin_amdgcn_readfirstlane(min(max(a.kv_offsets[b], 0), a.M));
        nk = __builtin_amdgcn_readfirstlane(min(max(a.kv_offsets[b + 1], k0), a.M)) - k0;
        rows = nq * G;
        row0 = block * block_rows;
        tiles = row0 < rows ? (limit(min(row0 + block_rows, rows) - 1) + kKeys - 1) / kKeys : 0;
    }
};

// Sums of a chunk: for each row the reference maximum and the weights' sum, and the output sums in accumulator order.
struct PromptParts {
    float2 *ml;  // [slot][kSplitRows]
    float *o;    // [slot][wavefront][D / 32][4][lane][4]
};

#ifndef ECOSPEC_GP_OCC
#define ECOSPEC_GP_OCC 3
#endif
// D: width of a head; W: wavefronts; R: row tiles of each; KT: key tiles a barrier; SPLIT: keys are cut into chunks.
template <int D, int W, int R, int KT, bool SPLIT>
__global__ __launch_bounds__(W * kWave, D == 64 ? ECOSPEC_GP_OCC : R == 1 ? 2 : 1) void prompt_kernel(GroupedPromptArgs a, int blocks, int most_chunks,
                                                                                PromptParts parts)
{
    constexpr int kThreads = W * kWave, kRows = 32 * R * W, kSteps = D / 16, kPanels = D / 64, kTiles = D / 32;
    constexpr int kTile = kKeys * D * 2, kLoads = 2 * kPanels;  // bytes of a tile; loads of a tile by a wavefront
    constexpr int kEdge = kRows / kKeys + 1;                    // most tiles that some rows of a workgroup see in part
    constexpr int kOperands = kSteps + 2 * kTiles;              // key and value operands of a tile
    constexpr int kRing = 8, kAhead = kRing - 1;                // of them in registers
    constexpr int kHeld = 4 * KT;                               // tiles of keys, and of values, in LDS
    constexpr int kBrings = KT * 4 / W;                         // tiles of a step that a wavefront loads a quarter of
    static_assert(kBrings * W == KT * 4, "every quarter is loaded");
    static_assert(kOperands % kRing == 0, "a tile's first operand has a fixed place");
    static_assert(!SPLIT || (R == 1 && W == kSplitWaves), "parts");
    constexpr int kProducts = kOperands * R, kPieces = 20 * R;  // of a tile
    struct Tiles {
        char k[kHeld][kTile];  // panel, row r, chunk c of 16 bytes at place c ^ (r >> 1 & 7)
        char v[kHeld][kTile];  // panel of 32 elements, row
        uint16_t some[kEdge][R][kThreads];  // which weights of a lane are not zero, in a tile with infinities or NaN
    };
    __shared__ __attribute__((aligned(16))) Tiles lds;

    const int pairs = a.B * a.Hkv;
    // Workgroups are dealt to the eight XCDs in turn: with pairs innermost a head's row blocks meet on few of them.  The
    // longest row blocks first, so that no long one is left for the end.
    const int pair = blockIdx.x % pairs, item = blockIdx.x / pairs;
    const int block = blocks - 1 - (SPLIT ? item / most_chunks : item), chunk = SPLIT ? item % most_chunks : 0;
    const Block blk(a, pair, block, kRows);
    if (blk.row0 >= blk.rows) return;
    const int chunks = SPLIT ? chunks_of(blk.tiles, most_chunks) : 1;
    if (SPLIT && chunk >= chunks) return;
    // From here on keys and tiles are counted from the chunk's first.
    const int from = SPLIT ? (int)((long)blk.tiles * chunk / chunks) : 0;
    const int tiles = SPLIT ? (int)((long)blk.tiles * (chunk + 1) / chunks) - from : blk.tiles;
    auto limit = [&](int row) { return min(max(blk.limit(row) - from * kKeys, 0), tiles * kKeys); };
    const int k0 = blk.k0 + from * kKeys, nk = min(blk.nk - from * kKeys, tiles * kKeys), rows = blk.rows, G = blk.G;

    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), col = lane % 32, half = lane / 32;
    const int edge = limit(blk.row0) / kKeys;  // first tile that some row of the workgroup does not see to its end
    const int first = blk.row0 + 32 * R * wave;
    const int all_see = __builtin_amdgcn_readfirstlane(limit(min(first, rows - 1)));  // keys that all rows of the wavefront see

    // ---- queries
    int mine[R];      // keys that the lane's rows see
    bf16x8 q[R][kSteps];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = min(first + 32 * r + col, rows - 1), token = row / G;
        mine[r] = limit(row);
        const uint16_t *src = a.q + (long)(blk.q0 + token) * a.q_stride + (blk.hk * G + row - token * G) * a.q_head + half * 8;
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
            u32x4 w = *reinterpret_cast<const u32x4 *>(src + st * 16);
            // The scale is positive from here on: the largest product is the largest score.
            if (a.scale < 0.f) w ^= 0x80008000u;
            q[r][st] = __builtin_bit_cast(bf16x8, w);
            asm volatile("" : "+a"(q[r][st]));
        }
    }

    // ---- loads: four wavefronts bring a tile, the w-th of them rows 8 w .. 8 w + 7 of each panel of its keys, and 16 rows of
    // panels of its values a load.  Rows past the last key, and tiles past the last, become zeros.
    const uint16_t *src_k = a.k + blk.hk * a.k_head + k0 * a.k_stride, *src_v = a.v + blk.hk * a.v_head + k0 * a.v_stride;
    const uint32_t stride_k = (uint32_t)a.k_stride * 2, stride_v = (uint32_t)a.v_stride * 2;
    const int w4 = wave % 4, mine0 = wave / 4;  // its quarter, and its first tile of a step
    const int e = 8 * w4 + lane / 8, place = (lane % 8) ^ (e >> 1 & 7);
    const int v_panel = D == 128 ? w4 : w4 / 2, v_row = D == 128 ? 0 : w4 % 2 * 16;
    uint32_t off_k[kBrings], off_v[kBrings];
#pragma unroll
    for (int i = 0; i < kBrings; ++i) {
        off_k[i] = (e + (mine0 + i) * kKeys) * stride_k + place * 16;
        off_v[i] = (v_row + (mine0 + i) * kKeys + lane / 4) * stride_v + v_panel * 64 + lane % 4 * 16;
    }
    const uint32_t low = 16 * stride_v;  // the lower half of a panel of values, for heads of 128
    const uint32_t ring_k = __builtin_amdgcn_readfirstlane(lds_addr(lds.k) + mine0 * kTile + w4 * 1024);
    const uint32_t ring_v = __builtin_amdgcn_readfirstlane(lds_addr(lds.v) + mine0 * kTile + v_panel * 2048 + v_row * 64);
    int left_k = nk, left_v = nk;  // keys from the step to load next on
    uint32_t to_k = ring_k, to_v = ring_v;
    u32x4 key_src, value_src;
    auto aim_keys = [&] {
        const int n = max(min(left_k, KT * kKeys), 0);
        key_src = rsrc_words(src_k, n ? (uint32_t)(n - 1) * stride_k + D * 2 : 0);
    };
    auto aim_values = [&] {
        const int n = max(min(left_v, KT * kKeys), 0);
        value_src = rsrc_words(src_v, n ? (uint32_t)(n - 1) * stride_v + D * 2 : 0);
    };
    auto keys_done = [&] {
        left_k -= KT * kKeys;
        if (left_k > 0) src_k += KT * kKeys / 2 * stride_k;
        to_k = to_k == ring_k + (kHeld - KT) * kTile ? ring_k : to_k + KT * kTile;
    };
    auto values_done = [&] {
        left_v -= KT * kKeys;
        if (left_v > 0) src_v += KT * kKeys / 2 * stride_v;
        to_v = to_v == ring_v + (kHeld - KT) * kTile ? ring_v : to_v + KT * kTile;
    };
    auto load = [&](int i, int n) {  // load n of the i-th of its tiles
        if (n < kPanels) load16_lds(key_src, off_k[i] + n * 128, to_k + i * kTile + n * (kKeys * 128));
        else if (n == kPanels) load16_lds(value_src, off_v[i], to_v + i * kTile);
        else load16_lds(value_src, off_v[i] + low, to_v + i * kTile + 1024);
    };
    auto load_keys = [&] {
        aim_keys();
#pragma unroll
        for (int i = 0; i < kBrings * kPanels; ++i) load(i / kPanels, i % kPanels);
        keys_done();
    };
    auto load_values = [&] {
        aim_values();
#pragma unroll
        for (int i = 0; i < kBrings * kPanels; ++i) load(i / kPanels, kPanels + i % kPanels);
        values_done();
    };
#pragma unroll 1
    for (int t = 0; t < KT + 2; t += KT) load_keys();
    load_values();
    // The values of tile -1, whose weights are zeros.
    for (int i = threadIdx.x; i < kTile / 16; i += kThreads) reinterpret_cast<u32x4 *>(lds.v[kHeld - 1])[i] = u32x4{0, 0, 0, 0};

    f32x16 o[R][kTiles];
    float m[R], l[R], base[R], down[R], bound[R];
    int scaled = 0;
    u32x4 p0[R][2] = {}, p1[R][2];  // weights of the tile before and of this one, in turn: 16 keys each
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int d = 0; d < kTiles; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[r][d][i] = 0.f;
        m[r] = bound[r] = -INFINITY;
        l[r] = base[r] = 0.f;
        down[r] = 1.f;
    }
    uint32_t odd_tiles = 0;  // edge tiles with infinities or NaN among the values
    const float scale2 = fmaxf(fabsf(a.scale) * kLog2e, 0x1p-126f);  // not zero: it meets infinities
    const float slack = kSlack / scale2;

    uint32_t k_at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) k_at[i] = (uint32_t)(col * 128 + ((2 * i + half) ^ (col >> 1 & 7)) * 16);
    const int i16 = lane % 16;
    const uint32_t v_at = (uint32_t)((4 * half + i16 / 4) * 64 + lane / 16 % 2 * 32 + i16 % 4 * 8);

    // Piece c of the weights of row tile r with scores s.  Register i is key 8 (i / 4) + 4 half + i % 4.
    float top[R], sum[R];
    auto weights = [&](f32x16 (&s)[R], u32x4 (&p)[R][2], int r, int c) {
        f32x16 &x = s[r];
        if (c == 0) {
            top[r] = max3(max3(x[0], x[1], x[2]), max3(x[3], x[4], x[5]), x[6]);
        } else if (c == 1) {
            top[r] = max3(top[r], max3(max3(x[7], x[8], x[9]), max3(x[10], x[11], x[12]), x[13]), max2(x[14], x[15]));
        } else if (c == 2) {
            if (r < R - 1) return;
            bool past = false;
#pragma unroll
            for (int i = 0; i < R; ++i) past |= top[i] > bound[i];
            if (__builtin_expect(__any(past), 0)) {
                // New reference maxima.  The output sums follow when the products under way are in them.
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    const float now = fmaxf(m[i], halves_max(top[i]) * scale2);
                    scaled |= __any(m[i] != -INFINITY);
                    base[i] = now == -INFINITY ? 0.f : now;
                    down[i] = __builtin_amdgcn_exp2f((m[i] == -INFINITY ? base[i] : m[i]) - base[i]);
                    l[i] *= down[i];
                    m[i] = now;
                    bound[i] = now == -INFINITY ? now : now / scale2 + slack;
                }
            }
        } else {
            const int e = c - 3;  // of 16 elements
            // Written out to stay here, where the compiler would sink it behind all products, and in this order: the result of
            // an exponential needs a wait state, which the instructions of the element before are.
            if (e < 16) {
                const float y = fmaf(x[e], scale2, -base[r]);
                asm volatile("v_exp_f32 %0, %1" : "=v"(x[e]) : "v"(y));
            }
            // The element before: its sum, and pairs to bf16.
            if (e > 0 && e <= 16) {
                const int i = e - 1;
                if (i == 1) asm volatile("v_add_f32 %0, %1, %2" : "=v"(sum[r]) : "v"(x[0]), "v"(x[1]));
                if (i > 1) asm volatile("v_add_f32 %0, %0, %1" : "+v"(sum[r]) : "v"(x[i]));
                if (i % 2) {
                    uint32_t w;
                    asm volatile("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(w) : "v"(x[i - 1]), "v"(x[i]));
                    p[r][i / 8][i % 8 / 2] = w;
                }
                if (i == 15) asm volatile("v_add_f32 %0, %0, %1" : "+v"(l[r]) : "v"(sum[r]));
            }
        }
    };
    // Operand f of a tile: its keys' steps, then its values' (16 keys, element tile).  From kOperands on the next tile's.
    uint32_t key_to = 0, value_to = (kHeld - 2) * kTile, key_at[4], value_at;
    bf16x8 ring[kRing];
    auto fetch = [&](int f) {
        const int x = f % kOperands;
        if (x == 0) {
            key_to = (key_to + kTile) % (kHeld * kTile);
#pragma unroll
            for (int i = 0; i < 4; ++i) key_at[i] = k_at[i] + key_to;
        }
        if (x == kSteps) {
            value_to = (value_to + kTile) % (kHeld * kTile);
            value_at = v_at + value_to;
        }
        if (x < kSteps) {
            ring[f % kRing] = *reinterpret_cast<const bf16x8 *>(lds.k[0] + key_at[x % 4] + x / 4 * (kKeys * 128));
        } else {
            const char *w = lds.v[0] + value_at + (x - kSteps) % kTiles * (kKeys * 64) + (x - kSteps) / kTiles * 16 * 64;
            const u32x2 lo = read_tr(w), hi = read_tr(w + 8 * 64);
            ring[f % kRing] = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
        }
    };
    // Products of a tile's keys into s, then of a tile's values by p, `between(c)` behind product c.
    auto products = [&](f32x16 (&s)[R], u32x4 (&p)[R][2], auto between) {
#pragma unroll
        for (int f = 0; f < kOperands; ++f) {
            fetch(f + kAhead);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                __builtin_amdgcn_sched_barrier(0);
                const int n = f - kSteps;
                if (f == 0) mfma_first(s[r], ring[0], q[r][0]);
                else if (f < kSteps) mfma_next<false>(s[r], ring[f % kRing], q[r][f]);
                else o[r][n % kTiles] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    ring[f % kRing], __builtin_bit_cast(bf16x8, p[r][n / kTiles]), o[r][n % kTiles], 0, 0, 0);
                between(f * R + r);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    // A step: tiles t .. t + KT - 1 follow.
    auto begin = [&](int t) {
        // The keys up to tile t + KT + 1 and the values up to tile t + KT - 1 have landed; every wavefront is past the scores of
        // tile t and the values of tile t - 2.
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kBrings * kLoads) : "memory");
        aim_keys();
        aim_values();
#pragma unroll 1
        for (int u = max(t, edge); u < min(t + KT, tiles); ++u) {
            // A weight of zero must not meet an infinity or NaN: where a tile that not all rows see to its end has one,
            // zeros take its place, and what it gives the rows that see it is added at the end.
            u32x4 *all = reinterpret_cast<u32x4 *>(lds.v[u % kHeld]);
            bool odd = false;
            for (int i = threadIdx.x; i < kTile / 16; i += kThreads) {
                u32x4 x = all[i];
                bool any = false;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const bool lo = not_finite(x[w]), hi = not_finite(x[w] >> 16);
                    x[w] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
                    any |= lo || hi;
                }
                if (any) all[i] = x;
                odd |= any;
            }
            if (__syncthreads_or(odd)) odd_tiles |= 1u << (u - edge);
        }
    };
    // One tile, the i-th of its step: s its scores, p its weights, next the scores of the tile after, was the weights of the
    // tile before.
    auto tile = [&](int t, int i, f32x16 (&s)[R], f32x16 (&next)[R], u32x4 (&p)[R][2], u32x4 (&was)[R][2]) {
        // The sums so far, for the reference maximum that the weights of tile t - 1 have.
        if (scaled) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int d = 0; d < kTiles; ++d) acc_scale(o[r][d], down[r]);
            scaled = 0;
        }
        if ((t + 1) * kKeys > all_see) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int left = mine[r] - t * kKeys - 4 * half;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (i / 4 * 8 + i % 4 >= left) s[r][i] = -INFINITY;
            }
        }
        products(next, was, [&](int c) {
#pragma unroll
            for (int j = c * kPieces / kProducts; j < (c + 1) * kPieces / kProducts; ++j) weights(s, p, j % R, j / R);
            // The loads behind the last products, every other.
            if (i < kBrings && c >= kProducts - 2 * kLoads && (kProducts - c) % 2 == 0) load(i, (c - (kProducts - 2 * kLoads)) / 2);
        });
        if (i == KT - 1) {
            keys_done();
            values_done();
        }
        if (odd_tiles >> max(t - edge, 0) & 1) {  // no bit is set before tile `edge`
#pragma unroll
            for (int r = 0; r < R; ++r) {
                uint32_t some = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float w = s[r][i];
                    asm volatile("" : "+v"(w));  // here, not ahead of the branch in every tile
                    some |= (w != 0.f ? 1u : 0u) << i;
                }
                if (t < tiles) lds.some[t - edge][r][threadIdx.x] = (uint16_t)some;
            }
        }
    };

    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    load_keys();
    load_values();
    f32x16 s0[R], s1[R];
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
        const bf16x8 k = *reinterpret_cast<const bf16x8 *>(lds.k[0] + k_at[st % 4] + st / 4 * (kKeys * 128));
#pragma unroll
        for (int r = 0; r < R; ++r) {
            asm volatile("s_nop 1");  // behind the queries' way to their registers
            if (st == 0) mfma_first(s0[r], k, q[r][0]);
            else mfma_next<true>(s0[r], k, q[r][st]);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) asm volatile("s_nop 15\n\ts_nop 7" : "+v"(s0[r]));
#pragma unroll
    for (int f = 0; f < kAhead; ++f) fetch(f);
    // Tiles 0 .. tiles: the last adds the values of the last but one.  (With two a step perhaps one more, of zeros.)
#pragma unroll 1
    for (int t = 0; t <= tiles; t += 2) {
        begin(t);
        tile(t, 0, s0, s1, p1, p0);
        if (KT == 1) {
            if (t == tiles) break;
            begin(t + 1);
        }
        tile(t + 1, KT - 1, s1, s0, p0, p1);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing is on its way to LDS when the workgroup ends

#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = first + 32 * r + col;
        l[r] = halves_sum(l[r]);
        const bool whole = !SPLIT || chunks == 1;
        const float inv = !whole ? 1.f : l[r] == 0.f ? 0.f : 1.f / l[r];
        const long slot = ((long)pair * blocks + block) * most_chunks + chunk;
        if (row >= rows) continue;
        const long at = (long)(blk.q0 + row / G) * a.H + blk.hk * G + row % G;
#pragma unroll
        for (int d = 0; d < kTiles; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 x = {o[r][d][4 * i] * inv, o[r][d][4 * i + 1] * inv, o[r][d][4 * i + 2] * inv, o[r][d][4 * i + 3] * inv};
                if (whole)
                    *reinterpret_cast<u32x2 *>(a.o + at * D + 32 * d + 8 * i + 4 * half) =
                        u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
                else
                    reinterpret_cast<f32x4 *>(parts.o)[(((slot * W + wave) * kTiles + d) * 4 + i) * kWave + lane] = x;
            }
        if (odd_tiles) {
            for (int n = 0; n < D / 2; ++n) {  // the lane's own elements, as above
                const int el = n / 16 * 32 + n % 16 / 4 * 8 + 4 * half + n % 4;
                float c = 0.f;
                for (int b = 0; b < kEdge; ++b) {
                    if (!(odd_tiles >> b & 1)) continue;
                    const int begin = (edge + b) * kKeys;
                    for (int j = 0; j < min(mine[r] - begin, kKeys); ++j) {
                        const uint16_t w = a.v[blk.hk * a.v_head + (long)(k0 + begin + j) * a.v_stride + el];
                        if (!not_finite(w)) continue;
                        const uint32_t is = lds.some[b][r][wave * kWave + j / 4 % 2 * 32 + col] >> (j / 8 * 4 + j % 4) & 1;
                        c = fmaf(is ? 1.f : 0.f, bf16_bits_to_f32(w), c);
                    }
                }
                if (c == 0.f) continue;
                if (whole) {
                    uint16_t *to = a.o + at * D + el;
                    *to = f32_to_bf16_bits(bf16_bits_to_f32(*to) + c);
                } else {
                    parts.o[((((slot * W + wave) * kTiles + n / 16) * 4 + n % 16 / 4) * kWave + lane) * 4 + n % 4] += c;
                }
            }
        }
        if (half) continue;
        if (!whole) parts.ml[slot * kSplitRows + wave * 32 + col] = float2{m[r], l[r]};
        else if (a.lse) a.lse[at] = l[r] == 0.f ? -INFINITY : (m[r] + __builtin_amdgcn_logf(l[r])) / kLog2e;
    }
}

// Adds up the chunks of a row block: a workgroup has 32 rows, a lane of a wavefront the four elements that registers 4 i .. of
// that lane of the accumulators hold.
template <int D>
__global__ __launch_bounds__(4 * kWave) void join_prompt_kernel(GroupedPromptArgs a, int blocks, int most_chunks, PromptParts parts)
{
    constexpr int kTiles = D / 32;
    const int of = blockIdx.x % kSplitWaves, pb = blockIdx.x / kSplitWaves, pair = pb / blocks;
    const Block blk(a, pair, pb % blocks, kSplitRows);
    const int chunks = chunks_of(blk.tiles, most_chunks), lane = lane_id(), i = threadIdx.x / kWave;
    const int row = blk.row0 + of * 32 + lane % 32;
    if (chunks == 1 || row >= blk.rows) return;
    const float2 *ml = parts.ml + (long)pb * most_chunks * kSplitRows + of * 32 + lane % 32;
    float top = -INFINITY;
#pragma unroll 8
    for (int c = 0; c < chunks; ++c) top = fmaxf(top, ml[c * kSplitRows].x);
    const float base = top == -INFINITY ? 0.f : top;
    float total = 0.f;
    f32x4 sum[kTiles] = {};
    const f32x4 *o = reinterpret_cast<const f32x4 *>(parts.o) + (((long)pb * most_chunks * kSplitWaves + of) * kTiles * 4 + i) * kWave + lane;
#pragma unroll 4
    for (int c = 0; c < chunks; ++c) {
        const float2 part = ml[c * kSplitRows];
        const float f = __builtin_amdgcn_exp2f(part.x - base);
        total = fmaf(part.y, f, total);
#pragma unroll
        for (int d = 0; d < kTiles; ++d) {
            const f32x4 v = o[((long)c * kSplitWaves * kTiles + d) * 4 * kWave];
#pragma unroll
            for (int n = 0; n < 4; ++n) sum[d][n] = fmaf(v[n], f, sum[d][n]);
        }
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const long at = (long)(blk.q0 + row / blk.G) * a.H + blk.hk * blk.G + row % blk.G;
#pragma unroll
    for (int d = 0; d < kTiles; ++d)
        *reinterpret_cast<u32x2 *>(a.o + at * D + 32 * d + 8 * i + lane / 32 * 4) =
            u32x2{pack_bf16x2(sum[d][0] * inv, sum[d][1] * inv), pack_bf16x2(sum[d][2] * inv, sum[d][3] * inv)};
    if (a.lse && i == 0 && lane < 32) a.lse[at] = total == 0.f ? -INFINITY : (base + __builtin_amdgcn_logf(total)) / kLog2e;
}

#ifndef ECOSPEC_GP_R
#define ECOSPEC_GP_R 1
#endif
#ifndef ECOSPEC_GP_W
#define ECOSPEC_GP_W 4
#endif
#ifndef ECOSPEC_GP_KT
#define ECOSPEC_GP_KT 1
#endif

template <int D>
hipError_t launch(const GroupedPromptArgs &a, void *workspace, hipStream_t stream)
{
    const long rows = (long)a.max_tokens * (a.H / a.Hkv);
    const int pairs = a.B * a.Hkv, few = (int)((rows + kSplitRows - 1) / kSplitRows);
    char *w = static_cast<char *>(workspace);
    const PromptParts parts{reinterpret_cast<float2 *>(w), reinterpret_cast<float *>(w + kSlots * kSplitRows * sizeof(float2))};
    const long room = kSlots / ((long)pairs * few), cut = (a.M + kKeys - 1) / kKeys / kMinTiles;
    const int chunks = (int)(room < cut ? room : cut);
    if (chunks > 1) {
        prompt_kernel<D, kSplitWaves, 1, 1, true><<<(unsigned)(pairs * few * chunks), kSplitWaves * kWave, 0, stream>>>(a, few, chunks, parts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        join_prompt_kernel<D><<<(unsigned)(pairs * few * kSplitWaves), 4 * kWave, 0, stream>>>(a, few, chunks, parts);
        return hipGetLastError();
    }
    constexpr int W = ECOSPEC_GP_W, R = ECOSPEC_GP_R, KT = ECOSPEC_GP_KT;
    const int blocks = (int)((rows + 32 * R * W - 1) / (32 * R * W));
    prompt_kernel<D, W, R, KT, false><<<(unsigned)((long)pairs * blocks), W * kWave, 0, stream>>>(a, blocks, 1, parts);
    return hipGetLastError();
}

}  // namespace

size_t grouped_prompt_workspace(int D) { return (size_t)kSlots * kSplitRows * (sizeof(float2) + D * sizeof(float)); }

hipError_t launch_grouped_prompt(const GroupedPromptArgs &a, int D, void *workspace, hipStream_t stream)
{
    return D == 64 ? launch<64>(a, workspace, stream) : launch<128>(a, workspace, stream);
}

}  // namespace ecospec
