// Attention of whole prompts with grouped heads: causal, sequences of different lengths side by side.
//
// The query rows of a sequence that read the same keys are its tokens times the heads of one key/value head, token by
// token: a workgroup takes consecutive ones, 32 R of each of four wavefronts.  So short sequences fill its rows too, and
// long ones have few keys that only some of the rows see.
//   Scores are transposed (S^T = K Q^T): a lane holds one row, its scores are the value product's operand as they stand
//   (O^T = V^T P^T), and V^T is read with the transposing LDS load.
//   Three tiles of 32 keys are under way: while the matrix cores multiply the keys of tile t + 1 and the values of tile
//   t - 1, the vector unit works out the weights of tile t, a piece behind each product.
//   Keys and values go from memory straight to LDS, two tiles before their products (rings of four tiles each), in
//   panels: of 64 elements for keys (rows of 128 bytes, chunks of 16 XORed with row bits, so that 16 rows' chunks, a quarter
//   of a read, lie in different banks), of 32 for values (rows of 64 bytes: half a read is 256 in a row).  One barrier a
//   tile, and operands are read seven products ahead, past it: keys land a tile earlier than that needs.
#include "attn_plan.hpp"
#include "step.hpp"

namespace ecospec {
namespace {

constexpr int kKeys = 32, kPromptWaves = 4, kPromptThreads = kPromptWaves * kWave;
constexpr float kSlack = 8.f;  // powers of two that weights may pass 1 by before their reference maximum moves

typedef __attribute__((ext_vector_type(4))) short s16x4;

__device__ __forceinline__ u32x2 read_tr(const char *p)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
}

__device__ __forceinline__ bool not_finite(uint32_t bf16) { return (bf16 & 0x7f80u) == 0x7f80u; }

// The score products, sums in vector registers, which the vector unit works on; a register written by the vector
// unit needs two wait states before a product reads it.
__device__ __forceinline__ void mfma_first(f32x16 &s, const bf16x8 &k, const bf16x8 &q)
{
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "v"(q));
}

__device__ __forceinline__ void mfma_next(f32x16 &s, const bf16x8 &k, const bf16x8 &q)
{
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "v"(q));
}

// D: width of a head; R: row tiles of a wavefront.
template <int D, int R>
__global__ __launch_bounds__(kPromptThreads, R == 1 ? 2 : 1) void prompt_kernel(GroupedPromptArgs a, int blocks)
{
    constexpr int kRows = 32 * R * kPromptWaves, kSteps = D / 16, kPanels = D / 64, kTiles = D / 32;
    constexpr int kTile = kKeys * D * 2, kLoads = 2 * kPanels;  // bytes of a tile; loads of a tile by a wavefront
    constexpr int kEdge = kRows / kKeys + 1;                    // most tiles that some rows of a workgroup see in part
    constexpr int kOperands = kSteps + 2 * kTiles;              // key and value operands of a tile
    constexpr int kRing = 8, kAhead = kRing - 1;                // of them in registers
    static_assert(kOperands % kRing == 0, "a tile's first operand has a fixed place");
    constexpr int kProducts = kOperands * R, kPieces = 20 * R;  // of a tile
    struct Tiles {
        char k[4][kTile];  // panel, row r, chunk c of 16 bytes at place c ^ (r >> 1 & 7)
        char v[4][kTile];  // panel of 32 elements, row
        uint16_t some[kEdge][R][kPromptThreads];  // which weights of a lane are not zero, in a tile with infinities or NaN
    };
    __shared__ __attribute__((aligned(16))) Tiles lds;

    const int G = a.H / a.Hkv, pairs = a.B * a.Hkv;
    // Workgroups are dealt to the eight XCDs in turn: with pairs innermost a head's row blocks meet on few of them.  The
    // longest row blocks first, so that no long one is left for the end.
    const int pair = blockIdx.x % pairs, block = blocks - 1 - (int)(blockIdx.x / pairs);
    const int b = pair / a.Hkv, hk = pair % a.Hkv;
    const int q0 = __builtin_amdgcn_readfirstlane(min(max(a.q_offsets[b], 0), a.N));
    const int nq = __builtin_amdgcn_readfirstlane(min(max(a.q_offsets[b + 1], q0), a.N)) - q0;
    const int k0 = __builtin_amdgcn_readfirstlane(min(max(a.kv_offsets[b], 0), a.M));
    const int nk = __builtin_amdgcn_readfirstlane(min(max(a.kv_offsets[b + 1], k0), a.M)) - k0;
    const int rows = nq * G, row0 = block * kRows;
    if (row0 >= rows) return;

    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), col = lane % 32, half = lane / 32;
    auto limit = [&](int row) { return min(max(row / G + 1 + nk - nq, 0), nk); };  // keys that a query row sees
    const int tiles = (limit(min(row0 + kRows, rows) - 1) + kKeys - 1) / kKeys;
    const int edge = limit(row0) / kKeys;  // first tile that some row of the workgroup does not see to its end
    const int first = row0 + 32 * R * wave;
    const int all_see = __builtin_amdgcn_readfirstlane(limit(min(first, rows - 1)));  // keys that all rows of the wavefront see

    // ---- queries
    int mine[R];      // keys that the lane's rows see
    bf16x8 q[R][kSteps];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = min(first + 32 * r + col, rows - 1), token = row / G;
        mine[r] = limit(row);
        const uint16_t *from = a.q + (long)(q0 + token) * a.q_stride + (hk * G + row - token * G) * a.q_head + half * 8;
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
            u32x4 w = *reinterpret_cast<const u32x4 *>(from + st * 16);
            // The scale is positive from here on: the largest product is the largest score.
            if (a.scale < 0.f) w ^= 0x80008000u;
            q[r][st] = __builtin_bit_cast(bf16x8, w);
        }
    }

    // ---- loads: wavefront w brings rows 8 w .. 8 w + 7 of each panel of a tile's keys, and 16 rows of panels of its values
    // a load.  Rows past the last key, and tiles past the last, become zeros.
    const uint16_t *src_k = a.k + hk * a.k_head + k0 * a.k_stride, *src_v = a.v + hk * a.v_head + k0 * a.v_stride;
    const uint32_t stride_k = (uint32_t)a.k_stride * 2, stride_v = (uint32_t)a.v_stride * 2;
    const int e = 8 * wave + lane / 8, place = (lane % 8) ^ (e >> 1 & 7);
    const uint32_t off_k = e * stride_k + place * 16;
    // Values: load n of wavefront w brings 16 rows (the upper ones for odd n) of a panel.
    const int v_panel = D == 128 ? wave : wave / 2, v_row = D == 128 ? 0 : wave % 2 * 16;
    const uint32_t off_v = (v_row + lane / 4) * stride_v + v_panel * 64 + lane % 4 * 16, off_low = off_v + 16 * stride_v;
    const uint32_t ring_k = __builtin_amdgcn_readfirstlane(lds_addr(lds.k) + wave * 1024);
    const uint32_t ring_v = __builtin_amdgcn_readfirstlane(lds_addr(lds.v) + v_panel * 2048 + v_row * 64);
    int left_k = nk, left_v = nk;  // keys from the tile to load next on
    uint32_t to_k = ring_k, to_v = ring_v;
    u32x4 key_src, value_src;
    auto aim_keys = [&] {
        const int n = max(min(left_k, kKeys), 0);
        key_src = rsrc_words(src_k, n ? (uint32_t)(n - 1) * stride_k + D * 2 : 0);
    };
    auto aim_values = [&] {
        const int n = max(min(left_v, kKeys), 0);
        value_src = rsrc_words(src_v, n ? (uint32_t)(n - 1) * stride_v + D * 2 : 0);
    };
    auto keys_done = [&] {
        left_k -= kKeys;
        if (left_k > 0) src_k += kKeys / 2 * stride_k;
        to_k = to_k == ring_k + 3 * kTile ? ring_k : to_k + kTile;
    };
    auto values_done = [&] {
        left_v -= kKeys;
        if (left_v > 0) src_v += kKeys / 2 * stride_v;
        to_v = to_v == ring_v + 3 * kTile ? ring_v : to_v + kTile;
    };
    auto load = [&](int n) {
        if (n < kPanels) load16_lds(key_src, off_k + n * 128, to_k + n * (kKeys * 128));
        else if (n == kPanels) load16_lds(value_src, off_v, to_v);
        else load16_lds(value_src, off_low, to_v + 1024);
    };
    auto load_keys = [&] {
        aim_keys();
#pragma unroll
        for (int n = 0; n < kPanels; ++n) load(n);
        keys_done();
    };
    auto load_values = [&] {
        aim_values();
#pragma unroll
        for (int n = kPanels; n < kLoads; ++n) load(n);
        values_done();
    };
#pragma unroll 1
    for (int t = 0; t < 3; ++t) load_keys();
    load_values();
    // The values of tile -1, whose weights are zeros.
    for (int i = threadIdx.x; i < kTile / 16; i += kPromptThreads) reinterpret_cast<u32x4 *>(lds.v[3])[i] = u32x4{0, 0, 0, 0};

    f32x16 o[R][kTiles];
    float m[R], l[R], down[R];
    int scaled[R];
    u32x4 p0[R][2] = {}, p1[R][2];  // weights of the tile before and of this one, in turn: 16 keys each
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int d = 0; d < kTiles; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[r][d][i] = 0.f;
        m[r] = -INFINITY;
        l[r] = 0.f;
        down[r] = 1.f;
        scaled[r] = 0;
    }
    uint32_t odd_tiles = 0;  // edge tiles with infinities or NaN among the values
    const float scale2 = fmaxf(fabsf(a.scale) * kLog2e, 0x1p-126f);  // not zero: it meets infinities

    uint32_t k_at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) k_at[i] = (uint32_t)(col * 128 + ((2 * i + half) ^ (col >> 1 & 7)) * 16);
    const int i16 = lane % 16;
    const uint32_t v_at = (uint32_t)((4 * half + i16 / 4) * 64 + lane / 16 % 2 * 32 + i16 % 4 * 8);

    // Piece c of the weights of row tile r with scores s.  Register i is key 8 (i / 4) + 4 half + i % 4.
    float top[R], base[R], sum[R];
    auto weights = [&](f32x16 &s, u32x4 (&p)[2], int r, int c) {
        if (c == 0) {
            top[r] = max3(max3(max3(s[0], s[1], s[2]), max3(s[3], s[4], s[5]), s[6]),
                          max3(max3(s[7], s[8], s[9]), max3(s[10], s[11], s[12]), s[13]), fmaxf(s[14], s[15]));
        } else if (c == 1) {
            top[r] = halves_max(top[r]) * scale2;
        } else if (c == 2) {
            int move = __any(top[r] > m[r] + kSlack);
            scaled[r] = move & __any(m[r] != -INFINITY);
            asm("" : "+v"(move));  // a select, not a branch
            const float now = move ? fmaxf(m[r], top[r]) : m[r];
            base[r] = now == -INFINITY ? 0.f : now;
            down[r] = __builtin_amdgcn_exp2f((m[r] == -INFINITY ? base[r] : m[r]) - base[r]);
            m[r] = now;
            sum[r] = 0.f;
        } else {
            const int e = c - 3;  // of 16 elements
            // Written out to stay here, where the compiler would sink it behind all products, and in this order: the result of
            // an exponential needs a wait state, which the instructions of the element before are.
            if (e < 16) {
                const float x = fmaf(s[e], scale2, -base[r]);
                asm volatile("v_exp_f32 %0, %1" : "=v"(s[e]) : "v"(x));
            }
            // The element before: its sum, and pairs to bf16.
            if (e > 0 && e <= 16) {
                const int i = e - 1;
                asm volatile("v_add_f32 %0, %0, %1" : "+v"(sum[r]) : "v"(s[i]));
                if (i % 2) {
                    uint32_t w;
                    asm volatile("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(w) : "v"(s[i - 1]), "v"(s[i]));
                    p[i / 8][i % 8 / 2] = w;
                }
                if (i == 15) l[r] = fmaf(l[r], down[r], sum[r]);
            }
        }
    };
    // Operand f of a tile: its keys' steps, then its values' (16 keys, element tile).  From kOperands on the next tile's.
    uint32_t key_to = 0, value_to = 2 * kTile, key_at[4], value_at;
    bf16x8 ring[kRing];
    auto fetch = [&](int f) {
        const int x = f % kOperands;
        if (x == 0) {
            key_to = key_to == 3 * kTile ? 0 : key_to + kTile;
#pragma unroll
            for (int i = 0; i < 4; ++i) key_at[i] = k_at[i] + key_to;
        }
        if (x == kSteps) {
            value_to = value_to == 3 * kTile ? 0 : value_to + kTile;
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
                else if (f < kSteps) mfma_next(s[r], ring[f % kRing], q[r][f]);
                else o[r][n % kTiles] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    ring[f % kRing], __builtin_bit_cast(bf16x8, p[r][n / kTiles]), o[r][n % kTiles], 0, 0, 0);
                between(f * R + r);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    // One tile: s its scores, p its weights, next the scores of the tile after, was the weights of the tile before.
    auto tile = [&](int t, f32x16 (&s)[R], f32x16 (&next)[R], u32x4 (&p)[R][2], u32x4 (&was)[R][2]) {
        // The keys of tile t + 2 and the values of tile t have landed; every wavefront is past the scores of tile t and the
        // values of tile t - 2.
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kLoads) : "memory");
        aim_keys();
        aim_values();
        if (t >= edge && t < tiles) {
            // A weight of zero must not meet an infinity or NaN: where a tile that not all rows see to its end has one,
            // zeros take its place, and what it gives the rows that see it is added at the end.
            u32x4 *all = reinterpret_cast<u32x4 *>(lds.v[t % 4]);
            bool odd = false;
            for (int i = threadIdx.x; i < kTile / 16; i += kPromptThreads) {
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
            if (__syncthreads_or(odd)) odd_tiles |= 1u << (t - edge);
        }
        // The sums so far, for the reference maximum that the weights of tile t - 1 have.
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (scaled[r]) {
#pragma unroll
                for (int d = 0; d < kTiles; ++d) acc_scale(o[r][d], down[r]);
                scaled[r] = 0;
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
            for (int j = c * kPieces / kProducts; j < (c + 1) * kPieces / kProducts; ++j) weights(s[j % R], p[j % R], j % R, j / R);
            // The loads behind the last products but one, every other.
            const int n = (c - (kProducts - 2 * kLoads)) / 2;
            if (c >= kProducts - 2 * kLoads && (c - kProducts) % 2 == 0) load(n);
        });
        keys_done();
        values_done();
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
            if (st == 0) mfma_first(s0[r], k, q[r][0]);
            else mfma_next(s0[r], k, q[r][st]);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) asm volatile("s_nop 15\n\ts_nop 7" : "+v"(s0[r]));
#pragma unroll
    for (int f = 0; f < kAhead; ++f) fetch(f);
    // Tiles 0 .. tiles: the last adds the values of the last but one.
#pragma unroll 1
    for (int t = 0; t <= tiles; t += 2) {
        tile(t, s0, s1, p1, p0);
        if (t + 1 <= tiles) tile(t + 1, s1, s0, p0, p1);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing is on its way to LDS when the workgroup ends

#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = first + 32 * r + col;
        l[r] = halves_sum(l[r]);
        if (row >= rows) continue;
        const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
        const long at = (long)(q0 + row / G) * a.H + hk * G + row % G;
#pragma unroll
        for (int d = 0; d < kTiles; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<u32x2 *>(a.o + at * D + 32 * d + 8 * i + 4 * half) =
                    u32x2{pack_bf16x2(o[r][d][4 * i] * inv, o[r][d][4 * i + 1] * inv),
                          pack_bf16x2(o[r][d][4 * i + 2] * inv, o[r][d][4 * i + 3] * inv)};
        if (a.lse && half == 0) a.lse[at] = l[r] == 0.f ? -INFINITY : (m[r] + __builtin_amdgcn_logf(l[r])) / kLog2e;
        if (!odd_tiles) continue;
        for (int n = 0; n < D / 2; ++n) {  // the lane's own elements, as above
            const int el = n / 16 * 32 + n % 16 / 4 * 8 + 4 * half + n % 4;
            float c = 0.f;
            for (int x = 0; x < kEdge; ++x) {
                if (!(odd_tiles >> x & 1)) continue;
                const int from = (edge + x) * kKeys;
                for (int j = 0; j < min(mine[r] - from, kKeys); ++j) {
                    const uint16_t w = a.v[hk * a.v_head + (long)(k0 + from + j) * a.v_stride + el];
                    if (!not_finite(w)) continue;
                    const uint32_t is = lds.some[x][r][wave * kWave + j / 4 % 2 * 32 + col] >> (j / 8 * 4 + j % 4) & 1;
                    c = fmaf(is ? 1.f : 0.f, bf16_bits_to_f32(w), c);
                }
            }
            if (c == 0.f) continue;
            uint16_t *to = a.o + at * D + el;
            *to = f32_to_bf16_bits(bf16_bits_to_f32(*to) + c);
        }
    }
}

template <int D, int R>
void launch(const GroupedPromptArgs &a, hipStream_t stream)
{
    const int blocks = (int)(((long)a.max_tokens * (a.H / a.Hkv) + 128 * R - 1) / (128 * R));
    prompt_kernel<D, R><<<(unsigned)(a.B * a.Hkv * blocks), kPromptThreads, 0, stream>>>(a, blocks);
}

}  // namespace

size_t grouped_prompt_workspace(int D) { return 256; }

hipError_t launch_grouped_prompt(const GroupedPromptArgs &a, int D, void *workspace, hipStream_t stream)
{
#ifndef ECOSPEC_GP_R
#define ECOSPEC_GP_R 1
#endif
    if (D == 64) launch<64, ECOSPEC_GP_R>(a, stream);
    else launch<128, ECOSPEC_GP_R>(a, stream);
    return hipGetLastError();
}

}  // namespace ecospec
