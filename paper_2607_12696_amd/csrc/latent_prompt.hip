// Latent attention of prompts, expanded form: per head 192-element keys (128 of its own, 64 rotary ones that all heads
// share) and 128-element values, causal.
//
// 640 operations a row, key and head against 512 bytes a key and head: bound by the matrix cores.  A workgroup takes 128
// consecutive queries of one head, 32 rows each of four wavefronts; two workgroups a compute unit, each with its own barriers.
//   Scores are transposed (S^T = K Q^T): a lane holds one row, its scores are the value product's operand as they stand
//   (O^T = V^T P^T), and V^T is read with the transposing LDS load.
//   Three tiles are under way: while the matrix cores multiply the keys of tile t + 1 and the values of tile t - 1, the
//   vector unit works out the weights of tile t, a piece behind each product.
//   Keys and values go from memory straight to LDS, two tiles ahead (rings of three tiles of keys, five of values), in
//   panels: of 64 elements for keys (rows of 128 bytes, chunks of 16 XORed with row bits, so that 16 rows' chunks, a quarter
//   of a read, lie in different banks), of 32 for values (rows of 64 bytes: half a read is 256 in a row).  So a read's
//   place in the tile is an immediate offset.  One barrier a tile of 32 keys.
//   The weights are rounded to bf16, the type of the value product's operands; their sum keeps fp32.  A weight is off by at
// most 2^-9 of itself, which takes the error of o against 64 bits from 1.6e-3 (its own rounding to bf16) to 2.2e-3 (root mean
// square); weights in two parts would double the value products.
// Measured: 5003 tokens of 128 heads 1.22 ms (842 TFLOP/s), 6 prompts of 563 to 1201 tokens, 16 heads, 75 us.  Workgroups of
// 256 queries, one a compute unit, load half as often but wait for each other more and leave more idle rows: 1.24 ms and
// 84 us.  In the long prompt the matrix cores are busy for half of the cycles and wavefronts wait for a quarter of theirs;
// power counts too (operands of zeros take a fifth less time).  The short ones are held by their longest row block: 47 tiles
// in series at 1.5 us, two workgroups sharing a compute unit.
#include "attn_plan.hpp"

namespace ecospec {
namespace {

constexpr int kDn = 128, kP = 64, kDv = 128, kDq = kDn + kP;
constexpr int kKeys = 32;
constexpr int kWaves = 4, kRows = 32 * kWaves, kThreads = 64 * kWaves;
constexpr int kSteps = kDq / 16;
constexpr int kRing = 4, kAhead = 3;  // key and value operands in registers
constexpr int kLoads = 5;             // loads of a tile by a wavefront
constexpr int kProducts = kSteps + 8;  // of a tile: scores, values
constexpr int kLoadFrom = kProducts - 2 * kLoads;  // a load behind every other product from here on
constexpr int kEdge = kRows / kKeys + 1;  // most tiles that some rows of a workgroup see in part
constexpr float kSlack = 8.f;

typedef __attribute__((ext_vector_type(4))) short s16x4;

__device__ __forceinline__ u32x2 read_tr(const char *p)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
}

__device__ __forceinline__ bool not_finite(uint32_t bf16) { return (bf16 & 0x7f80u) == 0x7f80u; }

constexpr int kPanel = kKeys * 128;              // 64 elements of a tile's keys
constexpr int kKeyTile = 3 * kPanel, kValueTile = kKeys * kDv * 2;

struct Tiles {
    char k[3][kKeyTile];    // panel, row r, chunk c of 16 bytes at place c ^ (r >> 1 & 7); the last panel is the rotary part
    char v[5][kValueTile];  // panel of 32 elements, row
    uint16_t some[kEdge][kThreads];  // which weights of a lane are not zero, in a tile with infinities or NaN
};

union Lds {
    char q[kWaves][32 * kDq * 2];  // the queries of each wavefront, before the loop: at c ^ (r >> 1 & 7)
    Tiles t;
};
static_assert(2 * sizeof(Lds) <= 160 * 1024, "two workgroups a compute unit");

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

__global__ __launch_bounds__(kThreads, 2) void prompt_kernel(PromptArgs a, int blocks)
{
    __shared__ __attribute__((aligned(16))) Lds lds;
    // A head's row blocks on one XCD; the longest of all heads first, so that no long one is left for the end.
    const int pairs = (a.B * a.H + 7) / 8, pair = blockIdx.x % 8 + 8 * (int)(blockIdx.x / 8 % pairs);
    const int block = blocks - 1 - (int)(blockIdx.x / 8 / pairs);
    if (pair >= a.B * a.H) return;
    const int b = pair / a.H, h = pair % a.H;
    const int q0 = __builtin_amdgcn_readfirstlane(min(max(a.q_offsets[b], 0), a.N));
    const int nq = __builtin_amdgcn_readfirstlane(min(max(a.q_offsets[b + 1], q0), a.N)) - q0;
    const int k0 = __builtin_amdgcn_readfirstlane(min(max(a.kv_offsets[b], 0), a.M));
    const int nk = __builtin_amdgcn_readfirstlane(min(max(a.kv_offsets[b + 1], k0), a.M)) - k0;
    const int row0 = block * kRows;
    if (row0 >= nq) return;

    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), col = lane % 32, half = lane / 32;
    auto limit = [&](int row) { return min(max(row + 1 + nk - nq, 0), nk); };  // keys that a query sees
    const int tiles = (limit(min(row0 + kRows, nq) - 1) + kKeys - 1) / kKeys;
    const int edge = limit(row0) / kKeys;  // first tile that some row of the workgroup does not see to its end
    const int first = row0 + 32 * wave;
    const int all_see = limit(first);      // keys that all rows of the wavefront see

    // ---- queries through LDS
    bf16x8 q[kSteps];
    {
        const int rows = max(min(nq - first, 32), 0), stride = a.H * kDq * 2;
        const u32x4 from = rsrc_words(a.q + ((long)(q0 + min(first, nq - 1)) * a.H + h) * kDq,
                                      rows ? (uint32_t)((rows - 1) * stride + kDq * 2) : 0);
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds_addr(lds.q[wave]));
#pragma unroll
        for (int n = 0; n < 12; ++n) {
            const int i = n * 64 + lane, r = i / 24, c = i % 24;
            load16_lds(from, (uint32_t)(r * stride + (c ^ (r >> 1 & 7)) * 16), to + n * 1024);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
            u32x4 w = *reinterpret_cast<const u32x4 *>(lds.q[wave] + col * kDq * 2 + ((2 * st + half) ^ (col >> 1 & 7)) * 16);
            // The scale is positive from here on: the largest product is the largest score.
            if (a.scale < 0.f) w ^= 0x80008000u;
            q[st] = __builtin_bit_cast(bf16x8, w);
        }
    }
    __syncthreads();

    // ---- loads: wavefront w brings rows 8 w .. 8 w + 7 of a tile's keys, a panel a load, and panel w of its values, 16 rows a
    // load.  Rows past the last key, and tiles past the last, become zeros.
    const uint16_t *src_k = a.k + h * a.k_head + k0 * a.k_stride, *src_v = a.v + h * a.v_head + k0 * a.v_stride;
    const uint16_t *rope = a.k_rope + (long)k0 * kP;
    const uint32_t stride_k = (uint32_t)a.k_stride * 2, stride_v = (uint32_t)a.v_stride * 2;
    const int e = 8 * wave + lane / 8, place = (lane % 8) ^ (e >> 1 & 7);
    const uint32_t off_k = e * stride_k + place * 16, off_rope = (uint32_t)(e * kP * 2 + place * 16);
    const uint32_t off_v = lane / 4 * stride_v + wave * 64 + lane % 4 * 16, off_low = off_v + 16 * stride_v;
    // The tile to load next: its place in memory and in the rings.
    const uint32_t ring_k = __builtin_amdgcn_readfirstlane(lds_addr(lds.t.k) + wave * 1024);
    const uint32_t ring_v = __builtin_amdgcn_readfirstlane(lds_addr(lds.t.v) + wave * 2048);
    int left_k = tiles ? nk : 0;  // keys from the tile on
    uint32_t to_k = ring_k, to_v = ring_v;
    u32x4 k_src, rope_src, v_src;
    auto aim = [&] {
        const int rows = max(min(left_k, kKeys), 0);
        k_src = rsrc_words(src_k, rows ? (uint32_t)(rows - 1) * stride_k + kDn * 2 : 0);
        rope_src = rsrc_words(rope, (uint32_t)rows * kP * 2);
        v_src = rsrc_words(src_v, rows ? (uint32_t)(rows - 1) * stride_v + kDv * 2 : 0);
    };
    auto advance = [&] {
        left_k -= kKeys;
        if (left_k > 0) {
            src_k += kKeys / 2 * stride_k;
            src_v += kKeys / 2 * stride_v;
            rope += kKeys * kP;
        }
        to_k = to_k == ring_k + 2 * kKeyTile ? ring_k : to_k + kKeyTile;
        to_v = to_v == ring_v + 4 * kValueTile ? ring_v : to_v + kValueTile;
    };
    auto load = [&](int n) {
        if (n == 0) load16_lds(k_src, off_k, to_k);
        else if (n == 1) load16_lds(k_src, off_k + 128, to_k + kPanel);
        else if (n == 2) load16_lds(rope_src, off_rope, to_k + 2 * kPanel);
        else if (n == 3) load16_lds(v_src, off_v, to_v);
        else load16_lds(v_src, off_low, to_v + 1024);
    };
#pragma unroll 1
    for (int t = 0; t < 2; ++t) {
        aim();
#pragma unroll
        for (int n = 0; n < kLoads; ++n) load(n);
        advance();
    }
    // The values of tile -1, whose weights are zeros.
    for (int i = threadIdx.x; i < kKeys * kDv * 2 / 16; i += kThreads) reinterpret_cast<u32x4 *>(lds.t.v[4])[i] = u32x4{0, 0, 0, 0};

    f32x16 o[kDv / 32];
#pragma unroll
    for (int d = 0; d < kDv / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float m = -INFINITY, l = 0.f, down = 1.f;
    int scaled = 0;
    bf16x8 p[2] = {};  // weights of the tile before: 16 keys each
    uint32_t odd_tiles = 0;  // edge tiles with infinities or NaN among the values
    const float scale2 = fmaxf(fabsf(a.scale) * kLog2e, 0x1p-126f);  // not zero: it meets infinities

    uint32_t k_at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) k_at[i] = (uint32_t)(col * 128 + ((2 * i + half) ^ (col >> 1 & 7)) * 16);
    const int i16 = lane % 16;
    const uint32_t v_at = (uint32_t)((4 * half + i16 / 4) * 64 + lane / 16 % 2 * 32 + i16 % 4 * 8);

    // Behind product c, a piece of the weights of the scores s of a tile.  Register i is key 8 (i / 4) + 4 half + i % 4.
    float top, base, sum;
    u32x4 packed[2];
    auto weights = [&](f32x16 &s, int c) {
        if (c == 0) {
            top = max3(max3(max3(s[0], s[1], s[2]), max3(s[3], s[4], s[5]), s[6]),
                       max3(max3(s[7], s[8], s[9]), max3(s[10], s[11], s[12]), s[13]), fmaxf(s[14], s[15]));
        } else if (c == 1) {
            top = halves_max(top) * scale2;
        } else if (c == 2) {
            int move = __any(top > m + kSlack);
            scaled = move & __any(m != -INFINITY);
            asm("" : "+v"(move));  // a select, not a branch
            const float now = move ? fmaxf(m, top) : m;
            base = now == -INFINITY ? 0.f : now;
            down = __builtin_amdgcn_exp2f((m == -INFINITY ? base : m) - base);
            m = now;
            sum = 0.f;
        } else {
            const int e = c - 3;  // of 16 elements
            if (e < 16) s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], scale2, -base));
            // The element before: its sum, and pairs to bf16.  Written out to stay here, where the compiler would sink them
            // behind all products; a piece later, because the result of an exp2 needs a wait state.
            if (e > 0 && e <= 16) {
                const int i = e - 1;
                asm volatile("v_add_f32 %0, %0, %1" : "+v"(sum) : "v"(s[i]));
                if (i % 2) {
                    uint32_t w;
                    asm volatile("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(w) : "v"(s[i - 1]), "v"(s[i]));
                    packed[i / 8][i % 8 / 2] = w;
                }
                if (i == 15) l = fmaf(l, down, sum);
            }
        }
    };
    static_assert(kProducts >= 20, "all pieces");
    // Operands of the tiles at these ring offsets.
    uint32_t key_at[4], value_at = v_at + 4 * kValueTile;
    auto k_frag = [&](int st) { return *reinterpret_cast<const bf16x8 *>(lds.t.k[0] + key_at[st % 4] + st / 4 * kPanel); };
    auto v_frag = [&](int n) {  // n: 4 * (16 keys) + element tile
        const char *w = lds.t.v[0] + value_at + n % 4 * (kKeys * 64) + n / 4 * 16 * 64;
        const u32x2 lo = read_tr(w), hi = read_tr(w + 8 * 64);
        return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
    };
    bf16x8 k[kRing], v[kAhead];
    auto first_keys = [&] {
#pragma unroll
        for (int st = 0; st < kRing - 1; ++st) k[st] = k_frag(st);
    };
    // Products of a tile's keys (the first ones fetched) into s, then of a tile's values, `between(c)` behind product c.
    auto products = [&](f32x16 &s, auto between) {
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
            if (st + kRing - 1 < kSteps) k[(st + kRing - 1) % kRing] = k_frag(st + kRing - 1);
            else v[st + kRing - 1 - kSteps] = v_frag(st + kRing - 1 - kSteps);
            __builtin_amdgcn_sched_barrier(0);
            if (st == 0) mfma_first(s, k[0], q[0]);
            else mfma_next(s, k[st % kRing], q[st]);
            between(st);
        }
        static_assert(kRing - 1 == kAhead, "the last steps fetch the first value operands");
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            __builtin_amdgcn_sched_barrier(0);
            o[n % 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[n % kAhead], p[n / 4], o[n % 4], 0, 0, 0);
            between(kSteps + n);
            if (n + kAhead < 8) v[n % kAhead] = v_frag(n + kAhead);
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    uint32_t key_to = 0, value_to = 4 * kValueTile;
    auto turn_rings = [&] {  // to the keys and the values after
        key_to = key_to == 2 * kKeyTile ? 0 : key_to + kKeyTile;
        value_to = value_to == 4 * kValueTile ? 0 : value_to + kValueTile;
#pragma unroll
        for (int i = 0; i < 4; ++i) key_at[i] = k_at[i] + key_to;
        value_at = v_at + value_to;
    };

    // One tile: s its scores, next the scores of the tile after.
    auto tile = [&](int t, f32x16 &s, f32x16 &next) {
        // Tile t + 1 has landed; every wavefront is past the scores of tile t and the values of tile t - 2.
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLoads) : "memory");
        first_keys();
        aim();
        if (t >= edge && t < tiles) {
            // A weight of zero must not meet an infinity or NaN: where a tile that not all rows see to its end has one,
            // zeros take its place, and what it gives the rows that see it is added at the end.
            u32x4 *all = reinterpret_cast<u32x4 *>(lds.t.v[t % 5]);
            bool odd = false;
            for (int i = threadIdx.x; i < kKeys * kDv * 2 / 16; i += kThreads) {
                u32x4 v = all[i];
                bool any = false;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const bool lo = not_finite(v[w]), hi = not_finite(v[w] >> 16);
                    v[w] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
                    any |= lo || hi;
                }
                if (any) all[i] = v;
                odd |= any;
            }
            if (__syncthreads_or(odd)) odd_tiles |= 1u << (t - edge);
        }
        // The sums so far, for the reference maximum that the weights of tile t - 1 have.
        if (scaled) {
#pragma unroll
            for (int d = 0; d < kDv / 32; ++d) acc_scale(o[d], down);
            scaled = 0;
        }
        if ((t + 1) * kKeys > all_see) {
            const int left = limit(first + col) - t * kKeys - 4 * half;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i / 4 * 8 + i % 4 >= left) s[i] = -INFINITY;
        }
        products(next, [&](int c) {
            weights(s, c);
            if (c >= kLoadFrom && (c - kLoadFrom) % 2 == 0) load((c - kLoadFrom) / 2);
        });
#pragma unroll
        for (int st = 0; st < 2; ++st) p[st] = __builtin_bit_cast(bf16x8, packed[st]);
        advance();
        turn_rings();
        if (odd_tiles >> max(t - edge, 0) & 1) {  // no bit is set before tile `edge`
            uint32_t some = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) some |= (s[i] != 0.f ? 1u : 0u) << i;
            lds.t.some[t - edge][threadIdx.x] = (uint16_t)some;
        }
    };

    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    aim();
#pragma unroll
    for (int n = 0; n < kLoads; ++n) load(n);
    advance();
    f32x16 s0, s1;
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) key_at[i] = k_at[i];
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
            if (st == 0) mfma_first(s0, k_frag(0), q[0]);
            else mfma_next(s0, k_frag(st), q[st]);
        }
        asm volatile("s_nop 15\n\ts_nop 7" : "+v"(s0));
    }
    key_to = kKeyTile;
#pragma unroll
    for (int i = 0; i < 4; ++i) key_at[i] = k_at[i] + kKeyTile;
    // Tiles 0 .. tiles: the last adds the values of the last but one.
#pragma unroll 1
    for (int t = 0; t <= tiles; t += 2) {
        tile(t, s0, s1);
        if (t + 1 <= tiles) tile(t + 1, s1, s0);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing is on its way to LDS when the workgroup ends

    const int row = first + col;
    l = halves_sum(l);
    if (row < nq) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const long at = (long)(q0 + row) * a.H + h;
#pragma unroll
        for (int d = 0; d < kDv / 32; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<u32x2 *>(a.o + at * kDv + 32 * d + 8 * i + 4 * half) =
                    u32x2{pack_bf16x2(o[d][4 * i] * inv, o[d][4 * i + 1] * inv),
                          pack_bf16x2(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv)};
        if (a.lse && half == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) / kLog2e;
    }
    if (!odd_tiles || row >= nq) return;
    for (int n = 0; n < 64; ++n) {  // the lane's own elements, as above
        const int el = n / 16 * 32 + n % 16 / 4 * 8 + 4 * half + n % 4;
        float c = 0.f;
        for (int e = 0; e < kEdge; ++e) {
            if (!(odd_tiles >> e & 1)) continue;
            const int at = (edge + e) * kKeys;
            for (int j = 0; j < min(limit(row) - at, kKeys); ++j) {
                const uint16_t v = a.v[h * a.v_head + (long)(k0 + at + j) * a.v_stride + el];
                if (!not_finite(v)) continue;
                const uint32_t some = lds.t.some[e][wave * kWave + j / 4 % 2 * 32 + col] >> (j / 8 * 4 + j % 4) & 1;
                c = fmaf(some ? 1.f : 0.f, bf16_bits_to_f32(v), c);
            }
        }
        if (c == 0.f) continue;
        uint16_t *to = a.o + ((long)(q0 + row) * a.H + h) * kDv + el;
        *to = f32_to_bf16_bits(bf16_bits_to_f32(*to) + c);
    }
}

}  // namespace

hipError_t launch_latent_prompt(const PromptArgs &a, hipStream_t stream)
{
    const int blocks = (a.max_tokens + kRows - 1) / kRows, pairs = (a.B * a.H + 7) / 8;
    prompt_kernel<<<(unsigned)(8 * pairs * blocks), kThreads, 0, stream>>>(a, blocks);
    return hipGetLastError();
}

}  // namespace ecospec
