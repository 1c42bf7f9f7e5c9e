// Latent attention of draft tokens, absorbed form: T * H query rows of a sequence over the same rows of 576 elements.
//
// 2 * (576 + 512) operations a row and key against 1152 bytes a key: with all 128 heads of a layer even one token is at
// the balance of the matrix cores and HBM, and more tokens are bound by the matrix cores.  A workgroup is one per compute
// unit: 128 rows, four wavefronts with the whole register file.
//   Scores: transposed (S^T = K Q^T, a lane holds one row), wavefront w having rows 32 w .. with their queries in 144
//   registers; every wavefront reads the tile's keys from LDS.
//   Values: wavefront w has elements 128 w .. of all 128 rows, in 256 accumulator registers, so each value is read from
//   LDS once; the weights P pass between the wavefronts through LDS as the product's operand (bf16, 8 KiB a tile).
//   The values' operand V^T is the key rows read with the transposing LDS load.
// Tiles of 32 keys go from memory straight to LDS (three buffers: the tile of the value product, the next one's scores,
// one in flight), chunks of 16 bytes XORed with the row's low bits so that neither kind of read meets a bank twice.  With
// one wavefront on a SIMD nothing else hides the softmax: it runs between the value products of the tile before.  One
// barrier a tile.
//   P is rounded to bf16, the type of the value product's operands; its sum keeps fp32.  A weight is off by at most 2^-9 of
// itself, which takes the error of o against 64 bits from 1.7e-3 (its own rounding to bf16) to 1.8e-3, and to 1.95e-3 for the
// 48 tokens below (root mean square); weights in two parts would double the value products.
//   Measured: trees of 4 to 16 tokens of 8 sequences over 6000 to 20000 tokens, 128 heads, 375 us with the join (867
// TFLOP/s; a large library product reaches 1250) and 359 back to back; 48 single tokens over 1300 to 6000 tokens 97 us (94),
// 16 of them the join of 67 MB of parts; one token of 16 heads over 4097 tokens 18 us, the fixed cost of two launches.
// Matrix cores are busy for 47% of the former's cycles; wavefronts wait for 35% of theirs, because a tile's loads go out
// behind the value products of a step and are waited for at its end.
#include "attn_plan.hpp"

namespace ecospec {
namespace {

constexpr int kR = 512, kW = 576;
constexpr int kRows = 128, kKeys = 32;  // at most
constexpr int kRowBytes = kW * 2, kChunks = kRowBytes / 16;  // 72 chunks of 16 bytes
constexpr int kTile = kKeys * kRowBytes;                     // 36864
constexpr int kSteps = kW / 16;
constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kAhead = 4, kRing = 2;  // operands of a group of score products; groups in registers, running or being read
constexpr int kLoadEvery = 2;
constexpr float kSlack = 8.f;  // powers of two by which weights may outgrow their reference before sums are scaled down

typedef __attribute__((ext_vector_type(4))) short s16x4;

// LDS has 64 banks and reads 256 bytes a cycle.  Chunk c of row r lies at place c ^ twist(r) of its row: rows are 72 chunks,
// so that two rows with the same place are half the banks apart, and the twist keeps 16 consecutive rows' chunks c (a
// quarter of a read of keys) and 4 rows' four neighbouring chunks (half a read of values) in different banks.
__device__ __forceinline__ uint32_t twist(uint32_t r) { return (r >> 1 & 1) << 2 | (r >> 2 & 3); }

__device__ __forceinline__ u32x2 read_tr(const char *p)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
}

// The score products, with their sums in vector registers (the accumulation registers are full): the compiler would give
// them accumulation registers.  Written out, they carry their own waits: a register written by the vector unit needs two
// wait states before a product reads it, a product's result 19 before the vector unit does.
__device__ __forceinline__ void mfma_first(f32x16 &s, const bf16x8 &a, const bf16x8 &b)
{
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(a), "v"(b));
}

__device__ __forceinline__ void mfma_next(f32x16 &s, const bf16x8 &a, const bf16x8 &b)
{
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(a), "v"(b));
}

__device__ __forceinline__ void mfma_wait(f32x16 &s) { asm volatile("s_nop 15\n\ts_nop 7" : "+v"(s)); }

__device__ __forceinline__ bool not_finite(uint32_t bf16) { return (bf16 & 0x7f80u) == 0x7f80u; }

struct Weights {
    u32x4 p[2][4][2][kWave];  // tile parity, row tile of 32, reduction step of 16 keys, lane
    float down[2][kRows];     // what the sums of a row are multiplied by before the tile is added
    int scaled[2][4];         // whether that is anything but 1 for a row tile
    float2 ml[kRows];
};

union Lds {
    char rows[4][kTile];  // the queries of each wavefront, before the loop
    struct {
        char tile[3][kTile];
        Weights w;
    };
};

// RT: row tiles of 32 rows that the workgroup has, wavefront w scoring tile w (fewer than four where a call has few rows).
template <int RT>
__global__ __launch_bounds__(kThreads, 1) void latent_attn_kernel(LatentArgs a, Shape shape, Parts parts)
{
    constexpr int kRows = 32 * RT;
    __shared__ __attribute__((aligned(16))) Lds lds;
    Item it;
    if (!plan_item(a, a.H, 1, shape, parts, it)) return;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), col = lane % 32, half = lane / 32;
    const int row0 = it.group * kRows, n_rows = it.n_tok * a.H;
    const int *table = a.block_table + (long)it.b * a.max_blocks;
    const int lp = 31 - __builtin_clz(a.page);
    const int cached = (it.len + kKeys - 1) / kKeys, drafts = min(it.n_tok, kMaxDrafts);
    const bool scoring = RT == 4 || wave < RT;

    // ---- rows to LDS: nine loads of 64 chunks bring eight rows.  Wavefront w brings rows 8 w .. 8 w + 7 of a tile, which
    // lie in one page.  Rows past the end become zeros.
    const int row8 = 8 * wave;
    uint32_t src[9];  // lane's byte offset from the first row
#pragma unroll
    for (int n = 0; n < 9; ++n) {
        const int i = n * 64 + lane, r = i / kChunks, c = i % kChunks;
        src[n] = (uint32_t)(r * kRowBytes + (c ^ twist(r + row8)) * 16);
    }
    // The page of the rows of tile t, unclamped: read a tile ahead, through a vector register, because a scalar load
    // would make every wait for LDS wait for it too.
    auto page_id = [&](int t) {
        int block = max(min(t * kKeys + row8, it.len - 1), 0) >> lp;
        asm volatile("" : "+v"(block));
        return table[block];
    };
    u32x4 rsrc;
    uint32_t dst;
    auto aim = [&](int t, int id) {  // the loads of tile t; past the chunk they bring nothing but zeros
        int key, rows;
        const uint16_t *base;
        if (t >= it.last) {
            rows = 0;
            base = a.q;
        } else if (t < cached) {
            id = __builtin_amdgcn_readfirstlane(min(max(id, 0), a.n_pages - 1));
            key = min(t * kKeys + row8, it.len - 1);
            rows = min(it.len - key, 8);
            base = a.pages + ((long)id * a.page + (key & (a.page - 1))) * kW;
        } else {
            key = min((t - cached) * kKeys + row8, drafts - 1);
            rows = min(drafts - key, 8);
            base = a.kv_new + (long)(it.t0 + key) * kW;
        }
        rsrc = rsrc_words(base, (uint32_t)(rows * kRowBytes));
        dst = __builtin_amdgcn_readfirstlane(lds_addr(lds.tile[(t - it.first) % 3]) + row8 * kRowBytes);
    };
    auto load = [&](int n) { load16_lds(rsrc, src[n], dst + n * 1024); };

    // Lane offsets of the LDS reads: keys (and queries), by the step's low bits; values, by the element tile's low bit.
    uint32_t k_at[4], v_at[2];
#pragma unroll
    for (int s = 0; s < 4; ++s) k_at[s] = (uint32_t)(col * kRowBytes + ((2 * s + half) ^ twist(col)) * 16);
    {
        const int i = lane % 16, key = 4 * half + i / 4;
#pragma unroll
        for (int d = 0; d < 2; ++d)
            v_at[d] = (uint32_t)(key * kRowBytes + (((4 * d + lane / 16 % 2 * 2 + i % 4 / 2) ^ twist(key)) + 16 * wave) * 16 + i % 2 * 8);
    }

    // ---- queries of the wavefront's 32 rows, consecutive in memory, through LDS
    int next_id = it.first < cached ? page_id(it.first) : 0;
    bf16x8 q[kSteps];
    if (scoring) {
        const int r = row0 + 32 * wave, rows = max(min(n_rows - r, 32), 0);
        const u32x4 from = rsrc_words(a.q + ((long)it.t0 * a.H + min(r, n_rows - 1)) * kW, (uint32_t)(rows * kRowBytes));
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds_addr(lds.rows[wave]));
#pragma unroll 1
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int n = 0; n < 9; ++n)  // src is for the wavefront's rows of a tile: twist(r + 8) again
                load16_lds(from, (src[n] ^ ((e ^ wave) & 1) * 32) + e * 8 * kRowBytes, to + e * 8 * kRowBytes + n * 1024);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[s] = *reinterpret_cast<const bf16x8 *>(lds.rows[wave] + k_at[s % 4] + s / 4 * 128);
    }
    __syncthreads();
    auto aim_next = [&](int t) {
        aim(t, next_id);
        if (t + 1 < cached) next_id = page_id(t + 1);
    };
    aim_next(it.first);
#pragma unroll
    for (int n = 0; n < 9; ++n) load(n);

    f32x16 o[RT][4];  // row tile, element tile
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[rt][d][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    int not_finite_drafts = 0;  // bit: draft tile
    const float scale2 = a.scale * kLog2e;
    Weights &ws = lds.w;

    // Scores of tile t, in powers of two; register i is key 8 (i / 4) + 4 half + i % 4.
    auto scores = [&](int t, float *x) {
        const char *tile = lds.tile[(t - it.first) % 3];
        bf16x8 k[kRing][kAhead];
        auto fetch = [&](int g) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int st = g * kAhead + i;
                k[g % kRing][i] = *reinterpret_cast<const bf16x8 *>(tile + k_at[st % 4] + st / 4 * 128);
            }
        };
        constexpr int kGroups = kSteps / kAhead;
#pragma unroll
        for (int g = 0; g < kRing - 1; ++g) fetch(g);
        f32x16 s;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            if (g + kRing - 1 < kGroups) fetch(g + kRing - 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (g == 0 && i == 0) mfma_first(s, k[0][0], q[0]);
                else mfma_next(s, k[g % kRing][i], q[g * kAhead + i]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        mfma_wait(s);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = s[i] * scale2;
        if (t >= cached) {
            const int r = row0 + 32 * wave + col;
            uint64_t see = 0;
            if (r < n_rows) see = (a.mask ? a.mask[it.t0 + r / a.H] : bits_below(r / a.H + 1)) & bits_below(drafts);
            const uint32_t bits = (uint32_t)(see >> (t - cached) * kKeys) >> 4 * half;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (!(bits >> (i / 4 * 8 + i % 4) & 1)) x[i] = -INFINITY;
        } else if ((t + 1) * kKeys > it.len) {
            const int left = it.len - t * kKeys - 4 * half;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i / 4 * 8 + i % 4 >= left) x[i] = -INFINITY;
        }
    };
    // Weights of the scores x of tile t, the running maximum and sum, and what the sums so far are scaled by: 32 pieces
    // without a branch, to run one behind each value product.
    float top, base, down, sum;
    auto weights = [&](int t, float *x, int piece) {
        const int par = (t - it.first) & 1;
        if (piece == 0) top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), x[6]));
        if (piece == 1) top = fmaxf(top, fmaxf(fmaxf(fmaxf(x[7], x[8]), fmaxf(x[9], x[10])), fmaxf(x[11], x[12])));
        if (piece == 2) top = halves_max(fmaxf(top, fmaxf(fmaxf(x[13], x[14]), x[15])));
        if (piece == 3) {
            int move = __any(top > m + kSlack);
            const int scaled = move & __any(m != -INFINITY);
            asm("" : "+v"(move));  // a select, not a branch
            const float now = move ? fmaxf(m, top) : m;
            base = now == -INFINITY ? 0.f : now;
            down = (m == -INFINITY ? base : m) - base;
            m = now;
            ws.scaled[par][wave] = scaled;
        }
        if (piece == 4) {
            down = __builtin_amdgcn_exp2f(down);
            ws.down[par][32 * wave + col] = down;
            sum = 0.f;
        }
        if (piece >= 5 && piece < 21) {
            const int i = piece - 5;
            x[i] = __builtin_amdgcn_exp2f(x[i] - base);
            sum += x[i];
        }
        if (piece == 21) ws.p[par][wave][0][lane] = __builtin_bit_cast(u32x4, pack_bf16x8(x));
        if (piece == 22) ws.p[par][wave][1][lane] = __builtin_bit_cast(u32x4, pack_bf16x8(x + 8));
        if (piece == 23) l = fmaf(l, down, sum);
    };
    // Whether the sums have to be scaled before tile t's values are added: read early.
    auto flags = [&](int t) { return *reinterpret_cast<const u32x4 *>(ws.scaled[(t - it.first) & 1]); };
    auto rescale = [&](int t, u32x4 scaled) {
        const int par = (t - it.first) & 1;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
            if (__builtin_amdgcn_readfirstlane(scaled[rt])) {
                const float f = ws.down[par][32 * rt + col];
#pragma unroll
                for (int d = 0; d < 4; ++d) acc_scale(o[rt][d], f);
            }
        if (t >= cached) {
            // A weight of zero must not meet an infinity or NaN: where a draft has one, zeros take its place, and what it
            // gives the rows that see it is added at the end.
            u32x4 *all = reinterpret_cast<u32x4 *>(lds.tile[(t - it.first) % 3]);
            bool odd = false;
            for (int i = threadIdx.x; i < kTile / 16; i += kThreads) {
                u32x4 v = all[i];
                bool some = false;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const bool lo = not_finite(v[w]), hi = not_finite(v[w] >> 16);
                    v[w] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
                    some |= lo || hi;
                }
                if (some) all[i] = v;
                odd |= some;
            }
            if (__syncthreads_or(odd)) not_finite_drafts |= 1 << (t - cached);
        }
    };
    // Adds tile t's values; `between(c)` runs behind product c of 8 * RT.
    auto values = [&](int t, auto between) {
        const int par = (t - it.first) & 1;
        const char *tile = lds.tile[(t - it.first) % 3];
        bf16x8 w[2][RT], v[2];
        auto fetch_w = [&](int st) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) w[st][rt] = __builtin_bit_cast(bf16x8, ws.p[par][rt][st][lane]);
        };
        auto fetch_v = [&](int g) {
            const char *p = tile + g % 4 / 2 * 128 + g / 4 * 16 * kRowBytes;
            const u32x2 lo = read_tr(p + v_at[g % 2]), hi = read_tr(p + (v_at[g % 2] ^ 32) + 8 * kRowBytes);  // twist(r + 8)
            v[g % 2] = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
        };
        fetch_w(0);
        fetch_v(0);
        fetch_v(1);
#pragma unroll
        for (int g = 0; g < 8; ++g) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                __builtin_amdgcn_sched_barrier(0);
                o[rt][g % 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[g % 2], w[g / 4][rt], o[rt][g % 4], 0, 0, 0);
                between(g * RT + rt);
            }
            if (g == 2) fetch_w(1);
            if (g + 2 < 8) fetch_v(g + 2);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // The loads so far have landed, and every wavefront is past the tile before.
    auto step = [] {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    auto all_weights = [&](int t, float *x) {
#pragma unroll
        for (int c = 0; c < 24; ++c) weights(t, x, c);
    };

    step();
    float x[16];
    if (scoring) {
        scores(it.first, x);
        all_weights(it.first, x);
    }
    aim_next(it.first + 1);
#pragma unroll
    for (int n = 0; n < 9; ++n) load(n);
    step();
    for (int t = it.first + 1; t < it.last; ++t) {
        aim_next(t + 1);
        const u32x4 scaled = flags(t - 1);
        if (scoring) scores(t, x);
        rescale(t - 1, scaled);
        // The next tile's loads go out between the value products, which leave LDS time for them.
        if (RT == 4) {
            values(t - 1, [&](int c) {
                if (c % kLoadEvery == 0 && c / kLoadEvery < 9) load(c / kLoadEvery);
                weights(t, x, c);
            });
        } else {
#pragma unroll
            for (int n = 0; n < 9; ++n) load(n);
            if (scoring) all_weights(t, x);
            values(t - 1, [](int) {});
        }
        step();
    }
    rescale(it.last - 1, flags(it.last - 1));
    values(it.last - 1, [](int) {});

    l = halves_sum(l);
    if (scoring && half == 0) ws.ml[32 * wave + col] = make_float2(l == 0.f ? -INFINITY : m, l);
    __syncthreads();
    const bool part = it.chunks > 1;
    float *part_o = parts.o + (long)it.slot * kRows * kR;
    if (part) {
        f32x4 *out = reinterpret_cast<f32x4 *>(part_o);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    out[(rt * 16 + 4 * wave + d) * 256 + i * 64 + lane] =
                        f32x4{o[rt][d][4 * i], o[rt][d][4 * i + 1], o[rt][d][4 * i + 2], o[rt][d][4 * i + 3]};
        if (threadIdx.x < kRows) parts.ml[(long)it.slot * kRows + threadIdx.x] = ws.ml[threadIdx.x];
    } else {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int r = row0 + 32 * rt + col;
            if (r >= n_rows) continue;
            const long at = (long)it.t0 * a.H + r;
            const float2 ml = ws.ml[32 * rt + col];
            const float inv = ml.y == 0.f ? 0.f : 1.f / ml.y;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<u32x2 *>(a.o + at * kR + 128 * wave + 32 * d + 8 * i + 4 * half) =
                        u32x2{pack_bf16x2(o[rt][d][4 * i] * inv, o[rt][d][4 * i + 1] * inv),
                              pack_bf16x2(o[rt][d][4 * i + 2] * inv, o[rt][d][4 * i + 3] * inv)};
            if (a.lse && wave == 0 && half == 0) a.lse[at] = ml.y == 0.f ? -INFINITY : (ml.x + __builtin_amdgcn_logf(ml.y)) / kLog2e;
        }
    }
    if (!not_finite_drafts) return;
    // What the infinities and NaN of drafts give the rows that see them, added to what was just written; the weights of the
    // draft tiles still lie in LDS.
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * kR; i += kThreads) {
        const int row = i / kR, el = i % kR, r = row0 + row;
        if (r >= n_rows) break;
        const uint64_t sees = (a.mask ? a.mask[it.t0 + r / a.H] : bits_below(r / a.H + 1)) & bits_below(drafts);
        float c = 0.f;
        for (int j = 0; j < drafts; ++j) {
            const int t = j / kKeys, k = j % kKeys;
            const uint16_t v = a.kv_new[(long)(it.t0 + j) * kW + el];
            if (!(not_finite_drafts >> t & 1) || !(sees >> j & 1) || !not_finite(v)) continue;
            const u32x4 &p = ws.p[(cached + t - it.first) & 1][row / 32][k / 16][k / 4 % 2 * 32 + row % 32];
            c = fmaf(bf16_bits_to_f32(reinterpret_cast<const uint16_t *>(&p)[k / 8 % 2 * 4 + k % 4]), bf16_bits_to_f32(v), c);
        }
        if (c == 0.f) continue;
        if (part) {
            part_o[((row / 32 * 16 + el / 32) * 256 + el % 32 / 8 * 64 + el / 4 % 2 * 32 + row % 32) * 4 + el % 4] += c;
        } else {
            uint16_t *p = a.o + ((long)it.t0 * a.H + r) * kR + el;
            *p = f32_to_bf16_bits(bf16_bits_to_f32(*p) + c);
        }
    }
}

// Row tiles of a workgroup: as few as hold the rows of an average sequence (of those that can have tokens at all).  Tiles
// without rows cost their products (32 tokens of 16 heads over up to 9000: 56 us with one tile, 88 with four); more
// workgroups for the same rows read the keys again (64 sequences of up to four such tokens: 106 us with two tiles, 137 with
// one, 140 with four; 48 tokens of 128 heads: 94 with four, 114 with two, 220 with one).
int row_tiles(int N, int B, int H)
{
    const long rows = (long)N * H, sequences = N < B ? N : B;
    return rows <= 32 * sequences ? 1 : rows <= 64 * sequences ? 2 : 4;
}

// Shortest chunk, in tiles: longer ones leave compute units idle (one token over 2047: 22 us, 24 with 4 and
// 28 with 8; over 8191 they are alike).
constexpr int kShort = 2;

// Two rounds of chunks (and a grid for them) are considered from chunks of kLong tiles on; whether a call can have them is
// known from the block table's width.
constexpr int kLong = 64;

bool may_be_long(long groups, int max_blocks, int page)
{
    return (double)groups * max_blocks * page >= (double)kLong * kKeys * kCus;
}

template <int RT>
hipError_t launch(const LatentArgs &a, void *workspace, hipStream_t stream)
{
    constexpr int kRows = 32 * RT;
    const long groups = group_bound(a.N, a.B, a.H, 1, kRows);
    Parts parts;
    const bool twice = may_be_long(groups, a.max_blocks, a.page);
    parts_at(workspace, groups, kCus, twice, kRows, kR, &parts);
    latent_attn_kernel<RT><<<(unsigned)grid_bound(groups, kCus, twice), kThreads, 0, stream>>>(
        a, Shape{kRows, kKeys, kShort, kCus, twice ? kLong : 0}, parts);
    launch_join<kRows, kR>(a, a.H, parts, groups, stream);
    return hipGetLastError();
}

}  // namespace

// Enough for every call of at most N tokens and B sequences: of all the row tiles that such a call can have, from those of
// a token a sequence to those of one sequence with all tokens; each one's need grows with N and B.
size_t latent_workspace(int N, int B, int H, int max_blocks, int page)
{
    size_t most = 0;
    for (int rt = row_tiles(1, 1, H); rt <= row_tiles(N < kMaxDrafts ? N : kMaxDrafts, 1, H); rt *= 2) {
        const long groups = group_bound(N, B, H, 1, 32 * rt);
        const size_t need = parts_at(nullptr, groups, kCus, may_be_long(groups, max_blocks, page), 32 * rt, kR, nullptr);
        most = need > most ? need : most;
    }
    return most;
}

hipError_t launch_latent_attn(const LatentArgs &a, void *workspace, hipStream_t stream)
{
    switch (row_tiles(a.N, a.B, a.H)) {
    case 1: return launch<1>(a, workspace, stream);
    case 2: return launch<2>(a, workspace, stream);
    default: return launch<4>(a, workspace, stream);
    }
}

}  // namespace ecospec
