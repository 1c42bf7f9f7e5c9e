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
#include "attn_plan.hpp"

namespace ecospec {
namespace {

constexpr int kR = 512, kW = 576;
constexpr int kRows = 128, kKeys = 32;
constexpr int kRowBytes = kW * 2, kChunks = kRowBytes / 16;  // 72 chunks of 16 bytes
constexpr int kTile = kKeys * kRowBytes;                     // 36864
constexpr int kSteps = kW / 16;
constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kAhead = 4, kRing = 3;  // operands of a group of score products; groups in registers, running or being read
constexpr float kSlack = 8.f;  // powers of two by which weights may outgrow their reference before sums are scaled down

typedef __attribute__((ext_vector_type(4))) short s16x4;

__device__ __forceinline__ u32x2 read_tr(const char *p)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
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

struct Lds {
    char tile[3][kTile];
    u32x4 p[2][4][2][kWave];  // weights: tile parity, row tile of 32, reduction step of 16 keys, lane
    float down[2][kRows];     // what the sums of a row are multiplied by before the tile is added
    int scaled[2][kWaves];    // whether that is anything but 1 for a row tile
    float2 ml[kRows];
};

__global__ __launch_bounds__(kThreads, 1) void latent_attn_kernel(LatentArgs a, Shape shape, Parts parts)
{
    __shared__ __attribute__((aligned(16))) Lds lds;
    Item it;
    if (!plan_item(a, a.H, 1, shape, parts, reinterpret_cast<int *>(lds.tile), it)) return;
    __syncthreads();
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), col = lane % 32, half = lane / 32;
    const int row0 = it.group * kRows, n_rows = it.n_tok * a.H;
    const int *table = a.block_table + (long)it.b * a.max_blocks;
    const int lp = 31 - __builtin_clz(a.page);
    const int cached = (it.len + kKeys - 1) / kKeys, drafts = min(it.n_tok, kMaxDrafts);

    // ---- tiles: wavefront w brings rows 8 w .. 8 w + 7, nine loads of 64 chunks; they lie in one page.
    const int row8 = 8 * wave;
    uint32_t src[9];  // lane's byte offset from the first row
#pragma unroll
    for (int n = 0; n < 9; ++n) {
        const int i = n * 64 + lane, r = i / kChunks, c = i % kChunks;
        src[n] = (uint32_t)(r * kRowBytes + (c ^ r) * 16);
    }
    // The page of the rows of tile t, unclamped: read a tile ahead, through a vector register, because a scalar load
    // would make every wait for LDS wait for it too.
    auto page_id = [&](int t) {
        int block = max(min(t * kKeys + row8, it.len - 1), 0) >> lp;
        asm volatile("" : "+v"(block));
        return table[block];
    };
    auto load = [&](int t, int id, int buf) {
        id = __builtin_amdgcn_readfirstlane(min(max(id, 0), a.n_pages - 1));
        int key, rows;
        const uint16_t *base;
        if (t < cached) {
            key = min(t * kKeys + row8, it.len - 1);
            rows = min(it.len - key, 8);
            base = a.pages + ((long)id * a.page + (key & (a.page - 1))) * kW;
        } else {
            key = min((t - cached) * kKeys + row8, drafts - 1);
            rows = min(drafts - key, 8);
            base = a.kv_new + (long)(it.t0 + key) * kW;
        }
        const u32x4 rsrc = rsrc_words(base, (uint32_t)(rows * kRowBytes));
        const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_addr(lds.tile[buf]) + row8 * kRowBytes);
#pragma unroll
        for (int n = 0; n < 9; ++n) load16_lds(rsrc, src[n], dst + n * 1024);  // rows past the end: zeros
    };

    int next_id = it.first < cached ? page_id(it.first) : 0;
#pragma unroll 1
    for (int t = it.first; t < min(it.first + 2, it.last); ++t) {
        load(t, next_id, t - it.first);
        if (t + 1 < cached) next_id = page_id(t + 1);
    }

    // ---- queries of the wavefront's 32 rows
    bf16x8 q[kSteps];
    {
        const int r = row0 + 32 * wave + col;
        const bool in = r < n_rows;
        const int tok = in ? r / a.H : 0;
        const uint16_t *p = a.q + ((long)(it.t0 + tok) * a.H + (in ? r % a.H : 0)) * kW + 8 * half;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[s] = *reinterpret_cast<const bf16x8 *>(p + 16 * s);
    }

    f32x16 o[4][4];  // row tile, element tile
#pragma unroll
    for (int rt = 0; rt < 4; ++rt)
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[rt][d][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    int not_finite_drafts = 0;  // bit: draft tile
    const float scale2 = a.scale * kLog2e;

    // Lane offsets of the LDS reads: keys, by the step's low bits; values, by the element tile's low bit.
    uint32_t k_at[4], v_at[2];
#pragma unroll
    for (int s = 0; s < 4; ++s) k_at[s] = (uint32_t)(col * kRowBytes + ((2 * s + half) ^ (col & 7)) * 16);
    {
        const int i = lane % 16, key = 4 * half + i / 4;
#pragma unroll
        for (int d = 0; d < 2; ++d)
            v_at[d] = (uint32_t)(key * kRowBytes + ((((4 * d + lane / 16 % 2 * 2 + i % 4 / 2) ^ key) + 16 * wave) * 16) + i % 2 * 8);
    }

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
    // Weights of the scores x of tile t, the running maximum and sum, and what the sums so far are scaled by; no branch,
    // so that it can run between the products of values().
    auto weights = [&](int t, float *x) {
        const int par = (t - it.first) & 1;
        float top = x[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
        top = halves_max(top);
        int move = __any(top > m + kSlack);
        asm("" : "+v"(move));  // a select, not a branch
        const float now = move ? fmaxf(m, top) : m, base = now == -INFINITY ? 0.f : now;
        const float down = __builtin_amdgcn_exp2f((m == -INFINITY ? base : m) - base);
        const int scaled = move & __any(m != -INFINITY);
        m = now;
        lds.down[par][32 * wave + col] = down;
        lds.scaled[par][wave] = scaled;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[i] = __builtin_amdgcn_exp2f(x[i] - base);
            sum += x[i];
        }
        l = fmaf(l, down, sum);
        lds.p[par][wave][0][lane] = __builtin_bit_cast(u32x4, pack_bf16x8(x));
        lds.p[par][wave][1][lane] = __builtin_bit_cast(u32x4, pack_bf16x8(x + 8));
    };
    // Before tile t's values are added.
    auto rescale = [&](int t) {
        const int par = (t - it.first) & 1;
#pragma unroll
        for (int rt = 0; rt < 4; ++rt)
            if (__builtin_amdgcn_readfirstlane(lds.scaled[par][rt])) {
                const float down = lds.down[par][32 * rt + col];
#pragma unroll
                for (int d = 0; d < 4; ++d) acc_scale(o[rt][d], down);
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
    auto values = [&](int t) {
        const int par = (t - it.first) & 1;
        const char *tile = lds.tile[(t - it.first) % 3];
        bf16x8 w[2][4], v[2];
        auto fetch_w = [&](int st) {
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) w[st][rt] = __builtin_bit_cast(bf16x8, lds.p[par][rt][st][lane]);
        };
        auto fetch_v = [&](int g) {
            const char *p = tile + v_at[g % 2] + g % 4 / 2 * 128 + g / 4 * 16 * kRowBytes;
            const u32x2 lo = read_tr(p), hi = read_tr(p + 8 * kRowBytes);
            v[g % 2] = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
        };
        fetch_w(0);
        fetch_v(0);
        fetch_v(1);
        fetch_w(1);
#pragma unroll
        for (int g = 0; g < 8; ++g) {
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) o[rt][g % 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[g % 2], w[g / 4][rt], o[rt][g % 4], 0, 0, 0);
            if (g + 2 < 8) fetch_v(g + 2);
        }
    };
    // Order of the instructions of values() and weights() in one block: operands two groups of products ahead, and the
    // softmax in the time that the products take.
    auto interleave = [] {
        __builtin_amdgcn_sched_group_barrier(0x100, 12, 0);
#pragma unroll
        for (int g = 0; g < 8; ++g) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
    };
    // The loads so far have landed, and every wavefront is past the tile before.
    auto step = [] {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };

    step();
    float x[16];
    scores(it.first, x);
    weights(it.first, x);
    step();
    for (int t = it.first + 1; t < it.last; ++t) {
        if (t + 1 < it.last) {
            load(t + 1, next_id, (t + 1 - it.first) % 3);
            if (t + 2 < cached) next_id = page_id(t + 2);
        }
        scores(t, x);
        rescale(t - 1);
        values(t - 1);
        weights(t, x);
        interleave();
        step();
    }
    rescale(it.last - 1);
    values(it.last - 1);

    l = halves_sum(l);
    if (half == 0) lds.ml[32 * wave + col] = make_float2(l == 0.f ? -INFINITY : m, l);
    __syncthreads();
    const bool part = it.chunks > 1;
    float *part_o = parts.o + (long)it.slot * kRows * kR;
    if (part) {
        f32x4 *out = reinterpret_cast<f32x4 *>(part_o);
#pragma unroll
        for (int rt = 0; rt < 4; ++rt)
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    out[(rt * 16 + 4 * wave + d) * 256 + i * 64 + lane] =
                        f32x4{o[rt][d][4 * i], o[rt][d][4 * i + 1], o[rt][d][4 * i + 2], o[rt][d][4 * i + 3]};
        if (threadIdx.x < kRows) parts.ml[(long)it.slot * kRows + threadIdx.x] = lds.ml[threadIdx.x];
    } else {
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
            const int r = row0 + 32 * rt + col;
            if (r >= n_rows) continue;
            const long at = (long)it.t0 * a.H + r;
            const float2 ml = lds.ml[32 * rt + col];
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
            const u32x4 &p = lds.p[(cached + t - it.first) & 1][row / 32][k / 16][k / 4 % 2 * 32 + row % 32];
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

}  // namespace

size_t latent_workspace(int N, int B, int H) { return parts_at(nullptr, group_bound(N, B, H, 1, kRows), kCus, kRows, kR, nullptr); }

hipError_t launch_latent_attn(const LatentArgs &a, void *workspace, hipStream_t stream)
{
    const long groups = group_bound(a.N, a.B, a.H, 1, kRows);
    Parts parts;
    parts_at(workspace, groups, kCus, kRows, kR, &parts);
    latent_attn_kernel<<<(unsigned)grid_bound(groups, kCus), kThreads, 0, stream>>>(a, Shape{kRows, kKeys, 2, kCus}, parts);
    join_kernel<kRows, kR><<<(unsigned)(groups * (kRows / 32) * (kR / 32)), 256, 0, stream>>>(a, a.H, parts);
    return hipGetLastError();
}

}  // namespace ecospec
