// Grouped-query attention of draft tokens over the 8-bit cache and over each other.
//
// Scores are computed transposed, S^T = K Q^T, so that a lane of the 32 x 32 x 16 product holds one query row and 16 of
// its 32 scores; the other half of the wavefront has the rest.  Row m of the K operand is key pi(m) = 16 ((m >> 2) & 1) +
// 4 (m >> 3) + (m & 3) of the tile, which puts keys 0..15 into the lower half's registers in order and keys 16..31 into
// the upper's: they are the value product's operand P^T (its reduction index is the key) without any move between lanes,
// and its other operand V^T takes 16 consecutive tokens of one element, 16 bytes of the cache as it lies.  So codes go
// from memory to registers and through the conversion to bf16 into the matrix cores; LDS holds only the queries.
//
// Bound by HBM (2 bytes a cached token, head and element) up to some 64 rows a key/value head.  Four wavefronts take the
// tiles of a workgroup's chunk in turn, each with its own running maximum and sums, joined at the end through LDS.
// The weights are rounded to bf16 for the value product, whose operands are of that type; their sum keeps fp32.  A weight is
// off by at most 2^-9 of itself, which takes the error of o against 64 bits from 1.7e-3 (its own rounding to bf16) to 2.2e-3
// and 2.4e-3 (root mean square, both cases below); weights in two parts would double the value products.
//   Measured: trees of up to 8 tokens of 16 sequences over 15000 to 60000 tokens, 64 heads of 64 on 8, 143 and 150 us on two
// cards (4.05 and 3.9 TB/s of cache); four tokens over 16383, 64 heads of 128 on 4, 23 us, most of it the fixed cost of two
// launches and of 456 parts.  Wavefronts are alive for three quarters of the former (chunks of 82 rounds at most, 75 on
// average), and the vector unit (conversions, exponentials and packing) is busy three quarters of that.  64 tokens of one
// sequence over 16383: 64 us with those heads of 128, 39 with those of 64; every 32 (64) rows read and convert the codes.
#include "attn_plan.hpp"

namespace ecospec {
namespace {

constexpr int kKeys = 32;  // of a tile
constexpr int kWaves = 4;
// Powers of two by which a row's weights may outgrow its reference maximum before the sums are scaled down: they are
// fp32, far from overflow, and the bf16 weights' rounding is relative.
constexpr float kSlack = 8.f;

// bf16 operand of eight codes, times the power of two of `scale`: exact.
__device__ __forceinline__ bf16x8 decode(uint32_t w0, uint32_t w1, float scale)
{
    u32x4 o;
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true));
    o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false));
    o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true));
    return __builtin_bit_cast(bf16x8, o);
}

// The score products, written out so that the first needs no sums of zeros; a register written by the vector unit needs
// two wait states before a product reads it.
__device__ __forceinline__ void mfma_first(f32x16 &s, const bf16x8 &k, const bf16x8 &q)
{
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "v"(q));
}

__device__ __forceinline__ void mfma_next(f32x16 &s, const bf16x8 &k, const bf16x8 &q)
{
    asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "v"(q));
}

// RT: row tiles of 32 rows; D: head width.
template <int D, int RT>
__global__ __launch_bounds__(256, 2) void cache_attn_kernel(CacheArgs a, Shape shape, Parts parts)
{
    constexpr int kRows = 32 * RT, kSteps = D / 16, kDt = D / 32;
    constexpr int kQ = RT * kSteps * 64 * 16;                // bytes of the queries, in operand order
    constexpr int kP = kWaves * kRows * kKeys * 2;           // weights of a draft tile, for non-finite drafts
    constexpr int kMerge = 2 * RT * kDt * 4096;              // two wavefronts' sums
    constexpr int kLds = kQ + kP > kMerge ? kQ + kP : kMerge;
    __shared__ __attribute__((aligned(16))) char lds[kLds];
    __shared__ float2 ml[kWaves][kRows];

    const int G = a.H / a.Hkv;
    Item it;
    if (!plan_item(a, G, a.Hkv, shape, parts, it)) return;
    const int kvh = it.group / it.row_tiles, row0 = it.group % it.row_tiles * kRows;
    const int n_rows = it.n_tok * G;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), col = lane % 32, half = lane / 32;

    // Queries: step s, lane (row, half): elements 32 (s / 2) + 16 half + 8 (s % 2) .. + 7, as the codes' 16 bytes give.
    u32x4 *q_lds = reinterpret_cast<u32x4 *>(lds);
    for (int i = threadIdx.x; i < RT * kSteps * 64; i += 256) {
        const int rt = i / (kSteps * 64), s = i / 64 % kSteps, l = i % 64;
        const int r = row0 + rt * 32 + l % 32;
        u32x4 v = {0, 0, 0, 0};
        if (r < n_rows) {
            const long at = (long)(it.t0 + r / G) * a.H + kvh * G + r % G;
            v = *reinterpret_cast<const u32x4 *>(a.q + at * D + 32 * (s / 2) + 16 * (l / 32) + 8 * (s % 2));
            if (a.scale < 0.f) v ^= 0x80008000u;
        }
        q_lds[i] = v;
    }
    __syncthreads();

    f32x16 o[RT][kDt];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -INFINITY;
        l[rt] = 0.f;
#pragma unroll
        for (int d = 0; d < kDt; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[rt][d][i] = 0.f;
    }

    const int pi = (col >> 2 & 1) * 16 + (col >> 3) * 4 + (col & 3);
    const int *table = a.block_table + (long)it.b * a.max_blocks;
    const int lp = 31 - __builtin_clz(a.page);
    const int cached = (it.len + kKeys - 1) / kKeys;  // tiles

    // Running maximum, weights and sums of one row tile's scores x, in powers of two once multiplied by `unit` > 0.  The
    // weights come out times 2^up, and `down_up` = 2^-up keeps that out of their sum.
    auto softmax = [&](int rt, f32x16 &x, float unit, float up, float down_up) {
        float tops[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
            tops[h] = max3(max3(x[8 * h], x[8 * h + 1], x[8 * h + 2]), max3(x[8 * h + 3], x[8 * h + 4], x[8 * h + 5]), x[8 * h + 6]);
        const float top = halves_max(max3(tops[0], tops[1], fmaxf(x[7], x[15])) * unit);
        if (__any(top > m[rt] + kSlack)) {
            const float now = fmaxf(m[rt], top);
            const float down = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[rt] - now);
            m[rt] = now;
            l[rt] *= down;
#pragma unroll
            for (int d = 0; d < kDt; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[rt][d][i] *= down;
        }
        const float base = (m[rt] == -INFINITY ? 0.f : m[rt]) - up;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], unit, -base));
            sum[i % 2] += x[i];
        }
        l[rt] = fmaf(sum[0] + sum[1], down_up, l[rt]);
    };
    // The sums of the score products are read by an instruction that the compiler does not see: 19 wait states after them.
    auto settle = [&](f32x16 (&s)[RT]) {
        if constexpr (RT == 2) asm volatile("s_nop 15\n\ts_nop 3" : "+v"(s[0]), "+v"(s[1]));
        else asm volatile("s_nop 15\n\ts_nop 3" : "+v"(s[0]));
    };

    // ---- cached tokens
    // Positive and not zero: the largest product is the largest score (a negative scale turned the queries' signs), and it
    // meets infinities.
    const float scale2 = fmaxf(fabsf(a.scale) * kLog2e, 0x1p-126f);
    struct Codes {  // of a tile: this lane's operands and scales
        u32x4 k[D / 32], v[kDt];
        float ks, vs;
    } ring[2];
    const long stride = (long)a.page * D;  // of a head's page
    // A tile's codes and scales are read two tiles of the wavefront ahead (one ahead: 2047 tokens 22 us instead of 20, long
    // caches alike), its pages three: this half's 16 keys for the values and the scales, the 16 of key pi for the keys.
    // Through vector registers: a scalar load would make every wait for LDS wait for it too.
    auto page_id = [&](int t, int group) { return table[min((t * kKeys + 16 * group) >> lp, a.max_blocks - 1)]; };
    auto head = [&](int id) { return (long)min(max(id, 0), a.n_pages - 1) * a.Hkv + kvh; };
    auto load_k = [&](Codes &c, int t, int id) {
        const uint8_t *p = a.k + head(id) * stride + ((t * kKeys + pi) & (a.page - 1)) * D + 16 * half;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) c.k[i] = *reinterpret_cast<const u32x4 *>(p + 32 * i);
    };
    auto load_v = [&](Codes &c, int t, int id) {
        const uint8_t *p = a.v + head(id) * stride + ((t * kKeys + 16 * half) & (a.page - 1)) + (long)col * a.page;
#pragma unroll
        for (int d = 0; d < kDt; ++d) c.v[d] = *reinterpret_cast<const u32x4 *>(p + (long)(32 * d) * a.page);
    };
    const int end = min(it.last, cached);
    int t = it.first + wave, k_id = 0, v_id = 0;
    auto load_scales = [&](Codes &c, int id) {
        c.ks = a.k_scale[head(id)];
        c.vs = a.v_scale[head(id)];
    };
    auto load_ids = [&](int t) {
        k_id = page_id(min(t, end - 1), pi >> 4);
        v_id = page_id(min(t, end - 1), half);
    };
    if (t < end) {
        load_ids(t);
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int k_of = k_id, v_of = v_id, at = min(t + n * kWaves, end - 1);
            load_ids(t + (n + 1) * kWaves);
            load_k(ring[n], at, k_of);
            load_v(ring[n], at, v_of);
            load_scales(ring[n], v_of);
        }
    }
    auto tile = [&](int t, Codes &c) {
        const float ks = c.ks * scale2;
        float vs = c.vs;
        const int next = t + 2 * kWaves;
        const int left = it.len - t * kKeys - 16 * half;  // of this half's 16 keys
        f32x16 s[RT];
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
            const bf16x8 k = decode(c.k[st / 2][st % 2 * 2], c.k[st / 2][st % 2 * 2 + 1], 1.f);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const bf16x8 q = __builtin_bit_cast(bf16x8, q_lds[(rt * kSteps + st) * 64 + lane]);
                if (st == 0) mfma_first(s[rt], k, q);
                else mfma_next(s[rt], k, q);
            }
        }
        const bool tail = (t + 1) * kKeys > it.len;
        if (tail) {
            // Past the cache's end lies whatever its pages held: no weight, and zeros for the values.
            if (left <= 0) vs = 0.f;
#pragma unroll
            for (int d = 0; d < kDt; ++d)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int n = left - 4 * w;
                    c.v[d][w] &= n >= 4 ? ~0u : n <= 0 ? 0u : (1u << 8 * n) - 1;
                }
        }
        const int id = v_id;
        if (next < end) {
            load_k(c, next, k_id);
            load_scales(c, id);
            load_ids(next + kWaves);
        }
        settle(s);
        if (tail)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (i >= left) s[rt][i] = -INFINITY;
        // The values' scale, one for a lane's 16 keys: its power of two goes into their conversion, the rest into the
        // exponent of the weights.
        const float rest = __uint_as_float(0x3f800000u | (__float_as_uint(vs) & 0x7fffffu));
        const float up = __builtin_amdgcn_logf(rest), down_up = __builtin_amdgcn_rcpf(rest);
        bf16x8 p[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            softmax(rt, s[rt], fmaxf(ks, 0x1p-126f), up, down_up);
#pragma unroll
            for (int i = 0; i < 16; ++i) p[rt][i / 8][i % 8] = static_cast<__bf16>(s[rt][i]);
        }
#pragma unroll
        for (int d = 0; d < kDt; ++d)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bf16x8 v = decode(c.v[d][2 * h], c.v[d][2 * h + 1], vs);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) o[rt][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[rt][h], o[rt][d], 0, 0, 0);
            }
        if (next < end) load_v(c, next, id);
    };
    for (; t < end; t += 2 * kWaves) {
        tile(t, ring[0]);
        if (t + kWaves < end) tile(t + kWaves, ring[1]);
    }

    // ---- drafts
    const int drafts = min(it.n_tok, kMaxDrafts);
    t = it.first + wave;
    if (t < end) t += (end - t + kWaves - 1) / kWaves * kWaves;
    for (; t < it.last; t += kWaves) {
        const int j0 = (t - cached) * kKeys;
        f32x16 s[RT];
        const uint16_t *kp = a.k_new + ((long)(it.t0 + min(j0 + pi, drafts - 1)) * a.Hkv + kvh) * D + 16 * half;
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
            const bf16x8 k = *reinterpret_cast<const bf16x8 *>(kp + 32 * (st / 2) + 8 * (st % 2));
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const bf16x8 q = __builtin_bit_cast(bf16x8, q_lds[(rt * kSteps + st) * 64 + lane]);
                if (st == 0) mfma_first(s[rt], k, q);
                else mfma_next(s[rt], k, q);
            }
        }
        settle(s);
        // Weights as the products' operand, and in LDS (row, draft) for drafts that are not finite.
        uint16_t *w = reinterpret_cast<uint16_t *>(lds + kQ) + wave * kRows * kKeys;
        bf16x8 p[RT][2];
        uint32_t all[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int r = row0 + rt * 32 + col;
            uint64_t see = 0;
            if (r < n_rows) {
                const int tok = r / G;
                see = (a.mask ? a.mask[it.t0 + tok] : bits_below(tok + 1)) & bits_below(drafts);
            }
            all[rt] = (uint32_t)(see >> j0);
            const uint32_t bits = all[rt] >> 16 * half;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (!(bits >> i & 1)) s[rt][i] = -INFINITY;
            softmax(rt, s[rt], scale2, 0.f, 1.f);
#pragma unroll
            for (int i = 0; i < 16; ++i) p[rt][i / 8][i % 8] = static_cast<__bf16>(s[rt][i]);
#pragma unroll
            for (int h = 0; h < 2; ++h) *reinterpret_cast<bf16x8 *>(w + (rt * 32 + col) * kKeys + 16 * half + 8 * h) = p[rt][h];
        }
        __builtin_amdgcn_wave_barrier();
        const int mine = drafts - j0 - 16 * half;
        const uint16_t *vp = a.v_new + ((long)(it.t0 + j0 + 16 * half) * a.Hkv + kvh) * D + col;
#pragma unroll
        for (int d = 0; d < kDt; ++d) {
            u32x4 vb[2];
            bool odd = false;
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
                const uint32_t lo = j < mine ? vp[(long)j * a.Hkv * D + 32 * d] : 0u;
                const uint32_t hi = j + 1 < mine ? vp[(long)(j + 1) * a.Hkv * D + 32 * d] : 0u;
                odd |= (lo & 0x7f80u) == 0x7f80u || (hi & 0x7f80u) == 0x7f80u;
                vb[j / 8][j % 8 / 2] = lo | hi << 16;
            }
            if (__any(odd)) {
                // A weight of zero must not meet an infinity or NaN: each row adds the drafts that it sees, one by one.
                for (int j = 0; j < min(drafts - j0, kKeys); ++j) {
                    const uint16_t *v = a.v_new + ((long)(it.t0 + j0 + j) * a.Hkv + kvh) * D + 32 * d + 4 * half;
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        const float f = bf16_bits_to_f32(*const_cast<volatile uint16_t *>(w + (rt * 32 + col) * kKeys + j));
                        if (all[rt] >> j & 1)
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[rt][d][i] = fmaf(f, bf16_bits_to_f32(v[i / 4 * 8 + i % 4]), o[rt][d][i]);
                    }
                }
                continue;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    o[rt][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vb[h]), p[rt][h], o[rt][d], 0, 0, 0);
        }
        __builtin_amdgcn_wave_barrier();
    }

    // ---- join the four wavefronts: 2 and 3 onto 0 and 1, then 1 onto 0
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] = halves_sum(l[rt]);
        if (half == 0) ml[wave][rt * 32 + col] = make_float2(m[rt], l[rt]);
    }
    __syncthreads();
    float base[RT], total[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w][rt * 32 + col].x);
        base[rt] = top == -INFINITY ? 0.f : top;
        total[rt] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float2 v = ml[w][rt * 32 + col];
            total[rt] = fmaf(v.y, __builtin_amdgcn_exp2f(v.x - base[rt]), total[rt]);
        }
        const float f = __builtin_amdgcn_exp2f(m[rt] - base[rt]);
#pragma unroll
        for (int d = 0; d < kDt; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[rt][d][i] *= f;
    }
    f32x4 *buf = reinterpret_cast<f32x4 *>(lds);
#pragma unroll
    for (int n = 2; n >= 1; n /= 2) {
        if (wave >= n && wave < 2 * n)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int d = 0; d < kDt; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        buf[(((wave - n) * RT + rt) * kDt + d) * 256 + i * 64 + lane] =
                            f32x4{o[rt][d][4 * i], o[rt][d][4 * i + 1], o[rt][d][4 * i + 2], o[rt][d][4 * i + 3]};
        __syncthreads();
        if (wave < n)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int d = 0; d < kDt; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x4 v = buf[((wave * RT + rt) * kDt + d) * 256 + i * 64 + lane];
#pragma unroll
                        for (int j = 0; j < 4; ++j) o[rt][d][4 * i + j] += v[j];
                    }
        __syncthreads();
    }
    if (wave) return;

    if (it.chunks > 1) {
        f32x4 *out = reinterpret_cast<f32x4 *>(parts.o) + (long)it.slot * RT * kDt * 256;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
            for (int d = 0; d < kDt; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    out[(rt * kDt + d) * 256 + i * 64 + lane] =
                        f32x4{o[rt][d][4 * i], o[rt][d][4 * i + 1], o[rt][d][4 * i + 2], o[rt][d][4 * i + 3]};
            if (half == 0)
                parts.ml[(long)it.slot * kRows + rt * 32 + col] = make_float2(total[rt] == 0.f ? -INFINITY : base[rt], total[rt]);
        }
        return;
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = row0 + rt * 32 + col;
        if (r >= n_rows) continue;
        const long at = (long)(it.t0 + r / G) * a.H + kvh * G + r % G;
        const float inv = total[rt] == 0.f ? 0.f : 1.f / total[rt];
#pragma unroll
        for (int d = 0; d < kDt; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<u32x2 *>(a.o + at * D + 32 * d + 8 * i + 4 * half) =
                    u32x2{pack_bf16x2(o[rt][d][4 * i] * inv, o[rt][d][4 * i + 1] * inv),
                          pack_bf16x2(o[rt][d][4 * i + 2] * inv, o[rt][d][4 * i + 3] * inv)};
        if (a.lse && half == 0) a.lse[at] = total[rt] == 0.f ? -INFINITY : (base[rt] + __builtin_amdgcn_logf(total[rt])) / kLog2e;
    }
}

// Row tiles of a workgroup: two for heads of 64 elements where the average row group has more than 32 rows (37 drafts over
// 130001 tokens: 142 us against 170 us with one); one for heads of 128, whose sums of two leave the loads no registers
// (16 sequences of four drafts over 16383 tokens: 49 us, 58 us with two).  The average is over the sequences that can have
// tokens at all.
int row_tiles(int N, int B, int per_token, int D) { return D == 64 && (long)N * per_token > 32L * (N < B ? N : B) ? 2 : 1; }

// Workgroups at once: two on a compute unit hide each other's waits (trees of 16 sequences: 148 us, with one 203, with three
// 161, all before the codes were read two tiles ahead; one sequence of four tokens: 23, 22 and 29).
constexpr int kSlots = 2 * kCus;

template <int D, int RT>
hipError_t launch(const CacheArgs &a, void *workspace, hipStream_t stream)
{
    const int G = a.H / a.Hkv;
    const long groups = group_bound(a.N, a.B, G, a.Hkv, 32 * RT);
    Parts parts;
    parts_at(workspace, groups, kSlots, false, 32 * RT, D, &parts);
    cache_attn_kernel<D, RT><<<(unsigned)grid_bound(groups, kSlots, false), 256, 0, stream>>>(
        a, Shape{32 * RT, kKeys, kWaves, kSlots, 0}, parts);
    launch_join<32 * RT, D>(a, G, parts, groups, stream);
    return hipGetLastError();
}

}  // namespace

// Enough for every call of at most N tokens and B sequences: of both counts of row tiles where such a call can have either,
// from a token a sequence to one sequence with all tokens; each one's need grows with N and B.
size_t cache_workspace(int N, int B, int H, int Hkv, int D)
{
    const int G = H / Hkv;
    size_t most = 0;
    for (int rt = row_tiles(1, 1, G, D); rt <= row_tiles(N < kMaxDrafts ? N : kMaxDrafts, 1, G, D); ++rt) {
        const size_t need = parts_at(nullptr, group_bound(N, B, G, Hkv, 32 * rt), kSlots, false, 32 * rt, D, nullptr);
        most = need > most ? need : most;
    }
    return most;
}

hipError_t launch_cache_attn(const CacheArgs &a, void *workspace, hipStream_t stream)
{
    if (a.D == 128) return launch<128, 1>(a, workspace, stream);
    return row_tiles(a.N, a.B, a.H / a.Hkv, a.D) == 2 ? launch<64, 2>(a, workspace, stream) : launch<64, 1>(a, workspace, stream);
}

}  // namespace ecospec
