// Attention of whole prompts with grouped heads: causal, sequences of different lengths side by side.
//
// The query rows of a sequence that read the same keys are its tokens times the heads of one key/value head, token by
// token: a workgroup takes 128 consecutive ones, 32 of each of four wavefronts.  So short sequences fill its rows too, and
// long ones have blocks keys that only some of the rows see.
//   One pass over the keys, in tiles of 32, with a running reference maximum and sum of weights for each row.  Scores are
//   transposed (S^T = K Q^T): a lane holds one row, its scores are the value product's operand as they stand
//   (O^T = V^T P^T), and V^T is read with the transposing LDS load.
//   Keys and values go from memory straight to LDS, a step (KT tiles) ahead, in panels: of 64 elements for keys (rows of 128
//   bytes, chunks of 16 XORed with row bits, so that 16 rows' chunks, a quarter of a read, lie in different banks), of 32 for
//   values (rows of 64 bytes: half a read is 256 in a row).  One barrier a step.
//   Products, maximum, exponentials and sums of a tile follow each other in a wavefront; what overlaps them is the other
//   wavefronts of its SIMD, of other workgroups, so registers are kept for four of them with heads of 64 and three with 128.
//   The weights are rounded to bf16 for the value product, as the matrix instruction takes them (their sum and the log-sum keep
//   fp32): outputs are 2.2e-3 of their size off, where fp32 weights and the rounding of the output leave 1.6e-3; two products, of
//   a weight and of what its rounding leaves, would be half as many again.
//   Where there are few row blocks, or sequences of keys far more than queries, each block's keys are cut into chunks, a
//   workgroup each, whose sums join_prompt_kernel adds up in order.
//   Measured: one prompt of 6007 tokens, 64 heads on 4 of 128, 524 to 538 us, up to 1.13 PFLOP/s (a bf16 product of 8192^3:
//   1.415): the matrix cores are busy 60% of the cycles and the vector unit issues in half of them, at 1.8 GHz, which the
//   power leaves (operands of zeros run at 2.2); six prompts of 706 to 1201 tokens, 64 heads on 8 of 64, 84 us: the vector
//   unit (five instructions a weight, half the products of a head of 128 to hide them), and wavefronts that end unevenly; 7
//   tokens over 4008 keys, 64 heads on 4 of 128, 14 us and 4.0 of the join: a chain of offsets, cuts, queries, first tile,
//   six tiles at 1.2 us (a lone wavefront's latency), parts; loads two and three steps ahead, or two and four tiles a step,
//   did not shorten it. With two wavefronts a SIMD, each with three tiles under way at once and a piece of the exponentials
//   behind each product (176 and 248 registers), the first two took 575 and 100 us; with 64 rows a wavefront, one a SIMD,
//   half the LDS reads, 580 and 143: one wavefront issues an instruction every seven cycles at best.
#include "attn_plan.hpp"
#include "step.hpp"

namespace ecospec {
namespace {

constexpr int kKeys = 32, kWaves = 4, kThreads = kWaves * kWave, kRows = 32 * kWaves;
// Most workgroups of a call whose keys are cut: all that registers leave room for, if chunks are long; else two a compute unit.
template <int D>
constexpr int kSlots = (D == 64 ? 4 : 3) * kCus;
constexpr int kFewSlots = 2 * kCus;
constexpr int kMinTiles = 6, kLongTiles = 32;  // of a chunk
constexpr int kJoinWaves = 8, kTogether = 4;   // most wavefronts of a joining workgroup; chunks that one takes together
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

// A number that is the same in all lanes, in a scalar register.
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }

// A sequence: its queries and keys.
struct Sequence {
    int q0, nq, k0, nk;
};

__device__ __forceinline__ Sequence sequence(const GroupedPromptArgs &a, int b)
{
    Sequence s;
    s.q0 = min(max(a.q_offsets[b], 0), a.N);
    s.nq = min(max(a.q_offsets[b + 1], s.q0), a.N) - s.q0;
    s.k0 = min(max(a.kv_offsets[b], 0), a.M);
    s.nk = min(max(a.kv_offsets[b + 1], s.k0), a.M) - s.k0;
    return s;
}

// That of a lane, or of the first one.
__device__ __forceinline__ Sequence uniform(const Sequence &s, int lane = 0)
{
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, lane); };
    return Sequence{of(s.q0), of(s.nq), of(s.k0), of(s.nk)};
}

// A workgroup's row block: its sequence and key/value head, and what its rows see.
struct Block : Sequence {
    int hk, rows, row0, tiles, G;

    __device__ __forceinline__ int limit(int row) const { return min(max(row / G + 1 + nk - nq, 0), nk); }  // keys of a query row

    __device__ __forceinline__ Block(const GroupedPromptArgs &a, const Sequence &s, int hk, int block) : Sequence(s), hk(hk)
    {
        G = a.H / a.Hkv;
        rows = nq * G;
        row0 = block * kRows;
        tiles = row0 < rows ? (limit(min(row0 + kRows, rows) - 1) + kKeys - 1) / kKeys : 0;
    }
};

__device__ __forceinline__ int wave_total(int v) { return __builtin_amdgcn_readlane(wave_inclusive_sum(v), kWave - 1); }

// How the keys of a call are cut: into chunks of about equal length, which follows from the lengths of all sequences, which only
// the device knows.  Every wavefront works it out for itself, a lane to a sequence; all members are uniform.
template <int D>
struct Cuts {
    struct Size {
        int blocks, tiles, chunks;  // row blocks of a head; tiles of the longest, and its chunks
    };
    const GroupedPromptArgs &a;
    int blocks;      // of a sequence, at most
    int length = 1;  // tiles of a chunk, at most
    Sequence mine;   // the lane's of the first 64

    __device__ __forceinline__ Sequence of(int b) const
    {
        return b < kWave ? mine : b < a.B ? sequence(a, b) : Sequence{0, 0, 0, 0};
    }

    __device__ __forceinline__ Size size(const Sequence &s) const
    {
        const int t = (s.nk + kKeys - 1) / kKeys;
        return Size{min((s.nq * (a.H / a.Hkv) + kRows - 1) / kRows, blocks), t, max((t + length - 1) / length, 1)};
    }

    // Places of a sequence's chunks among the parts, if it is cut.
    __device__ __forceinline__ int slots(const Size &s) const { return s.chunks > 1 ? s.blocks * a.Hkv * s.chunks : 0; }

    __device__ __forceinline__ Cuts(const GroupedPromptArgs &a, int blocks) : a(a), blocks(blocks)
    {
        const int lane = lane_id();
        mine = lane < a.B ? sequence(a, lane) : Sequence{0, 0, 0, 0};
        float work = 0.f;
        for (int b = lane; b < a.B + lane; b += kWave) {
            const Sequence q = of(b);
            const Size s = size(q);
            // A row block sees half of its sequence's queries' keys less than the last one, on average.
            work += (float)(s.blocks * a.Hkv) * max((float)s.tiles - (float)q.nq / (2 * kKeys), 1.f);
        }
        work = wave_sum(work);
        // Chunks that fill the card, if they are long beside their sums (64 heads on 8 of 64, 20000 keys behind: 200 tokens 94
        // us, by two workgroups a compute unit 104), else few (64 on 4 of 128, 20000 behind: 16 tokens 30 us, by three 34).
        const float n = work >= (float)kLongTiles * kSlots<D> ? kSlots<D> : kFewSlots;
        length = __builtin_amdgcn_readfirstlane(max((int)ceilf(work / n), kMinTiles));
        for (;; length += length / 8 + 1) {
            int sum = 0;
            for (int b = lane; b < a.B + lane; b += kWave) sum += slots(size(of(b)));
            if (wave_total(sum) <= kSlots<D>) break;
        }
    }

    // Sequence, head, row block and chunk of a workgroup, and the place of the row block's first chunk; false: nothing to do.
    __device__ __forceinline__ bool find(int item, int &b, Sequence &seq, int &hk, int &block, int &chunk, int &slot) const
    {
        slot = 0;
        for (int b0 = 0; b0 < a.B; b0 += kWave) {
            const Sequence q = of(b0 + lane_id());
            const Size s = size(q);
            const int items = s.blocks * a.Hkv * s.chunks, upto = wave_inclusive_sum(items), places = wave_inclusive_sum(slots(s));
            const uint64_t past = __ballot(upto > item);
            if (past) {
                const int l = (int)__builtin_ctzll(past), n = __builtin_amdgcn_readlane(s.blocks, l);
                const int chunks = __builtin_amdgcn_readlane(s.chunks, l);
                item -= __builtin_amdgcn_readlane(upto - items, l);
                b = b0 + l;
                seq = uniform(q, l);
                hk = item % a.Hkv;
                // The longest row blocks first.
                block = n - 1 - item / a.Hkv / chunks;
                chunk = item / a.Hkv % chunks;
                slot += __builtin_amdgcn_readlane(places - slots(s), l) + (hk * n + block) * chunks;
                return true;
            }
            item -= __builtin_amdgcn_readlane(upto, kWave - 1);
            slot += __builtin_amdgcn_readlane(places, kWave - 1);
        }
        return false;
    }
};

// Wavefronts that join so many chunks: a block's own, as far as the launch has them.  (Those, and the chunks' length, follow
// from all of a call's sequences: the same call gives the same sums, another batch may order a sequence's differently.)
__host__ __device__ inline int join_waves(int chunks) { return min((chunks + kTogether - 1) / kTogether, kJoinWaves); }

// Sums of a chunk: for each row the reference maximum and the weights' sum, and the output sums in accumulator order.
struct PromptParts {
    float2 *ml;  // [slot][kRows]
    float *o;    // [slot][wavefront][D / 8][lane][4]
    int2 *cut;   // [sequence and head][row block]: the first chunk's slot, and how many
};

typedef __attribute__((ext_vector_type(2))) float f32x2;

__device__ __forceinline__ uint32_t to_bf16x2(float lo, float hi)  // one conversion
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// D: width of a head; KT: key tiles a barrier; SPLIT: keys are cut into chunks.
template <int D, int KT, bool SPLIT>
__global__ __launch_bounds__(kThreads, D == 64 ? 4 : 3) void prompt_kernel(GroupedPromptArgs a, int blocks,
                                                                           PromptParts parts)
{
    constexpr int kSteps = D / 16, kPanels = D / 64, kTiles = D / 32;
    constexpr int kTile = kKeys * D * 2;         // bytes of a tile
    constexpr int kEdge = kRows / kKeys + 1;                    // most tiles that some rows of a workgroup see in part
    constexpr int kRing = 4;                                    // operands of a product in registers
    struct Tiles {
        char k[2][KT][kTile];  // panel, row r, chunk c of 16 bytes at place c ^ (r >> 1 & 7)
        char v[2][KT][kTile];  // panel of 32 elements, row
        uint16_t some[kEdge][kThreads];  // which weights of a lane are not zero, in a tile with infinities or NaN
    };
    __shared__ __attribute__((aligned(16))) Tiles lds;

    int b, hk, block, chunk = 0, slot = 0, chunks = 1;
    int length = 0;
    Sequence seq;
    if (SPLIT) {
        const Cuts<D> cuts(a, blocks);
        if (!cuts.find(blockIdx.x, b, seq, hk, block, chunk, slot)) return;
        length = cuts.length;
    } else {
        // Workgroups are dealt to the eight XCDs in turn: with pairs innermost a head's row blocks meet on blocks of them.  The
        // longest row blocks first, so that no long one is left for the end.
        const int pairs = a.B * a.Hkv, pair = blockIdx.x % pairs;
        block = blocks - 1 - blockIdx.x / pairs;
        b = pair / a.Hkv;
        hk = pair % a.Hkv;
        seq = uniform(sequence(a, b));
    }
    const Block blk(a, seq, hk, block);
    if (blk.row0 >= blk.rows) return;
    if (SPLIT) {
        chunks = max((blk.tiles + length - 1) / length, 1);
        if (chunk >= chunks) return;
        if (chunk == 0 && threadIdx.x == 0) parts.cut[(b * a.Hkv + hk) * blocks + block] = int2{slot, chunks};
        slot += chunk;
    }
    // From here on keys and tiles are counted from the chunk's first.
    const int from = SPLIT ? (int)((long)blk.tiles * chunk / chunks) : 0;
    const int tiles = SPLIT ? (int)((long)blk.tiles * (chunk + 1) / chunks) - from : blk.tiles;
    auto limit = [&](int row) { return min(max(blk.limit(row) - from * kKeys, 0), tiles * kKeys); };
    const int k0 = blk.k0 + from * kKeys, nk = min(blk.nk - from * kKeys, tiles * kKeys), rows = blk.rows, G = blk.G;

    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), col = lane % 32, half = lane / 32;
    const int edge = limit(blk.row0) / kKeys;  // first tile that some row of the workgroup does not see to its end
    const int first = blk.row0 + 32 * wave;
    const int all_see = __builtin_amdgcn_readfirstlane(limit(min(first, rows - 1)));  // keys that all rows of the wavefront see

    // ---- queries
    const int my_row = min(first + col, rows - 1), token = my_row / G, mine = limit(my_row);
    bf16x8 q[kSteps];
    {
        const uint16_t *src = a.q + (long)(blk.q0 + token) * a.q_stride + (blk.hk * G + my_row - token * G) * a.q_head + half * 8;
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
            u32x4 w = *reinterpret_cast<const u32x4 *>(src + st * 16);
            // The scale is positive from here on: the largest product is the largest score.
            if (a.scale < 0.f) w ^= 0x80008000u;
            q[st] = __builtin_bit_cast(bf16x8, w);
        }
    }

    // ---- loads: wavefront w brings rows 8 w .. 8 w + 7 of each panel of a tile's keys, and 16 rows of panels of its values a
    // load.  Rows past the last key, and tiles past the last, become zeros.
    const uint16_t *src_k = a.k + blk.hk * a.k_head + k0 * a.k_stride, *src_v = a.v + blk.hk * a.v_head + k0 * a.v_stride;
    const uint32_t stride_k = (uint32_t)a.k_stride * 2, stride_v = (uint32_t)a.v_stride * 2;
    const int e = 8 * wave + lane / 8, place = (lane % 8) ^ (e >> 1 & 7);
    const int v_panel = D == 128 ? wave : wave / 2, v_row = D == 128 ? 0 : wave % 2 * 16;
    const uint32_t off_k = e * stride_k + place * 16, off_v = (v_row + lane / 4) * stride_v + v_panel * 64 + lane % 4 * 16;
    const uint32_t next_k = kKeys * stride_k, next_v = kKeys * stride_v, low = 16 * stride_v;
    const uint32_t ring_k = __builtin_amdgcn_readfirstlane(lds_addr(lds.k) + wave * 1024);
    const uint32_t ring_v = __builtin_amdgcn_readfirstlane(lds_addr(lds.v) + v_panel * 2048 + v_row * 64);
    int left = nk;  // keys from the step to load next on
    auto load_step = [&](int buffer) {
        const int n = max(min(left, KT * kKeys), 0);
        const u32x4 ks = rsrc_words(src_k, n ? (uint32_t)(n - 1) * stride_k + D * 2 : 0);
        const u32x4 vs = rsrc_words(src_v, n ? (uint32_t)(n - 1) * stride_v + D * 2 : 0);
        const uint32_t to_k = ring_k + buffer * KT * kTile, to_v = ring_v + buffer * KT * kTile;
#pragma unroll
        for (int i = 0; i < KT; ++i) {
#pragma unroll
            for (int p = 0; p < kPanels; ++p) load16_lds(ks, off_k + i * next_k + p * 128, to_k + i * kTile + p * (kKeys * 128));
            load16_lds(vs, off_v + i * next_v, to_v + i * kTile);
            if (D == 128) load16_lds(vs, off_v + i * next_v + low, to_v + i * kTile + 1024);
        }
        left -= KT * kKeys;
        if (left > 0) {
            src_k += KT * kKeys / 2 * stride_k;
            src_v += KT * kKeys / 2 * stride_v;
        }
    };
    load_step(0);

    f32x16 o[kTiles];
    float m = -INFINITY, bound = -INFINITY, l = 0.f, base = 0.f;
#pragma unroll
    for (int d = 0; d < kTiles; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    uint32_t odd_tiles = 0;  // edge tiles with infinities or NaN among the values
    const float scale2 = uniform(fmaxf(fabsf(a.scale) * kLog2e, 0x1p-126f));  // not zero: it meets infinities
    const float slack = uniform(kSlack / scale2);
    uint32_t k_at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) k_at[i] = (uint32_t)(col * 128 + ((2 * i + half) ^ (col >> 1 & 7)) * 16);
    const int i16 = lane % 16;
    const uint32_t v_at = (uint32_t)((4 * half + i16 / 4) * 64 + lane / 16 % 2 * 32 + i16 % 4 * 8);

    // Tile t, its keys and values at kt and vt in LDS.  Register i of the scores is key 8 (i / 4) + 4 half + i % 4.
    auto tile = [&](int t, const char *kt, const char *vt) {
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
        {
            bf16x8 ring[kRing];
            auto key = [&](int st) {
                ring[st % kRing] = *reinterpret_cast<const bf16x8 *>(kt + k_at[st % 4] + st / 4 * (kKeys * 128));
            };
#pragma unroll
            for (int st = 0; st < kRing - 1; ++st) key(st);
#pragma unroll
            for (int st = 0; st < kSteps; ++st) {
                if (st + kRing - 1 < kSteps) key(st + kRing - 1);
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[st % kRing], q[st], s, 0, 0, 0);
            }
        }
        bf16x8 ring[kRing];
        auto value = [&](int n) {
            const char *w = vt + v_at + n % kTiles * (kKeys * 64) + n / kTiles * 16 * 64;
            const u32x2 lo = read_tr(w), hi = read_tr(w + 8 * 64);
            ring[n % kRing] = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
        };
#pragma unroll
        for (int n = 0; n < kRing - 1; ++n) value(n);
        asm volatile("s_nop 15\n\ts_nop 3" : "+v"(s));  // from a product to instructions written out
        if ((t + 1) * kKeys > all_see) {
            const int seen = mine - t * kKeys - 4 * half;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i / 4 * 8 + i % 4 >= seen) s[i] = -INFINITY;
        }
        const float top = max3(max3(max3(max3(s[0], s[1], s[2]), max3(s[3], s[4], s[5]), s[6]), max3(s[7], s[8], s[9]), s[10]),
                               max3(s[11], s[12], s[13]), max2(s[14], s[15]));
        if (__builtin_expect(__any(top > bound), 0)) {
            // A new reference maximum for each row.
            const float now = fmaxf(m, halves_max(top) * scale2);
            base = now == -INFINITY ? 0.f : now;
            const float down = __builtin_amdgcn_exp2f((m == -INFINITY ? base : m) - base);
            l *= down;
#pragma unroll
            for (int d = 0; d < kTiles; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= down;
            m = now;
            bound = now == -INFINITY ? now : now / scale2 + slack;
        }
        float sum = 0.f;
        u32x4 p[2];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale2, -base));
            s[i + 1] = __builtin_amdgcn_exp2f(fmaf(s[i + 1], scale2, -base));
            sum = i ? sum + s[i] : s[i];
            sum += s[i + 1];
            p[i / 8][i % 8 / 2] = to_bf16x2(s[i], s[i + 1]);
        }
        l += sum;
        if (t >= edge && odd_tiles >> (t - edge) & 1) {  // a step's bits come before its first tile, which may be before `edge`
            uint32_t set = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float w = s[i];
                asm volatile("" : "+v"(w));  // here, not ahead of the branch in every tile
                set |= (w != 0.f ? 1u : 0u) << i;
            }
            lds.some[t - edge][threadIdx.x] = (uint16_t)set;
        }
#pragma unroll
        for (int n = 0; n < 2 * kTiles; ++n) {
            if (n + kRing - 1 < 2 * kTiles) value(n + kRing - 1);
            const bf16x8 weights = __builtin_bit_cast(bf16x8, p[n / kTiles]);
            o[n % kTiles] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[n % kRing], weights, o[n % kTiles], 0, 0, 0);
        }
    };
    // Tiles t .. t + KT - 1, in this buffer.
    auto step = [&](int t, int buffer) {
        // They have landed, and every wavefront is past the step before, whose buffer the next one's loads take.
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        load_step(buffer ^ 1);
#pragma unroll 1
        for (int u = max(t, edge); u < min(t + KT, tiles); ++u) {
            // A weight of zero must not meet an infinity or NaN: where a tile that not all rows see to its end has one,
            // zeros take its place, and what it gives the rows that see it is added at the end.
            u32x4 *all = reinterpret_cast<u32x4 *>(lds.v[buffer][u - t]);
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
#pragma unroll
        for (int i = 0; i < KT; ++i)
            if (KT == 1 || t + i < tiles) tile(t + i, lds.k[buffer][i], lds.v[buffer][i]);
    };
    if (SPLIT) {
        // Few steps, whose first costs its instructions' way to the compute unit: one copy of them (4 to 8 tiles a workgroup, a
        // call of 18.5 to 21.9 us becomes 18.1 to 21.2; in long runs two copies are 3% faster).
#pragma unroll 1
        for (int t = 0, buffer = 0; t < tiles; t += KT, buffer ^= 1) step(t, buffer);
    } else {
#pragma unroll 1
        for (int t = 0; t < tiles; t += 2 * KT) {
            step(t, 0);
            if (t + KT >= tiles) break;
            step(t + KT, 1);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing is on its way to LDS when the workgroup ends

    const int row = first + col;
    l = halves_sum(l);
    const bool whole = !SPLIT || chunks == 1;
    const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
    if (row >= rows) return;
    const long at = (long)(blk.q0 + row / G) * a.H + blk.hk * G + row % G;
#pragma unroll
    for (int d = 0; d < kTiles; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4 x = {o[d][4 * i] * inv, o[d][4 * i + 1] * inv, o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv};
            if (whole)
                *reinterpret_cast<u32x2 *>(a.o + at * D + 32 * d + 8 * i + 4 * half) =
                    u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
            else
                reinterpret_cast<f32x4 *>(parts.o)[((((long)slot * kWaves + wave) * kTiles + d) * 4 + i) * kWave + lane] = x;
        }
    if (odd_tiles) {
        for (int n = 0; n < D / 2; ++n) {  // the lane's own elements, as above
            const int el = n / 16 * 32 + n % 16 / 4 * 8 + 4 * half + n % 4;
            float c = 0.f;
            for (int b = 0; b < kEdge; ++b) {
                if (!(odd_tiles >> b & 1)) continue;
                const int begin = (edge + b) * kKeys;
                for (int j = 0; j < min(mine - begin, kKeys); ++j) {
                    const uint16_t w = a.v[blk.hk * a.v_head + (long)(k0 + begin + j) * a.v_stride + el];
                    if (!not_finite(w)) continue;
                    const uint32_t is = lds.some[b][wave * kWave + j / 4 % 2 * 32 + col] >> (j / 8 * 4 + j % 4) & 1;
                    c = fmaf(is ? 1.f : 0.f, bf16_bits_to_f32(w), c);
                }
            }
            if (c == 0.f) continue;
            if (whole) {
                uint16_t *to = a.o + at * D + el;
                *to = f32_to_bf16_bits(bf16_bits_to_f32(*to) + c);
            } else {
                parts.o[(((((long)slot * kWaves + wave) * kTiles + n / 16) * 4 + n % 16 / 4) * kWave + lane) * 4 + n % 4] += c;
            }
        }
    }
    if (half) return;
    if (!whole) parts.ml[slot * kRows + wave * 32 + col] = float2{m, l};
    else if (a.lse) a.lse[at] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) / kLog2e;
}

// Adds up the chunks of a row block: a workgroup has 32 rows by 8 elements, what registers 4 i .. 4 i + 3 of one element tile
// of the accumulators hold; its wavefronts, one for each four chunks and at most eight, take chunks in turn, four together, in
// one pass with a running reference maximum.  What bounds it: latency (offsets, one read for 32 chunks, barrier).  7 tokens over
// 4008 keys, 21 chunks, 5.5 MB: 4.0 us (31 chunks 4.1, with the references read first, behind a barrier of their own, 6.4).
// The whole call for 3 tokens over 30003 keys, 8 heads on one, 234 chunks, takes 17 us (by four wavefronts 3 more; eight chunks
// together, or 16 wavefronts, are no better here and 5 us worse for 50 tokens over 20050 keys, 64 heads on 4).  Eight wavefronts
// where two chunks are joined cost 15 us of 42, for 29 prompts of up to 364 tokens, two heads.
template <int D>
__global__ __launch_bounds__(kJoinWaves *kWave) void join_prompt_kernel(GroupedPromptArgs a, int blocks, PromptParts parts)
{
    constexpr int kGroups = D / 32 * 4;
    __shared__ f32x4 sums[kJoinWaves - 1][kWave];
    __shared__ float2 totals[kJoinWaves - 1][kWave];
    const int group = blockIdx.x % kGroups, of = blockIdx.x / kGroups % kWaves, pb = blockIdx.x / (kGroups * kWaves);
    const int pair = pb / blocks, b = pair / a.Hkv, hk = pair % a.Hkv, block = pb % blocks;
    const Block blk(a, uniform(sequence(a, b)), hk, block);
    if (blk.row0 + of * 32 >= blk.rows) return;
    const int2 cut = parts.cut[pb];
    const int chunks = cut.y, lane = lane_id(), wave = threadIdx.x / kWave;
    const int row = blk.row0 + of * 32 + lane % 32;
    // One chunk: it is written already.  (The bounds: offsets that decrease, which no call may have, can leave a block without.)
    if (chunks < 2 || (uint32_t)cut.x >= kSlots<D> || chunks > kSlots<D> - cut.x) return;
    const int waves = min(join_waves(chunks), (int)blockDim.x / kWave);  // the others have nothing to do
    const long slot = cut.x;
    const float2 *ml = parts.ml + slot * kRows + of * 32 + lane % 32;
    const f32x4 *o = reinterpret_cast<const f32x4 *>(parts.o) + ((slot * kWaves + of) * kGroups + group) * kWave + lane;
    constexpr long kStep = kWaves * kGroups * kWave;
    float top = -INFINITY, base = 0.f, total = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    auto reach = [&](float to) {  // a reference maximum of at least `to`
        const float now = fmaxf(top, to), next = now == -INFINITY ? 0.f : now;
        const float down = __builtin_amdgcn_exp2f((top == -INFINITY ? next : top) - next);
        total *= down;
#pragma unroll
        for (int n = 0; n < 4; ++n) sum[n] *= down;
        top = now;
        base = next;
    };
    auto add = [&](float m, float l, const f32x4 &v) {
        const float f = __builtin_amdgcn_exp2f(m - base);
        total = fmaf(l, f, total);
#pragma unroll
        for (int n = 0; n < 4; ++n) sum[n] = fmaf(v[n], f, sum[n]);
    };
#pragma unroll 1
    for (int c0 = wave; wave < waves && c0 < chunks; c0 += kTogether * waves) {
        float2 part[kTogether];
        f32x4 v[kTogether];
#pragma unroll
        for (int i = 0; i < kTogether; ++i) {
            const int c = min(c0 + i * waves, chunks - 1);
            part[i] = ml[c * kRows];
            v[i] = o[c * kStep];
        }
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < kTogether; ++i) {
            if (c0 + i * waves >= chunks) {  // the last one again
                part[i] = float2{-INFINITY, 0.f};
                v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            most = fmaxf(most, part[i].x);
        }
        reach(most);
#pragma unroll
        for (int i = 0; i < kTogether; ++i) add(part[i].x, part[i].y, v[i]);
    }
    if (wave) {
        sums[wave - 1][lane] = sum;
        totals[wave - 1][lane] = float2{top, total};
    }
    __syncthreads();
    if (wave || row >= blk.rows) return;
    float most = -INFINITY;
    for (int w = 0; w < waves - 1; ++w) most = fmaxf(most, totals[w][lane].x);
    reach(most);
    for (int w = 0; w < waves - 1; ++w) add(totals[w][lane].x, totals[w][lane].y, sums[w][lane]);
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const long at = (long)(blk.q0 + row / blk.G) * a.H + blk.hk * blk.G + row % blk.G;
    *reinterpret_cast<u32x2 *>(a.o + at * D + 8 * group + lane / 32 * 4) =
        u32x2{pack_bf16x2(sum[0] * inv, sum[1] * inv), pack_bf16x2(sum[2] * inv, sum[3] * inv)};
    if (a.lse && group == 0 && lane < 32) a.lse[at] = total == 0.f ? -INFINITY : (base + __builtin_amdgcn_logf(total)) / kLog2e;
}

// Two tiles a barrier where LDS has room for all the wavefronts that registers allow (heads of 64: 85 us with one, 83 with two;
// heads of 128: two would leave two workgroups a compute unit, 560 us instead of 535).
template <int D>
constexpr int kTilesAStep = D == 64 ? 2 : 1;

template <int D>
hipError_t launch(const GroupedPromptArgs &a, void *workspace, hipStream_t stream)
{
    const long rows = (long)a.max_tokens * (a.H / a.Hkv);
    const int pairs = a.B * a.Hkv, blocks = (int)((rows + kRows - 1) / kRows);
    char *w = static_cast<char *>(workspace);
    PromptParts parts;
    parts.ml = reinterpret_cast<float2 *>(w);
    parts.o = reinterpret_cast<float *>(parts.ml + kSlots<D> * kRows);
    parts.cut = reinterpret_cast<int2 *>(parts.o + (size_t)kSlots<D> * kRows * D);
    const long groups = (long)pairs * blocks, tiles = a.M / ((long)a.B * kKeys);  // of the average sequence
    constexpr int KT = kTilesAStep<D>;
    // Cut where there are few row blocks; or not so many, and keys behind that are more than the queries: of several sequences,
    // which may differ much, the longest would take all the time.  (24 of up to 66 tokens, half of them behind up to 9176 keys,
    // 32 heads on 2 of 128: 76 us, uncut 222.)  Not where keys are few: 30 of up to 246 tokens, 4 heads on 2 of 128, take 13.9
    // us, cut 19.3.
    const bool few = tiles >= kLongTiles * (kSlots<D> / groups) ? kSlots<D> / groups > 1 : kFewSlots / groups > 1;
    const bool ragged = a.B > 1 && groups <= kSlots<D> && a.M >= 2L * a.N;
    if (tiles >= 8 && (few || ragged)) {
        // Workgroups for every chunk that the device may make: row blocks that are not cut, and parts.
        const long heads = (long)a.Hkv * blocks, most = heads * ((a.M / kKeys + a.B) / kMinTiles + 1 + a.B);
        const int grid = (int)min(groups + kSlots<D>, most), spread = (int)((a.B > 1 ? 2 : 1) * kSlots<D> / groups) + 1;
        prompt_kernel<D, KT, true><<<(unsigned)grid, kThreads, 0, stream>>>(a, blocks, parts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        join_prompt_kernel<D><<<(unsigned)(groups * kWaves * (D / 8)), join_waves(spread) * kWave, 0, stream>>>(a, blocks, parts);
        return hipGetLastError();
    }
    prompt_kernel<D, KT, false><<<(unsigned)groups, kThreads, 0, stream>>>(a, blocks, parts);
    return hipGetLastError();
}

}  // namespace

size_t grouped_prompt_workspace(int D)
{
    return (size_t)(D == 64 ? kSlots<64> : kSlots<128>) * (kRows * (sizeof(float2) + D * sizeof(float)) + sizeof(int2));
}

hipError_t launch_grouped_prompt(const GroupedPromptArgs &a, int D, void *workspace, hipStream_t stream)
{
    return D == 64 ? launch<64>(a, workspace, stream) : launch<128>(a, workspace, stream);
}

}  // namespace ecospec
