// Attention of whole prompts with grouped heads: causal, sequences of different lengths side by side.
//
// The query rows of a sequence that read the same keys are its tokens times the heads of one key/value head, token by
// token: a workgroup takes 128 consecutive ones, 32 of each of four wavefronts.  So short sequences fill its rows too, and
// long ones have few keys that only some of the rows see.
//   Scores are transposed (S^T = K Q^T): a lane holds one row, its scores are the value product's operand as they stand
//   (O^T = V^T P^T), and V^T is read with the transposing LDS load.
//   Keys and values go from memory straight to LDS, in panels: of 64 elements for keys (rows of 128 bytes, chunks of 16
//   XORed with row bits, so that 16 rows' chunks, a quarter of a read, lie in different banks), of 32 for values (rows of 64
//   bytes: half a read is 256 in a row).
#include "attn_plan.hpp"
#include "step.hpp"

namespace ecospec {
namespace {

constexpr int kKeys = 32, kPromptWaves = 4, kRows = 32 * kPromptWaves, kPromptThreads = kPromptWaves * kWave;

typedef __attribute__((ext_vector_type(4))) short s16x4;

__device__ __forceinline__ u32x2 read_tr(const char *p)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
}

__device__ __forceinline__ bool not_finite(uint32_t bf16) { return (bf16 & 0x7f80u) == 0x7f80u; }

template <int D>
__global__ __launch_bounds__(kPromptThreads) void prompt_kernel(GroupedPromptArgs a, int blocks)
{
    constexpr int kSteps = D / 16, kTile = kKeys * D * 2, kTiles = D / 32;
    constexpr int kEdge = kRows / kKeys + 1;  // most tiles that some rows of a workgroup see in part
    __shared__ __attribute__((aligned(16))) char lds_k[kTile];  // panel, row r, chunk c of 16 bytes at place c ^ (r >> 1 & 7)
    __shared__ __attribute__((aligned(16))) char lds_v[kTile];  // panel of 32 elements, row
    __shared__ uint16_t some[kEdge][kPromptThreads];  // which weights of a lane are not zero, in a tile with infinities or NaN
    const int G = a.H / a.Hkv, pairs = a.B * a.Hkv;
    const int pair = blockIdx.x / blocks, block = blocks - 1 - blockIdx.x % blocks;
    if (pair >= pairs) return;
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
    const int row = row0 + 32 * wave + col, mine = limit(min(row, rows - 1));
    const long at = (long)(q0 + min(row, rows - 1) / G), head = hk * G + min(row, rows - 1) % G;

    bf16x8 q[kSteps];
#pragma unroll
    for (int st = 0; st < kSteps; ++st)
        q[st] = *reinterpret_cast<const bf16x8 *>(a.q + at * a.q_stride + head * a.q_head + st * 16 + half * 8);

    f32x16 o[kTiles];
#pragma unroll
    for (int d = 0; d < kTiles; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    const float scale2 = a.scale * kLog2e;
    uint32_t odd_tiles = 0;  // edge tiles with infinities or NaN among the values

    const int i16 = lane % 16;
    const uint32_t v_at = (uint32_t)((4 * half + i16 / 4) * 64 + lane / 16 % 2 * 32 + i16 % 4 * 8);
    for (int t = 0; t < tiles; ++t) {
        __syncthreads();
        const int left = min(nk - t * kKeys, kKeys);
        for (int i = threadIdx.x; i < kTile / 16; i += kPromptThreads) {
            const int r = i / (D / 8), c = i % (D / 8);
            const long key = k0 + t * kKeys + r;
            u32x4 kx = {0, 0, 0, 0}, vx = {0, 0, 0, 0};
            if (r < left) {
                kx = *reinterpret_cast<const u32x4 *>(a.k + key * a.k_stride + hk * a.k_head + c * 8);
                vx = *reinterpret_cast<const u32x4 *>(a.v + key * a.v_stride + hk * a.v_head + c * 8);
            }
            *reinterpret_cast<u32x4 *>(lds_k + c / 8 * (kKeys * 128) + r * 128 + ((c % 8) ^ (r >> 1 & 7)) * 16) = kx;
            *reinterpret_cast<u32x4 *>(lds_v + c / 4 * (kKeys * 64) + r * 64 + c % 4 * 16) = vx;
        }
        __syncthreads();
        if (t >= edge) {
            // A weight of zero must not meet an infinity or NaN: where a tile that not all rows see to its end has one,
            // zeros take its place, and what it gives the rows that see it is added at the end.
            u32x4 *all = reinterpret_cast<u32x4 *>(lds_v);
            bool odd = false;
            for (int i = threadIdx.x; i < kTile / 16; i += kPromptThreads) {
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
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
            const bf16x8 k = *reinterpret_cast<const bf16x8 *>(lds_k + st / 4 * (kKeys * 128) + col * 128 + ((st % 4 * 2 + half) ^ (col >> 1 & 7)) * 16);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[st], s, 0, 0, 0);
        }
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i] = t * kKeys + i / 4 * 8 + 4 * half + i % 4 < mine ? s[i] * scale2 : -INFINITY;
            top = fmaxf(top, s[i]);
        }
        top = fmaxf(m, halves_max(top));
        const float base = top == -INFINITY ? 0.f : top, down = __builtin_amdgcn_exp2f((m == -INFINITY ? base : m) - base);
        m = top;
        float p[16], sum = 0.f;
        uint32_t set = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            p[i] = __builtin_amdgcn_exp2f(s[i] - base);
            sum += p[i];
            set |= (p[i] != 0.f ? 1u : 0u) << i;
        }
        l = fmaf(l, down, sum);
        if (t >= edge && odd_tiles >> (t - edge) & 1) some[t - edge][threadIdx.x] = (uint16_t)set;
#pragma unroll
        for (int d = 0; d < kTiles; ++d) {
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= down;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const char *w = lds_v + d * (kKeys * 64) + n * 16 * 64 + v_at;
                const u32x2 lo = read_tr(w), hi = read_tr(w + 8 * 64);
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]}),
                                                               pack_bf16x8(p + 8 * n), o[d], 0, 0, 0);
            }
        }
    }

    l = halves_sum(l);
    if (row >= rows) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const long to = at * a.H + head;
#pragma unroll
    for (int d = 0; d < kTiles; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<u32x2 *>(a.o + to * D + 32 * d + 8 * i + 4 * half) =
                u32x2{pack_bf16x2(o[d][4 * i] * inv, o[d][4 * i + 1] * inv), pack_bf16x2(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv)};
    if (a.lse && half == 0) a.lse[to] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) / kLog2e;
    if (!odd_tiles) return;
    for (int n = 0; n < D / 2; ++n) {  // the lane's own elements, as above
        const int el = n / 16 * 32 + n % 16 / 4 * 8 + 4 * half + n % 4;
        float c = 0.f;
        for (int e = 0; e < kEdge; ++e) {
            if (!(odd_tiles >> e & 1)) continue;
            const int first = (edge + e) * kKeys;
            for (int j = 0; j < min(mine - first, kKeys); ++j) {
                const uint16_t v = a.v[hk * a.v_head + (long)(k0 + first + j) * a.v_stride + el];
                if (!not_finite(v)) continue;
                const uint32_t is = some[e][wave * kWave + j / 4 % 2 * 32 + col] >> (j / 8 * 4 + j % 4) & 1;
                c = fmaf(is ? 1.f : 0.f, bf16_bits_to_f32(v), c);
            }
        }
        if (c == 0.f) continue;
        uint16_t *x = a.o + to * D + el;
        *x = f32_to_bf16_bits(bf16_bits_to_f32(*x) + c);
    }
}

}  // namespace

size_t grouped_prompt_workspace(int D) { return 256; }

hipError_t launch_grouped_prompt(const GroupedPromptArgs &a, int D, void *workspace, hipStream_t stream)
{
    const int blocks = (int)(((long)a.max_tokens * (a.H / a.Hkv) + kRows - 1) / kRows);
    const unsigned grid = (unsigned)(a.B * a.Hkv * blocks);
    if (D == 64) prompt_kernel<64><<<grid, kPromptThreads, 0, stream>>>(a, blocks);
    else prompt_kernel<128><<<grid, kPromptThreads, 0, stream>>>(a, blocks);
    return hipGetLastError();
}

}  // namespace ecospec
