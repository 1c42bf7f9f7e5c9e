// Latent attention of prompts, expanded form: per head 192-element keys (128 of its own, 64 rotary ones that all heads
// share) and 128-element values, causal.
//
// 640 operations a row, key and head against 512 bytes a key and head: bound by the matrix cores.  A workgroup takes 256
// consecutive queries of one head, 32 each of eight wavefronts, two on a SIMD, and tiles of 64 keys from LDS.
//   Scores are transposed (S^T = K Q^T): a lane holds one row, its scores are the value product's operand as they stand
//   (O^T = V^T P^T), and V^T is read with the transposing LDS load.
//   The two wavefronts of a SIMD work in turn: while the first four multiply keys, the other four do the softmax and the
//   value product of the tile before, so that the matrix cores and the vector unit are both in use; a barrier after each
//   half step keeps them apart.
//   Keys and values go from memory straight to LDS, two buffers each, issued two half steps before they are read; chunks
//   of 16 bytes are XORed with row bits so that 16 rows' chunks (a quarter of a read) lie in different banks.
#include "attn_plan.hpp"

namespace ecospec {
namespace {

constexpr int kDn = 128, kP = 64, kDv = 128, kDq = kDn + kP;
constexpr int kKeys = 64;
constexpr int kWaves = 8, kRows = 32 * kWaves, kThreads = 64 * kWaves;
constexpr int kSteps = kDq / 16;
constexpr int kRing = 4;  // steps of score operands in registers
constexpr float kSlack = 8.f;

typedef __attribute__((ext_vector_type(4))) short s16x4;

__device__ __forceinline__ u32x2 read_tr(const char *p)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
}

__device__ __forceinline__ bool not_finite(uint32_t bf16) { return (bf16 & 0x7f80u) == 0x7f80u; }

__device__ __forceinline__ bf16x8 finite(bf16x8 v)
{
    u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] &= (not_finite(w[i]) ? 0u : 0xffffu) | (not_finite(w[i] >> 16) ? 0u : 0xffff0000u);
    return __builtin_bit_cast(bf16x8, w);
}

struct Lds {
    char k[2][kKeys * kDn * 2];     // row r, chunk c of 16 bytes at place c ^ (r & 15)
    char rope[2][kKeys * kP * 2];   // at c ^ (r >> 1 & 7)
    char v[2][kKeys * kDv * 2];     // at c ^ (r & 3) << 2
    uint16_t p[kWaves][2][32][kKeys];  // weights of even and odd tiles with infinities or NaN among the values
};

__global__ __launch_bounds__(kThreads, 2) void prompt_kernel(PromptArgs a, int blocks)
{
    __shared__ __attribute__((aligned(16))) Lds lds;
    // All row blocks of a head on one XCD, one after the other, so that its L2 has the head's keys; long ones first.
    const int pair = blockIdx.x % 8 + 8 * (int)(blockIdx.x / 8 / blocks), block = blocks - 1 - (int)(blockIdx.x / 8) % blocks;
    if (pair >= a.B * a.H) return;
    const int b = pair / a.H, h = pair % a.H;
    const int q0 = min(max(a.q_offsets[b], 0), a.N), nq = min(max(a.q_offsets[b + 1], q0), a.N) - q0;
    const int k0 = min(max(a.kv_offsets[b], 0), a.M), nk = min(max(a.kv_offsets[b + 1], k0), a.M) - k0;
    const int row0 = block * kRows;
    if (row0 >= nq) return;

    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), col = lane % 32, half = lane / 32;
    auto limit = [&](int row) { return min(max(row + 1 + nk - nq, 0), nk); };  // keys that a query sees
    const int tiles = (limit(min(row0 + kRows, nq) - 1) + kKeys - 1) / kKeys;
    const int first = row0 + 32 * wave, row = first + col;
    const int all_see = limit(first), some_see = first < nq ? limit(min(first + 32, nq) - 1) : 0;  // of the wavefront's rows
    const int mine = limit(row);

    // ---- loads: wavefront w brings rows 8 w .. 8 w + 7 of a tile
    uint32_t k_off[2], v_off[2], rope_off;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int r = 8 * wave + 4 * e + lane / 16;
        k_off[e] = (uint32_t)(r * (uint32_t)a.k_stride * 2 + ((lane % 16) ^ (r & 15)) * 16);
        v_off[e] = (uint32_t)(r * (uint32_t)a.v_stride * 2 + ((lane % 16) ^ (r & 3) << 2) * 16);
    }
    {
        const int r = 8 * wave + lane / 8;
        rope_off = (uint32_t)(r * kP * 2 + ((lane % 8) ^ (r >> 1 & 7)) * 16);
    }
    const uint16_t *kh = a.k + h * a.k_head + k0 * a.k_stride, *vh = a.v + h * a.v_head + k0 * a.v_stride;
    const uint16_t *rh = a.k_rope + (long)k0 * kP;
    // Rows past the last key become zeros; tiles past the last bring nothing but zeros.
    auto load_k = [&](int t) {
        const int rows = t < tiles ? min(nk - t * kKeys, kKeys) : 0, at = min(t, tiles - 1) * kKeys;
        const u32x4 r = rsrc_words(kh + at * a.k_stride, rows ? (uint32_t)((rows - 1) * a.k_stride + kDn) * 2 : 0);
        const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_addr(lds.k[t & 1]) + wave * 2048);
        load16_lds(r, k_off[0], dst);
        load16_lds(r, k_off[1], dst + 1024);
        load16_lds(rsrc_words(rh + (long)at * kP, (uint32_t)rows * kP * 2), rope_off,
                   __builtin_amdgcn_readfirstlane(lds_addr(lds.rope[t & 1]) + wave * 1024));
    };
    auto load_v = [&](int t) {
        const int rows = t < tiles ? min(nk - t * kKeys, kKeys) : 0, at = min(t, tiles - 1) * kKeys;
        const u32x4 r = rsrc_words(vh + at * a.v_stride, rows ? (uint32_t)((rows - 1) * a.v_stride + kDv) * 2 : 0);
        const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_addr(lds.v[t & 1]) + wave * 2048);
        load16_lds(r, v_off[0], dst);
        load16_lds(r, v_off[1], dst + 1024);
    };

    bf16x8 q[kSteps];
    {
        const uint16_t *p = a.q + ((long)(q0 + min(row, nq - 1)) * a.H + h) * kDq + 8 * half;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[s] = *reinterpret_cast<const bf16x8 *>(p + 16 * s);
    }
    if (tiles) {
        load_k(0);
        load_v(0);
    }

    f32x16 o[kDv / 32], s[2];
#pragma unroll
    for (int d = 0; d < kDv / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    int not_finite_tiles = 0, last_odd = 0;  // bit: even or odd tile; a wavefront sees at most two tiles in part
    const float scale2 = a.scale * kLog2e;

    const uint32_t k_at = (uint32_t)(col * 256 + (half ^ (col & 15)) * 16), rope_at = (uint32_t)(col * 128 + (half ^ (col >> 1 & 7)) * 16);
    const int i16 = lane % 16;
    const uint32_t v_at = (uint32_t)((4 * half + i16 / 4) * 256 + ((lane / 16 % 2 * 2 + i16 % 4 / 2) ^ (i16 / 4) << 2) * 16 + i16 % 2 * 8);

    auto scores = [&](int t) {
        if (t * kKeys >= some_see) return;
        const char *k = lds.k[t & 1], *rope = lds.rope[t & 1];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
        bf16x8 f[kRing][2];  // operands of a step's two products
        auto fetch = [&](int st) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const char *p = st < 8 ? k + (k_at ^ (st * 32)) + kt * 32 * 256 : rope + (rope_at ^ ((st - 8) * 32)) + kt * 32 * 128;
                f[st % kRing][kt] = *reinterpret_cast<const bf16x8 *>(p);
            }
        };
#pragma unroll
        for (int st = 0; st < kRing - 1; ++st) fetch(st);
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
            if (st + kRing - 1 < kSteps) fetch(st + kRing - 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[st % kRing][kt], q[st], s[kt], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Register i of key tile kt is key 32 kt + 8 (i / 4) + 4 half + i % 4.
    auto values = [&](int t) {
        if (t * kKeys >= some_see) return;
        const char *v = lds.v[t & 1];
        const bool part = (t + 1) * kKeys > all_see;
        float x[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = s[i / 16][i % 16] * scale2;
        if (part) {
            const int left = mine - t * kKeys - 4 * half;
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i / 4 * 8 + i % 4 >= left) x[i] = -INFINITY;
        }
        float top = x[0];
#pragma unroll
        for (int i = 1; i < 32; ++i) top = fmaxf(top, x[i]);
        top = halves_max(top);
        if (__any(top > m + kSlack)) {
            const float now = fmaxf(m, top), down = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= down;
#pragma unroll
            for (int d = 0; d < kDv / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= down;
        }
        const float base = m == -INFINITY ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            x[i] = __builtin_amdgcn_exp2f(x[i] - base);
            sum += x[i];
        }
        l += sum;
        bf16x8 p[4];
#pragma unroll
        for (int st = 0; st < 4; ++st) p[st] = pack_bf16x8(x + 8 * st);
        bool odd = false;
        if (part) {
            // A weight of zero must not meet an infinity or NaN: where the tile has one, zeros take its place, and what it
            // gives the rows that see it is added at the end.
            for (int i = lane; i < kKeys * kDv * 2 / 16; i += kWave) {
                const u32x4 w = reinterpret_cast<const u32x4 *>(v)[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) odd |= not_finite(w[j]) || not_finite(w[j] >> 16);
            }
            odd = __any(odd);
            if (odd) {
                not_finite_tiles |= 1 << (t & 1);
                last_odd = t;
#pragma unroll
                for (int i = 0; i < 32; i += 4)
                    *reinterpret_cast<u32x2 *>(&lds.p[wave][t & 1][col][i / 4 * 8 + 4 * half]) = u32x2{pack_bf16x2(x[i], x[i + 1]), pack_bf16x2(x[i + 2], x[i + 3])};
            }
        }
        bf16x8 f[3];
        auto fetch = [&](int n) {
            const char *w = v + (v_at ^ (n % 4 * 64)) + n / 4 * 16 * 256;
            const u32x2 lo = read_tr(w), hi = read_tr(w + 8 * 256);
            f[n % 3] = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
        };
        fetch(0);
        fetch(1);
#pragma unroll
        for (int n = 0; n < 16; ++n) {
            if (n + 2 < 16) fetch(n + 2);
            if (odd) f[n % 3] = finite(f[n % 3]);
            __builtin_amdgcn_sched_barrier(0);
            o[n % 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n % 3], p[n / 4], o[n % 4], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // Half step 2 t: the first four wavefronts take the scores of tile t, the others the values of tile t - 1; half step
    // 2 t + 1: values of tile t and scores of tile t.  Every wavefront issues its share of keys t + 1 in half step 2 t (they
    // have landed at the end of 2 t + 1) and of values t + 1 in half step 2 t + 1 (at the end of 2 t + 2).
    const bool second = wave >= 4;
    auto keys_step = [&] {  // ends a half step that issued keys (three loads): the values before them have landed
        asm volatile("s_waitcnt vmcnt(3) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    auto values_step = [&] {
        asm volatile("s_waitcnt vmcnt(2) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (second && tiles) {
        load_k(1);
        keys_step();
    }
    for (int t = 0; t < tiles; ++t) {
        if (second) load_v(t + 1);
        else load_k(t + 1);
        scores(t);
        if (second) values_step();
        else keys_step();
        if (second) load_k(t + 2);
        else load_v(t + 1);
        values(t);
        if (second) {
            if (t + 1 < tiles) keys_step();
        } else {
            values_step();
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing is on its way to LDS when the workgroup ends

    if (row >= nq) return;
    l = halves_sum(l);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const long at = (long)(q0 + row) * a.H + h;
#pragma unroll
    for (int d = 0; d < kDv / 32; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<u32x2 *>(a.o + at * kDv + 32 * d + 8 * i + 4 * half) =
                u32x2{pack_bf16x2(o[d][4 * i] * inv, o[d][4 * i + 1] * inv), pack_bf16x2(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv)};
    if (a.lse && half == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) / kLog2e;
    if (!not_finite_tiles) return;
    for (int n = 0; n < 64; ++n) {  // the lane's own elements, as above
        const int el = n / 16 * 32 + n % 16 / 4 * 8 + 4 * half + n % 4;
        float c = 0.f;
        for (int t = max(last_odd - 1, 0); t <= last_odd; ++t) {
            if (!(not_finite_tiles >> (t & 1) & 1)) continue;
            for (int j = 0; j < min(mine - t * kKeys, kKeys); ++j) {
                const uint16_t e = vh[(long)(t * kKeys + j) * a.v_stride + el];
                if (not_finite(e)) c = fmaf(bf16_bits_to_f32(lds.p[wave][t & 1][col][j]), bf16_bits_to_f32(e), c);
            }
        }
        if (c == 0.f) continue;
        uint16_t *p = a.o + at * kDv + el;
        *p = f32_to_bf16_bits(bf16_bits_to_f32(*p) + c);
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
