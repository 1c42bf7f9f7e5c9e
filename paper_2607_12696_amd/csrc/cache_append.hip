// Append to the 8-bit key/value cache: per touched page and head one scale,
// the smallest power of two that holds what the page has had so far.
//
// What bounds it: memory.  A token's head is 2 D bytes read and D written, for
// keys and for values, and a page's scale must be known before its first code
// is written.  So one workgroup takes the keys or the values of one head in
// one page and keeps the page's new tokens in registers between the maximum
// and the codes: every value is read once.  A thread has 4 slots by 8 elements
// (4 loads of 16 bytes), for every page size and D, so the workgroup is as
// large as its page asks for, and a small page does not leave waves idle.
// Keys are stored as 8 bytes a slot.  Values lie element by element: 4 slots
// of an element make one word, words turn in LDS, and 16 slots are stored at
// once.
// Measured: 15001 tokens of 4 heads of 128 11.8 us in the kernel (3.9 TB/s; byte
// by byte 55); 4 sequences of 5 tokens, 8 heads of 64, 5.4 us, four dependent
// reads (lengths, block, tokens, old codes) and the launch.
#include "attn.hpp"
#include "device.hpp"

namespace ecospec {
namespace {

constexpr int kMaxPage = 128;

typedef unsigned short half_pair __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b)  // of two 16-bit numbers each
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(half_pair, a), __builtin_bit_cast(half_pair, b)));
}

// bf16 of a register's low or high half.
__device__ __forceinline__ float lo_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// 4 e4m3fn codes, ties to even.  The values are at most 448 or NaN.
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d)
{
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

// q, the nearest float to a number that is q plus something of r's sign, to the
// nearest with an odd last bit: rounded to a code then, it gives what the
// number itself would (24 bits lie well past the code's 4).
__device__ __forceinline__ float sticky(float q, float r)
{
    const uint32_t bits = __float_as_uint(q);
    if (!(fabsf(q) > 0x1p-20f) || !(fabsf(q) < 0x1p20f) || r == 0.f || (bits & 1u)) return q;
    return __uint_as_float((r < 0.f) == (q < 0.f) ? bits + 1 : bits - 1);
}

// The codes of a word at a scale that is larger by 1 / down.
__device__ __forceinline__ uint32_t recode4(uint32_t w, float down)
{
    float v[4] = {__builtin_amdgcn_cvt_f32_fp8((int)w, 0), __builtin_amdgcn_cvt_f32_fp8((int)w, 1),
                  __builtin_amdgcn_cvt_f32_fp8((int)w, 2), __builtin_amdgcn_cvt_f32_fp8((int)w, 3)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float p = v[i] * down;
        v[i] = sticky(p, fmaf(v[i], down, -p));
    }
    return code4(v[0], v[1], v[2], v[3]);
}

template <int D>
__global__ __launch_bounds__(kMaxPage * D / 32) void append_kernel(AppendArgs a)
{
    constexpr int C = D / 8;  // threads to a slot's elements
    __shared__ __align__(16) uint8_t turned[D * (kMaxPage + 16) + 8 * kMaxPage];
    __shared__ uint32_t part[kMaxPage * D / 32 / kWave];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int h = blockIdx.x % a.Hkv;
    const bool values = blockIdx.y;
    const int room = a.max_blocks * a.page;

    // The workgroup's page: the touched pages of all sequences in order.
    int nth = blockIdx.x / a.Hkv, b0 = 0, t0, n, len, upto;
    for (;; b0 += kWave) {
        if (b0 >= a.B) return;
        const int b = b0 + lane;
        t0 = n = len = 0;
        if (b < a.B) {
            t0 = min(max(a.token_offsets[b], 0), a.N);
            len = min(max(a.cache_len[b], 0), room);
            n = min(min(max(a.token_offsets[b + 1], t0), a.N) - t0, room - len);
        }
        upto = n ? (len + n - 1) / a.page - len / a.page + 1 : 0;
#pragma unroll
        for (int s = 1; s < kWave; s <<= 1) {
            const int x = __shfl_up(upto, s, kWave);
            upto += lane >= s ? x : 0;
        }
        const int all = __builtin_amdgcn_readlane(upto, kWave - 1);
        if (nth < all) break;
        nth -= all;
    }
    const int mine = __builtin_popcountll(__builtin_amdgcn_ballot_w64(upto <= nth));  // lanes before the page's
    nth -= mine ? __builtin_amdgcn_readlane(upto, mine - 1) : 0;
    t0 = __builtin_amdgcn_readlane(t0, mine);
    n = __builtin_amdgcn_readlane(n, mine);
    len = __builtin_amdgcn_readlane(len, mine);

    const int blk = len / a.page + nth, begin = blk * a.page;
    const int kept = max(len - begin, 0), end = min(len + n - begin, a.page);  // the new tokens' slots
    const int id = min(max(a.block_table[(long)(b0 + mine) * a.max_blocks + blk], 0), a.n_pages - 1);
    const uint16_t *src = (values ? a.v_new : a.k_new) + h * D;
    uint8_t *dst = (values ? a.v : a.k) + ((long)id * a.Hkv + h) * a.page * D;
    float *scale = (values ? a.v_scale : a.k_scale) + (long)id * a.Hkv + h;

    // Its tokens, and the largest finite magnitude as the bits of a bf16.
    const int c = threadIdx.x % C, slot = threadIdx.x / C * 4;
    uint4 x[4];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = make_uint4(0, 0, 0, 0);
        if (slot + i < kept || slot + i >= end) continue;
        const int e = t0 + begin + slot + i - len;
        const int row = a.rows ? min(max(a.rows[e], 0), a.n_rows - 1) : e;
        x[i] = *reinterpret_cast<const uint4 *>(src + (long)row * a.Hkv * D + c * 8);
    }
    const float was = kept ? *scale : 0.f;
    auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f(x[i].x), f(x[i].y), f(x[i].z), f(x[i].w);
    };
    each([&](uint32_t w) { top = max_pair(top, w & 0x7fff7fffu); });
    top = max(top & 0xffffu, top >> 16);
    const bool special = top >= 0x7f80u;
    if (special) {
        top = 0;
        each([&](uint32_t w) {
            const uint32_t l = w & 0x7fffu, u = w >> 16 & 0x7fffu;
            top = max(top, max(l < 0x7f80u ? l : 0u, u < 0x7f80u ? u : 0u));
        });
    }
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, s, kWave));
    if (lane == 0) part[wave] = top;
    __syncthreads();
    for (int w = 0; w < (int)blockDim.x / kWave; ++w) top = max(top, part[w]);

    // top = m * 2^e with 1 <= m < 2, 448 = 1.75 * 2^8.
    const int e = max((int)(top >> 7) - 127 - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0), -126);
    const float unit = fmaxf(was, __uint_as_float((uint32_t)(e + 127) << 23));
    const float inv = 1.f / unit, down = was / unit;
    const bool grows = kept && unit > was;
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = j % 2 ? hi_half(w[j / 2]) : lo_half(w[j / 2]);
    }
    if ((__float_as_uint(unit) & 0x7fffffu) == 0) {  // a power of two: the product is the quotient
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] *= inv;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float q = v[i][j] / unit;
                v[i][j] = sticky(q, fmaf(-q, unit, v[i][j]));
            }
    }
    if (special) {  // infinities are past 448, what is finite is not
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (v[i][j] > 448.f) v[i][j] = 448.f;
                if (v[i][j] < -448.f) v[i][j] = -448.f;
            }
    }

    if (!values) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint2 *at = reinterpret_cast<uint2 *>(dst + (long)(slot + i) * D + c * 8);
            if (slot + i >= kept && slot + i < end) {
                *at = make_uint2(code4(v[i][0], v[i][1], v[i][2], v[i][3]), code4(v[i][4], v[i][5], v[i][6], v[i][7]));
            } else if (grows && slot + i < a.page) {
                const uint2 old = *at;
                *at = make_uint2(recode4(old.x, down), recode4(old.y, down));
            }
        }
    } else {
        // Element 8 c + j lies in row j * C + c of LDS, rows 16 bytes apart from
        // the page's length and each j by another page: 64 banks at a time, in
        // and out.
        const int pitch = a.page + 16;
        auto row_of = [&](int el) { return turned + ((el % 8) * C + el / 8) * pitch + (el % 8) * a.page; };
        if (slot < a.page)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                *reinterpret_cast<uint32_t *>(row_of(8 * c + j) + slot) = code4(v[0][j], v[1][j], v[2][j], v[3][j]);
        __syncthreads();
        const int chunks = a.page / 16;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = threadIdx.x + i * blockDim.x, el = at / chunks, s0 = at % chunks * 16;
            if (el >= D) break;
            uint4 *out = reinterpret_cast<uint4 *>(dst + (long)el * a.page + s0);
            const bool any = s0 < end && s0 + 16 > kept, whole = s0 >= kept && s0 + 16 <= end;
            if (!any && !grows) continue;
            uint4 w = make_uint4(0, 0, 0, 0);
            if (any) w = *reinterpret_cast<const uint4 *>(row_of(el) + s0);
            if (!whole) {  // the page is this workgroup's own: what others have of the 16 slots stays
                uint4 old = *out;
                if (grows)
                    old = make_uint4(recode4(old.x, down), recode4(old.y, down), recode4(old.z, down), recode4(old.w, down));
                auto merge = [&](uint32_t had, uint32_t now, int s) {
                    const int from = min(max(kept - s, 0), 4), to = min(max(end - s, 0), 4);
                    const uint32_t m = from < to ? (uint32_t)((1ull << 8 * to) - (1ull << 8 * from)) : 0u;
                    return (now & m) | (had & ~m);
                };
                w = make_uint4(merge(old.x, w.x, s0), merge(old.y, w.y, s0 + 4), merge(old.z, w.z, s0 + 8),
                               merge(old.w, w.w, s0 + 12));
            }
            *out = w;
        }
    }
    if (threadIdx.x == 0) *scale = unit;
}

// Pages that a call can touch: no sequence more than its longest possible run
// of tokens does, and all together no more than whole pages of all tokens and
// two ends each.
long touched(const AppendArgs &a)
{
    const long each = ((long)a.max_tokens + a.page - 2) / a.page + 1;
    const long one_by_one = a.B * each, together = a.N / a.page + 2L * a.B;
    return one_by_one < together ? one_by_one : together;
}

int threads(const AppendArgs &a)
{
    const int t = a.page * a.D / 32;
    return t < kWave ? kWave : t;
}

}  // namespace

bool cache_append_fits(const AppendArgs &a)
{
    return touched(a) * a.Hkv * threads(a) <= 1L << 31;
}

hipError_t launch_cache_append(const AppendArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)(touched(a) * a.Hkv), 2);
    if (a.D == 64)
        append_kernel<64><<<grid, threads(a), 0, stream>>>(a);
    else
        append_kernel<128><<<grid, threads(a), 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace ecospec
