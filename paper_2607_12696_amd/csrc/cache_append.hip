// Append to the 8-bit key/value cache: per touched page and head one scale,
// the smallest power of two that holds what the page has had so far.
#include "attn.hpp"
#include "device.hpp"

namespace ecospec {
namespace {

__device__ __forceinline__ float e4m3_value(uint32_t code)
{
    return __builtin_amdgcn_cvt_f32_fp8((int)code, 0);
}

__device__ __forceinline__ uint32_t e4m3_code(float v)
{
    if (v > 448.f) v = 448.f;
    if (v < -448.f) v = -448.f;
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false) & 0xffu;
}

// One workgroup per (touched page, head, keys or values).
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a, int most)
{
    __shared__ float part[4];
    const int h = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv / most, nth = blockIdx.x / a.Hkv % most;
    const bool values = blockIdx.y;
    const int t0 = min(max(a.token_offsets[b], 0), a.N), t1 = min(max(a.token_offsets[b + 1], t0), a.N);
    const int len = min(max(a.cache_len[b], 0), a.max_blocks * a.page);
    const int blk = len / a.page + nth;
    const int first = max(len, blk * a.page);                                       // first new position of the page
    const int last = min(len + (t1 - t0), min(blk + 1, a.max_blocks) * a.page);     // and its end
    if (first >= last) return;
    const int id = min(max(a.block_table[(long)b * a.max_blocks + blk], 0), a.n_pages - 1);
    const uint16_t *src = values ? a.v_new : a.k_new;
    uint8_t *dst = (values ? a.v : a.k) + ((long)id * a.Hkv + h) * a.page * a.D;
    float *scale = (values ? a.v_scale : a.k_scale) + (long)id * a.Hkv + h;
    const int kept = first - blk * a.page, n = (last - first) * a.D;
    auto value = [&](int i) {
        const int e = t0 + (first - len) + i / a.D;
        const int row = a.rows ? min(max(a.rows[e], 0), a.n_rows - 1) : e;
        return bf16_bits_to_f32(src[((long)row * a.Hkv + h) * a.D + i % a.D]);
    };
    float top = 0.f;
    for (int i = threadIdx.x; i < n; i += 256) {
        const float v = fabsf(value(i));
        if (v < INFINITY) top = fmaxf(top, v);
    }
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) top = fmaxf(top, __shfl_xor(top, s, kWave));
    if (lane_id() == 0) part[threadIdx.x / kWave] = top;
    const float was = kept ? *scale : 0.f;
    __syncthreads();
    top = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    // top = m * 2^e with 1 <= m < 2, 448 = 1.75 * 2^8.
    const uint32_t bits = __float_as_uint(top);
    int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    if (e < -126) e = -126;
    const float need = ldexpf(1.f, e), unit = fmaxf(was, need);
    if (kept && unit > was) {
        const float down = was / unit;
        for (int i = threadIdx.x; i < a.page * a.D; i += 256) {
            const int slot = values ? i % a.page : i / a.D;
            if (slot < kept || slot >= kept + (last - first)) dst[i] = (uint8_t)e4m3_code(e4m3_value(dst[i]) * down);
        }
    }
    const float inv = 1.f / unit;
    for (int i = threadIdx.x; i < n; i += 256) {
        const int slot = kept + i / a.D, el = i % a.D;
        dst[values ? (long)el * a.page + slot : (long)slot * a.D + el] = (uint8_t)e4m3_code(value(i) * inv);
    }
    if (threadIdx.x == 0) *scale = unit;
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs &a, hipStream_t stream)
{
    const int most = (a.max_tokens + a.page - 2) / a.page + 1;  // pages that a sequence can touch
    append_kernel<<<dim3((unsigned)(a.B * most * a.Hkv), 2), 256, 0, stream>>>(a, most);
    return hipGetLastError();
}

}  // namespace ecospec
