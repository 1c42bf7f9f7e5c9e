// Grouped-query attention of draft tokens over the 8-bit cache.
#include "row_attn.hpp"

namespace ecospec {
namespace {

template <int D>
struct CacheRow : PagedRow {
    const CacheArgs &a;
    int kvh;
    float q[D / kWave];
    __device__ CacheRow(const CacheArgs &args) : PagedRow(args), a(args)
    {
        kvh = h / (a.H / a.Hkv);
        for (int i = 0; i < D / kWave; ++i)
            q[i] = bf16_bits_to_f32(a.q[((long)t * a.H + h) * D + lane_id() * (D / kWave) + i]);
    }
    __device__ static float code(uint8_t c) { return __builtin_amdgcn_cvt_f32_fp8((int)c, 0); }
    __device__ float dot(int j, int lane) const
    {
        float s = 0.f;
        const int e0 = lane * (D / kWave);
        if (j < len) {
            const long head = page_of(j) * a.Hkv + kvh;
            for (int i = 0; i < D / kWave; ++i) s = fmaf(q[i], code(a.k[(head * page + j % page) * D + e0 + i]), s);
            return s * a.k_scale[head];
        }
        const uint16_t *k = a.k_new + ((long)(t0 + j - len) * a.Hkv + kvh) * D + e0;
        for (int i = 0; i < D / kWave; ++i) s = fmaf(q[i], bf16_bits_to_f32(k[i]), s);
        return s;
    }
    __device__ float value(int j, int e) const
    {
        if (j < len) {
            const long head = page_of(j) * a.Hkv + kvh;
            return code(a.v[(head * D + e) * page + j % page]) * a.v_scale[head];
        }
        return bf16_bits_to_f32(a.v_new[((long)(t0 + j - len) * a.Hkv + kvh) * D + e]);
    }
};

template <int D>
__global__ __launch_bounds__(256) void cache_row_kernel(CacheArgs a)
{
    const CacheRow<D> r(a);
    row_attention<D>(r, a.scale, a.o + (long)blockIdx.x * D, a.lse ? a.lse + blockIdx.x : nullptr);
}

}  // namespace

size_t cache_workspace(int, int, int, int, int) { return 256; }

hipError_t launch_cache_attn(const CacheArgs &a, void *, hipStream_t stream)
{
    if (a.D == 64)
        cache_row_kernel<64><<<(unsigned)(a.N * a.H), 256, 0, stream>>>(a);
    else
        cache_row_kernel<128><<<(unsigned)(a.N * a.H), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace ecospec
