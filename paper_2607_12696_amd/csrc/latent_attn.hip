// Latent attention of draft tokens, absorbed form.
#include "row_attn.hpp"

namespace ecospec {
namespace {

constexpr int kR = 512, kP = 64, kW = kR + kP;

struct LatentRow : PagedRow {
    const LatentArgs &a;
    float q[kW / kWave];
    __device__ LatentRow(const LatentArgs &args) : PagedRow(args), a(args)
    {
        for (int i = 0; i < kW / kWave; ++i)
            q[i] = bf16_bits_to_f32(a.q[((long)t * a.H + h) * kW + lane_id() * (kW / kWave) + i]);
    }
    __device__ const uint16_t *row(int j) const
    {
        return j < len ? a.pages + (page_of(j) * page + j % page) * kW : a.kv_new + (long)(t0 + j - len) * kW;
    }
    __device__ float dot(int j, int lane) const
    {
        const uint16_t *k = row(j) + lane * (kW / kWave);
        float s = 0.f;
        for (int i = 0; i < kW / kWave; ++i) s = fmaf(q[i], bf16_bits_to_f32(k[i]), s);
        return s;
    }
    __device__ float value(int j, int e) const { return bf16_bits_to_f32(row(j)[e]); }
};

__global__ __launch_bounds__(256) void latent_row_kernel(LatentArgs a)
{
    const LatentRow r(a);
    row_attention<kR>(r, a.scale, a.o + (long)blockIdx.x * kR, a.lse ? a.lse + blockIdx.x : nullptr);
}

}  // namespace

size_t latent_workspace(int, int, int) { return 256; }

hipError_t launch_latent_attn(const LatentArgs &a, void *, hipStream_t stream)
{
    latent_row_kernel<<<(unsigned)(a.N * a.H), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace ecospec
