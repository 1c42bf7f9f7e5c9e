// Latent attention of prompts, expanded form.
#include "row_attn.hpp"

namespace ecospec {
namespace {

constexpr int kDn = 128, kP = 64, kDv = 128, kDq = kDn + kP;

struct PromptRow {
    const PromptArgs &a;
    int t, h, k0, n;
    float q[kDq / kWave];
    __device__ PromptRow(const PromptArgs &args) : a(args)
    {
        t = blockIdx.x / a.H;
        h = blockIdx.x % a.H;
        const int b = sequence_of(a.q_offsets, a.B, t);
        const int q0 = a.q_offsets[b], q1 = a.q_offsets[b + 1];
        k0 = min(max(a.kv_offsets[b], 0), a.M);
        const int k1 = min(max(a.kv_offsets[b + 1], k0), a.M);
        n = min(max(t - q0 + 1 + (k1 - k0) - (q1 - q0), 0), k1 - k0);
        for (int i = 0; i < kDq / kWave; ++i) q[i] = bf16_bits_to_f32(a.q[((long)t * a.H + h) * kDq + lane_id() * 3 + i]);
    }
    __device__ int keys() const { return n; }
    __device__ bool seen(int) const { return true; }
    __device__ float dot(int j, int lane) const
    {
        float s = 0.f;
        for (int i = 0; i < kDq / kWave; ++i) {
            const int e = lane * 3 + i;
            const uint16_t k = e < kDn ? a.k[(k0 + j) * a.k_stride + h * a.k_head + e] : a.k_rope[(long)(k0 + j) * kP + e - kDn];
            s = fmaf(q[i], bf16_bits_to_f32(k), s);
        }
        return s;
    }
    __device__ float value(int j, int e) const { return bf16_bits_to_f32(a.v[(k0 + j) * a.v_stride + h * a.v_head + e]); }
};

__global__ __launch_bounds__(256) void prompt_row_kernel(PromptArgs a)
{
    const PromptRow r(a);
    row_attention<kDv>(r, a.scale, a.o + (long)blockIdx.x * kDv, a.lse ? a.lse + blockIdx.x : nullptr);
}

}  // namespace

hipError_t launch_latent_prompt(const PromptArgs &a, hipStream_t stream)
{
    prompt_row_kernel<<<(unsigned)(a.N * a.H), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace ecospec
