// Residual addition and root-mean-square norm with an optional 8-bit output.
//   v = x + residual;  u = v * rsqrt(mean(v^2) + eps) * weight
// Bound by memory: 2 bytes an element of each of x, residual, sum and y, 1 of the
// codes, a few operations each.  One workgroup a row, which stays in registers
// between the sum of squares and the outputs: every input is read once and the
// norm is never rounded to bf16 before it is coded.  The sum of squares is fp32,
// a tree over the workgroup; v stays fp32 although `sum` is stored in bf16, so
// the norm has one rounding.  Measured: 6001 rows of 2880 with MX codes 25 us
// (6.3 TB/s, part of it from the memory-side cache), 4 rows of 7168 4 us; 6001
// rows of 7168 74 us with codes by row and 61 without codes.  Narrow rows leave
// threads idle: 20000 of 512 19 us, 60000 of 128 44 us (1.4 TB/s).
#include "attn.hpp"
#include "device.hpp"

namespace ecospec {
namespace {

enum { Q_NONE = 0, Q_GROUP = 1, Q_MX = 2, Q_ROW = 3 };

struct NormArgs {
    const uint16_t *x, *residual, *weight;
    uint16_t *sum, *y;
    uint8_t *q;
    void *scales;
    int d, qfmt;
    float eps;
};

__device__ __forceinline__ void unpack8(const u32x4 &w, float *f)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ u32x4 pack8(const float *f)
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    return w;
}

// Code of v (already divided by its scale): saturating, NaN kept.
__device__ __forceinline__ float saturate(float v)
{
    if (v > 448.f) v = 448.f;
    if (v < -448.f) v = -448.f;
    return v;
}

// The quotient f / scale by its rounded reciprocal and one correction, which brings it to the nearest fp32 number: a product
// with the reciprocal alone can leave a tie between two codes.  An infinite scale (inv 0) is passed as 0: quotients 0 and NaN.
// Zeros keep their sign.
__device__ __forceinline__ float quotient(float f, float scale, float inv)
{
    const float q = f * inv;
    return fmaf(fmaf(q, scale, -f), -inv, q);
}

// Squares are summed of v / 128, so that the sum over the widest row (16384 elements) overflows no sooner than their
// mean does.  Where the mean does, or is so small that squares may have lost bits below fp32's smallest normal number, the
// row is summed again times a power of two that brings it back.  (Rows like that need an epsilon of nearly nothing, or
// elements past 2^64: others go on with the sum they have.)
constexpr float kDown = 0x1p-7f;
constexpr float kLeast = 0x1p-80f;  // an element of the root mean square adds 2^-14 of this, 32 bits above the smallest normal
constexpr float kUp = 0x1p100f;     // a row below kLeast has elements below 2^-33: 2^67, their squares / 128^2 sum to 2^120
constexpr float kBack = 0x1p-70f;   // elements below 2^128: 2^58

template <int STEP>
__device__ __forceinline__ float lanes_max(float m)
{
#pragma unroll
    for (int s = 1; s < STEP; s <<= 1) m = fmaxf(m, __shfl_xor(m, s, kWave));
    return m;
}

template <int THREADS, int VPT>
__global__ __launch_bounds__(THREADS) void rmsnorm_kernel(NormArgs a)
{
    constexpr int kWaves = THREADS / kWave;
    __shared__ float part[2][kWaves];
    const long row = blockIdx.x;
    const int vecs = a.d / 8;
    const u32x4 *x = reinterpret_cast<const u32x4 *>(a.x + row * a.d);
    const u32x4 *r = reinterpret_cast<const u32x4 *>(a.residual + row * a.d);
    float v[VPT][8];
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = i * THREADS + threadIdx.x;
        if (at < vecs) {
            unpack8(x[at], v[i]);
            if (a.residual) {
                float f[8];
                unpack8(r[at], f);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] += f[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float t = v[i][j] * kDown;
                ss = fmaf(t, t, ss);
            }
        }
    }
    ss = wave_sum(ss);
    if (lane_id() == 0) part[0][threadIdx.x / kWave] = ss;
    __syncthreads();
    ss = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) ss += part[0][w];
    float mean = ss / ((float)a.d * kDown * kDown) + a.eps, by = 1.f;
    if (!(mean >= kLeast && mean < INFINITY)) {
        by = mean < kLeast ? kUp : kBack;
        ss = 0.f;
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            if (i * THREADS + threadIdx.x < vecs)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float t = v[i][j] * (by * kDown);
                    ss = fmaf(t, t, ss);
                }
        ss = wave_sum(ss);
        if (lane_id() == 0) part[1][threadIdx.x / kWave] = ss;
        __syncthreads();
        ss = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) ss += part[1][w];
        mean = ss / ((float)a.d * kDown * kDown) + a.eps * by * by;
        __syncthreads();
    }
    const float rinv = 1.f / sqrtf(mean);
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = i * THREADS + threadIdx.x;
        if (at < vecs) {
            if (a.sum) reinterpret_cast<u32x4 *>(a.sum + row * a.d)[at] = pack8(v[i]);
            float w[8];
            unpack8(reinterpret_cast<const u32x4 *>(a.weight)[at], w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[i][j] *= by;
                v[i][j] *= rinv * w[j];
                top = fmaxf(top, fabsf(v[i][j]));
            }
            if (a.y) reinterpret_cast<u32x4 *>(a.y + row * a.d)[at] = pack8(v[i]);
        }
    }
    if (a.qfmt == Q_NONE) return;
    if (a.qfmt == Q_ROW) {
        top = lanes_max<64>(top);
        if (lane_id() == 0) part[1][threadIdx.x / kWave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, part[1][w]);
        if (threadIdx.x == 0) static_cast<float *>(a.scales)[row] = fmaxf(top, 0x1p-100f) / 448.f;
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = i * THREADS + threadIdx.x;
        const bool in = at < vecs;
        float m = 0.f;
        if (in)
#pragma unroll
            for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(v[i][j]));
        float inv, scale = 0.f;
        if (a.qfmt == Q_MX) {
            m = lanes_max<4>(m);  // 32 elements
            int e = (int)(__float_as_uint(m) >> 23) - 127 - 8;
            if (e < -127) e = -127;
            inv = ldexpf(1.f, -e);  // the product is the quotient
            if (in && (at & 3) == 0) static_cast<uint8_t *>(a.scales)[row * (a.d / 32) + at / 4] = (uint8_t)(e + 127);
        } else {
            m = a.qfmt == Q_ROW ? top : lanes_max<16>(m);  // 128 elements
            const float s = fmaxf(m, 0x1p-100f) / 448.f;
            inv = 1.f / s;
            if (s < INFINITY) scale = s;
            if (a.qfmt == Q_GROUP && in && (at & 15) == 0)
                static_cast<float *>(a.scales)[row * ((a.d + 127) / 128) + at / 16] = s;
        }
        if (!in) continue;
        float f[8];
        if (a.qfmt == Q_MX) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = saturate(v[i][j] * inv);
        } else {  // at most 448 but for a rounding, and what is below 464 becomes 448
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = quotient(v[i][j], scale, inv);
        }
        u32x2 c;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h], f[4 * h + 1], 0, false);
            c[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h + 2], f[4 * h + 3], w, true);
        }
        reinterpret_cast<u32x2 *>(a.q + row * a.d)[at] = c;
    }
}

}  // namespace

hipError_t launch_add_rmsnorm(const uint16_t *x, const uint16_t *residual, const uint16_t *weight, int T, int d,
                              float eps, int qfmt, uint16_t *sum, uint16_t *y, uint8_t *q, void *scales,
                              hipStream_t stream)
{
    const NormArgs a{x, residual, weight, sum, y, q, scales, d, qfmt, eps};
    // As many threads as the row has vectors of 8, up to the largest workgroup.  One vector a thread beats fewer threads
    // with more: 4 rows of 7168 take 3.9 us in the kernel, 4.4 us with two a thread and 6.2 us with four; 6001 rows 72 us
    // against 76 and 83.  Threads without one cost: 6001 rows of 2880 take 26 us, 32 us with 1024 threads; 20000 rows of
    // 1536 take 47 us, 73 us with 512 threads.
    if (d <= 2048)
        rmsnorm_kernel<256, 1><<<T, 256, 0, stream>>>(a);
    else if (d <= 4096)
        rmsnorm_kernel<512, 1><<<T, 512, 0, stream>>>(a);
    else if (d <= 8192)
        rmsnorm_kernel<1024, 1><<<T, 1024, 0, stream>>>(a);
    else
        rmsnorm_kernel<1024, 2><<<T, 1024, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace ecospec
