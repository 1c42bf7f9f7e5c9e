// Internal launchers of the norm, attention and cache kernels; attn_abi.cpp
// validates arguments and then calls these.  All enqueue on `stream`, allocate
// nothing and return the hipError_t of the launch.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

namespace ecospec {

constexpr int kMaxDrafts = 64;  // draft tokens of a sequence: one bit each in its tree masks

hipError_t launch_add_rmsnorm(const uint16_t *x, const uint16_t *residual, const uint16_t *weight, int T, int d,
                              float eps, int qfmt, uint16_t *sum, uint16_t *y, uint8_t *q, void *scales,
                              hipStream_t stream);

// Draft tokens and the paged cache's bookkeeping, shared by both cached forms.
struct PagedArgs {
    int N, B, H;
    int n_pages, page, max_blocks;
    const int32_t *token_offsets, *block_table, *cache_len;
    const uint64_t *mask;  // or null: causal
    float scale;
    uint16_t *o;
    float *lse;  // or null
};

struct LatentArgs : PagedArgs {
    const uint16_t *q, *kv_new, *pages;
};
size_t latent_workspace(int N, int B, int H, int max_blocks, int page);
hipError_t launch_latent_attn(const LatentArgs &a, void *workspace, hipStream_t stream);

struct CacheArgs : PagedArgs {
    int Hkv, D;
    const uint16_t *q, *k_new, *v_new;
    const uint8_t *k, *v;
    const float *k_scale, *v_scale;
};
size_t cache_workspace(int N, int B, int H, int Hkv, int D);
hipError_t launch_cache_attn(const CacheArgs &a, void *workspace, hipStream_t stream);

struct AppendArgs {
    int N, B, n_rows, max_tokens;
    int Hkv, D, n_pages, page, max_blocks;
    const uint16_t *k_new, *v_new;
    const int32_t *rows, *token_offsets, *block_table, *cache_len;
    uint8_t *k, *v;
    float *k_scale, *v_scale;
};
bool cache_append_fits(const AppendArgs &a);  // the launch's grid
hipError_t launch_cache_append(const AppendArgs &a, hipStream_t stream);

struct PromptArgs {
    int N, M, B, H, max_tokens;
    const int32_t *q_offsets, *kv_offsets;
    const uint16_t *q, *k, *k_rope, *v;
    int64_t k_stride, k_head, v_stride, v_head;
    float scale;
    uint16_t *o;
    float *lse;  // or null
};
hipError_t launch_latent_prompt(const PromptArgs &a, hipStream_t stream);

}  // namespace ecospec
