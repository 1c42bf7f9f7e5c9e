// Internal launchers of the kernels at the two ends of a decoding step (pages,
// prompts of grouped heads, log probabilities); step_abi.cpp validates arguments
// and then calls these.  All enqueue on `stream`, allocate nothing and return
// the hipError_t of the launch.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

namespace ecospec {

constexpr int kMaxSequences = 1024;

struct PagesArgs {
    int B, N, n_pages, page, max_blocks;
    int32_t *block_table, *free_pages;
    const int32_t *cache_len, *keep_len, *token_offsets, *n_free;  // keep_len or null
    int32_t *new_len, *n_free_out, *refused;
    int64_t *slots;      // or null
    int32_t *positions;  // or null
};
hipError_t launch_pages_update(const PagesArgs &a, hipStream_t stream);

struct RowsArgs {
    int N, n_rows;
    long slots_end;  // n_pages * page
    uint16_t *pages;
    const uint16_t *kv_new;
    const int32_t *rows;  // or null
    const int64_t *slots;
};
constexpr int kLatentRow = 576;  // elements
hipError_t launch_latent_append(const RowsArgs &a, hipStream_t stream);

struct GroupedPromptArgs {
    int N, M, B, H, Hkv, max_tokens;
    const int32_t *q_offsets, *kv_offsets;
    const uint16_t *q, *k, *v;
    int64_t q_stride, q_head, k_stride, k_head, v_stride, v_head;
    float scale;
    uint16_t *o;
    float *lse;  // or null
};
size_t grouped_prompt_workspace(int D);
hipError_t launch_grouped_prompt(const GroupedPromptArgs &a, int D, void *workspace, hipStream_t stream);

struct LogprobArgs {
    const void *logits;
    int64_t stride;
    int N, V, M, k;
    float scale;
    const int32_t *tokens;
    float *logprob, *lse, *entropy, *top_logprob;  // each or null
    int32_t *top_idx;
};
size_t logprobs_workspace();
hipError_t launch_token_logprobs(const LogprobArgs &a, bool bf16, void *workspace, hipStream_t stream);

}  // namespace ecospec
