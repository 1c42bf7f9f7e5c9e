// C ABI of the two ends of a decoding step (pages, prompts of grouped heads, log
// probabilities): argument validation, then one launch sequence each.  No
// allocation, no synchronisation.
#include "ecospec_moe.h"

#include <hip/hip_runtime_api.h>
#include <math.h>

#include "step.hpp"

namespace ecospec {
void set_last_error(const char *msg);
}

namespace {

moe_status_t from_hip(hipError_t e)
{
    if (e == hipSuccess) return MOE_OK;
    ecospec::set_last_error(hipGetErrorString(e));
    return MOE_ERR_HIP;
}

// The stream's device is the current one for the launches of a call: a kernel is looked up on the current device.
struct OnDeviceOf {
    int was = -1;
    explicit OnDeviceOf(void *stream)
    {
        int now = 0;
        hipDevice_t of = 0;
        if (!stream || hipGetDevice(&now) != hipSuccess || hipStreamGetDevice((hipStream_t)stream, &of) != hipSuccess) return;
        if (now != of && hipSetDevice(of) == hipSuccess) was = now;
    }
    ~OnDeviceOf()
    {
        if (was >= 0) (void)hipSetDevice(was);
    }
    OnDeviceOf(const OnDeviceOf &) = delete;
    OnDeviceOf &operator=(const OnDeviceOf &) = delete;
};

bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// A range of memory that a call reads or writes; null: none.
struct Range {
    const void *at;
    size_t bytes;
};

bool overlap(const Range &x, const Range &y)
{
    const uintptr_t a = (uintptr_t)x.at, b = (uintptr_t)y.at;
    return x.at && y.at && a < b + y.bytes && b < a + x.bytes;
}

// Whether something that a call writes overlaps anything else of it.
template <size_t OUT, size_t IN>
bool any_overlap(const Range (&out)[OUT], const Range (&in)[IN])
{
    for (size_t i = 0; i < OUT; ++i) {
        for (const Range &x : in)
            if (overlap(out[i], x)) return true;
        for (size_t j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return true;
    }
    return false;
}

bool page_ok(int page) { return page == 16 || page == 32 || page == 64 || page == 128; }

constexpr int kMaxTokens = 1 << 30;        // of one page update
constexpr int kMaxAppended = 1 << 24;      // rows of one append
constexpr int kMaxHeads = 1024;
constexpr long kMaxPromptRows = 1L << 30;  // query rows (token, head)
constexpr int64_t kMaxStride = 1L << 23;   // elements between a prompt's keys: a tile is addressed in 32 bits
constexpr int kMaxLogitRows = 1 << 22, kMaxVocabulary = 1 << 24, kMaxGiven = 1 << 16, kMaxTop = 64;
constexpr float kMaxScale = 0x1p126f;  // of logits: twice its product with log2 e is a number

}  // namespace

extern "C" {

moe_status_t moe_pages_update(const moe_page_pool_t *p, const int32_t *keep_len, const int32_t *token_offsets, int N,
                              int32_t *new_len, int32_t *n_free_out, int32_t *refused, int64_t *slots,
                              int32_t *positions, void *stream)
{
    if (!p || !p->block_table || !p->cache_len || !p->free_pages || !p->n_free || !token_offsets || !new_len || !n_free_out ||
        !refused)
        return MOE_ERR_INVALID_ARG;
    if (p->B < 1 || p->B > ecospec::kMaxSequences || p->n_pages < 1 || p->max_blocks < 1 || !page_ok(p->page))
        return MOE_ERR_INVALID_ARG;
    if ((long)p->max_blocks * p->page > 1L << 30 || N < 1 || N > kMaxTokens) return MOE_ERR_INVALID_ARG;
    if (!aligned(slots, 8)) return MOE_ERR_INVALID_ARG;
    // Workgroups read the counts while others write the new ones.
    const size_t B = p->B, n = N;
    const Range out[] = {{new_len, B * 4}, {n_free_out, 4}, {refused, 4}, {slots, n * 8}, {positions, n * 4},
                         {p->block_table, B * p->max_blocks * 4}, {p->free_pages, (size_t)p->n_pages * 4}};
    const Range in[] = {{p->cache_len, B * 4}, {keep_len, B * 4}, {token_offsets, (B + 1) * 4}, {p->n_free, 4}};
    if (any_overlap(out, in)) return MOE_ERR_INVALID_ARG;
    ecospec::PagesArgs a{};
    a.B = p->B;
    a.N = N;
    a.n_pages = p->n_pages;
    a.page = p->page;
    a.max_blocks = p->max_blocks;
    a.block_table = p->block_table;
    a.free_pages = p->free_pages;
    a.cache_len = p->cache_len;
    a.keep_len = keep_len;
    a.token_offsets = token_offsets;
    a.n_free = p->n_free;
    a.new_len = new_len;
    a.n_free_out = n_free_out;
    a.refused = refused;
    a.slots = slots;
    a.positions = positions;
    const OnDeviceOf device(stream);
    return from_hip(ecospec::launch_pages_update(a, (hipStream_t)stream));
}

moe_status_t moe_latent_append(void *pages, int n_pages, int page, int r, int p, const void *kv_new, int n_rows,
                               const int32_t *rows, int N, const int64_t *slots, void *stream)
{
    if (!pages || !kv_new || !slots || n_pages < 1 || !page_ok(page) || r < 1 || p < 0 || N < 1 || n_rows < 1)
        return MOE_ERR_INVALID_ARG;
    if (!rows && n_rows < N) return MOE_ERR_INVALID_ARG;
    if (!aligned(pages, 16) || !aligned(kv_new, 16) || !aligned(slots, 8)) return MOE_ERR_INVALID_ARG;
    if (r != 512 || p != 64 || N > kMaxAppended) return MOE_ERR_UNSUPPORTED;
    const size_t row = (size_t)(r + p) * 2;
    const Range out[] = {{pages, (size_t)n_pages * page * row}};
    const Range in[] = {{kv_new, n_rows * row}, {rows, (size_t)N * 4}, {slots, (size_t)N * 8}};
    if (any_overlap(out, in)) return MOE_ERR_INVALID_ARG;
    ecospec::RowsArgs a{};
    a.N = N;
    a.n_rows = n_rows;
    a.slots_end = (long)n_pages * page;
    a.pages = static_cast<uint16_t *>(pages);
    a.kv_new = static_cast<const uint16_t *>(kv_new);
    a.rows = rows;
    a.slots = slots;
    const OnDeviceOf device(stream);
    return from_hip(ecospec::launch_latent_append(a, (hipStream_t)stream));
}

moe_status_t moe_grouped_prompt_workspace_size(int D, size_t *bytes)
{
    if (!bytes || D < 1) return MOE_ERR_INVALID_ARG;
    if (D != 64 && D != 128) return MOE_ERR_UNSUPPORTED;
    *bytes = ecospec::grouped_prompt_workspace(D);
    return MOE_OK;
}

moe_status_t moe_grouped_prompt(const moe_grouped_prompt_t *p, void *o, float *lse, void *workspace,
                                size_t workspace_bytes, void *stream)
{
    if (!p || !o || !workspace || !p->q || !p->k || !p->v || !p->q_offsets || !p->kv_offsets) return MOE_ERR_INVALID_ARG;
    if (p->N < 1 || p->M < 1 || p->B < 1 || p->B > ecospec::kMaxSequences || p->max_tokens < 1) return MOE_ERR_INVALID_ARG;
    if (p->Hkv < 1 || p->Hkv > 256 || p->H < 1 || p->H > kMaxHeads || p->H % p->Hkv || p->D < 1) return MOE_ERR_INVALID_ARG;
    if (!isfinite(p->scale)) return MOE_ERR_INVALID_ARG;
    const void *ptr[] = {p->q, p->k, p->v, o};
    for (const void *x : ptr)
        if (!aligned(x, 16)) return MOE_ERR_INVALID_ARG;
    if (!aligned(workspace, 256) || !aligned(lse, 4)) return MOE_ERR_INVALID_ARG;
    const int64_t str[] = {p->q_stride, p->q_head, p->k_stride, p->k_head, p->v_stride, p->v_head};
    for (int64_t x : str)
        if (x < 0 || x % 8) return MOE_ERR_INVALID_ARG;
    if (p->k_stride > kMaxStride || p->v_stride > kMaxStride) return MOE_ERR_UNSUPPORTED;
    if (p->D != 64 && p->D != 128) return MOE_ERR_UNSUPPORTED;
    const int most = p->max_tokens < p->N ? p->max_tokens : p->N;
    if ((long)p->N * p->H > kMaxPromptRows || (long)p->B * p->H * most > kMaxPromptRows) return MOE_ERR_UNSUPPORTED;  // the grid
    if (workspace_bytes < ecospec::grouped_prompt_workspace(p->D)) return MOE_ERR_WORKSPACE;
    auto spans = [&](const void *x, int n, int64_t stride, int heads, int64_t head) {
        return Range{x, ((size_t)(n - 1) * stride + (size_t)(heads - 1) * head + p->D) * 2};
    };
    const size_t rows = (size_t)p->N * p->H, table = (size_t)(p->B + 1) * 4;
    const Range out[] = {{o, rows * p->D * 2}, {lse, rows * 4}, {workspace, ecospec::grouped_prompt_workspace(p->D)}};
    const Range in[] = {spans(p->q, p->N, p->q_stride, p->H, p->q_head), spans(p->k, p->M, p->k_stride, p->Hkv, p->k_head),
                        spans(p->v, p->M, p->v_stride, p->Hkv, p->v_head), {p->q_offsets, table}, {p->kv_offsets, table}};
    if (any_overlap(out, in)) return MOE_ERR_INVALID_ARG;
    ecospec::GroupedPromptArgs a{};
    a.N = p->N;
    a.M = p->M;
    a.B = p->B;
    a.H = p->H;
    a.Hkv = p->Hkv;
    a.max_tokens = most;
    a.q_offsets = p->q_offsets;
    a.kv_offsets = p->kv_offsets;
    a.q = static_cast<const uint16_t *>(p->q);
    a.k = static_cast<const uint16_t *>(p->k);
    a.v = static_cast<const uint16_t *>(p->v);
    a.q_stride = p->q_stride;
    a.q_head = p->q_head;
    a.k_stride = p->k_stride;
    a.k_head = p->k_head;
    a.v_stride = p->v_stride;
    a.v_head = p->v_head;
    a.scale = p->scale;
    a.o = static_cast<uint16_t *>(o);
    a.lse = lse;
    const OnDeviceOf device(stream);
    return from_hip(ecospec::launch_grouped_prompt(a, p->D, workspace, (hipStream_t)stream));
}

moe_status_t moe_token_logprobs_workspace_size(int N, size_t *bytes)
{
    if (!bytes || N < 1 || N > kMaxLogitRows) return MOE_ERR_INVALID_ARG;
    *bytes = ecospec::logprobs_workspace();
    return MOE_OK;
}

moe_status_t moe_token_logprobs(const void *logits, int dtype, int64_t stride, int N, int V, float scale,
                                const int32_t *tokens, int M, int k, float *logprob, float *lse, float *entropy,
                                int32_t *top_idx, float *top_logprob, void *workspace, size_t workspace_bytes,
                                void *stream)
{
    if (!logits || !workspace || N < 1 || N > kMaxLogitRows || V < 1 || V > kMaxVocabulary || stride < V)
        return MOE_ERR_INVALID_ARG;
    if (dtype != MOE_F32 && dtype != MOE_BF16) return MOE_ERR_INVALID_ARG;
    if (!isfinite(scale) || !(scale > 0.f)) return MOE_ERR_INVALID_ARG;
    if (k < 0 || k > kMaxTop || k > V || M < 0 || M > kMaxGiven || (long)N * M > 1L << 30) return MOE_ERR_INVALID_ARG;
    if ((M == 0) != (tokens == nullptr) || (M == 0) != (logprob == nullptr)) return MOE_ERR_INVALID_ARG;
    if ((k == 0) != (top_idx == nullptr) || (k == 0 && top_logprob)) return MOE_ERR_INVALID_ARG;
    if (!logprob && !lse && !entropy && !top_idx) return MOE_ERR_INVALID_ARG;
    if (!aligned(logits, dtype == MOE_BF16 ? 2 : 4) || !aligned(workspace, 256)) return MOE_ERR_INVALID_ARG;
    if (scale > kMaxScale) return MOE_ERR_UNSUPPORTED;
    if (workspace_bytes < ecospec::logprobs_workspace()) return MOE_ERR_WORKSPACE;
    const size_t n = N;
    const Range out[] = {{logprob, n * M * 4}, {lse, n * 4}, {entropy, n * 4}, {top_idx, n * k * 4}, {top_logprob, n * k * 4},
                         {workspace, ecospec::logprobs_workspace()}};
    const Range in[] = {{logits, ((n - 1) * (size_t)stride + V) * (dtype == MOE_BF16 ? 2 : 4)}, {tokens, n * M * 4}};
    if (any_overlap(out, in)) return MOE_ERR_INVALID_ARG;
    ecospec::LogprobArgs a{};
    a.logits = logits;
    a.stride = stride;
    a.N = N;
    a.V = V;
    a.M = M;
    a.k = k;
    a.scale = scale;
    a.tokens = tokens;
    a.logprob = logprob;
    a.lse = lse;
    a.entropy = entropy;
    a.top_logprob = top_logprob;
    a.top_idx = top_idx;
    const OnDeviceOf device(stream);
    return from_hip(ecospec::launch_token_logprobs(a, dtype == MOE_BF16, workspace, (hipStream_t)stream));
}

}  // extern "C"
