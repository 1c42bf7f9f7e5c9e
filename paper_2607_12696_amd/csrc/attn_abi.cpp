// C ABI of the norm, the attention and the 8-bit cache: argument validation,
// then one launch sequence each.  No allocation, no synchronisation.
#include "ecospec_moe.h"

#include <hip/hip_runtime_api.h>
#include <math.h>

#include "attn.hpp"

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

bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

constexpr int kMaxBatch = 1024;
constexpr int kMaxHeads = 1024;
constexpr long kMaxRows = 1L << 24;  // query rows (token, head) of a call
constexpr int kMaxWidth = 16384;     // of a normalised row
constexpr int kMaxNormRows = 1 << 21;  // by 1024 threads: a launch's 2^31
constexpr long kMaxPromptRows = 1L << 30;
constexpr int64_t kMaxStride = 1L << 23;  // elements between a prompt's keys

bool page_ok(int page) { return page == 16 || page == 32 || page == 64 || page == 128; }

moe_status_t check_pages(int n_pages, int page, int max_blocks, const int32_t *table, const int32_t *len)
{
    if (!table || !len || n_pages < 1 || max_blocks < 1 || !page_ok(page)) return MOE_ERR_INVALID_ARG;
    if ((long)max_blocks * page > 1L << 30) return MOE_ERR_INVALID_ARG;  // positions are 32-bit
    return MOE_OK;
}

moe_status_t check_latent(const moe_latent_cache_t *c)
{
    if (!c || !c->pages || !aligned(c->pages, 16) || c->r < 1 || c->p < 0) return MOE_ERR_INVALID_ARG;
    const moe_status_t st = check_pages(c->n_pages, c->page, c->max_blocks, c->block_table, c->cache_len);
    if (st != MOE_OK) return st;
    return c->r == 512 && c->p == 64 ? MOE_OK : MOE_ERR_UNSUPPORTED;
}

moe_status_t check_cache(const moe_cache_t *c)
{
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || c->k == c->v) return MOE_ERR_INVALID_ARG;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || c->Hkv < 1 || c->Hkv > 256 || c->D < 1) return MOE_ERR_INVALID_ARG;
    const moe_status_t st = check_pages(c->n_pages, c->page, c->max_blocks, c->block_table, c->cache_len);
    if (st != MOE_OK) return st;
    return c->D == 64 || c->D == 128 ? MOE_OK : MOE_ERR_UNSUPPORTED;
}

moe_status_t check_call(int N, int B, int H)
{
    if (N < 1 || B < 1 || B > kMaxBatch || H < 1 || H > kMaxHeads || (long)N * H > kMaxRows) return MOE_ERR_INVALID_ARG;
    if (N > (long)ecospec::kMaxDrafts * B) return MOE_ERR_INVALID_ARG;  // some sequence has more than a mask names
    return MOE_OK;
}

void set_paged(ecospec::PagedArgs &a, const moe_drafts_t *d, int H, float scale, void *o, float *lse)
{
    a.N = d->N;
    a.B = d->B;
    a.H = H;
    a.token_offsets = d->token_offsets;
    a.mask = d->mask;
    a.scale = scale;
    a.o = static_cast<uint16_t *>(o);
    a.lse = lse;
}

// slots: null where places follow from block_table and cache_len.
moe_status_t append(const moe_cache_t *cache, const void *k_new, const void *v_new, int n_rows, const int32_t *rows, int N, int B,
                    const int32_t *token_offsets, int max_tokens, const int64_t *slots, void *stream)
{
    const moe_status_t st = check_cache(cache);
    if (st != MOE_OK) return st;
    if (!k_new || !v_new || !token_offsets || N < 1 || n_rows < 1 || B < 1 || B > kMaxBatch || max_tokens < 1)
        return MOE_ERR_INVALID_ARG;
    if (!rows && n_rows < N) return MOE_ERR_INVALID_ARG;
    if (!aligned(k_new, 16) || !aligned(v_new, 16)) return MOE_ERR_INVALID_ARG;
    ecospec::AppendArgs a{};
    a.N = N;
    a.B = B;
    a.n_rows = n_rows;
    a.max_tokens = max_tokens < N ? max_tokens : N;
    a.Hkv = cache->Hkv;
    a.D = cache->D;
    a.n_pages = cache->n_pages;
    a.page = cache->page;
    a.max_blocks = cache->max_blocks;
    a.k_new = static_cast<const uint16_t *>(k_new);
    a.v_new = static_cast<const uint16_t *>(v_new);
    a.rows = rows;
    a.token_offsets = token_offsets;
    a.slots = slots;
    a.block_table = cache->block_table;
    a.cache_len = cache->cache_len;
    a.k = cache->k;
    a.v = cache->v;
    a.k_scale = cache->k_scale;
    a.v_scale = cache->v_scale;
    if (!ecospec::cache_append_fits(a)) return MOE_ERR_UNSUPPORTED;
    return from_hip(ecospec::launch_cache_append(a, (hipStream_t)stream));
}

}  // namespace

extern "C" {

moe_status_t moe_add_rmsnorm(const void *x, const void *residual, const void *weight, int T, int d, float eps,
                             int qfmt, void *sum, void *y, void *q, void *scales, void *stream)
{
    if (!x || !weight || T < 1 || d < 1 || !(eps >= 0.f) || isinf(eps)) return MOE_ERR_INVALID_ARG;
    if (qfmt < MOE_Q_NONE || qfmt > MOE_Q_FP8_ROW) return MOE_ERR_INVALID_ARG;
    if ((qfmt == MOE_Q_NONE) != (q == nullptr) || (q == nullptr) != (scales == nullptr)) return MOE_ERR_INVALID_ARG;
    if (!sum && !y && !q) return MOE_ERR_INVALID_ARG;
    // A workgroup reads its row before it writes it, so only whole-buffer aliases of the inputs work.
    if (y && (y == residual || y == sum)) return MOE_ERR_INVALID_ARG;
    if (q && (q == x || q == residual || q == sum || q == y || q == scales)) return MOE_ERR_INVALID_ARG;
    const void *ptr[] = {x, residual, weight, sum, y, q};
    for (const void *p : ptr)
        if (!aligned(p, 16)) return MOE_ERR_INVALID_ARG;
    if (!aligned(scales, 4)) return MOE_ERR_INVALID_ARG;
    if (d % 32 || d > kMaxWidth || T > kMaxNormRows) return MOE_ERR_UNSUPPORTED;
    return from_hip(ecospec::launch_add_rmsnorm(
        static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(residual),
        static_cast<const uint16_t *>(weight), T, d, eps, qfmt, static_cast<uint16_t *>(sum),
        static_cast<uint16_t *>(y), static_cast<uint8_t *>(q), scales, (hipStream_t)stream));
}

moe_status_t moe_latent_attn_workspace_size(const moe_latent_cache_t *cache, int N, int B, int H, size_t *bytes)
{
    if (!bytes) return MOE_ERR_INVALID_ARG;
    moe_status_t st = check_latent(cache);
    if (st != MOE_OK) return st;
    if ((st = check_call(N, B, H)) != MOE_OK) return st;
    *bytes = ecospec::latent_workspace(N, B, H, cache->max_blocks, cache->page);
    return MOE_OK;
}

moe_status_t moe_latent_attn(const moe_latent_cache_t *cache, const moe_drafts_t *drafts, const void *q,
                             const void *kv_new, int H, float scale, void *o, float *lse, void *workspace,
                             size_t workspace_bytes, void *stream)
{
    if (!drafts || !drafts->token_offsets || !q || !kv_new || !o || !workspace || !isfinite(scale))
        return MOE_ERR_INVALID_ARG;
    moe_status_t st = check_latent(cache);
    if (st != MOE_OK) return st;
    if ((st = check_call(drafts->N, drafts->B, H)) != MOE_OK) return st;
    if (o == q || !aligned(q, 16) || !aligned(kv_new, 16) || !aligned(o, 16) || !aligned(workspace, 256))
        return MOE_ERR_INVALID_ARG;
    if (workspace_bytes < ecospec::latent_workspace(drafts->N, drafts->B, H, cache->max_blocks, cache->page)) return MOE_ERR_WORKSPACE;
    ecospec::LatentArgs a{};
    set_paged(a, drafts, H, scale, o, lse);
    a.n_pages = cache->n_pages;
    a.page = cache->page;
    a.max_blocks = cache->max_blocks;
    a.block_table = cache->block_table;
    a.cache_len = cache->cache_len;
    a.q = static_cast<const uint16_t *>(q);
    a.kv_new = static_cast<const uint16_t *>(kv_new);
    a.pages = static_cast<const uint16_t *>(cache->pages);
    return from_hip(ecospec::launch_latent_attn(a, workspace, (hipStream_t)stream));
}

moe_status_t moe_latent_prompt(const moe_prompt_t *p, void *o, float *lse, void *stream)
{
    if (!p || !o || !p->q || !p->k || !p->k_rope || !p->v || !p->q_offsets || !p->kv_offsets) return MOE_ERR_INVALID_ARG;
    if (p->N < 1 || p->M < 1 || p->B < 1 || p->B > kMaxBatch || p->H < 1 || p->H > kMaxHeads || p->max_tokens < 1)
        return MOE_ERR_INVALID_ARG;
    if (!isfinite(p->scale) || o == p->q || p->dn < 1 || p->p < 0 || p->dv < 1) return MOE_ERR_INVALID_ARG;
    const void *ptr[] = {p->q, p->k, p->k_rope, p->v, o};
    for (const void *x : ptr)
        if (!aligned(x, 16)) return MOE_ERR_INVALID_ARG;
    const int64_t str[] = {p->k_stride, p->k_head, p->v_stride, p->v_head};
    for (int64_t x : str)
        if (x < 0 || x % 8) return MOE_ERR_INVALID_ARG;
    // A tile of 64 keys is addressed through a 32-bit buffer range.
    if (p->k_stride > kMaxStride || p->v_stride > kMaxStride) return MOE_ERR_UNSUPPORTED;
    if (p->dn != 128 || p->p != 64 || p->dv != 128) return MOE_ERR_UNSUPPORTED;
    const long most = p->max_tokens < p->N ? p->max_tokens : p->N;
    if ((long)p->N * p->H > kMaxPromptRows || (long)p->B * p->H * most > kMaxPromptRows) return MOE_ERR_UNSUPPORTED;  // the grid
    ecospec::PromptArgs a{};
    a.N = p->N;
    a.M = p->M;
    a.B = p->B;
    a.H = p->H;
    a.max_tokens = p->max_tokens < p->N ? p->max_tokens : p->N;
    a.q_offsets = p->q_offsets;
    a.kv_offsets = p->kv_offsets;
    a.q = static_cast<const uint16_t *>(p->q);
    a.k = static_cast<const uint16_t *>(p->k);
    a.k_rope = static_cast<const uint16_t *>(p->k_rope);
    a.v = static_cast<const uint16_t *>(p->v);
    a.k_stride = p->k_stride;
    a.k_head = p->k_head;
    a.v_stride = p->v_stride;
    a.v_head = p->v_head;
    a.scale = p->scale;
    a.o = static_cast<uint16_t *>(o);
    a.lse = lse;
    return from_hip(ecospec::launch_latent_prompt(a, (hipStream_t)stream));
}

moe_status_t moe_cache_append(const moe_cache_t *cache, const void *k_new, const void *v_new, int n_rows,
                              const int32_t *rows, int N, int B, const int32_t *token_offsets, int max_tokens,
                              void *stream)
{
    return append(cache, k_new, v_new, n_rows, rows, N, B, token_offsets, max_tokens, nullptr, stream);
}

moe_status_t moe_cache_append_slots(const moe_cache_t *cache, const void *k_new, const void *v_new, int n_rows,
                                    const int32_t *rows, int N, int B, const int32_t *token_offsets, int max_tokens,
                                    const int64_t *slots, void *stream)
{
    if (!slots || !aligned(slots, 8)) return MOE_ERR_INVALID_ARG;
    return append(cache, k_new, v_new, n_rows, rows, N, B, token_offsets, max_tokens, slots, stream);
}

moe_status_t moe_cache_attn_workspace_size(const moe_cache_t *cache, int N, int B, int H, size_t *bytes)
{
    if (!bytes) return MOE_ERR_INVALID_ARG;
    moe_status_t st = check_cache(cache);
    if (st != MOE_OK) return st;
    if ((st = check_call(N, B, H)) != MOE_OK) return st;
    if (H % cache->Hkv) return MOE_ERR_INVALID_ARG;
    *bytes = ecospec::cache_workspace(N, B, H, cache->Hkv, cache->D);
    return MOE_OK;
}

moe_status_t moe_cache_attn(const moe_cache_t *cache, const moe_drafts_t *drafts, const void *q, const void *k_new,
                            const void *v_new, int H, float scale, void *o, float *lse, void *workspace,
                            size_t workspace_bytes, void *stream)
{
    if (!drafts || !drafts->token_offsets || !q || !k_new || !v_new || !o || !workspace || !isfinite(scale))
        return MOE_ERR_INVALID_ARG;
    moe_status_t st = check_cache(cache);
    if (st != MOE_OK) return st;
    if ((st = check_call(drafts->N, drafts->B, H)) != MOE_OK) return st;
    if (H % cache->Hkv) return MOE_ERR_INVALID_ARG;
    if (o == q || !aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(o, 16) ||
        !aligned(workspace, 256))
        return MOE_ERR_INVALID_ARG;
    if (workspace_bytes < ecospec::cache_workspace(drafts->N, drafts->B, H, cache->Hkv, cache->D))
        return MOE_ERR_WORKSPACE;
    ecospec::CacheArgs a{};
    set_paged(a, drafts, H, scale, o, lse);
    a.n_pages = cache->n_pages;
    a.page = cache->page;
    a.max_blocks = cache->max_blocks;
    a.block_table = cache->block_table;
    a.cache_len = cache->cache_len;
    a.Hkv = cache->Hkv;
    a.D = cache->D;
    a.q = static_cast<const uint16_t *>(q);
    a.k_new = static_cast<const uint16_t *>(k_new);
    a.v_new = static_cast<const uint16_t *>(v_new);
    a.k = cache->k;
    a.v = cache->v;
    a.k_scale = cache->k_scale;
    a.v_scale = cache->v_scale;
    return from_hip(ecospec::launch_cache_attn(a, workspace, (hipStream_t)stream));
}

}  // extern "C"
