// The paged cache as the kernels see it, and the host's checks of what describes it: shared by sp_cache_append and
// sp_attend.
#pragma once

#include "sp_common.hpp"

namespace sp {

constexpr int kCacheBlock = SP_CACHE_BLOCK;

// One layer's pools behind a block table. Strides in elements.
struct CacheView {
    const int32_t *table;       // [B][table_stride]
    int64_t table_stride;
    int64_t n_pages, page_tokens, page_stride, stride_head, stride_token;
    int32_t n_q_heads, n_kv_heads, group;
};

inline bool cache_is_e4m3(const sp_cache_desc &d) { return d.cache_type == SP_CACHE_E4M3; }

inline sp_status check_cache(const sp_cache_desc *d)
{
    if (!d) return fail(SP_ERR_INVALID_ARG, "desc is null");
    if (d->n_q_heads < 1 || d->n_kv_heads < 1 || d->n_q_heads % d->n_kv_heads != 0)
        return fail(SP_ERR_INVALID_ARG, "n_q_heads = %d must be a positive multiple of n_kv_heads = %d", d->n_q_heads, d->n_kv_heads);
    if (d->cache_type != SP_CACHE_BF16 && d->cache_type != SP_CACHE_E4M3)
        return fail(SP_ERR_INVALID_ARG, "cache_type = %d is neither SP_CACHE_BF16 nor SP_CACHE_E4M3", d->cache_type);
    if (d->head_dim != 64 && d->head_dim != 128) return fail(SP_ERR_UNSUPPORTED, "head_dim = %d is neither 64 nor 128", d->head_dim);
    if (d->n_q_heads / d->n_kv_heads > 16)
        return fail(SP_ERR_UNSUPPORTED, "%d query heads share a kv head, at most 16 are supported", d->n_q_heads / d->n_kv_heads);
    if (d->n_kv_heads > 4096) return fail(SP_ERR_UNSUPPORTED, "n_kv_heads = %d exceeds 4096", d->n_kv_heads);
    if (d->n_pages < 1 || d->n_pages >= (int64_t(1) << 31))
        return fail(SP_ERR_INVALID_ARG, "n_pages = %lld outside 1..2^31-1", (long long)d->n_pages);
    if (d->page_tokens < 1 || d->page_tokens % kCacheBlock != 0 || d->page_tokens > (1 << 24))
        return fail(SP_ERR_INVALID_ARG, "page_tokens = %lld is not a positive multiple of %d of at most 2^24",
                    (long long)d->page_tokens, kCacheBlock);
    const int64_t unit = cache_is_e4m3(*d) ? 16 : 8, most = int64_t(1) << 40;
    const int64_t strides[3] = {d->page_stride, d->stride_head, d->stride_token};
    for (int64_t s : strides)
        if (s < 0 || s > most || s % unit != 0)
            return fail(SP_ERR_INVALID_ARG, "cache stride %lld is not a multiple of %lld elements in 0..2^40", (long long)s,
                        (long long)unit);
    if (d->stride_token < d->head_dim)
        return fail(SP_ERR_INVALID_ARG, "stride_token = %lld is less than head_dim = %d", (long long)d->stride_token, d->head_dim);
    if (d->stride_token > (1 << 24))
        return fail(SP_ERR_INVALID_ARG, "stride_token = %lld exceeds 2^24", (long long)d->stride_token);
    if (d->n_kv_heads > 1 && d->stride_head < d->head_dim)
        return fail(SP_ERR_INVALID_ARG, "stride_head = %lld is less than head_dim = %d", (long long)d->stride_head, d->head_dim);
    if (d->n_pages > 1 && d->page_stride < d->head_dim)
        return fail(SP_ERR_INVALID_ARG, "page_stride = %lld is less than head_dim = %d", (long long)d->page_stride, d->head_dim);
    return SP_OK;
}

// Pointers of the pools and their scales.
inline sp_status check_pools(const sp_cache_desc &d, const void *k, const void *v, const float *ks, const float *vs)
{
    if (!k || !v) return fail(SP_ERR_INVALID_ARG, "k_pool_dev or v_pool_dev is null");
    if ((uintptr_t)k % 16 != 0 || (uintptr_t)v % 16 != 0) return fail(SP_ERR_INVALID_ARG, "cache pools must be 16-byte aligned");
    if (cache_is_e4m3(d)) {
        if (!ks || !vs) return fail(SP_ERR_INVALID_ARG, "an E4M3 cache needs k_scale_dev and v_scale_dev");
        if ((uintptr_t)ks % 4 != 0 || (uintptr_t)vs % 4 != 0) return fail(SP_ERR_INVALID_ARG, "scales must be 4-byte aligned");
    }
    return SP_OK;
}

// offsets_host[0 .. B]; *total = offsets[B], *longest = the most tokens of one request.
inline sp_status check_ragged(const int64_t *off, int32_t B, int64_t *total, int64_t *longest)
{
    if (B < 0 || B > 4096) return fail(SP_ERR_INVALID_ARG, "B = %d outside 0..4096", B);
    if (!off) return fail(SP_ERR_INVALID_ARG, "offsets_host is null");
    if (off[0] != 0) return fail(SP_ERR_INVALID_ARG, "offsets_host[0] = %lld must be 0", (long long)off[0]);
    int64_t most = 0;
    for (int32_t b = 0; b < B; ++b) {
        if (off[b + 1] < off[b]) return fail(SP_ERR_INVALID_ARG, "offsets_host decreases at %d", b + 1);
        const int64_t n = off[b + 1] - off[b];
        most = n > most ? n : most;
    }
    if (off[B] >= (int64_t(1) << 31)) return fail(SP_ERR_INVALID_ARG, "%lld rows exceed 2^31-1", (long long)off[B]);
    *total = off[B];
    *longest = most;
    return SP_OK;
}

inline CacheView view_of(const sp_cache_desc &d, const int32_t *table, int64_t table_stride)
{
    return {table, table_stride, d.n_pages, d.page_tokens, d.page_stride, d.stride_head, d.stride_token,
            d.n_q_heads, d.n_kv_heads, d.n_q_heads / d.n_kv_heads};
}

}  // namespace sp
