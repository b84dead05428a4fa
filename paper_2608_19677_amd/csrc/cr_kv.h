// Internal helpers of the paged key/value caches (cr_pages.hip, cr_kvq.hip, cr_attn.hip). Not part of the ABI.
#pragma once

#include "cr_common.h"

namespace cr {

// The cache as kernels take it: strides in elements of 2 bytes.
struct KvPages {
    const uint16_t* k;
    const uint16_t* v;
    int64_t layer_stride, page_stride, head_stride, token_stride;
    uint32_t heads, dim, log_tokens, num_pages, layers;
};

inline uint32_t log2_of(uint32_t p2) { return (uint32_t)__builtin_ctz(p2); }

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
inline bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

inline bool good_stride(int64_t s) { return s >= 0 && (s & 7) == 0 && s < ((int64_t)1 << 31); }

inline bool good_rows(const cr_rows& r)
{
    return r.p && aligned16(r.p) && good_stride(r.token_stride) && good_stride(r.head_stride);
}

// The scalars alone (for size queries) and the whole handle.
inline bool good_cache_sizes(const cr_kv_cache* c)
{
    return c && c->dtype <= CR_F16 && c->heads >= 1 && c->heads <= CR_MAX_HEADS && (c->dim == 64 || c->dim == 128) &&
           c->page_tokens >= 1 && c->page_tokens <= CR_MAX_PAGE_TOKENS && (c->page_tokens & (c->page_tokens - 1)) == 0 &&
           c->num_pages >= 1 && c->num_pages <= CR_MAX_PAGES && c->layers >= 1 && c->layers <= CR_MAX_LAYERS;
}

inline bool good_cache(const cr_kv_cache* c)
{
    return good_cache_sizes(c) && c->k && c->v && aligned16(c->k) && aligned16(c->v) && c->layer_stride >= 0 && (c->layer_stride & 7) == 0 &&
           good_stride(c->page_stride) && good_stride(c->head_stride) && good_stride(c->token_stride);
}

inline KvPages kv_pages(const cr_kv_cache* c)
{
    return KvPages{(const uint16_t*)c->k, (const uint16_t*)c->v, c->layer_stride, c->page_stride, c->head_stride,
                   c->token_stride, c->heads, c->dim, log2_of(c->page_tokens), c->num_pages, c->layers};
}

// The cache held in 8 bits. Scales go by pairs, the keys' exponent and the values'.
struct KvqPages {
    const uint8_t* k;
    const uint8_t* v;
    const uint16_t* scale;
    int64_t layer_stride, page_stride, head_stride, token_stride;  // in bytes
    uint32_t heads, dim, log_tokens, log_block, num_pages;
};

inline bool good_cache_sizes(const cr_kvq_cache* c)
{
    return c && c->dtype <= CR_F16 && c->code <= CR_E5M2 && c->heads >= 1 && c->heads <= CR_MAX_HEADS && (c->dim == 64 || c->dim == 128) &&
           c->page_tokens >= 1 && c->page_tokens <= CR_MAX_PAGE_TOKENS && (c->page_tokens & (c->page_tokens - 1)) == 0 &&
           c->block_tokens >= 1 && c->block_tokens <= CR_MAX_BLOCK_TOKENS && c->block_tokens <= c->page_tokens &&
           (c->block_tokens & (c->block_tokens - 1)) == 0 && c->num_pages >= 1 && c->num_pages <= CR_MAX_PAGES && c->layers >= 1 &&
           c->layers <= CR_MAX_LAYERS;
}

inline bool good_bytes(int64_t s) { return s >= 0 && (s & 15) == 0 && s < ((int64_t)1 << 31); }

inline bool good_cache(const cr_kvq_cache* c)
{
    return good_cache_sizes(c) && c->k && c->v && aligned16(c->k) && aligned16(c->v) && c->scale && ((uintptr_t)c->scale & 1u) == 0 &&
           c->layer_stride >= 0 && (c->layer_stride & 15) == 0 && good_bytes(c->page_stride) && good_bytes(c->head_stride) &&
           good_bytes(c->token_stride);
}

// Pairs of scales of a page, all heads, and of a layer.
inline uint32_t scales_of_page(const cr_kvq_cache* c) { return c->heads * (c->page_tokens / c->block_tokens); }
inline uint64_t scales_of_layer(const cr_kvq_cache* c) { return (uint64_t)c->num_pages * scales_of_page(c); }

inline KvqPages kvq_pages(const cr_kvq_cache* c, uint32_t layer)
{
    const int64_t at = (int64_t)layer * c->layer_stride;
    return KvqPages{(const uint8_t*)c->k + at, (const uint8_t*)c->v + at, (const uint16_t*)c->scale + layer * scales_of_layer(c),
                    c->layer_stride, c->page_stride, c->head_stride, c->token_stride, c->heads, c->dim, log2_of(c->page_tokens),
                    log2_of(c->block_tokens), c->num_pages};
}

// Place of the scales of a token of a page.
__device__ __forceinline__ uint64_t scale_at(uint32_t page, uint32_t heads, uint32_t head, uint32_t tok, uint32_t log_tokens, uint32_t log_block)
{
    return (((uint64_t)page * heads + head) << (log_tokens - log_block)) + (tok >> log_block);
}

// Pages of n tokens.
__host__ __device__ __forceinline__ uint32_t pages_of(uint32_t n, uint32_t log_tokens)
{
    return (n >> log_tokens) + ((n & ((1u << log_tokens) - 1u)) != 0u);
}

// Largest i in [0, n) with f(i) <= t, for f non-decreasing with f(0) <= t (otherwise an index in
// range); uniform over the wavefront. 64 places are looked at in one step, so up to 64
// sequences cost one load latency and 4,096 two.
template <typename F>
__device__ __forceinline__ uint32_t wave_find(uint32_t n, uint64_t t, F f)
{
    uint32_t lo = 0;
    while (n > 1) {
        const uint32_t step = (n + 63u) / 64u;
        const uint32_t at = lane_id() * step;
        const uint64_t m = ballot(at < n && f(lo + at) <= t);
        const uint32_t i = m ? 63u - (uint32_t)__builtin_clzll(m) : 0u;
        lo += i * step;
        n = min(step, n - i * step);
    }
    return lo;
}

}  // namespace cr
