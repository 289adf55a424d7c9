// libmmvseg: the calls on a paged cache of 8-bit values with a scale for each block of slots and head (include/mmvseg.h): append, reading
// back, attention of single tokens.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "mmvseg.h"

#include "values.h"
#include "block_cache.h"
#include "paged_attention.h"
#include "call_checks.h"
#include "attention_host.h"
#include "block_host.h"

extern "C" {

mmv_status mmv_block_append(uint64_t tokens, const void *d_k, uint64_t k_stride, const void *d_v, uint64_t v_stride, mmv_type type,
                            const int64_t *d_slots, const mmv_block_cache *cache, void *hip_stream) {
    if (const mmv_status st = check_block_cache(cache)) return st;
    if (!valid_value_type(type) || tokens >= kMostAppended) return MMV_ERR_INVALID_ARG;
    const uint64_t values = (uint64_t)cache->heads * cache->dim;
    if ((tokens > 1 && (k_stride < values || v_stride < values)) || k_stride % 8 || v_stride % 8) return MMV_ERR_INVALID_ARG;
    if (tokens == 0) return MMV_OK;
    if (!d_k || !d_v || !d_slots) return MMV_ERR_NULL;
    if (!aligned_to(d_k, 16) || !aligned_to(d_v, 16) || !aligned_to(d_slots, 8)) return MMV_ERR_INVALID_ARG;
    if (cache->pages == 0) return MMV_OK;
    BlockAppendParams P = {};
    P.c = block_cache_params(*cache);
    P.x[0] = d_k, P.x[1] = d_v, P.stride[0] = k_stride, P.stride[1] = v_stride, P.slots = d_slots, P.tokens = (uint32_t)tokens;
    return block_append_call(P, type, cache->type == MMV_TYPE_I8, (hipStream_t)hip_stream);
}

mmv_status mmv_block_read(uint64_t n, uint64_t tokens, const int32_t *d_offsets, const int32_t *d_first, const int32_t *d_table, uint64_t table_width,
                          uint64_t table_stride, const mmv_block_cache *cache, mmv_type type, void *d_k, uint64_t k_stride, void *d_v, uint64_t v_stride,
                          void *hip_stream) {
    if (const mmv_status st = check_block_cache(cache)) return st;
    if (!valid_value_type(type) || n >= kMostRequests || tokens >= k2to31 || table_width >= k2to31 || (n > 1 && table_stride < table_width)) return MMV_ERR_INVALID_ARG;
    const uint64_t values = (uint64_t)cache->heads * cache->dim;
    if ((tokens > 1 && (k_stride < values || v_stride < values)) || k_stride % 8 || v_stride % 8) return MMV_ERR_INVALID_ARG;
    if (n == 0 || tokens == 0) return MMV_OK;
    if (!d_offsets || (!d_table && table_width) || !d_k || !d_v) return MMV_ERR_NULL;
    if (!aligned_to(d_offsets, 4) || !aligned_to(d_first, 4) || !aligned_to(d_table, 4) || !aligned_to(d_k, 16) || !aligned_to(d_v, 16)) return MMV_ERR_INVALID_ARG;
    BlockReadParams P = {};
    P.c = block_cache_params(*cache);
    P.offsets = d_offsets, P.first = d_first, P.table = d_table, P.table_stride = table_stride, P.table_width = (uint32_t)table_width;
    P.n = (uint32_t)n, P.tokens = (uint32_t)tokens, P.token_pieces = (uint32_t)(values / 8), P.page = divider(cache->page);
    P.k = d_k, P.v = d_v, P.k_stride = k_stride, P.v_stride = v_stride;
    return block_read_call(P, type, cache->type == MMV_TYPE_I8, (hipStream_t)hip_stream);
}

mmv_status mmv_block_attention(uint64_t n, uint32_t q_heads, const void *d_q, uint64_t q_stride, mmv_type type, const mmv_block_cache *cache,
                               const int32_t *d_table, uint64_t table_width, uint64_t table_stride, const int32_t *d_context, float scale, uint32_t window,
                               void *d_out, float *d_lse, void *d_ws, size_t ws_bytes, void *hip_stream) {
    if (const mmv_status st = check_block_cache(cache)) return st;
    if (!valid_value_type(type) || table_width >= k2to31 || !attention_sizes(n, q_heads, cache->heads, cache->dim, table_width * cache->page) ||
        (n > 1 && table_stride < table_width) || q_stride % 8 || (n > 1 && q_stride < (uint64_t)q_heads * cache->dim))
        return MMV_ERR_INVALID_ARG;
    if (n == 0) return MMV_OK;
    if (!d_q || (!d_table && table_width) || !d_context || !d_out) return MMV_ERR_NULL;
    if (!aligned_to(d_q, 16) || !aligned_to(d_out, 16) || !aligned_to(d_table, 4) || !aligned_to(d_context, 4) || !aligned_to(d_lse, 4)) return MMV_ERR_INVALID_ARG;
    if (const mmv_status st = check_workspace(d_ws, ws_bytes, attention_workspace(n, q_heads, cache->heads, cache->dim, table_width * cache->page))) return st;
    AttentionParams P = {};
    P.q = d_q, P.k = cache->d_k, P.v = cache->d_v, P.q_stride = q_stride;
    P.page_stride = (uint32_t)cache->page_stride, P.head_stride = cache->head_stride, P.slot_stride = (uint32_t)cache->slot_stride;
    P.table = d_table, P.context = d_context, P.table_stride = table_stride;
    P.max_context = cache->pages ? (uint32_t)(table_width * cache->page) : 0u;   // (no pages: nothing to look at)
    P.out = d_out, P.lse = d_lse;
    P.n = (uint32_t)n, P.q_heads = q_heads, P.heads = cache->heads, P.group = q_heads / cache->heads, P.dim = cache->dim;
    P.page = cache->page, P.pages = (uint32_t)cache->pages, P.window = window;
    P.block_groups = divider(cache->block / 8), P.head_scales = cache->page / cache->block, P.k_scales = cache->d_k_scales, P.v_scales = cache->d_v_scales;
    P.score_by = scale * kLog2e, P.out_by = 1.f;
    return block_attention_over(P, type, cache->type, d_ws, (hipStream_t)hip_stream);
}

}  // extern "C"
