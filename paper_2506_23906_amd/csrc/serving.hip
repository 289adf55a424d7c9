// libmmvseg: the calls of a serving step over a ragged batch (include/mmvseg.h): page tables and slots, cache append,
// attention of single tokens over a paged cache, linear attention with decay over prompts and for single tokens.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mmvseg.h"

#include "values.h"
#include "pages.h"
#include "paged_attention.h"
#include "decay.h"
#include "serving_host.h"

extern "C" {

size_t mmv_page_tables_workspace_bytes(uint64_t n) { return n < kMostRequests ? tables_workspace(n) : 0; }

mmv_status mmv_page_tables(uint64_t n, const int32_t *d_cached, const int32_t *d_new, const int32_t *d_free, uint64_t free_count,
                           int32_t *d_table, uint64_t table_width, uint64_t table_stride, uint32_t page, uint64_t max_tokens,
                           int32_t *d_offsets, int32_t *d_context, int64_t *d_slots, int32_t *d_positions, int64_t *d_used,
                           void *d_ws, size_t ws_bytes, void *hip_stream) {
    if (n >= kMostRequests || max_tokens >= k2to31 || free_count >= k2to31 || table_width >= k2to31 || page < 1 || page > 65536 || (n > 1 && table_stride < table_width))
        return MMV_ERR_INVALID_ARG;
    if (!d_offsets || !d_used || (n && (!d_cached || !d_new || !d_context)) || (free_count && !d_free) || (n && table_width && !d_table) ||
        (max_tokens && (!d_slots || !d_positions)))
        return MMV_ERR_NULL;
    for (const void *p : {(const void *)d_cached, (const void *)d_new, (const void *)d_free, (const void *)d_table, (const void *)d_offsets, (const void *)d_context, (const void *)d_positions})
        if (!aligned_to(p, 4)) return MMV_ERR_INVALID_ARG;
    if (!aligned_to(d_slots, 8) || !aligned_to(d_used, 8)) return MMV_ERR_INVALID_ARG;
    if (const mmv_status st = check_workspace(d_ws, ws_bytes, tables_workspace(n))) return st;
    TablesParams P = {};
    P.n = (uint32_t)n, P.page = divider(page), P.max_tokens = (uint32_t)max_tokens, P.free_count = (uint32_t)free_count;
    P.table_width = d_table ? (uint32_t)table_width : 0u, P.table_stride = table_stride;
    P.cached = d_cached, P.fresh = d_new, P.free_pages = d_free, P.table = d_table;
    P.offsets = d_offsets, P.context = d_context, P.positions = d_positions, P.slots = d_slots, P.used = d_used;
    return tables_call(P, d_ws, (hipStream_t)hip_stream);
}

mmv_status mmv_cache_append(uint64_t tokens, const void *d_k, uint64_t k_stride, const void *d_v, uint64_t v_stride, mmv_type type,
                            const int64_t *d_slots, const mmv_paged_cache *cache, void *hip_stream) {
    if (const mmv_status st = check_cache(cache, type)) return st;
    if (tokens >= k2to31) return MMV_ERR_INVALID_ARG;
    const uint64_t values = (uint64_t)cache->heads * cache->dim;
    if (tokens > 1 && (k_stride < values || v_stride < values)) return MMV_ERR_INVALID_ARG;
    if (k_stride % 8 || v_stride % 8) return MMV_ERR_INVALID_ARG;
    if (tokens == 0) return MMV_OK;
    if (!d_k || !d_v || !d_slots) return MMV_ERR_NULL;
    if (!aligned_to(d_k, 16) || !aligned_to(d_v, 16) || !aligned_to(d_slots, 8)) return MMV_ERR_INVALID_ARG;
    if (cache->pages == 0) return MMV_OK;
    return append_call(tokens, d_k, k_stride, d_v, v_stride, type, d_slots, *cache, (hipStream_t)hip_stream);
}

size_t mmv_paged_attention_workspace_bytes(uint64_t n, uint32_t q_heads, uint32_t heads, uint32_t dim, uint64_t max_context) {
    if (!attention_sizes(n, q_heads, heads, dim, max_context)) return 0;
    return attention_workspace(n, q_heads, heads, dim, max_context);
}

mmv_status mmv_paged_attention(uint64_t n, uint32_t q_heads, const void *d_q, uint64_t q_stride, mmv_type type,
                               const mmv_paged_cache *cache, const int32_t *d_table, uint64_t table_width, uint64_t table_stride,
                               const int32_t *d_context, float scale, uint32_t window, void *d_out, float *d_lse,
                               void *d_ws, size_t ws_bytes, void *hip_stream) {
    if (const mmv_status st = check_cache(cache, type)) return st;
    if (table_width >= k2to31 || !attention_sizes(n, q_heads, cache->heads, cache->dim, table_width * cache->page) || (n > 1 && table_stride < table_width) ||
        q_stride % 8 || (n > 1 && q_stride < (uint64_t)q_heads * cache->dim))
        return MMV_ERR_INVALID_ARG;
    if (cache->page % 8) return MMV_ERR_UNSUPPORTED;
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
    P.score_by = scale * cache->k_scale * kLog2e, P.out_by = cache->v_scale;
    return attention_call(P, type, cache->type, d_ws, (hipStream_t)hip_stream);
}

size_t mmv_decay_attention_workspace_bytes(uint64_t n, uint64_t tokens, uint32_t heads, uint32_t dk, uint32_t dv) {
    if (!decay_sizes(n, tokens, heads, heads, dk, dv)) return 0;
    return decay_workspace(n, tokens, heads, dk, dv);
}

mmv_status mmv_decay_attention(uint64_t n, uint64_t tokens, uint32_t heads, uint32_t kv_heads, uint32_t dk, uint32_t dv,
                               const void *d_q, uint64_t q_stride, const void *d_k, uint64_t k_stride, const void *d_v, uint64_t v_stride,
                               mmv_type type, const int32_t *d_offsets, const float *d_log_decay, float scale,
                               const float *d_state_in, float *d_state_out, uint64_t states, const int32_t *d_state_index,
                               void *d_out, void *d_ws, size_t ws_bytes, void *hip_stream) {
    if (!decay_sizes(n, tokens, heads, kv_heads, dk, dv)) return MMV_ERR_INVALID_ARG;
    DecayParams P = {};
    if (const mmv_status st = decay_params(P, n, tokens, heads, kv_heads, dk, dv, d_q, q_stride, d_k, k_stride, d_v, v_stride, type, d_log_decay, scale, d_state_in,
                                           d_state_out, states, d_state_index, d_out))
        return st;
    if (n == 0) return MMV_OK;
    if (!d_offsets) return MMV_ERR_NULL;
    if (!aligned_to(d_offsets, 4)) return MMV_ERR_INVALID_ARG;
    if (const mmv_status st = check_workspace(d_ws, ws_bytes, decay_workspace(n, tokens, heads, dk, dv))) return st;
    P.offsets = d_offsets;
    return decay_call(P, type, d_ws, (hipStream_t)hip_stream);
}

mmv_status mmv_decay_step(uint64_t n, uint32_t heads, uint32_t kv_heads, uint32_t dk, uint32_t dv,
                          const void *d_q, uint64_t q_stride, const void *d_k, uint64_t k_stride, const void *d_v, uint64_t v_stride,
                          mmv_type type, const float *d_log_decay, float scale,
                          const float *d_state_in, float *d_state_out, uint64_t states, const int32_t *d_state_index,
                          void *d_out, void *hip_stream) {
    if (!decay_sizes(n, n, heads, kv_heads, dk, dv)) return MMV_ERR_INVALID_ARG;
    DecayParams P = {};
    if (const mmv_status st = decay_params(P, n, n, heads, kv_heads, dk, dv, d_q, q_stride, d_k, k_stride, d_v, v_stride, type, d_log_decay, scale, d_state_in, d_state_out,
                                           states, d_state_index, d_out))
        return st;
    if (n == 0) return MMV_OK;
    return decay_step_call(P, type, (hipStream_t)hip_stream);
}

}  // extern "C"
