// libmmvseg, part of the translation unit serving.hip (included there, in order).
// Host side of a serving step's calls: argument checks, workspaces, launches.
#pragma once

namespace {

constexpr uint64_t k2to31 = 1ull << 31;
constexpr uint64_t kMostRequests = 1ull << 22;
constexpr uint32_t kMostHeads = 1024;

inline uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
inline size_t round256(size_t b) { return (b + 255) & ~(size_t)255; }
inline bool aligned_to(const void *p, uintptr_t by) { return (uintptr_t)p % by == 0; }
inline mmv_status launched() { return hipGetLastError() == hipSuccess ? MMV_OK : MMV_ERR_HIP; }
inline bool valid_value_type(int t) { return t == MMV_TYPE_F16 || t == MMV_TYPE_BF16; }
inline mmv_status check_workspace(const void *ws, size_t bytes, size_t needed) {
    if (!needed) return MMV_OK;
    if (!ws) return MMV_ERR_NULL;
    return ((uintptr_t)ws & 255u) || bytes < needed ? MMV_ERR_WORKSPACE : MMV_OK;
}

inline size_t tables_workspace(uint64_t n) { return n <= kTablesLocal ? 0 : round256(8 * n); }

// The cache itself, and that values of `type` can go into it and be multiplied with it.
inline mmv_status check_cache(const mmv_paged_cache *c, int type) {
    if (!c) return MMV_ERR_NULL;
    const int own = c->type;
    if (!valid_value_type(type) || (own != MMV_TYPE_E4M3 && own != type)) return MMV_ERR_INVALID_ARG;
    if (c->page < 1 || c->page > 65536 || c->heads < 1 || c->heads > kMostHeads || c->dim < 8 || c->dim > 256 || c->dim % 8) return MMV_ERR_INVALID_ARG;
    if (c->pages >= k2to31 || c->pages * c->page >= k2to31 || c->page_stride % 8 || c->head_stride % 8 || c->slot_stride % 8) return MMV_ERR_INVALID_ARG;
    // (the largest offset, in bytes, of a cache of 2^31 slots is far below 2^63: strides up to 2^30 are sense)
    if (c->page_stride > (1ull << 40) || c->head_stride > (1ull << 40) || c->slot_stride > (1ull << 40)) return MMV_ERR_INVALID_ARG;
    if (own == MMV_TYPE_E4M3 ? !(c->k_scale > 0.f && c->v_scale > 0.f && c->k_scale < INFINITY && c->v_scale < INFINITY) : !(c->k_scale == 1.f && c->v_scale == 1.f)) return MMV_ERR_INVALID_ARG;
    if (c->pages && (!c->d_k || !c->d_v)) return MMV_ERR_NULL;
    return aligned_to(c->d_k, 16) && aligned_to(c->d_v, 16) ? MMV_OK : MMV_ERR_INVALID_ARG;
}

mmv_status append_call(uint64_t tokens, const void *k, uint64_t k_stride, const void *v, uint64_t v_stride, int type, const int64_t *slots,
                       const mmv_paged_cache &c, hipStream_t s) {
    AppendParams P = {};
    P.k = k, P.v = v, P.k_stride = k_stride, P.v_stride = v_stride, P.slots = slots;
    P.cache_k = c.d_k, P.cache_v = c.d_v, P.page_stride = c.page_stride, P.head_stride = c.head_stride, P.slot_stride = c.slot_stride;
    P.page = c.page, P.num_slots = (uint32_t)(c.pages * c.page), P.head_pieces = c.dim / 8, P.pieces = c.heads * P.head_pieces;
    P.total = tokens * P.pieces;
    P.k_by = (float)(1.0 / c.k_scale), P.v_by = (float)(1.0 / c.v_scale);
    const uint64_t blocks = ceil_div(P.total, 256);
    if (blocks >= k2to31) return MMV_ERR_INVALID_ARG;
    if (c.type == MMV_TYPE_E4M3) {
        if (type == MMV_TYPE_F16) cache_append_kernel<f16_t, true><<<(unsigned)blocks, 256, 0, s>>>(P);
        else cache_append_kernel<bf16_t, true><<<(unsigned)blocks, 256, 0, s>>>(P);
    } else {
        cache_append_kernel<bf16_t, false><<<(unsigned)blocks, 256, 0, s>>>(P);   // (bits are copied: one kernel for both types)
    }
    return launched();
}

inline bool attention_sizes(uint64_t n, uint32_t q_heads, uint32_t heads, uint32_t dim, uint64_t max_context) {
    return n < kMostRequests && heads >= 1 && heads <= kMostHeads && q_heads >= heads && q_heads % heads == 0 && q_heads / heads <= 16 && dim >= 8 && dim <= 256 && dim % 8 == 0 &&
           max_context < k2to31 && n * q_heads < k2to31;
}
inline size_t attention_workspace(uint64_t, uint32_t, uint32_t, uint32_t, uint64_t) { return 0; }
mmv_status attention_call(const AttentionParams &P, int type, int cache_type, void *, hipStream_t s) {
    const unsigned blocks = P.n * P.q_heads;
    if (type == MMV_TYPE_F16) {
        if (cache_type == MMV_TYPE_E4M3) paged_attention_kernel<f16_t, e4m3_t><<<blocks, 64, 0, s>>>(P);
        else paged_attention_kernel<f16_t, f16_t><<<blocks, 64, 0, s>>>(P);
    } else {
        if (cache_type == MMV_TYPE_E4M3) paged_attention_kernel<bf16_t, e4m3_t><<<blocks, 64, 0, s>>>(P);
        else paged_attention_kernel<bf16_t, bf16_t><<<blocks, 64, 0, s>>>(P);
    }
    return launched();
}

inline bool decay_sizes(uint64_t n, uint64_t tokens, uint32_t heads, uint32_t kv_heads, uint32_t dk, uint32_t dv) {
    return n < kMostRequests && tokens < k2to31 && heads >= 1 && heads <= kMostHeads && kv_heads >= 1 && kv_heads <= heads && heads % kv_heads == 0 && dk >= 8 && dk <= kMostDk &&
           dk % 8 == 0 && dv >= 8 && dv <= kMostDv && dv % 8 == 0 && n * heads < k2to31;
}
mmv_status decay_params(DecayParams &P, uint64_t n, uint64_t tokens, uint32_t heads, uint32_t kv_heads, uint32_t dk, uint32_t dv, const void *q, uint64_t q_stride, const void *k,
                        uint64_t k_stride, const void *v, uint64_t v_stride, int type, const float *log_decay, float scale, const float *state_in, float *state_out,
                        uint64_t states, const int32_t *state_index, void *out) {
    if (!valid_value_type(type) || states >= k2to31 || q_stride % 8 || k_stride % 8 || v_stride % 8) return MMV_ERR_INVALID_ARG;
    if (tokens > 1 && (q_stride < (uint64_t)heads * dk || k_stride < (uint64_t)kv_heads * dk || v_stride < (uint64_t)kv_heads * dv)) return MMV_ERR_INVALID_ARG;
    if (!state_index && (state_in || state_out) && states < n) return MMV_ERR_INVALID_ARG;
    if (tokens && n && (!q || !k || !v || !out)) return MMV_ERR_NULL;
    if (n && !log_decay) return MMV_ERR_NULL;
    for (const void *p : {q, k, v, (const void *)out, (const void *)state_in, (const void *)state_out})
        if (!aligned_to(p, 16)) return MMV_ERR_INVALID_ARG;
    if (!aligned_to(log_decay, 4) || !aligned_to(state_index, 4)) return MMV_ERR_INVALID_ARG;
    const uint64_t bytes = states * heads * dk * dv * 4;
    if (state_in && state_out && state_in != state_out && (uintptr_t)state_in < (uintptr_t)state_out + bytes && (uintptr_t)state_out < (uintptr_t)state_in + bytes)
        return MMV_ERR_INVALID_ARG;
    P.q = q, P.k = k, P.v = v, P.q_stride = q_stride, P.k_stride = k_stride, P.v_stride = v_stride, P.tokens = tokens;
    P.log_decay = log_decay, P.state_in = state_in, P.state_out = state_out, P.state_index = state_index, P.states = states, P.out = out;
    P.n = (uint32_t)n, P.heads = heads, P.group = heads / kv_heads, P.dk = dk, P.dv = dv, P.scale = scale;
    return MMV_OK;
}
inline size_t decay_workspace(uint64_t, uint64_t, uint32_t, uint32_t, uint32_t) { return 0; }
mmv_status decay_call(const DecayParams &P, int type, void *, hipStream_t s) {
    if (type == MMV_TYPE_F16) decay_kernel<f16_t><<<P.n * P.heads, kMostDv, 0, s>>>(P);
    else decay_kernel<bf16_t><<<P.n * P.heads, kMostDv, 0, s>>>(P);
    return launched();
}
mmv_status decay_step_call(const DecayParams &P, int type, hipStream_t s) { return decay_call(P, type, nullptr, s); }

}  // namespace
