// libmmvseg, part of the translation unit serving.hip (included there, in order).
// Attention of one token per row over a paged cache.
#pragma once

namespace {

struct AttentionParams {
    const void *q, *k, *v;
    uint64_t q_stride;                             // elements
    uint64_t page_stride, head_stride, slot_stride;
    const int32_t *table, *context;
    uint64_t table_stride, max_context;
    void *out;
    float *lse;
    uint32_t n, q_heads, heads, group, dim, page, pages, window;
    float score_by, out_by;
};

// One wave for a row and query head: a lane takes a position for the scores, then four components of the output.
template <typename T, typename C> __global__ __launch_bounds__(64) void paged_attention_kernel(AttentionParams P) {
    __shared__ float query[256], weight[64];
    __shared__ uint64_t at_lds[64];
    const uint32_t row = blockIdx.x / P.q_heads, qh = blockIdx.x % P.q_heads, lane = threadIdx.x;
    const T *q = (const T *)P.q + row * P.q_stride + (uint64_t)qh * P.dim;
    for (uint32_t c = lane; c < 256; c += 64) query[c] = c < P.dim ? to_f32(q[c]) : 0.f;
    __syncthreads();
    int64_t length = P.context[row];
    if (length < 0) length = 0;
    if ((uint64_t)length > P.max_context) length = (int64_t)P.max_context;
    const int64_t begin = P.window && length > P.window ? length - P.window : 0;
    const uint64_t head = (uint64_t)(qh / P.group) * P.head_stride;
    float most = -INFINITY, sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t first = begin; first < length; first += 64) {
        const int64_t p = first + lane;
        float s = -INFINITY;
        uint64_t at = ~0ull;
        if (p < length) {
            const int32_t id = P.table[row * P.table_stride + p / P.page];
            if ((uint32_t)id < P.pages) {
                at = (uint64_t)id * P.page_stride + head + (uint64_t)(p % P.page) * P.slot_stride;
                const C *k = (const C *)P.k + at;
                s = 0.f;
                for (uint32_t c = 0; c < P.dim; ++c) s += query[c] * to_f32(k[c]);
                s *= P.score_by;
            }
        }
        float m = s;
        for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
        m = fmaxf(m, most);
        const float base = m == -INFINITY ? 0.f : m;
        const float w = at == ~0ull ? 0.f : expf(s - base), by = expf(most - base);
        most = m;
        sum *= by;
        for (int i = 0; i < 4; ++i) o[i] *= by;
        weight[lane] = w;
        at_lds[lane] = at;
        __syncthreads();
        for (int j = 0; j < 64; ++j) {
            const uint64_t a = at_lds[j];
            if (a == ~0ull) continue;
            const float wj = weight[j];
            sum += wj;
            const C *v = (const C *)P.v + a;
            for (int i = 0; i < 4; ++i) {
                const uint32_t c = lane + 64 * i;
                if (c < P.dim) o[i] += wj * to_f32(v[c]);
            }
        }
        __syncthreads();
    }
    const float by = sum == 0.f ? 0.f : P.out_by / sum;
    for (int i = 0; i < 4; ++i) {
        const uint32_t c = lane + 64 * i;
        if (c < P.dim) ((T *)P.out)[((uint64_t)row * P.q_heads + qh) * P.dim + c] = from_f32<T>(o[i] * by);
    }
    if (P.lse && lane == 0) P.lse[(uint64_t)row * P.q_heads + qh] = most == -INFINITY && sum == 0.f ? -INFINITY : most + logf(sum);
}

}  // namespace
