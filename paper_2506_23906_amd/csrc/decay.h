// libmmvseg, part of the translation unit serving.hip (included there, in order).
// Linear attention with a decay for each head.
#pragma once

namespace {

struct DecayParams {
    const void *q, *k, *v;
    uint64_t q_stride, k_stride, v_stride, tokens;   // strides in elements
    const int32_t *offsets;                          // null: one token for each request
    const float *log_decay;
    const float *state_in;
    float *state_out;
    const int32_t *state_index;
    uint64_t states;
    void *out;
    uint32_t n, heads, group, dk, dv;
    float scale;
};
constexpr uint32_t kMostDk = 128, kMostDv = 256;

// The state that request r starts from and leaves, ~0 for none.
__device__ __forceinline__ uint64_t state_of(const DecayParams &P, uint32_t r) {
    const int64_t i = P.state_index ? P.state_index[r] : r;
    return i >= 0 && (uint64_t)i < P.states ? (uint64_t)i : ~0ull;
}
__device__ __forceinline__ float head_decay(const DecayParams &P, uint32_t h) {
    const float d = P.log_decay[h];
    return d < -1e30f ? -1e30f : d;   // (0 * -infinity is no exponent)
}
struct Span {
    uint32_t begin, end;
};
__device__ __forceinline__ Span span_of(const DecayParams &P, uint32_t r) {
    if (!P.offsets) return {r, r + 1};
    const int64_t most = (int64_t)P.tokens;
    int64_t a = P.offsets[r], b = P.offsets[r + 1];
    a = a < 0 ? 0 : a > most ? most : a;
    b = b < a ? a : b > most ? most : b;
    return {(uint32_t)a, (uint32_t)b};
}

// One workgroup for a request and head, token by token: a thread has a column of the state.
template <typename T> __global__ __launch_bounds__(kMostDv) void decay_kernel(DecayParams P) {
    __shared__ float query[kMostDk], key[kMostDk];
    const uint32_t r = blockIdx.x / P.heads, h = blockIdx.x % P.heads, c = threadIdx.x, kv = h / P.group;
    const Span span = span_of(P, r);
    const uint64_t state = state_of(P, r), matrix = (uint64_t)P.dk * P.dv;
    const float decay = expf(head_decay(P, h));
    float S[kMostDk];
#pragma unroll
    for (uint32_t i = 0; i < kMostDk; ++i)
        S[i] = P.state_in && state != ~0ull && i < P.dk && c < P.dv ? P.state_in[(state * P.heads + h) * matrix + (uint64_t)i * P.dv + c] : 0.f;
    for (uint32_t t = span.begin; t < span.end; ++t) {
        __syncthreads();
        if (c < kMostDk) {
            query[c] = c < P.dk ? to_f32(((const T *)P.q)[t * P.q_stride + (uint64_t)h * P.dk + c]) : 0.f;
            key[c] = c < P.dk ? to_f32(((const T *)P.k)[t * P.k_stride + (uint64_t)kv * P.dk + c]) : 0.f;
        }
        __syncthreads();
        const float v = c < P.dv ? to_f32(((const T *)P.v)[t * P.v_stride + (uint64_t)kv * P.dv + c]) : 0.f;
        float o = 0.f;
#pragma unroll
        for (uint32_t i = 0; i < kMostDk; ++i) {
            S[i] = S[i] * decay + key[i] * v;
            o += query[i] * S[i];
        }
        if (c < P.dv) ((T *)P.out)[((uint64_t)t * P.heads + h) * P.dv + c] = from_f32<T>(o * P.scale);
    }
    if (P.state_out && state != ~0ull && c < P.dv)
#pragma unroll
        for (uint32_t i = 0; i < kMostDk; ++i)
            if (i < P.dk) P.state_out[(state * P.heads + h) * matrix + (uint64_t)i * P.dv + c] = S[i];
}

}  // namespace
