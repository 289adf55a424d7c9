// libmmvseg, part of the translation unit delta.hip (included there, in order).
// The gated delta rule.
#pragma once

namespace {

struct DeltaParams {
    const void *q, *k, *v;
    uint64_t q_stride, k_stride, v_stride, tokens;   // strides in elements
    const int32_t *offsets;                          // null: one token for each request
    const float *log_decay, *beta;                   // [tokens][heads]
    const float *state_in;
    float *state_out;
    const int32_t *state_index;
    uint64_t states;
    void *out;
    uint32_t n, heads, group, dk, dv;
    uint32_t first;                                  // request of a launch
    float scale;
};
constexpr uint32_t kMostDk = 128, kMostDv = 256;
// e^g with an error of fp32's last bit: the exponent in two parts.  Below e^-200, 0 in fp32, the same as there (0 * -infinity is no exponent).
__device__ __forceinline__ float at_least_200(float g) { return g < -200.f ? -200.f : g; }
__device__ __forceinline__ float exp_of(float g) {
    constexpr float kLog2e = 1.44269504f, kRest = 1.92596299e-8f;
    g = at_least_200(g);
    const float x = g * kLog2e, rest = __builtin_fmaf(g, kLog2e, -x) + g * kRest, y = __builtin_amdgcn_exp2f(x);
    return x < 127.f ? __builtin_fmaf(y, rest * 0.693147181f, y) : y;
}

// The state that request r starts from and leaves, ~0 for none.
__device__ __forceinline__ uint64_t state_of(const DeltaParams &P, uint32_t r) {
    const int64_t i = P.state_index ? P.state_index[r] : r;
    return i >= 0 && (uint64_t)i < P.states ? (uint64_t)i : ~0ull;
}
struct Span {
    uint32_t begin, end;
};
__device__ __forceinline__ Span span_of(const DeltaParams &P, uint32_t r) {
    if (!P.offsets) return {r, r + 1};
    const int64_t most = (int64_t)P.tokens;
    int64_t a = P.offsets[r], b = P.offsets[r + 1];
    a = a < 0 ? 0 : a > most ? most : a;
    b = b < a ? a : b > most ? most : b;
    return {(uint32_t)a, (uint32_t)b};
}

// ---- token by token ------------------------------------------------------------------------------------------------
//
//   S' = e^g S,   u = beta (v - k S'),   S = S' + k u^T,   out = scale q S = scale (q S' + (q . k) u)
// One token is bound by reading and writing the state: 8 dk dv bytes for 6 dk dv operations.  A workgroup has a slice of at most 128 columns of one state, a thread four
// columns (16 bytes) of every `step`-th row, all loaded before the first is used.  The threads of the same columns are neighbouring lanes: k S' and q S' are added up
// over them without LDS, and every one of them has the sums that its rows' update needs.
template <typename T, int kRows> __global__ __launch_bounds__(256) void delta_tokens_kernel(DeltaParams P, uint32_t slices, uint32_t slice, uint32_t step) {
    __shared__ float query[2][kMostDk], key[2][kMostDk];
    const uint32_t tid = threadIdx.x, unit = blockIdx.x / slices, r = P.first + unit / P.heads, h = unit % P.heads, shared = h / P.group;
    const uint32_t first = tid & (step - 1), c = (blockIdx.x - unit * slices) * slice + tid / step * 4;
    const bool live = tid / step * 4 < slice && c < P.dv;
    const uint64_t state = state_of(P, r), at = (state * P.heads + h) * ((uint64_t)P.dk * P.dv) + c;
    const bool have = state != ~0ull;
    const Span span = span_of(P, r);
    f32x4 S[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const uint32_t d = first + i * step;
        S[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
        if (P.state_in && have && live && d < P.dk) S[i] = __builtin_nontemporal_load((const f32x4 *)(P.state_in + at + (uint64_t)d * P.dv));
    }
    for (uint32_t t = span.begin; t < span.end; ++t) {
        const uint32_t buffer = t & 1;
        if (tid < P.dk) {
            query[buffer][tid] = to_f32(((const T *)P.q)[t * P.q_stride + (uint64_t)shared * P.dk + tid]);
            key[buffer][tid] = to_f32(((const T *)P.k)[t * P.k_stride + (uint64_t)shared * P.dk + tid]);
        }
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        const T *pv = (const T *)P.v + t * P.v_stride + (uint64_t)h * P.dv + c;
        if (live) v = (f32x4){to_f32(pv[0]), to_f32(pv[1]), to_f32(pv[2]), to_f32(pv[3])};
        const float decay = exp_of(P.log_decay[(uint64_t)t * P.heads + h]), beta = P.beta[(uint64_t)t * P.heads + h];
        __syncthreads();   // (one barrier a token: the other buffer is written behind it)
        f32x4 by_key = {0.f, 0.f, 0.f, 0.f}, by_query = by_key;
        float both = 0.f;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const uint32_t d = first + i * step;
            const float kd = d < P.dk ? key[buffer][d] : 0.f, qd = d < P.dk ? query[buffer][d] : 0.f;
            S[i] *= decay;
            by_key += kd * S[i], by_query += qd * S[i], both += qd * kd;
        }
        for (uint32_t d = 1; d < step; d <<= 1) {
#pragma unroll
            for (int j = 0; j < 4; ++j) by_key[j] += __shfl_xor(by_key[j], d), by_query[j] += __shfl_xor(by_query[j], d);
            both += __shfl_xor(both, d);
        }
        const f32x4 u = beta * (v - by_key);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const uint32_t d = first + i * step;
            if (d < P.dk) S[i] += key[buffer][d] * u;
        }
        if (live && first == 0) {
            const f32x4 o = P.scale * (by_query + both * u);
            *(u32x2 *)((T *)P.out + ((uint64_t)t * P.heads + h) * P.dv + c) = (u32x2){pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
        }
    }
    if (!P.state_out || !have || !live) return;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const uint32_t d = first + i * step;
        if (d < P.dk) __builtin_nontemporal_store(S[i], (f32x4 *)(P.state_out + at + (uint64_t)d * P.dv));
    }
}

}  // namespace
