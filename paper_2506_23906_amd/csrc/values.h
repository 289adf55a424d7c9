// libmmvseg, part of the translation unit serving.hip (included there, in order).
// The 16-bit values of queries, caches and states' inputs, their products on the matrix cores and terms of 16 bits; moves between lanes.
#pragma once

namespace {

using f16_t = _Float16;
using bf16_t = __bf16;

__device__ __forceinline__ float to_f32(f16_t v) { return (float)v; }
__device__ __forceinline__ float to_f32(bf16_t v) { return __builtin_bit_cast(float, (uint32_t)__builtin_bit_cast(uint16_t, v) << 16); }
template <typename T> __device__ __forceinline__ T from_f32(float v) { return (T)v; }   // to the nearest, ties to even

// Every lane reads the lane that the control word names (row_shr n = 0x110 + n inside rows of 16 lanes, row_bcast 15 / 31 = 0x142 / 0x143);
// one that has no source, or whose row is not in kRowMask, reads 0.
template <int kCtrl, int kRowMask> __device__ __forceinline__ uint32_t dpp_or_zero(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, kRowMask, 0xF, false);
}

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ uint64_t uniform64(uint64_t v) { return ((uint64_t)uniform((uint32_t)(v >> 32)) << 32) | uniform((uint32_t)v); }
__device__ __forceinline__ uint32_t lane_value(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }

// Uniform loads through the scalar cache: they are not waited for along with vector loads.
__device__ __forceinline__ int32_t scalar_load(const int32_t *p) { return *(const __attribute__((address_space(4))) int32_t *)(uintptr_t)p; }

// Buffer loads and stores: what lies at or beyond `bytes` reads 0 and is not written (the whole offset has to be the lane's own).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, 0x00027000);
}

// Division of numbers below 2^31 by one of at most 2^17: a shift, or the upper half of a product and a shift (the factor is too large by less than 2^-31 of
// itself, so the quotient is exact).
struct Divider {
    uint32_t by, shift, divisor;
    __device__ __forceinline__ uint32_t quotient(uint32_t v) const { return by ? __umulhi(v, by) >> shift : v >> shift; }
};
inline Divider divider(uint32_t d) {
    uint32_t bits = 0;
    while ((1u << bits) < d) ++bits;
    if ((1u << bits) == d) return {0, bits, d};
    return {(uint32_t)(((1ull << (31 + bits)) + d - 1) / d), bits - 1, d};
}

// Lengths that the device alone knows.
__device__ __forceinline__ uint32_t length_of(int32_t v) { return v < 0 ? 0u : (uint32_t)v; }

// ---- products of 16-bit values -------------------------------------------------------------------------------------

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ f32x4 mfma_16x16x32(bf16_t, u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_16x16x32(f16_t, u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b) {
    typedef T pair __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, (pair){from_f32<T>(a), from_f32<T>(b)});
}
__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) { return mfma_16x16x32(bf16_t(), a, b, c); }
__device__ __forceinline__ float low_half(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }
// Two values into kTerms words of bf16 pairs: the upper halves of what is left each time, the last of it rounded.
template <int kTerms> __device__ __forceinline__ void take_apart(float a, float b, uint32_t (&to)[kTerms]) {
#pragma unroll
    for (int i = 0; i + 1 < kTerms; ++i) {
        to[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u);
        a -= high_half(__builtin_bit_cast(uint32_t, a)), b -= high_half(__builtin_bit_cast(uint32_t, b));
    }
    to[kTerms - 1] = pack2<bf16_t>(a, b);
}
// A word of two inputs as its bf16 terms.
template <typename T, int kTerms> __device__ __forceinline__ void input_terms(uint32_t w, uint32_t (&to)[kTerms]) {
    if constexpr (kTerms == 1) {
        to[0] = w;
    } else {
        typedef f16_t pair __attribute__((ext_vector_type(2)));
        const pair h = __builtin_bit_cast(pair, w);
        take_apart<kTerms>((float)h[0], (float)h[1], to);
    }
}

}  // namespace
