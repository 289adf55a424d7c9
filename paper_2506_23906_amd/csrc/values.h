// libmmvseg, part of the translation unit serving.hip (included there, in order).
// The 16-bit values of queries, caches and states' inputs; moves between lanes.
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

}  // namespace
