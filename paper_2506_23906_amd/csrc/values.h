// libmmvseg, part of the translation unit serving.hip (included there, in order).
// The 16- and 8-bit values of queries, caches and states' inputs.
#pragma once

namespace {

using f16_t = _Float16;
using bf16_t = __bf16;
struct e4m3_t {
    uint8_t bits;
};

__device__ __forceinline__ float to_f32(f16_t v) { return (float)v; }
__device__ __forceinline__ float to_f32(bf16_t v) { return __builtin_bit_cast(float, (uint32_t)__builtin_bit_cast(uint16_t, v) << 16); }
__device__ __forceinline__ float to_f32(e4m3_t v) { return __builtin_amdgcn_cvt_f32_fp8((int)v.bits, 0); }
template <typename T> __device__ __forceinline__ T from_f32(float v) { return (T)v; }   // to the nearest, ties to even

}  // namespace
