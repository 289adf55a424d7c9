// libmmvseg, part of the translation units of a serving step's calls (included there, in order).
// Host side: limits, argument checks and launches that the calls of a serving step share.
#pragma once

namespace {

constexpr uint64_t k2to31 = 1ull << 31;
constexpr uint64_t kMostRequests = 1ull << 22;
constexpr uint32_t kMostHeads = 1024;
constexpr uint64_t kMostStride = 1ull << 24;   // of tokens, in elements, for the recurrence: 64 of them in 32-bit byte offsets

inline uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
inline size_t round256(size_t b) { return (b + 255) & ~(size_t)255; }
inline bool aligned_to(const void *p, uintptr_t by) { return (uintptr_t)p % by == 0; }
inline mmv_status launched() { return hipGetLastError() == hipSuccess ? MMV_OK : MMV_ERR_HIP; }
// A launch has fewer than 2^32 threads: so many rows (requests, blocks) of `each` workgroups go into one.
inline uint32_t most_of_a_launch(uint32_t threads, uint64_t each) { return (uint32_t)(((1ull << 32) - 1) / threads / each); }
inline bool valid_value_type(int t) { return t == MMV_TYPE_F16 || t == MMV_TYPE_BF16; }
inline mmv_status check_workspace(const void *ws, size_t bytes, size_t needed) {
    if (!needed) return MMV_OK;
    if (!ws) return MMV_ERR_NULL;
    return ((uintptr_t)ws & 255u) || bytes < needed ? MMV_ERR_WORKSPACE : MMV_OK;
}
constexpr uint32_t kUnits = 256;   // compute units of an MI355X

}  // namespace
