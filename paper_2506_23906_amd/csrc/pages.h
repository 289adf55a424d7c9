// libmmvseg, part of the translation unit serving.hip (included there, in order).
// Page tables and slots from the requests' lengths; new keys and values into the paged cache.
#pragma once

namespace {

// ---- page tables ---------------------------------------------------------------------------------------------------
//
// Two exclusive sums over the requests (tokens, pages taken), then every token finds its request by bisection among the
// first tokens.  Up to kTablesLocal requests every workgroup makes the sums itself, in LDS: the lengths are a few KB that
// come from the L2, and a launch of their own would take longer than the whole call.  Beyond, one workgroup leaves them in
// the workspace.  The call is bound by its launch and by the chain lengths -> sums -> bisection -> slot.
constexpr uint32_t kTablesLocal = 2048;
constexpr int kTablesThreads = 256;
constexpr uint32_t kTablesTokens = 4 * kTablesThreads;   // tokens of a workgroup
constexpr uint32_t kInt32Max = 0x7fffffffu;

struct TablesParams {
    uint32_t n, page, max_tokens, free_count, table_width;
    uint64_t table_stride;
    const int32_t *cached, *fresh, *free_pages;
    int32_t *table, *offsets, *context, *positions;
    int64_t *slots, *used;
    uint32_t *ends, *taken;   // (beyond kTablesLocal) inclusive sum of tokens, exclusive sum of pages taken
};

struct Sum2 {
    uint64_t tokens, pages;
};
__device__ __forceinline__ uint64_t shift_up64(uint64_t v, int by, int lane) {
    const uint64_t o = __shfl_up(v, by);
    return lane >= by ? o : 0;
}
// Inclusive sums over the threads of a workgroup; `total` is the sum over all of them.
template <int kThreads> __device__ __forceinline__ Sum2 block_scan(Sum2 v, Sum2 *lds, Sum2 &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        v.tokens += shift_up64(v.tokens, d, lane);
        v.pages += shift_up64(v.pages, d, lane);
    }
    if (lane == 63) lds[wave] = v;
    __syncthreads();
    Sum2 before = {0, 0};
    total = {0, 0};
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        const Sum2 s = lds[w];
        if (w < wave) before.tokens += s.tokens, before.pages += s.pages;
        total.tokens += s.tokens, total.pages += s.pages;
    }
    __syncthreads();
    return {v.tokens + before.tokens, v.pages + before.pages};
}
__device__ __forceinline__ uint32_t cut32(uint64_t v) { return v > kInt32Max ? kInt32Max : (uint32_t)v; }
__device__ __forceinline__ uint32_t length_of(int32_t v) { return v < 0 ? 0u : (uint32_t)v; }
// Pages that request r takes: those that hold its positions, less those that hold the cached ones.
__device__ __forceinline__ uint32_t pages_taken(uint32_t cached, uint32_t fresh, uint32_t page) {
    const uint32_t held = (uint32_t)(((uint64_t)cached + page - 1) / page);
    return (uint32_t)(((uint64_t)cached + fresh + page - 1) / page) - held;
}

// Sums over all requests, kThreads at a time: ends[r] and taken[r], cut at 2^31 - 1 (a token number never reaches that).
template <int kThreads> __device__ __forceinline__ Sum2 sum_requests(const TablesParams &P, uint32_t *ends, uint32_t *taken, Sum2 *lds) {
    Sum2 carry = {0, 0};
    for (uint32_t first = 0; first < P.n; first += kThreads) {
        const uint32_t r = first + threadIdx.x;
        Sum2 own = {0, 0}, total;
        if (r < P.n) {
            const uint32_t fresh = length_of(P.fresh[r]);
            own = {fresh, pages_taken(length_of(P.cached[r]), fresh, P.page)};
        }
        const Sum2 s = block_scan<kThreads>(own, lds, total);
        if (r < P.n) {
            ends[r] = cut32(carry.tokens + s.tokens);
            taken[r] = cut32(carry.pages + s.pages - own.pages);
        }
        carry.tokens += total.tokens, carry.pages += total.pages;
    }
    return carry;
}
__device__ __forceinline__ void write_request(const TablesParams &P, uint32_t r, uint32_t end) {
    P.offsets[r + 1] = (int32_t)end;
    P.context[r] = (int32_t)cut32((uint64_t)length_of(P.cached[r]) + length_of(P.fresh[r]));
}
__device__ __forceinline__ void write_totals(const TablesParams &P, Sum2 total) {
    P.used[0] = (int64_t)total.pages;
    P.used[1] = (int64_t)total.tokens;
    P.offsets[0] = 0;
}

__global__ __launch_bounds__(1024) void sum_requests_kernel(TablesParams P) {
    __shared__ Sum2 lds[16];
    const Sum2 total = sum_requests<1024>(P, P.ends, P.taken, lds);
    if (threadIdx.x == 0) write_totals(P, total);
}

template <bool kLocal> __global__ __launch_bounds__(kTablesThreads) void page_tables_kernel(TablesParams P) {
    __shared__ uint32_t lds_ends[kLocal ? kTablesLocal : 1], lds_taken[kLocal ? kTablesLocal : 1];
    __shared__ Sum2 lds[kTablesThreads / 64];
    const uint32_t *ends = P.ends, *taken = P.taken;
    if constexpr (kLocal) {
        const Sum2 total = sum_requests<kTablesThreads>(P, lds_ends, lds_taken, lds);
        if (blockIdx.x == 0 && threadIdx.x == 0) write_totals(P, total);
        __syncthreads();
        ends = lds_ends, taken = lds_taken;
    }
    for (uint32_t r = blockIdx.x * kTablesThreads + threadIdx.x; r < P.n; r += gridDim.x * kTablesThreads) write_request(P, r, ends[r]);
    const uint32_t all = P.n ? ends[P.n - 1] : 0u;
#pragma unroll
    for (uint32_t i = 0; i < kTablesTokens; i += kTablesThreads) {
        const uint64_t t64 = (uint64_t)blockIdx.x * kTablesTokens + i + threadIdx.x;
        if (t64 >= P.max_tokens) return;
        const uint32_t t = (uint32_t)t64;
        int64_t slot = -1;
        int32_t position = -1;
        if (t < all) {
            uint32_t lo = 0, hi = P.n - 1;   // the first request that ends behind t
            while (lo < hi) {
                const uint32_t mid = (lo + hi) >> 1;
                if (ends[mid] > t) hi = mid;
                else lo = mid + 1;
            }
            const uint32_t cached = length_of(P.cached[lo]), fresh = length_of(P.fresh[lo]);
            const uint64_t at = (uint64_t)cached + (t - (lo ? ends[lo - 1] : 0u));
            (void)fresh;
            if (at <= kInt32Max) {
                position = (int32_t)at;
                const uint32_t where = (uint32_t)at / P.page, place = (uint32_t)at % P.page, held = (uint32_t)(((uint64_t)cached + P.page - 1) / P.page);
                if (where < P.table_width) {
                    int32_t *const entry = P.table + (uint64_t)lo * P.table_stride + where;
                    int32_t id = -1;
                    if (where < held) {
                        id = *entry;
                    } else {
                        const uint64_t which = (uint64_t)taken[lo] + (where - held);
                        if (which < P.free_count) {
                            id = P.free_pages[which];
                            if (place == 0) *entry = id;
                        }
                    }
                    if (id >= 0) slot = (int64_t)id * P.page + place;
                }
            }
        }
        P.slots[t] = slot;
        P.positions[t] = position;
    }
}

// ---- cache append -------------------------------------------------------------------------------------------------
//
// A thread moves eight values of the key and the same eight of the value: 16-byte loads, 16-byte stores (8 bytes into an
// 8-bit cache).  Bound by memory; a slot's eight-value pieces are neighbours, so stores are whole runs of dim values.
struct AppendParams {
    const void *k, *v;
    uint64_t k_stride, v_stride;   // elements
    const int64_t *slots;
    void *cache_k, *cache_v;
    uint64_t page_stride, head_stride, slot_stride, total;   // total: threads with work
    uint32_t page, num_slots, pieces, head_pieces;           // pieces of eight values of a token, of a head
    float k_by, v_by;
};

__device__ __forceinline__ float clamp_e4m3(float x) { return x > 448.f ? 448.f : x < -448.f ? -448.f : x; }   // (NaN stays)
template <typename T> __device__ __forceinline__ uint2 to_e4m3(const T *x, float by) {
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float a = clamp_e4m3(to_f32(x[4 * i]) * by), b = clamp_e4m3(to_f32(x[4 * i + 1]) * by);
        const float c = clamp_e4m3(to_f32(x[4 * i + 2]) * by), d = clamp_e4m3(to_f32(x[4 * i + 3]) * by);
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        p = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, p, true);
        w[i] = (uint32_t)p;
    }
    return make_uint2(w[0], w[1]);
}

template <typename T, bool kE4m3> __global__ __launch_bounds__(256) void cache_append_kernel(AppendParams P) {
    const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= P.total) return;
    const uint64_t t = id / P.pieces;
    const uint32_t piece = (uint32_t)(id - t * P.pieces), h = piece / P.head_pieces, c = piece - h * P.head_pieces;
    const int64_t slot = P.slots[t];
    if ((uint64_t)slot >= P.num_slots) return;
    const uint32_t p = (uint32_t)slot / P.page, in_page = (uint32_t)slot - p * P.page;
    const uint64_t to = (uint64_t)p * P.page_stride + (uint64_t)h * P.head_stride + (uint64_t)in_page * P.slot_stride + 8 * c;
    const uint4 k = *(const uint4 *)((const T *)P.k + t * P.k_stride + 8 * piece), v = *(const uint4 *)((const T *)P.v + t * P.v_stride + 8 * piece);
    if constexpr (kE4m3) {
        *(uint2 *)((uint8_t *)P.cache_k + to) = to_e4m3((const T *)&k, P.k_by);
        *(uint2 *)((uint8_t *)P.cache_v + to) = to_e4m3((const T *)&v, P.v_by);
    } else {
        *(uint4 *)((T *)P.cache_k + to) = k;
        *(uint4 *)((T *)P.cache_v + to) = v;
    }
}

}  // namespace
