// libmmvseg, part of the translation unit serving.hip (included there, in order).
// Page tables and slots from the requests' lengths; new keys and values into the paged cache.
#pragma once

namespace {

// ---- page tables ---------------------------------------------------------------------------------------------------
//
// Two exclusive sums over the requests (tokens, pages taken), then every token finds its request by bisection among the
// first tokens.  Up to kTablesLocal requests every workgroup makes the sums itself, in LDS: the lengths are a few KB that
// come from the L2, and a launch of their own would take longer than the whole call.  Beyond, one workgroup leaves them in
// the workspace.  The call is bound by its launch and by the chain lengths -> sums -> bisection -> page -> slot: 256 decoding
// requests take 3.3 us on the GPU, 100 prompts of 180000 tokens 4.5.  One token a thread: four consecutive ones, with one bisection and wide
// stores, made both slower (4.4 and 5.0), as did sums by shuffles through LDS (6.4 for the prompts, where every workgroup makes them).
constexpr uint32_t kTablesLocal = 2048;
constexpr int kTablesThreads = 256;
constexpr uint32_t kInt32Max = 0x7fffffffu;

struct TablesParams {
    uint32_t n, max_tokens, free_count, table_width;
    Divider page;
    uint64_t table_stride;
    const int32_t *cached, *fresh, *free_pages;
    int32_t *table, *offsets, *context, *positions;
    int64_t *slots, *used;
    uint32_t *ends, *taken;   // (beyond kTablesLocal) inclusive sum of tokens, exclusive sum of pages taken
};

struct Sum2 {
    uint64_t tokens, pages;
};
template <int kCtrl, int kRowMask> __device__ __forceinline__ uint64_t dpp64(uint64_t v) {
    return ((uint64_t)dpp_or_zero<kCtrl, kRowMask>((uint32_t)(v >> 32)) << 32) | dpp_or_zero<kCtrl, kRowMask>((uint32_t)v);
}
__device__ __forceinline__ uint64_t wave_upto64(uint64_t v) {   // inclusive sums over the lanes
    v += dpp64<0x111, 0xF>(v);
    v += dpp64<0x112, 0xF>(v);
    v += dpp64<0x114, 0xF>(v);
    v += dpp64<0x118, 0xF>(v);
    v += dpp64<0x142, 0xA>(v);
    return v + dpp64<0x143, 0xC>(v);
}
// Inclusive sums over the threads of a workgroup; `total` is the sum over all of them.
template <int kThreads> __device__ __forceinline__ Sum2 block_scan(Sum2 v, Sum2 *lds, Sum2 &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    v.tokens = wave_upto64(v.tokens), v.pages = wave_upto64(v.pages);
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
// Pages that hold `positions` (up to 2^32): a quotient of positions - 1 below 2^31, or of its halves.
__device__ __forceinline__ uint32_t pages_of(uint64_t positions, const Divider &page) {
    if (positions == 0) return 0;
    const uint64_t last = positions - 1;
    return (last >> 31 ? (uint32_t)(last / page.divisor) : page.quotient((uint32_t)last)) + 1;
}

// Sums over all requests, kThreads at a time: ends[r] and taken[r], cut at 2^31 - 1 (a token number never reaches that), and the cached lengths beside them.
template <int kThreads> __device__ __forceinline__ Sum2 sum_requests(const TablesParams &P, uint32_t *ends, uint32_t *taken, uint32_t *cached, Sum2 *lds) {
    Sum2 carry = {0, 0};
    for (uint32_t first = 0; first < P.n; first += kThreads) {
        const uint32_t r = first + threadIdx.x;
        Sum2 own = {0, 0}, total;
        if (r < P.n) {
            const uint32_t fresh = length_of(P.fresh[r]), old = length_of(P.cached[r]);
            own = {fresh, pages_of((uint64_t)old + fresh, P.page) - pages_of(old, P.page)};
            if (cached) cached[r] = old;
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
__device__ __forceinline__ void write_totals(const TablesParams &P, Sum2 total) {
    P.used[0] = (int64_t)total.pages;
    P.used[1] = (int64_t)total.tokens;
    P.offsets[0] = 0;
}

__global__ __launch_bounds__(1024) void sum_requests_kernel(TablesParams P) {
    __shared__ Sum2 lds[16];
    const Sum2 total = sum_requests<1024>(P, P.ends, P.taken, nullptr, lds);
    if (threadIdx.x == 0) write_totals(P, total);
}

template <bool kLocal> __global__ __launch_bounds__(kTablesThreads) void page_tables_kernel(TablesParams P) {
    __shared__ uint32_t lds_ends[kLocal ? kTablesLocal : 1], lds_taken[kLocal ? kTablesLocal : 1], lds_cached[kLocal ? kTablesLocal : 1];
    __shared__ Sum2 lds[kTablesThreads / 64];
    const uint32_t *ends = P.ends, *taken = P.taken;
    if constexpr (kLocal) {
        const Sum2 total = sum_requests<kTablesThreads>(P, lds_ends, lds_taken, lds_cached, lds);
        if (blockIdx.x == 0 && threadIdx.x == 0) write_totals(P, total);
        __syncthreads();
        ends = lds_ends, taken = lds_taken;
    }
    const auto cached_of = [&](uint32_t r) __attribute__((always_inline)) { return kLocal ? lds_cached[kLocal ? r : 0] : length_of(P.cached[r]); };
    const uint64_t own = (uint64_t)blockIdx.x * kTablesThreads + threadIdx.x;
    for (uint64_t r = own; r < P.n; r += (uint64_t)gridDim.x * kTablesThreads) {
        P.offsets[r + 1] = (int32_t)ends[r];
        P.context[r] = (int32_t)cut32((uint64_t)cached_of((uint32_t)r) + length_of(P.fresh[r]));
    }
    if (own >= P.max_tokens) return;
    const uint32_t t = (uint32_t)own, all = P.n ? ends[P.n - 1] : 0u;
    int64_t slot = -1;
    int32_t position = -1;
    if (t < all) {
        uint32_t r = 0, hi = P.n - 1;   // the first request that ends behind t
        while (r < hi) {
            const uint32_t mid = (r + hi) >> 1;
            if (ends[mid] > t) hi = mid;
            else r = mid + 1;
        }
        const uint32_t cached = cached_of(r);
        const uint64_t at = (uint64_t)cached + (t - (r ? ends[r - 1] : 0u));
        if (at <= kInt32Max) {
            position = (int32_t)at;
            const uint32_t where = P.page.quotient((uint32_t)at), held = pages_of(cached, P.page), place = (uint32_t)at - where * P.page.divisor;
            const uint64_t which = (uint64_t)taken[r] + (where - held);   // (of the free pages, behind those that the request has)
            int32_t *const entry = P.table + (uint64_t)r * P.table_stride + where;
            if (where < P.table_width && (where < held || which < P.free_count)) {
                const int32_t id = where < held ? *entry : P.free_pages[which];
                if (where >= held && place == 0) *entry = id;
                if (id >= 0) slot = (int64_t)id * P.page.divisor + place;
            }
        }
    }
    P.slots[t] = slot;
    P.positions[t] = position;
}

// ---- cache append -------------------------------------------------------------------------------------------------
//
// A thread moves eight values of the key and the same eight of the value: 16-byte loads, 16-byte stores (8 bytes into an
// 8-bit cache).  Bound by memory; a slot's eight-value pieces are neighbours, so stores are whole runs of dim values.
// 16385 tokens of 8 heads of 128 into an e4m3 cache 18.5 us, 5.4 TB/s; 256 tokens 2.6, a launch's life.
struct AppendParams {
    const void *k, *v;
    uint64_t k_stride, v_stride;   // elements
    const int64_t *slots;
    void *cache_k, *cache_v;
    uint64_t page_stride, head_stride, slot_stride;
    uint32_t total, num_slots;     // total: threads with work
    Divider page, pieces, head_pieces;   // pieces of eight values of a token, of a head
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
    const uint32_t id = blockIdx.x * 256 + threadIdx.x;
    if (id >= P.total) return;
    const uint32_t t = P.pieces.quotient(id), piece = id - t * P.pieces.divisor, h = P.head_pieces.quotient(piece), c = piece - h * P.head_pieces.divisor;
    const uint4 k = *(const uint4 *)((const T *)P.k + t * P.k_stride + 8 * piece), v = *(const uint4 *)((const T *)P.v + t * P.v_stride + 8 * piece);
    const int64_t slot = P.slots[t];
    if ((uint64_t)slot >= P.num_slots) return;
    const uint32_t p = P.page.quotient((uint32_t)slot), in_page = (uint32_t)slot - p * P.page.divisor;
    const uint64_t to = (uint64_t)p * P.page_stride + (uint64_t)h * P.head_stride + (uint64_t)in_page * P.slot_stride + 8 * c;
    if constexpr (kE4m3) {
        *(uint2 *)((uint8_t *)P.cache_k + to) = to_e4m3((const T *)&k, P.k_by);
        *(uint2 *)((uint8_t *)P.cache_v + to) = to_e4m3((const T *)&v, P.v_by);
    } else {
        *(uint4 *)((T *)P.cache_k + to) = k;
        *(uint4 *)((T *)P.cache_v + to) = v;
    }
}

}  // namespace
