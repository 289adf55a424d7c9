// libmmvseg, part of the translation unit block.hip (included there, in order).
// A cache of 8-bit values with a scale for each block of slots and head: written, and read back.
#pragma once

namespace {

struct BlockCacheParams {
    void *k, *v;
    float *k_scales, *v_scales;                        // [pages][heads][blocks of a page]
    uint64_t page_stride, head_stride, slot_stride;    // values
    uint32_t heads, page_blocks, block, num_slots, pages;
    Divider page_of_block, slots, pieces;              // blocks of a page, slots of a block, dim / 8
};

// Eight values of 8 bits (two words) as fp32, and back: to the nearest, ties to even, at most +-127 or +-448 (NaN stays one in e4m3).
template <bool kInt8> __device__ __forceinline__ void to_floats(uint2 w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t u = i ? w.y : w.x;
        if constexpr (kInt8) {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * i + j] = (float)(int8_t)(u >> (8 * j));
        } else {
            typedef float pair __attribute__((ext_vector_type(2)));
            const pair a = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, true);
            x[4 * i] = a[0], x[4 * i + 1] = a[1], x[4 * i + 2] = b[0], x[4 * i + 3] = b[1];
        }
    }
}
template <bool kInt8> __device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
    if constexpr (kInt8) {
        const auto code = [](float x) __attribute__((always_inline)) { return (uint32_t)(int)__builtin_rintf(fminf(fmaxf(x, -127.f), 127.f)); };
        const uint32_t lo = __builtin_amdgcn_perm(code(b), code(a), 0x0c0c0400u), hi = __builtin_amdgcn_perm(code(d), code(c), 0x0c0c0400u);
        return lo | hi << 16;
    } else {
        const auto most = [](float x) __attribute__((always_inline)) { return x > 448.f ? 448.f : x < -448.f ? -448.f : x; };
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(most(a), most(b), 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(most(c), most(d), w, true);
    }
}
template <bool kInt8> __device__ __forceinline__ uint2 to_codes(const float (&x)[8], float by) {
    return make_uint2(to_codes<kInt8>(x[0] * by, x[1] * by, x[2] * by, x[3] * by), to_codes<kInt8>(x[4] * by, x[5] * by, x[6] * by, x[7] * by));
}
template <typename T> __device__ __forceinline__ void values_of(uint4 w, float (&x)[8]) {
    const T *t = (const T *)&w;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_f32(t[i]);
}

// ---- writing -------------------------------------------------------------------------------------------------------
//
// The unit of work is a run: neighbouring tokens whose slots lie in one block.  A wave has the runs that begin among `window` tokens, for one head,
// the keys or the values: it finds the largest value, makes the block's scale, rounds what the block holds already to that scale where it grows, and
// writes.  Up to kHeld x 64 pieces of eight values stay in registers from the first read on; what is beyond is read twice.  Bound by memory and by the chain slots -> values -> largest
// -> scale -> codes of each run: 17600 tokens of 8 heads of 128 22.9 us in blocks of 16 (4.7 TB/s), 25.1 of 32; 256 tokens of as many requests 4.4.
struct BlockAppendParams {
    BlockCacheParams c;
    const void *x[2];              // keys, values
    uint64_t stride[2];            // from token to token, in values
    const int64_t *slots;
    uint32_t tokens, window, first_window, windows;   // windows: of a launch
};
constexpr float kLeastLargest = 0x1p-100f;   // what the largest value of a run counts as at least: the scale's reciprocal is finite

template <typename T> constexpr uint32_t kInfinity = __is_same(T, bf16_t) ? 0x7F80u : 0x7C00u;   // bits; above them: not a number
// Bits of the largest magnitude of eight values (as whole numbers: the order of floats), two side by side.
__device__ __forceinline__ uint32_t larger_halves(uint32_t a, uint32_t b) {
    typedef uint16_t pair __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(pair, a), __builtin_bit_cast(pair, b)));
}
__device__ __forceinline__ uint32_t largest_bits(uint4 w) {
    constexpr uint32_t kAbs = 0x7FFF7FFFu;
    return larger_halves(larger_halves(w.x & kAbs, w.y & kAbs), larger_halves(w.z & kAbs, w.w & kAbs));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
    return uniform(v);
}

template <int kHeld, typename T, bool kInt8> __global__ __launch_bounds__(256) void block_append_kernel(BlockAppendParams P) {
    const BlockCacheParams &C = P.c;
    const uint32_t lane = threadIdx.x & 63, unit = uniform(blockIdx.x * 4 + (threadIdx.x >> 6)), pair = unit >> 1, which = unit & 1;
    const uint32_t in_launch = pair / C.heads, h = pair - in_launch * C.heads;
    if (in_launch >= P.windows) return;
    const uint32_t pieces = C.pieces.divisor, from = (P.first_window + in_launch) * P.window;
    const T *const x = (const T *)(which ? P.x[1] : P.x[0]) + (uint64_t)h * pieces * 8;
    const uint64_t stride = which ? P.stride[1] : P.stride[0];
    uint8_t *const codes = (uint8_t *)(which ? C.v : C.k);
    float *const scales = which ? C.v_scales : C.k_scales;
    const auto block_of = [&](int64_t slot) __attribute__((always_inline)) { return (uint64_t)slot < C.num_slots ? (int32_t)C.slots.quotient((uint32_t)slot) : -1; };
    const auto slot_of = [&](uint64_t t) __attribute__((always_inline)) { return t < P.tokens ? P.slots[t] : (int64_t)-1; };
    // lane l: token from - 1 + l
    const int64_t slot = from + lane ? slot_of((uint64_t)from + lane - 1) : -1;
    const int32_t own = block_of(slot), before = __shfl_up(own, 1);
    uint64_t starts = __ballot(lane >= 1 && lane <= P.window && own >= 0 && own != before);
    while (starts) {
        const int l = __builtin_ctzll(starts);
        starts &= starts - 1;
        const int32_t block = (int32_t)lane_value((uint32_t)own, l);
        const uint32_t first = from + l - 1, first_slot = (uint32_t)block * C.block;
        const uint32_t page = C.page_of_block.quotient((uint32_t)block), in_page = (uint32_t)block - page * C.page_blocks;
        uint8_t *const to = codes + (uint64_t)page * C.page_stride + (uint64_t)h * C.head_stride + (uint64_t)in_page * C.block * C.slot_stride;
        float *const scale_at = scales + ((uint64_t)page * C.heads + h) * C.page_blocks + in_page;
        const float held_scale = *scale_at;
        // the run's tokens, and whether the block's first slot is among theirs
        const uint64_t here = __ballot(own == block) >> l, firsts = __ballot((uint64_t)slot == first_slot) >> l;
        uint32_t count = here == ~0ull ? 64 : __builtin_ctzll(~here);
        bool anew = (firsts & (count == 64 ? ~0ull : (1ull << count) - 1)) != 0;
        if (count == 64 - (uint32_t)l) {
            for (;;) {
                const int64_t s = slot_of((uint64_t)first + count + lane);
                const uint64_t same = __ballot(block_of(s) == block);
                const uint32_t more = same == ~0ull ? 64 : __builtin_ctzll(~same);
                anew |= (__ballot((uint64_t)s == first_slot) & (more == 64 ? ~0ull : (1ull << more) - 1)) != 0;
                count += more;
                if (more < 64) break;
            }
        }
        const uint32_t items = count * pieces;   // (fewer than 2^31: fewer than 2^26 tokens)
        const auto item = [&](uint32_t id) __attribute__((always_inline)) {
            const uint32_t row = C.pieces.quotient(id), piece = id - row * pieces;
            return *(const uint4 *)(x + (uint64_t)(first + row) * stride + 8 * piece);
        };
        uint4 held[kHeld];
        uint32_t largest = 0;
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            held[i] = make_uint4(0, 0, 0, 0);
            if (lane + 64 * i < items) held[i] = item(lane + 64 * i);
        }
#pragma unroll
        for (int i = 0; i < kHeld; ++i) largest = larger_halves(largest, largest_bits(held[i]));
        for (uint32_t id = lane + 64 * kHeld; id < items; id += 64) largest = larger_halves(largest, largest_bits(item(id)));
        uint32_t bits = wave_max(max(largest & 0xFFFFu, largest >> 16));
        bool not_a_number = false;
        if (bits >= kInfinity<T>) {   // (seldom) infinities count as the type's largest value, what is not a number does not count
            not_a_number = bits > kInfinity<T>;
            uint32_t most = 0;
            for (uint32_t id = lane; id < items; id += 64) {
                const uint4 w = item(id);
                const uint16_t *b = (const uint16_t *)&w;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t u = b[i] & 0x7FFFu;
                    most = max(most, u > kInfinity<T> ? 0u : min(u, kInfinity<T> - 1));
                }
            }
            bits = wave_max(most);
        }
        const float top = to_f32(__builtin_bit_cast(T, (uint16_t)bits));
        float wanted = fmaxf(top, kLeastLargest) * (kInt8 ? 1.f / 127.f : 1.f / 448.f);
        if (kInt8 && not_a_number) wanted = NAN;   // (whole numbers have no code for it: the whole block is none)
        const float scale = anew || held_scale < wanted ? wanted : held_scale == held_scale && wanted != wanted ? wanted : held_scale;
        const float inverse = 1.f / scale;
        if (!anew && held_scale < scale) {
            const float by = held_scale * inverse;
            const uint32_t all = C.block * pieces;
            for (uint32_t id = lane; id < all; id += 64) {
                const uint32_t row = C.pieces.quotient(id), piece = id - row * pieces;
                uint2 *const at = (uint2 *)(to + (uint64_t)row * C.slot_stride + 8 * piece);
                float y[8];
                to_floats<kInt8>(*at, y);
                *at = to_codes<kInt8>(y, by);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (stored before the run's own rows, some of which lie there too)
        }
        const auto store = [&](uint32_t id, uint4 w) __attribute__((always_inline)) {
            const uint32_t row = C.pieces.quotient(id), piece = id - row * pieces;
            const uint32_t in_block = (uint32_t)P.slots[first + row] - first_slot;
            float y[8];
            values_of<T>(w, y);
            *(uint2 *)(to + (uint64_t)in_block * C.slot_stride + 8 * piece) = to_codes<kInt8>(y, inverse);
        };
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (lane + 64 * i < items) store(lane + 64 * i, held[i]);
        for (uint32_t id = lane + 64 * kHeld; id < items; id += 64) store(id, item(id));
        if (lane == 0) *scale_at = scale;
    }
}

// ---- reading -------------------------------------------------------------------------------------------------------
//
// A lane brings eight values of a key and of a value of one token at a time; a token has as many neighbouring lanes as it has such pieces (a power of two, at most the wave), so that tokens of
// few heads share a wave.  The wave finds the request of its first token among 64 at a time, a lane goes on from there (100000 free places in between 8.7 us, one after the other 6800).  What is written is not read again soon: it goes past the caches.
// Bound by memory: 62000 tokens of 8 heads of 128 70.9 us (384 MB, 5.4 TB/s; a copy 6.5); 100 tokens, where the search and the table's entry wait for each other, 2.9 us.
struct BlockReadParams {
    BlockCacheParams c;
    const int32_t *offsets, *first, *table;
    uint64_t table_stride;
    uint32_t n, tokens, table_width, first_token;      // first_token: of a launch
    uint32_t token_pieces, lanes;                      // heads * dim / 8; lanes of a token: 2^lanes
    Divider page;                                      // slots of a page
    void *k, *v;
    uint64_t k_stride, v_stride;
};

template <typename T, bool kInt8> __global__ __launch_bounds__(256) void block_read_kernel(BlockReadParams P) {
    const BlockCacheParams &C = P.c;
    const uint32_t lane = threadIdx.x & 63, t0 = P.first_token + (uniform(blockIdx.x * 4 + (threadIdx.x >> 6)) << (6 - P.lanes)), t = t0 + (lane >> P.lanes);
    if (t0 >= P.tokens) return;
    // the last request that begins at t0 or before it: 64 at a time, then the beginnings from it on, one a lane
    uint32_t from = 0;
    for (uint32_t size = P.n; size > 64;) {
        const uint32_t step = (size + 63) / 64, probe = lane * step;
        const uint64_t not_behind = __ballot(probe < size && P.offsets[from + probe] <= (int32_t)t0);
        const uint32_t last = not_behind == ~0ull ? 63u : max(1u, (uint32_t)__builtin_ctzll(~not_behind)) - 1;
        from += last * step, size = min(step, size - last * step);
    }
    const int32_t begins = from + lane <= P.n ? P.offsets[from + lane] : 0x7fffffff;   // (behind the last one: where that ends)
    const uint64_t not_behind = __ballot(from + lane < P.n && begins <= (int32_t)t0);
    const uint32_t l = not_behind == ~0ull ? 63u : max(1u, (uint32_t)__builtin_ctzll(~not_behind)) - 1;
    uint32_t r = from + l;
    int32_t begin = (int32_t)lane_value((uint32_t)begins, l), end = l < 63 ? (int32_t)lane_value((uint32_t)begins, l + 1) : P.offsets[r + 1];
    if (end <= (int32_t)t && r + 1 < P.n) {   // the next one mostly; behind free places in steps that double, then by bisection
        uint32_t step = 1;
        for (++r; step < P.n - r && P.offsets[r + step] <= (int32_t)t; step *= 2) r += step;
        for (uint32_t behind = r + min(step, P.n - r); behind - r > 1;) {
            const uint32_t middle = r + (behind - r) / 2;
            (P.offsets[middle] <= (int32_t)t ? r : behind) = middle;
        }
        begin = P.offsets[r], end = P.offsets[r + 1];
    }
    if ((int32_t)t < begin || (int32_t)t >= end || t >= P.tokens) return;   // (nobody's)
    const int64_t position = (int64_t)t - begin + (P.first ? P.first[r] : 0);
    const uint32_t where = position >= 0 && position <= 0x7fffffff ? P.page.quotient((uint32_t)position) : ~0u;
    uint32_t page = ~0u;
    if (where < P.table_width) page = (uint32_t)P.table[(uint64_t)r * P.table_stride + where];
    const bool there = page < C.pages;
    const uint32_t slot = there ? (uint32_t)position - where * P.page.divisor : 0u;
    const uint64_t codes_at = (uint64_t)page * C.page_stride + (uint64_t)slot * C.slot_stride, scales_at = (uint64_t)page * C.heads * C.page_blocks + C.slots.quotient(slot);
    for (uint32_t inside = lane & ((1u << P.lanes) - 1); inside < P.token_pieces; inside += 1u << P.lanes) {
        const uint32_t h = C.pieces.quotient(inside), piece = inside - h * C.pieces.divisor;
        uint2 codes[2] = {make_uint2(0, 0), make_uint2(0, 0)};
        float by[2] = {0.f, 0.f};
        if (there) {
            const uint64_t at = codes_at + (uint64_t)h * C.head_stride + 8 * piece, scale = scales_at + (uint64_t)h * C.page_blocks;
            codes[0] = *(const uint2 *)((const uint8_t *)C.k + at), codes[1] = *(const uint2 *)((const uint8_t *)C.v + at);
            by[0] = C.k_scales[scale], by[1] = C.v_scales[scale];
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            float y[8];
            to_floats<kInt8>(codes[x], y);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] *= by[x];
            const u32x4 w = {pack2<T>(y[0], y[1]), pack2<T>(y[2], y[3]), pack2<T>(y[4], y[5]), pack2<T>(y[6], y[7])};
            __builtin_nontemporal_store(w, (u32x4 *)((T *)(x ? P.v : P.k) + t * (x ? P.v_stride : P.k_stride) + 8 * inside));
        }
    }
}

}  // namespace
