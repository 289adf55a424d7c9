// libmmvseg, part of the translation unit serving.hip (included there, in order).
// Attention of one token per row over a paged cache: split over the positions, parts joined.
#pragma once

namespace {

// ---- paged attention ----------------------------------------------------------------------------------------------
//
// Bound by the bytes of the keys and values: each is read once, for all the query heads that share it, straight into
// registers in the layout that the matrix cores take.  The unit of work is a tile of 32 positions of one (row, cache head); all
// tiles of all rows are one list, row after row, and every wave takes an equal run of it, whatever the lengths are:
// the rows are the segments of that list.  A wave keeps the running maximum and sum of its current segment; a segment
// that lies within one wave's run is written at once, one that several waves share leaves partial results (maximum, sum,
// unnormalised output) in the workspace, two for a wave at most, and a second launch joins them.
//
// A tile on the matrix cores (16x16x32), lane = 16 g + r:
//   scores   S^T = K Q^T: row r of A is the key of position 8 (r / 4) + 4 t + r % 4 (t = 0, 1: two products), its 8 dims of a step those of
//            g.  The result's lane (g, query r) then has the positions 8 g + 4 t + i: eight consecutive ones, and they are
//   output   O^T = V^T P^T: ... the eight that the lane holds of B here, so probabilities go from one product to the next in their
//            registers.  A lane loads 8 components of 8 consecutive positions' values (rows of the cache, coalesced)
//            and exchanges 16-bit halves between pairs of positions: one v_perm for two values.
// No LDS and no barrier in the loop.  Query heads beyond the group's are zero columns: the matrix cores have the time (about a tenth of
// what the loads take).  Whole calls: 48 ragged rows of up to 8192 positions (330 MB in bf16) 68.2 us, 62 of them in the list's kernel, 5.3 TB/s;
// 16 of up to 65536 (717 MB in e4m3) 123 us, 117 of them, 6.1 TB/s; one row of 1000 9.5 us, the lives of two launches.
struct AttentionParams {
    const void *q, *k, *v;
    uint64_t q_stride, head_stride;                // elements
    uint32_t page_stride, slot_stride;
    const int32_t *table, *context;
    uint64_t table_stride;
    void *out;
    float *lse;
    float *part_out, *part_ml;                     // [2 * workers][group][dim], [2 * workers][group][2]
    uint32_t *sums;                                // [n + 1] tiles of a head before every row, and of all
    uint32_t n, q_heads, heads, group, dim, page, pages, window, max_context, workers;
    uint32_t first_row;                            // of a joining launch
    Divider page_groups;                           // page / 8
    float score_by, out_by;                        // scale * k_scale * log2(e), v_scale / 2^kScaleBits
};
constexpr uint32_t kTile = 32;                     // positions
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

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
// Two of a word's four 8-bit values as 16-bit ones (exact).
template <bool kHigh> __device__ __forceinline__ uint32_t widen(bf16_t, uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.f, kHigh));
}
template <bool kHigh> __device__ __forceinline__ uint32_t widen(f16_t, uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.f, kHigh));
}
// Probabilities meet the values in 16 bits, as the matrix cores take both operands of one type, and as terms, each what is cut off at the type's precision of what the ones before it
// left, the last one rounded: three in bf16 (24 bits), two in fp16 (22).  Rounded once they would add as much error as the rounding of the result (1.4 times the error of exact
// ones in bf16, 1.2 times in fp16); bf16's third term, below that rounding by 2^-8, takes no time (48 ragged rows 68.1 us with two, 68.4 with three; 123.3 and 123.4 of 8-bit values).
// No term is zero beside a first one that is not (kInfinite: but for 8-bit caches, which hold no infinities): a value's infinity times a probability stays that
// infinity, and what has no weight adds nothing.  In bf16 each is at least 2^-30 of the probability.  fp16 has few exponents: there probabilities are scaled by 2^12 (which the result's
// factor takes back), above a base that lies at most 2^3 below them, so that the largest product's is 2^15, fp16's full precision goes down to 2^-26 of the largest probability and its
// least value is 2^-36 of that, which is also what the second term is at least; scaled by nothing, a tail of 65536 positions at 2^-25 of one beside it (2^-9 of the result) was lost.
template <typename T> constexpr int kScaleBits = __is_same(T, bf16_t) ? 0 : 12;
template <typename T> constexpr float kMostAbove = __is_same(T, bf16_t) ? 8.f : 3.f;   // of a score above the base, in bits
template <typename T> constexpr int kTerms = __is_same(T, bf16_t) ? 3 : 2;
template <bool kInfinite> __device__ __forceinline__ void probability_terms(bf16_t, float a, float b, uint32_t (&to)[3]) {
    const float least_a = a * 0x1p-30f, least_b = b * 0x1p-30f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t x = __builtin_bit_cast(uint32_t, a), y = __builtin_bit_cast(uint32_t, b);
        to[i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
        a -= __builtin_bit_cast(float, x & 0xFFFF0000u), b -= __builtin_bit_cast(float, y & 0xFFFF0000u);
        if (kInfinite) a = fmaxf(a, least_a), b = fmaxf(b, least_b);
    }
    to[2] = pack2<bf16_t>(a, b);
}
template <bool kInfinite> __device__ __forceinline__ void probability_terms(f16_t, float a, float b, uint32_t (&to)[2]) {
    typedef f16_t pair __attribute__((ext_vector_type(2)));
    a *= 0x1p12f, b *= 0x1p12f;
    to[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
    const pair cut = __builtin_bit_cast(pair, to[0]);
    const float cut_a = (float)cut[0], cut_b = (float)cut[1];
    to[1] = kInfinite ? pack2<f16_t>(fmaxf(a - cut_a, fminf(cut_a, 0x1p-24f)), fmaxf(b - cut_b, fminf(cut_b, 0x1p-24f))) : pack2<f16_t>(a - cut_a, b - cut_b);
}
// Largest / sum over the four lanes that differ in g.
__device__ __forceinline__ float over_g_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float over_g_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

struct RowTiles {
    uint32_t begin, end, first, count;   // positions [begin, end), tiles first .. first + count - 1
};
__device__ __forceinline__ RowTiles row_tiles(const AttentionParams &P, int32_t context) {
    const uint32_t end = min(length_of(context), P.max_context), begin = P.window && end > P.window ? end - P.window : 0u;
    const uint32_t first = begin / kTile;
    return {begin, end, first, (end + kTile - 1) / kTile - first};
}
// Inclusive sums over the lanes of a wave.
__device__ __forceinline__ uint32_t wave_upto(uint32_t v) {
    v += dpp_or_zero<0x111, 0xF>(v);
    v += dpp_or_zero<0x112, 0xF>(v);
    v += dpp_or_zero<0x114, 0xF>(v);
    v += dpp_or_zero<0x118, 0xF>(v);
    v += dpp_or_zero<0x142, 0xA>(v);
    return v + dpp_or_zero<0x143, 0xC>(v);
}
// Tiles of a wave's run.  (The list has less than 2^32 tiles: checked on the host.)
__device__ __forceinline__ uint32_t run_of(uint32_t tiles, uint32_t workers) { return tiles / workers + (tiles % workers ? 1u : 0u); }

// Where a wave is in the list of tiles (the same in all its lanes).
struct Place {
    uint32_t row, head, tile, first, last;   // the segment's tiles: first .. last - 1
    uint32_t begin, end;                     // its positions
};
// Uniform loads through the scalar cache: they are not waited for along with the loads of keys and values.
__device__ __forceinline__ int32_t scalar_load(const int32_t *p) { return *(const __attribute__((address_space(4))) int32_t *)(uintptr_t)p; }
__device__ __forceinline__ void enter_row(const AttentionParams &P, Place &at, int32_t context) {
    const RowTiles t = row_tiles(P, context);
    at.first = t.first, at.last = t.first + t.count, at.begin = t.begin, at.end = t.end;
}

template <int KS> constexpr int dims_per_lane() { return KS <= 2 ? 4 : KS <= 4 ? 8 : KS <= 6 ? 12 : 16; }
template <int KS> constexpr int certain_pieces() { return KS <= 2 ? 1 : KS == 3 ? 9 : KS == 4 ? 13 : KS == 5 ? 17 : 21; }   // of 8 dims, of any dim that takes this KS

// kExact: dim = 32 KS, and a slot's values lie behind those of the slot before.  kStream: loads that leave the caches to others.
template <int KS, bool kExact, bool kStream, typename T, bool kE4m3> struct Tile {
    static constexpr int kDims = dims_per_lane<KS>();
    static constexpr int kSize = kE4m3 ? 1 : 2;
    static constexpr int kKeyWords = kE4m3 ? 2 : 4, kValueWords = kE4m3 ? kDims / 4 : kDims / 2;
    uint32_t k[2][KS][kKeyWords], v[8][kValueWords];
    const char *pk, *pv;
    uint32_t pages_ok;   // bit i: the page of positions 8 i .. 8 i + 7 is there

    // Addresses of a tile's rows for this lane.  Pages are looked up for 8 positions at a time: those of the lane's keys are the
    // (r / 4)th of the tile's four, those of its values and scores the g-th.
    __device__ __forceinline__ void find(const AttentionParams &P, const Place &at, uint32_t g, uint32_t r) {
        const int32_t *row = P.table + (uint64_t)at.row * P.table_stride;
        uint64_t off[4];
        pages_ok = 0;
        if (P.page_groups.divisor % 4 == 0) {   // a tile lies in one page
            const uint32_t group = at.tile * 4, page = page_of(P, group);
            off[0] = place_of(P, scalar_load(row + page), group - page * P.page_groups.divisor, 15u);
#pragma unroll
            for (int i = 1; i < 4; ++i) off[i] = off[0] + (uint64_t)(8 * i) * slot_stride(P);
        } else {
            int32_t id[4];
            uint32_t inside[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t group = at.tile * 4 + i, page = page_of(P, group);
                id[i] = -1;
                if (group * 8 < at.end) id[i] = scalar_load(row + page);   // (behind it the row may end)
                inside[i] = group - page * P.page_groups.divisor;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) off[i] = place_of(P, id[i], inside[i], 1u << i);
        }
        const uint64_t head = (uint64_t)at.head * P.head_stride;
        const uint64_t ok_ = head + pick(off, r >> 2) + (r & 3) * slot_stride(P), ov = head + pick(off, g);
        pk = (const char *)P.k + kSize * ok_;
        pv = (const char *)P.v + kSize * ov;
    }
    // Where eight positions begin in a page (relative to the head), and that it is there.  What is read for a page that is not, from page 0, is not used.
    __device__ __forceinline__ uint64_t place_of(const AttentionParams &P, int32_t id, uint32_t inside, uint32_t bits) {
        const bool ok = (uint32_t)id < P.pages;
        pages_ok |= ok ? bits : 0u;
        return (uint64_t)(ok ? (uint32_t)id : 0u) * P.page_stride + (uint64_t)(inside * 8) * slot_stride(P);
    }
    static __device__ __forceinline__ uint64_t pick(const uint64_t (&off)[4], uint32_t i) {
        const uint64_t a = i & 1 ? off[1] : off[0], b = i & 1 ? off[3] : off[2];
        return i & 2 ? b : a;
    }
    static __device__ __forceinline__ uint32_t page_of(const AttentionParams &P, uint32_t g8) { return P.page_groups.quotient(g8); }
    static __device__ __forceinline__ uint32_t slot_stride(const AttentionParams &P) { return kExact ? 32 * KS : P.slot_stride; }
    template <int kWords> static __device__ __forceinline__ void load(uint32_t (&to)[kWords], const char *p) {
        typedef uint32_t words __attribute__((ext_vector_type(kWords)));
        words w;
        if constexpr (kStream) w = __builtin_nontemporal_load((const words *)p);
        else w = *(const words *)p;
#pragma unroll
        for (int i = 0; i < kWords; ++i) to[i] = w[i];
    }
    __device__ __forceinline__ void load_keys(const AttentionParams &P, uint32_t g) {
        const uint32_t pieces = P.dim / 8;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const char *p = pk + (uint32_t)(t * 4 * kSize) * slot_stride(P);
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                if constexpr (kExact && kE4m3) {   // 16 bytes for two steps: the dims of a step are those of this layout, of the queries too
                    if (s % 2 == 0) {
                        uint32_t both[4];
                        load(both, p + s * 32 + g * 16);
                        k[t][s][0] = both[0], k[t][s][1] = both[1], k[t][s + 1][0] = both[2], k[t][s + 1][1] = both[3];
                    }
                } else {
                    uint32_t piece = s * 4 + g;
                    if (!kExact && s * 4 + 3 >= certain_pieces<KS>()) piece = piece < pieces ? piece : 0;
                    load(k[t][s], p + piece * 8 * kSize);
                }
            }
        }
    }
    __device__ __forceinline__ void load_values(const AttentionParams &P, uint32_t r) {
        constexpr int kFirst = kDims >= 8 ? 8 : 4, kSecond = kDims - kFirst;   // components of the lane's one or two pieces
        const uint32_t first = kExact || r * kFirst < P.dim ? r * kFirst : 0;
        const uint32_t second = kExact || 128 + r * (kSecond ? kSecond : 1) < P.dim ? 128 + r * (kSecond ? kSecond : 1) : 0;
        constexpr int kWordsFirst = kFirst * kSize / 4, kWordsSecond = kSecond * kSize / 4;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const char *p = pv + (uint32_t)(j * kSize) * slot_stride(P);
            uint32_t a[kWordsFirst];
            load(a, p + first * kSize);
#pragma unroll
            for (int w = 0; w < kWordsFirst; ++w) v[j][w] = a[w];
            if constexpr (kSecond > 0) {
                uint32_t b[kWordsSecond];
                load(b, p + second * kSize);
#pragma unroll
                for (int w = 0; w < kWordsSecond; ++w) v[j][kWordsFirst + w] = b[w];
            }
        }
    }
    // The lane's dims of step s: 8 from this one on.
    static __device__ __forceinline__ uint32_t step_dim(int s, uint32_t g) { return kExact && kE4m3 ? (s / 2) * 64 + g * 16 + (s % 2) * 8 : s * 32 + g * 8; }
    __device__ __forceinline__ void scores(const AttentionParams &P, const u32x4 (&q)[KS], uint32_t g, f32x4 (&S)[2]) const {
        const uint32_t pieces = P.dim / 8;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            S[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                u32x4 a;
                if constexpr (kE4m3) {
                    a = (u32x4){widen<false>(T(), k[t][s][0]), widen<true>(T(), k[t][s][0]), widen<false>(T(), k[t][s][1]), widen<true>(T(), k[t][s][1])};
                } else {
                    a = (u32x4){k[t][s][0], k[t][s][1], k[t][s][2], k[t][s][3]};
                }
                if (!kExact && s * 4 + 3 >= certain_pieces<KS>()) {   // (what was read twice, times zeros of the query: it may be infinite)
                    const uint32_t keep = (uint32_t)(s * 4) + g < pieces ? ~0u : 0u;
#pragma unroll
                    for (int i = 0; i < 4; ++i) a[i] &= keep;
                }
                S[t] = mfma_16x16x32(T(), a, q[s], S[t]);
            }
        }
    }
    // Component c of the lane's values as the eight positions of a product's operand.
    template <int c> __device__ __forceinline__ u32x4 column() const {
        u32x4 a;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            if constexpr (kE4m3) {
                constexpr uint32_t at = c & 3;
                const uint32_t both = __builtin_amdgcn_perm(v[2 * m + 1][c / 4], v[2 * m][c / 4], at < 2 ? 0x05010400u : 0x07030602u);   // two components of both positions
                a[m] = widen<(at & 1) != 0>(T(), both);
            } else {
                a[m] = __builtin_amdgcn_perm(v[2 * m + 1][c / 2], v[2 * m][c / 2], c % 2 ? 0x07060302u : 0x05040100u);
            }
        }
        return a;
    }
    template <int c = 0> __device__ __forceinline__ void add_values(const u32x4 (&p)[kTerms<T>], f32x4 (&O)[kDims]) const {
        if constexpr (c < kDims) {
            const u32x4 a = column<c>();
#pragma unroll
            for (int i = 0; i < kTerms<T>; ++i) O[c] = mfma_16x16x32(T(), a, p[i], O[c]);
            add_values<c + 1>(p, O);
        }
    }
};

// Four consecutive or eight components of a query's output, from the lane's registers: component c of lane index i (0 .. 3 here: 4 g + i).
template <int kDims> __device__ __forceinline__ uint32_t dim_of(int c, uint32_t r) {
    constexpr int kFirst = kDims >= 8 ? 8 : 4, kSecond = kDims - kFirst;
    return c < kFirst ? r * kFirst + c : 128 + r * kSecond + (c - kFirst);
}
// What a wave has of a segment: the result where it has all of it, else a part for join_attention_kernel: in place 2 * worker where
// the segment began in an earlier wave's run, in 2 * worker + 1 where it begins in this one's and goes on.
template <int kDims, typename T> __device__ __forceinline__ void write_segment(const AttentionParams &P, const Place &at, uint32_t worker, bool begun, bool ended, uint32_t g, uint32_t r,
                                                                             float most, float sum, const f32x4 (&O)[kDims], T) {
    if (r >= P.group) return;   // (a column of zeros)
    const uint64_t query = (uint64_t)at.row * P.q_heads + at.head * P.group + r;
    if (!begun && ended) {
        const float by = sum == 0.f ? 0.f : P.out_by / sum;
        T *out = (T *)P.out + query * P.dim;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < kDims; c += 4) {
                const uint32_t d = dim_of<kDims>(c, 4 * g + i);
                if (d < P.dim) *(u32x2 *)(out + d) = (u32x2){pack2<T>(O[c][i] * by, O[c + 1][i] * by), pack2<T>(O[c + 2][i] * by, O[c + 3][i] * by)};
            }
        if (P.lse && g == 0) P.lse[query] = most == -INFINITY && sum == 0.f ? -INFINITY : (most + __builtin_amdgcn_logf(sum)) * kLn2;
        return;
    }
    const uint64_t part = (uint64_t)(2 * worker + (begun ? 0 : 1)) * P.group + r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < kDims; c += 4) {
            const uint32_t d = dim_of<kDims>(c, 4 * g + i);
            if (d < P.dim) *(f32x4 *)(P.part_out + part * P.dim + d) = (f32x4){O[c][i], O[c + 1][i], O[c + 2][i], O[c + 3][i]};
        }
    if (g == 0) P.part_ml[2 * part] = most, P.part_ml[2 * part + 1] = sum;
}

// `left` tiles of the list from a place on; at the end of every segment, and of the run, finish(place, begun, ended, maximum, sum, output) has what the wave has of it: begun:
// the segment began before the run (given for the first one), ended: it ends here.
template <int KS, bool kExact, bool kStream, typename T, bool kE4m3, typename Finish>
__device__ __forceinline__ void attention_run(const AttentionParams &P, Place at, uint32_t left, bool begun, uint32_t g, uint32_t r, Finish finish) {
    using TileT = Tile<KS, kExact, kStream, T, kE4m3>;
    constexpr int kDims = TileT::kDims;
            TileT tile;
            tile.find(P, at, g, r);
            tile.load_keys(P, g);
            tile.load_values(P, r);
            u32x4 q[KS];
            f32x4 O[kDims];
            float most = -INFINITY, sum = 0.f, recent = 0.f;   // (the probabilities of up to 32 tiles are added up before they meet the rest: of small ones beside a large sum little is lost)
            bool fresh = true;
            for (;;) {
                if (fresh) {   // a new segment: its queries
                    fresh = false;
                    const T *pq = (const T *)P.q + (uint64_t)at.row * P.q_stride + (uint64_t)(at.head * P.group + r) * P.dim;
    #pragma unroll
                    for (int s = 0; s < KS; ++s) {
                        const uint32_t d = TileT::step_dim(s, g);
                        q[s] = (u32x4){0, 0, 0, 0};
                        if (r < P.group && d < P.dim) q[s] = *(const u32x4 *)(pq + d);
                    }
    #pragma unroll
                    for (int c = 0; c < kDims; ++c) O[c] = (f32x4){0.f, 0.f, 0.f, 0.f};
                    most = -INFINITY, sum = 0.f, recent = 0.f;
                }
                f32x4 S[2];
                tile.scores(P, q, g, S);
                float s[8];
    #pragma unroll
                for (int i = 0; i < 8; ++i) s[i] = S[i / 4][i % 4] * P.score_by;
                const uint32_t pages_ok = tile.pages_ok;
                // the next tile's place; its keys are on their way while this one's values are multiplied
                const Place now = at;
                --left;
                if (left && ++at.tile == at.last) {
                    if (++at.head == P.heads) {
                        at.head = 0;
                        do {
                            ++at.row;
                            enter_row(P, at, scalar_load(P.context + at.row));
                        } while (at.first == at.last);   // (a row without positions; a later one has some, as `left` says)
                    }
                    at.tile = at.first;
                }
                if (pages_ok != 15u || now.tile * kTile < now.begin || (now.tile + 1) * kTile > now.end) {
                    uint32_t keep = 0;
    #pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t p = now.tile * kTile + 8 * g + i;
                        if (((pages_ok >> g) & 1) && p >= now.begin && p < now.end) keep |= 1u << i;
                        s[i] = (keep >> i) & 1 ? s[i] : -INFINITY;
                    }
    #pragma unroll
                    for (int j = 0; j < 8; ++j)   // (0 times what lies there need not be 0)
    #pragma unroll
                        for (int w = 0; w < TileT::kValueWords; ++w) tile.v[j][w] = (keep >> j) & 1 ? tile.v[j][w] : 0u;
                }
                tile.find(P, at, g, r);   // (behind the run's last tile: that one again, not used)
                tile.load_keys(P, g);
                float top = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
                // Scores a few bits above the base need no new one (nothing overflows: 16-bit floats reach 2^15).
                if (__any(top > most + kMostAbove<T>)) {
                    const float m = fmaxf(over_g_max(top), most), by = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(most - m);
                    most = m;
                    sum *= by, recent *= by;
    #pragma unroll
                    for (int c = 0; c < kDims; ++c) O[c] *= by;
                }
                const float base = most == -INFINITY ? 0.f : most;
    #pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s[i] = __builtin_amdgcn_exp2f(s[i] - base);
                    recent += s[i];
                }
                u32x4 p[kTerms<T>];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t terms[kTerms<T>];
                    probability_terms<!kE4m3>(T(), s[2 * i], s[2 * i + 1], terms);
#pragma unroll
                    for (int t = 0; t < kTerms<T>; ++t) p[t][i] = terms[t];
                }
                tile.add_values(p, O);
                tile.load_values(P, r);
                const bool ended = now.tile + 1 == now.last;
                if (now.tile % 32 == 31 || ended || !left) sum += recent, recent = 0.f;
                if (ended || !left) {
                    finish(now, begun, ended, most, over_g_sum(sum), O);
                    fresh = true, begun = false;
                }
                if (!left) break;
            }
}

template <int KS, bool kExact, bool kStream, typename T, bool kE4m3> __global__ __launch_bounds__(256, KS > 4 ? 1 : 2) void paged_attention_kernel(AttentionParams P) {
    constexpr int kDims = dims_per_lane<KS>();
    const uint32_t lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    const uint32_t worker = uniform(blockIdx.x * 4 + (threadIdx.x >> 6));
    // the list's length, this wave's run of it, and where that begins
    const int32_t first_context = lane < P.n ? P.context[lane] : 0;
    const uint32_t first_counts = row_tiles(P, first_context).count;
    const uint32_t first_upto = wave_upto(first_counts);
    uint32_t all_rows = lane_value(first_upto, 63);
    if (P.n > 64) {
        uint32_t more = 0;
        for (uint32_t i = 64 + lane; i < P.n; i += 64) more += row_tiles(P, P.context[i]).count;
        all_rows += lane_value(wave_upto(more), 63);
    }
    const uint32_t all = all_rows * P.heads, run = run_of(all, P.workers), start = (uint32_t)min((uint64_t)worker * run, (uint64_t)all);
    uint32_t left = min(run, all - start);
    if (worker == 0 || left) {
        uint32_t before = 0, row = 0, rows_before = 0, row_context = 0;
        const uint32_t target = start / P.heads;
        bool found = false;
        for (uint32_t first = 0; first < P.n && (worker == 0 || !found); first += 64) {
            const uint32_t i = first + lane;
            const int32_t context = first == 0 ? first_context : i < P.n ? P.context[i] : 0;
            const uint32_t own = row_tiles(P, context).count;
            const uint32_t upto = first == 0 ? first_upto : wave_upto(own);
            if (worker == 0 && i < P.n) P.sums[i] = before + upto - own;
            const uint64_t hit = __ballot(before + upto > target);
            if (hit && !found) {
                const int l = __builtin_ctzll(hit);
                found = true;
                row = first + l;
                row_context = lane_value((uint32_t)context, l);
                rows_before = before + lane_value(upto - own, l);
            }
            before += lane_value(upto, 63);
        }
        if (worker == 0 && lane == 0) P.sums[P.n] = all_rows;
        if (!left) return;
        Place at;
        at.row = uniform(row);
        enter_row(P, at, (int32_t)row_context);
        const uint32_t inside = start - rows_before * P.heads, count = at.last - at.first;
        at.head = uniform(inside / count);
        at.tile = at.first + uniform(inside % count);
        attention_run<KS, kExact, kStream, T, kE4m3>(P, at, left, at.tile != at.first, g, r,
                                                     [&](const Place &now, bool begun, bool ended, float most, float sum, const f32x4 (&O)[kDims]) __attribute__((always_inline)) {
                                                         write_segment<kDims>(P, now, worker, begun, ended, g, r, most, sum, O, T());
                                                     });
    }
}

// Joining parts: the largest maximum is the base, and every part counts, with weight 2^(its maximum - the base), whatever that is.  A part of scores that are no numbers has no
// maximum (-infinity) but a sum that is none either, and 0 times that stays no number, as it does for a wave that has the whole segment; a part without positions adds zeros.

// Where no segment has more tiles than a few for each of at most eight waves (four beyond 128 dims, which take more than half of a SIMD's registers): a workgroup has
// one, and joins its waves' parts in LDS.  One launch, and no sums over the rows ahead of the first load.
constexpr uint32_t whole_waves_most(uint32_t dim) { return dim <= 128 ? 8 : 4; }
template <int KS, bool kExact, bool kStream, typename T, bool kE4m3> __global__ __launch_bounds__(64 * whole_waves_most(32 * KS), KS > 4 ? 1 : 2) void whole_attention_kernel(AttentionParams P) {
    constexpr int kDims = dims_per_lane<KS>();
    constexpr uint32_t kWholeWaves = whole_waves_most(32 * KS);
    __shared__ float ml[kWholeWaves][16][2];
    extern __shared__ __align__(16) float parts[];   // [waves][group][dim]
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), waves = blockDim.x / 64, g = lane >> 4, r = lane & 15;
    Place at;
    at.row = uniform(blockIdx.x / P.heads), at.head = blockIdx.x - at.row * P.heads;
    enter_row(P, at, scalar_load(P.context + at.row));
    const uint32_t count = at.last - at.first, run = (count + waves - 1) / waves, start = min(wave * run, count), left = min(run, count - start);
    if (left) {
        at.tile = at.first + start;
        attention_run<KS, kExact, kStream, T, kE4m3>(P, at, left, false, g, r,
                                                     [&](const Place &, bool, bool, float most, float sum, const f32x4 (&O)[kDims]) __attribute__((always_inline)) {
                                                         if (run == count) write_segment<kDims>(P, at, 0, false, true, g, r, most, sum, O, T());   // (this wave has all of it)
                                                         if (r >= P.group || run == count) return;
                                                         float *const part = parts + (wave * P.group + r) * P.dim;
#pragma unroll
                                                         for (int i = 0; i < 4; ++i)
#pragma unroll
                                                             for (int c = 0; c < kDims; c += 4) {
                                                                 const uint32_t d = dim_of<kDims>(c, 4 * g + i);
                                                                 if (d < P.dim) *(f32x4 *)(part + d) = (f32x4){O[c][i], O[c + 1][i], O[c + 2][i], O[c + 3][i]};
                                                             }
                                                         if (g == 0) ml[wave][r][0] = most, ml[wave][r][1] = sum;
                                                     });
    }
    if (run == count && count) return;
    __syncthreads();
    // (every thread makes the waves' factors anew: one more barrier for making them once takes longer)
    const uint64_t first = (uint64_t)at.row * P.q_heads + (uint64_t)at.head * P.group;
    const uint32_t used = count ? (count + run - 1) / run : 0;
    for (uint32_t id = tid; id < P.group * P.dim; id += 64 * waves) {
        const uint32_t q = id / P.dim;
        float most[kWholeWaves], top = -INFINITY, total = 0.f, x = 0.f;
#pragma unroll
        for (uint32_t w = 0; w < kWholeWaves; ++w) {
            most[w] = w < used ? ml[w][q][0] : -INFINITY;
            top = fmaxf(top, most[w]);
        }
        const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (uint32_t w = 0; w < kWholeWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(most[w] - base);
            if (w < used) total += f * ml[w][q][1], x += f * parts[w * P.group * P.dim + id];
        }
        ((T *)P.out)[first * P.dim + id] = from_f32<T>(total == 0.f ? 0.f : x * (P.out_by / total));
        if (P.lse && id == q * P.dim) P.lse[first + q] = total == 0.f && top == -INFINITY ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kLn2;
    }
}

// Joins the parts of the segments that several waves share, and writes the rows without positions: a workgroup for a row and query head.  Its
// kWaves waves take every kWaves-th part each, eight of them under way at a time.  Bound by its life: 3 to 5 us (row sums, then parts, then LDS).
template <typename T, int kWaves> __global__ __launch_bounds__(64 * kWaves) void join_attention_kernel(AttentionParams P) {
    __shared__ float lds[kWaves][256 + 2];
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), id = P.first_row * P.q_heads + blockIdx.x;
    const uint32_t row = id / P.q_heads, qh = id - row * P.q_heads, h = qh / P.group, q = qh - h * P.group;
    const uint32_t before = (uint32_t)scalar_load((const int32_t *)P.sums + row), behind = (uint32_t)scalar_load((const int32_t *)P.sums + row + 1);
    const uint32_t all = (uint32_t)scalar_load((const int32_t *)P.sums + P.n) * P.heads, tiles = behind - before;
    T *out = (T *)P.out + (uint64_t)id * P.dim;
    if (tiles == 0) {
        for (uint32_t d = threadIdx.x; d < P.dim; d += 64 * kWaves) out[d] = from_f32<T>(0.f);
        if (P.lse && threadIdx.x == 0) P.lse[id] = -INFINITY;
        return;
    }
    const uint32_t from = before * P.heads + h * tiles, run = run_of(all, P.workers), first = from / run, last = (from + tiles - 1) / run;
    if (first == last) return;   // (written by that wave)
    // (the segment begins in the first wave's run: its part is that wave's second one)
    const auto place = [&](uint32_t w) __attribute__((always_inline)) { return (uint64_t)(2 * w + (w == first ? 1 : 0)) * P.group + q; };
    float most = -INFINITY, sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (uint32_t w0 = first + wave; w0 <= last; w0 += 8 * kWaves) {
        float part[8][4], m[8], l[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint64_t at = place(min(w0 + kWaves * i, last));
            m[i] = P.part_ml[2 * at], l[i] = P.part_ml[2 * at + 1];
#pragma unroll
            for (int c = 0; c < 4; ++c) part[i][c] = lane + 64 * c < P.dim ? P.part_out[at * P.dim + lane + 64 * c] : 0.f;
        }
        float top = most;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (w0 + kWaves * i > last) m[i] = -INFINITY;
            top = fmaxf(top, m[i]);
        }
        const float base = top == -INFINITY ? 0.f : top, by = __builtin_amdgcn_exp2f(most - base);
        most = top, sum *= by;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] *= by;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float f = __builtin_amdgcn_exp2f(m[i] - base);
            if (w0 + kWaves * i <= last) {
                sum += f * l[i];
#pragma unroll
                for (int c = 0; c < 4; ++c) o[c] += f * part[i][c];
            }
        }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) lds[wave][lane + 64 * c] = o[c];
    if (lane == 0) lds[wave][256] = most, lds[wave][257] = sum;
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds[w][256]);
    const float base = top == -INFINITY ? 0.f : top;
    for (uint32_t d = threadIdx.x; d < P.dim; d += 64 * kWaves) {
        float total = 0.f, x = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(lds[w][256] - base);
            total += f * lds[w][257], x += f * lds[w][d];
        }
        out[d] = from_f32<T>(total == 0.f ? 0.f : x * (P.out_by / total));
        if (P.lse && d == 0) P.lse[id] = total == 0.f && top == -INFINITY ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kLn2;
    }
}

}  // namespace
