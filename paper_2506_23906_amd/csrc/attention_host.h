// libmmvseg, part of the translation units of a serving step's calls (included there, in order).
// Host side of attention over a paged cache: which kernel, how many waves, workspaces, launches.
#pragma once

namespace {

inline bool attention_sizes(uint64_t n, uint32_t q_heads, uint32_t heads, uint32_t dim, uint64_t max_context) {
    return n < kMostRequests && heads >= 1 && heads <= kMostHeads && q_heads >= heads && q_heads % heads == 0 && q_heads / heads <= 16 && dim >= 8 && dim <= 256 && dim % 8 == 0 &&
           max_context < k2to31 && n * q_heads < k2to31 && n * heads * ceil_div(max_context, kTile) < 2 * k2to31;
}
// Waves that share the list of tiles: as many as keep 64 KB of keys and values under way on every compute unit (a wave has a tile of both at a time), or
// one for every tile there can be.  32 rows of 16000, us with 4 / 8 waves on a compute unit: 128 16-bit values (16 KB a tile) 316 / 322,
// 128 8-bit ones 183 / 164, 64 16-bit ones 178 / 169; 12 and more waves are slower everywhere (48 ragged rows of 128 16-bit values 72 -> 75).
inline uint32_t attention_workers(uint64_t n, uint32_t heads, uint32_t dim, uint64_t max_context, bool eight) {
    const uint32_t tile_bytes = 2 * kTile * dim * (eight ? 1 : 2);
    const uint64_t tiles = n * heads * ceil_div(max_context, kTile), most = 4ull * kUnits * (tile_bytes > 8192 ? 1 : tile_bytes > 4096 ? 2 : 4);
    const uint64_t w = tiles < most ? tiles : most;
    return w < 1 ? 1u : (uint32_t)w;
}
struct AttentionLayout {
    size_t ml, out, total;
};
inline AttentionLayout attention_layout(uint64_t n, uint32_t q_heads, uint32_t heads, uint32_t dim, uint64_t max_context, bool eight) {
    const size_t parts = 2ull * attention_workers(n, heads, dim, max_context, eight) * (q_heads / heads);
    AttentionLayout L;
    L.ml = round256(4 * (n + 1));
    L.out = L.ml + round256(8 * parts);
    L.total = L.out + round256(4 * parts * dim);
    return L;
}
// (for a cache of either size of values)
inline size_t attention_workspace(uint64_t n, uint32_t q_heads, uint32_t heads, uint32_t dim, uint64_t max_context) { return attention_layout(n, q_heads, heads, dim, max_context, true).total; }

// One workgroup for a segment, of as many waves as it can have tiles (by the table, or the window); 0: the list of tiles.  Us, list / whole segments:
// 8 segments of 100 positions 9.4 / 5.6, of 250 9.4 / 7.9, of 500 9.5 / 10.5; 64 ragged ones up to 500 9.8 / 9.2, up to 1000 10.7 / 14.0; 384 in a window
// of 1024 15.0 / 13.9; 1024 of 350 51.3 / 49.5; 2048 up to 1000 74.8 / 90.8.  So: two tiles for a wave at most, or more where the segments
// keep the device busy by themselves; and not many rounds of workgroups, each of which begins with loads that nothing hides.
inline uint32_t whole_waves(const AttentionParams &P) {
    const uint64_t positions = P.window && P.window < P.max_context ? (uint64_t)P.window + kTile - 1 : P.max_context;
    const uint64_t tiles = positions ? ceil_div(positions, kTile) : 1, most = whole_waves_most(P.dim), waves = tiles < most ? tiles : most, steps = ceil_div(tiles, waves);
    const uint64_t segments = (uint64_t)P.n * P.heads, rounds = ceil_div(segments * waves, 2 * kUnits * most);
    return (steps <= 2 || segments >= kUnits) && steps * rounds <= 6 && P.group * P.dim <= 2048 ? (uint32_t)waves : 0u;   // (their parts fit 64 KB of LDS)
}
template <int KS, bool kExact, bool kStream, typename T, int kCache> void launch_attention_kernel(const AttentionParams &P, hipStream_t s) {
    if (const uint32_t waves = whole_waves(P))
        whole_attention_kernel<KS, kExact, kStream, T, kCache><<<P.n * P.heads, 64 * waves, waves * P.group * P.dim * 4, s>>>(P);
    else
        paged_attention_kernel<KS, kExact, kStream, T, kCache><<<(P.workers + 3) / 4, 256, 0, s>>>(P);
}
template <bool kStream, typename T, int kCache> void launch_attention(const AttentionParams &P, hipStream_t s) {
    const bool packed = P.slot_stride == P.dim;
    if (P.dim == 64 && packed) launch_attention_kernel<2, true, kStream, T, kCache>(P, s);
    else if (P.dim == 128 && packed) launch_attention_kernel<4, true, kStream, T, kCache>(P, s);
    else if (P.dim == 256 && packed) launch_attention_kernel<8, true, kStream, T, kCache>(P, s);
    else if (P.dim <= 64) launch_attention_kernel<2, false, kStream, T, kCache>(P, s);
    else if (P.dim <= 96) launch_attention_kernel<3, false, kStream, T, kCache>(P, s);
    else if (P.dim <= 128) launch_attention_kernel<4, false, kStream, T, kCache>(P, s);
    else if (P.dim <= 160) launch_attention_kernel<5, false, kStream, T, kCache>(P, s);
    else launch_attention_kernel<8, false, kStream, T, kCache>(P, s);
}
// A cache that the chip's own (256 MB on the memory side) cannot keep until the next call is read past it.  Us without / with: 48 rows of 330 MB 71.9 ->
// 68.8, 16 rows of 730 MB 136 -> 123, 13 rows of 160 MB 36.7 -> 35.2; but 24 rows of 56 MB, three such caches in turn, 14.9 -> 16.5.
constexpr uint64_t kStreamBytes = 128ull << 20;
template <typename T, int kCache> void launch_attention_over(const AttentionParams &P, hipStream_t s) {
    const uint64_t bytes = 2ull * P.pages * P.page * P.heads * P.dim * (eight_bits(kCache) ? 1 : 2);
    if (bytes > kStreamBytes) launch_attention<true, T, kCache>(P, s);
    else launch_attention<false, T, kCache>(P, s);
}
// Many segments have few parts each and fill the device with two waves a workgroup; fewer segments have more parts, which four waves take at
// once.  Two and four waves, of whole calls: 96 rows of 20 query heads 37.5 and 41.1 us, 100 of 14 12.5 and 13.0; 67 rows of 16 19.5 and
// 17.2, 7 of 32 24.9 and 17.0.
constexpr uint32_t kManyJoins = 1280;

template <typename T> mmv_status launch_join(AttentionParams P, hipStream_t s) {
    if (P.n * P.q_heads <= kManyJoins) {
        join_attention_kernel<T, 4><<<P.n * P.q_heads, 256, 0, s>>>(P);
        return launched();
    }
    const uint32_t most = most_of_a_launch(128, P.q_heads);
    for (; P.first_row < P.n; P.first_row += most) {
        join_attention_kernel<T, 2><<<(P.n - P.first_row < most ? P.n - P.first_row : most) * P.q_heads, 128, 0, s>>>(P);
        if (const mmv_status st = launched()) return st;
    }
    return MMV_OK;
}

// One call over a cache of the kind kCache.
template <typename T, int kCache> mmv_status attention_call(AttentionParams P, void *d_ws, hipStream_t s) {
    const AttentionLayout L = attention_layout(P.n, P.q_heads, P.heads, P.dim, P.max_context, eight_bits(kCache));
    P.sums = (uint32_t *)d_ws, P.part_ml = (float *)((char *)d_ws + L.ml), P.part_out = (float *)((char *)d_ws + L.out);
    P.workers = attention_workers(P.n, P.heads, P.dim, P.max_context, eight_bits(kCache));
    P.page_groups = divider(P.page / 8);
    P.out_by *= 1.f / (1 << kScaleBits<ValueOperand<T, kCache>>);
    launch_attention_over<T, kCache>(P, s);
    if (const mmv_status st = launched()) return st;
    return whole_waves(P) ? MMV_OK : launch_join<T>(P, s);   // (nothing to join)
}

}  // namespace
