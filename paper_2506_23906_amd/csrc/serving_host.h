// libmmvseg, part of the translation unit serving.hip (included there, in order).
// Host side of a serving step's calls: argument checks, workspaces, launches.
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

inline size_t tables_workspace(uint64_t n) { return n <= kTablesLocal ? 0 : round256(8 * n); }

mmv_status tables_call(TablesParams P, void *d_ws, hipStream_t s) {
    const uint64_t blocks = ceil_div(P.max_tokens, kTablesThreads);
    const unsigned grid = blocks ? (unsigned)blocks : 1;
    if (P.n <= kTablesLocal) {
        page_tables_kernel<true><<<grid, kTablesThreads, 0, s>>>(P);
        return launched();
    }
    P.ends = (uint32_t *)d_ws, P.taken = P.ends + P.n;
    sum_requests_kernel<<<1, 1024, 0, s>>>(P);
    if (const mmv_status st = launched()) return st;
    page_tables_kernel<false><<<grid, kTablesThreads, 0, s>>>(P);
    return launched();
}

// The cache itself, and that values of `type` can go into it and be multiplied with it.
inline mmv_status check_cache(const mmv_paged_cache *c, int type) {
    if (!c) return MMV_ERR_NULL;
    const int own = c->type;
    if (!valid_value_type(type) || (own != MMV_TYPE_E4M3 && own != type)) return MMV_ERR_INVALID_ARG;
    if (c->page < 1 || c->page > 65536 || c->heads < 1 || c->heads > kMostHeads || c->dim < 8 || c->dim > 256 || c->dim % 8) return MMV_ERR_INVALID_ARG;
    if (c->pages >= k2to31 || c->pages * c->page >= k2to31 || c->page_stride % 8 || c->head_stride % 8 || c->slot_stride % 8) return MMV_ERR_INVALID_ARG;
    // (kernels hold the strides of pages and slots in 32 bits, the bytes of seven slots too; heads may lie further apart)
    if (c->page_stride >= k2to31 || c->head_stride > (1ull << 40) || c->slot_stride >= (1ull << 28)) return MMV_ERR_INVALID_ARG;
    if (own == MMV_TYPE_E4M3 ? !(c->k_scale > 0.f && c->v_scale > 0.f && c->k_scale < INFINITY && c->v_scale < INFINITY) : !(c->k_scale == 1.f && c->v_scale == 1.f)) return MMV_ERR_INVALID_ARG;
    if (c->pages && (!c->d_k || !c->d_v)) return MMV_ERR_NULL;
    return aligned_to(c->d_k, 16) && aligned_to(c->d_v, 16) ? MMV_OK : MMV_ERR_INVALID_ARG;
}

mmv_status append_call(uint64_t tokens, const void *k, uint64_t k_stride, const void *v, uint64_t v_stride, int type, const int64_t *slots,
                       const mmv_paged_cache &c, hipStream_t s) {
    AppendParams P = {};
    P.k_stride = k_stride, P.v_stride = v_stride;
    P.cache_k = c.d_k, P.cache_v = c.d_v, P.page_stride = c.page_stride, P.head_stride = c.head_stride, P.slot_stride = c.slot_stride;
    P.page = divider(c.page), P.num_slots = (uint32_t)(c.pages * c.page), P.head_pieces = divider(c.dim / 8), P.pieces = divider(c.heads * (c.dim / 8));
    P.k_by = (float)(1.0 / c.k_scale), P.v_by = (float)(1.0 / c.v_scale);
    const uint64_t most = (k2to31 - 256) / P.pieces.divisor;   // tokens of a launch: its pieces have numbers below 2^31
    for (uint64_t first = 0; first < tokens; first += most) {
        P.total = (uint32_t)((tokens - first < most ? tokens - first : most) * P.pieces.divisor);
        P.k = (const char *)k + 2 * first * k_stride, P.v = (const char *)v + 2 * first * v_stride, P.slots = slots + first;
        const unsigned blocks = (unsigned)ceil_div(P.total, 256);
        if (c.type != MMV_TYPE_E4M3) cache_append_kernel<bf16_t, false><<<blocks, 256, 0, s>>>(P);   // (bits are copied: one kernel for both types)
        else if (type == MMV_TYPE_F16) cache_append_kernel<f16_t, true><<<blocks, 256, 0, s>>>(P);
        else cache_append_kernel<bf16_t, true><<<blocks, 256, 0, s>>>(P);
        if (const mmv_status st = launched()) return st;
    }
    return MMV_OK;
}

inline bool attention_sizes(uint64_t n, uint32_t q_heads, uint32_t heads, uint32_t dim, uint64_t max_context) {
    return n < kMostRequests && heads >= 1 && heads <= kMostHeads && q_heads >= heads && q_heads % heads == 0 && q_heads / heads <= 16 && dim >= 8 && dim <= 256 && dim % 8 == 0 &&
           max_context < k2to31 && n * q_heads < k2to31 && n * heads * ceil_div(max_context, kTile) < 2 * k2to31;
}
// Waves that share the list of tiles: as many as keep 64 KB of keys and values under way on every compute unit (a wave has a tile of both at a time), or
// one for every tile there can be.  32 rows of 16000, us with 4 / 8 waves on a compute unit: 128 16-bit values (16 KB a tile) 316 / 322,
// 128 8-bit ones 183 / 164, 64 16-bit ones 178 / 169; 12 and more waves are slower everywhere (48 ragged rows of 128 16-bit values 72 -> 75).
constexpr uint32_t kUnits = 256;   // compute units of an MI355X
inline uint32_t attention_workers(uint64_t n, uint32_t heads, uint32_t dim, uint64_t max_context, bool e4m3) {
    const uint32_t tile_bytes = 2 * kTile * dim * (e4m3 ? 1 : 2);
    const uint64_t tiles = n * heads * ceil_div(max_context, kTile), most = 4ull * kUnits * (tile_bytes > 8192 ? 1 : tile_bytes > 4096 ? 2 : 4);
    const uint64_t w = tiles < most ? tiles : most;
    return w < 1 ? 1u : (uint32_t)w;
}
struct AttentionLayout {
    size_t ml, out, total;
};
inline AttentionLayout attention_layout(uint64_t n, uint32_t q_heads, uint32_t heads, uint32_t dim, uint64_t max_context, bool e4m3) {
    const size_t parts = 2ull * attention_workers(n, heads, dim, max_context, e4m3) * (q_heads / heads);
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
template <int KS, bool kExact, bool kStream, typename T, bool kE4m3> void launch_attention_kernel(const AttentionParams &P, hipStream_t s) {
    if (const uint32_t waves = whole_waves(P))
        whole_attention_kernel<KS, kExact, kStream, T, kE4m3><<<P.n * P.heads, 64 * waves, waves * P.group * P.dim * 4, s>>>(P);
    else
        paged_attention_kernel<KS, kExact, kStream, T, kE4m3><<<(P.workers + 3) / 4, 256, 0, s>>>(P);
}
template <bool kStream, typename T, bool kE4m3> void launch_attention(const AttentionParams &P, hipStream_t s) {
    const bool packed = P.slot_stride == P.dim;
    if (P.dim == 64 && packed) launch_attention_kernel<2, true, kStream, T, kE4m3>(P, s);
    else if (P.dim == 128 && packed) launch_attention_kernel<4, true, kStream, T, kE4m3>(P, s);
    else if (P.dim == 256 && packed) launch_attention_kernel<8, true, kStream, T, kE4m3>(P, s);
    else if (P.dim <= 64) launch_attention_kernel<2, false, kStream, T, kE4m3>(P, s);
    else if (P.dim <= 96) launch_attention_kernel<3, false, kStream, T, kE4m3>(P, s);
    else if (P.dim <= 128) launch_attention_kernel<4, false, kStream, T, kE4m3>(P, s);
    else if (P.dim <= 160) launch_attention_kernel<5, false, kStream, T, kE4m3>(P, s);
    else launch_attention_kernel<8, false, kStream, T, kE4m3>(P, s);
}
// A cache that the chip's own (256 MB on the memory side) cannot keep until the next call is read past it.  Us without / with: 48 rows of 330 MB 71.9 ->
// 68.8, 16 rows of 730 MB 136 -> 123, 13 rows of 160 MB 36.7 -> 35.2; but 24 rows of 56 MB, three such caches in turn, 14.9 -> 16.5.
constexpr uint64_t kStreamBytes = 128ull << 20;
template <typename T, bool kE4m3> void launch_attention_over(const AttentionParams &P, hipStream_t s) {
    const uint64_t bytes = 2ull * P.pages * P.page * P.heads * P.dim * (kE4m3 ? 1 : 2);
    if (bytes > kStreamBytes) launch_attention<true, T, kE4m3>(P, s);
    else launch_attention<false, T, kE4m3>(P, s);
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

mmv_status attention_call(AttentionParams P, int type, int cache_type, void *d_ws, hipStream_t s) {
    const bool e4m3 = cache_type == MMV_TYPE_E4M3;
    const AttentionLayout L = attention_layout(P.n, P.q_heads, P.heads, P.dim, P.max_context, e4m3);
    P.sums = (uint32_t *)d_ws, P.part_ml = (float *)((char *)d_ws + L.ml), P.part_out = (float *)((char *)d_ws + L.out);
    P.workers = attention_workers(P.n, P.heads, P.dim, P.max_context, e4m3);
    P.page_groups = divider(P.page / 8);
    P.out_by *= type == MMV_TYPE_F16 ? 1.f / (1 << kScaleBits<f16_t>) : 1.f;
    if (type == MMV_TYPE_F16) e4m3 ? launch_attention_over<f16_t, true>(P, s) : launch_attention_over<f16_t, false>(P, s);
    else e4m3 ? launch_attention_over<bf16_t, true>(P, s) : launch_attention_over<bf16_t, false>(P, s);
    if (const mmv_status st = launched()) return st;
    if (whole_waves(P)) return MMV_OK;   // (nothing to join)
    return type == MMV_TYPE_F16 ? launch_join<f16_t>(P, s) : launch_join<bf16_t>(P, s);
}

inline bool decay_sizes(uint64_t n, uint64_t tokens, uint32_t heads, uint32_t kv_heads, uint32_t dk, uint32_t dv) {
    return n < kMostRequests && tokens < k2to31 && heads >= 1 && heads <= kMostHeads && kv_heads >= 1 && kv_heads <= heads && heads % kv_heads == 0 && dk >= 8 && dk <= kMostDk &&
           dk % 8 == 0 && dv >= 8 && dv <= kMostDv && dv % 8 == 0 && n * heads < k2to31;
}
mmv_status decay_params(DecayParams &P, uint64_t n, uint64_t tokens, uint32_t heads, uint32_t kv_heads, uint32_t dk, uint32_t dv, const void *q, uint64_t q_stride, const void *k,
                        uint64_t k_stride, const void *v, uint64_t v_stride, int type, const float *log_decay, float scale, const float *state_in, float *state_out,
                        uint64_t states, const int32_t *state_index, void *out) {
    if (!valid_value_type(type) || states >= k2to31 || q_stride % 8 || k_stride % 8 || v_stride % 8) return MMV_ERR_INVALID_ARG;
    if (tokens > 1 && (q_stride < (uint64_t)heads * dk || k_stride < (uint64_t)kv_heads * dk || v_stride < (uint64_t)kv_heads * dv)) return MMV_ERR_INVALID_ARG;
    if (q_stride > kMostStride || k_stride > kMostStride || v_stride > kMostStride) return MMV_ERR_INVALID_ARG;
    if (!state_index && (state_in || state_out) && states < n) return MMV_ERR_INVALID_ARG;
    if (tokens && n && (!q || !k || !v || !out)) return MMV_ERR_NULL;
    if (n && !log_decay) return MMV_ERR_NULL;
    for (const void *p : {q, k, v, (const void *)out, (const void *)state_in, (const void *)state_out})
        if (!aligned_to(p, 16)) return MMV_ERR_INVALID_ARG;
    if (!aligned_to(log_decay, 4) || !aligned_to(state_index, 4)) return MMV_ERR_INVALID_ARG;
    const uint64_t bytes = states * heads * dk * dv * 4;
    if (state_in && state_out && state_in != state_out && (uintptr_t)state_in < (uintptr_t)state_out + bytes && (uintptr_t)state_out < (uintptr_t)state_in + bytes)
        return MMV_ERR_INVALID_ARG;
    P.q = q, P.k = k, P.v = v, P.q_stride = q_stride, P.k_stride = k_stride, P.v_stride = v_stride, P.tokens = tokens;
    if (tokens <= 1) P.q_stride = (uint64_t)heads * dk, P.k_stride = (uint64_t)kv_heads * dk, P.v_stride = (uint64_t)kv_heads * dv;   // (not checked above: no second token)
    P.log_decay = log_decay, P.state_in = state_in, P.state_out = state_out, P.state_index = state_index, P.states = states, P.out = out;
    P.n = (uint32_t)n, P.heads = heads, P.group = heads / kv_heads, P.dk = dk, P.dv = dv, P.scale = scale;
    return MMV_OK;
}
// Blocks of prompts (the least tokens of one, how many of a head): one for each request, or so many that the workgroups make whole rounds of what the
// device holds at once.  One round has the fewest states to add up and to pass on; but every request's last block is shorter than the others, which
// leaves a part of a single round idle where a request has few blocks, so more than a third as many requests as blocks take two rounds.  Us with one
// round / two / three, 128 columns: 16 heads (32 blocks of a round), 4 requests of up to 16000 tokens 103 / 120 / 137, 8 179 / 197 / 216, 10 237 / 238 /
// 255, 16 417 / 357 / 369, 12 of up to 32768 468 / 456 / 472; 8 heads (64 blocks), 16 of up to 8000 121 / 139 / 148, 24 174 / 185 / 199.
// The workgroups that fit are bf16's.  fp16's take twice the LDS for keys and queries, and one fits where two do (beyond 64 key components), two where three do: what is one round here is two of
// theirs.  Counting those that fit gives half the blocks, whose unequal ends cost about what the states save: us with bf16's count / fp16's own, 16 heads of 128 x 128, 4
// requests of up to 16000 267 / 285, 24 of 4000 382 / 371, 80 of 3000 749 / 576, 12 of 32768 1325 / 1404; 64 x 64 657 / 567; 8 heads of 80 x 112, 30 of 8000 424 / 458.
// A block is as short as one chunk while the chunks of all heads are less than about one round (three prompts of 900 tokens, 8 heads, blocks of
// 64 / 128 / 256 tokens at least 18.1 / 20.6 / 27.3; of 2500 tokens 23.8 / 24.9 / 33.2), beyond two chunks: below that the states' traffic shows (5000
// tokens, 16 heads 39.2 / 34.2 / 35.2).  Up to 256 tokens a block for each request: one launch (one prompt of 200: 14.7, with blocks 16.4; of 300: 17.5, 16.0).
constexpr uint32_t kOneBlock = 256;
constexpr uint64_t kFewTokens = 20480;   // times heads
constexpr uint32_t prompt_waves(uint32_t dv) { return dv <= 64 ? 4 : dv <= 128 ? 8 : dv <= 160 ? 10 : 16; }
// slots: the states that are kept, those of requests of several blocks alone (1000 prompts of 100 tokens, 16 heads of 128 x 128: 66 MB; one for every block 1.1 GB).
struct DecayBlocks {
    uint32_t block, blocks, slots;
    bool split;
};
inline DecayBlocks decay_blocks(uint64_t n, uint64_t tokens, uint32_t heads, uint32_t dk, uint32_t dv) {
    if (tokens <= kOneBlock) return {kOneBlock, (uint32_t)n, 0, false};
    const uint32_t by_waves = 16 / prompt_waves(dv), by_lds = dk <= 64 ? 3 : 2, on_unit = by_waves < by_lds ? by_waves : by_lds;   // workgroups on a compute unit, of bf16
    const uint64_t round = kUnits * on_unit / heads;
    uint64_t blocks = 3 * n <= round ? round : 2 * round;
    if (blocks < n + blocks / 2) blocks = n + blocks / 2;
    if (blocks == n) ++blocks;
    const uint64_t least = tokens * heads <= kFewTokens ? kChunk : 2 * kChunk;
    uint64_t block = least;
    if (n > 64) {   // enough for any lengths: requests need at most one block each and tokens / block
        block = ceil_div(ceil_div(tokens, blocks - n), kChunk) * kChunk;
        if (block < least) block = least;
    }
    const uint64_t slots = 2 * tokens / block;   // (a length of more than one block fills more than half of its blocks)
    return {(uint32_t)block, (uint32_t)blocks, (uint32_t)(slots < blocks ? slots : blocks), true};
}
inline size_t decay_workspace(uint64_t n, uint64_t tokens, uint32_t heads, uint32_t dk, uint32_t dv) {
    const DecayBlocks b = decay_blocks(n, tokens, heads, dk, dv);
    return b.split ? round256((size_t)b.slots * heads * dk * dv * 4) : 0;
}
template <int KD, int NW, typename T, bool kStates> mmv_status launch_blocks(PromptParams P, hipStream_t s) {
    const uint32_t most = most_of_a_launch(64 * NW, P.d.heads);
    for (; P.first_block < P.blocks; P.first_block += most) {
        decay_prompt_kernel<KD, NW, T, kStates><<<(P.blocks - P.first_block < most ? P.blocks - P.first_block : most) * P.d.heads, 64 * NW, 0, s>>>(P);
        if (const mmv_status st = launched()) return st;
    }
    return MMV_OK;
}
inline mmv_status launch_block_states(PromptParams P, hipStream_t s) {
    const uint32_t each = (uint32_t)ceil_div((uint64_t)P.d.dk * P.d.dv, 1024) * P.d.heads, most = most_of_a_launch(256, each);
    for (; P.first_request < P.d.n; P.first_request += most) {
        decay_blocks_kernel<<<(P.d.n - P.first_request < most ? P.d.n - P.first_request : most) * each, 256, 0, s>>>(P);
        if (const mmv_status st = launched()) return st;
    }
    return MMV_OK;
}
template <int KD, int NW, typename T> mmv_status launch_prompts(const PromptParams &P, hipStream_t s) {
    if (P.block_states) {
        if (const mmv_status st = launch_blocks<KD, NW, T, true>(P, s)) return st;
        if (const mmv_status st = launch_block_states(P, s)) return st;
    }
    return launch_blocks<KD, NW, T, false>(P, s);
}
template <int KD, typename T> mmv_status launch_prompts_of(const PromptParams &P, hipStream_t s) {
    switch (prompt_waves(P.d.dv)) {
        case 4: return launch_prompts<KD, 4, T>(P, s);
        case 8: return launch_prompts<KD, 8, T>(P, s);
        case 10: return launch_prompts<KD, 10, T>(P, s);
        default: return launch_prompts<KD, 16, T>(P, s);
    }
}
mmv_status decay_call(const DecayParams &d, int type, void *d_ws, hipStream_t s) {
    PromptParams P = {};
    P.d = d;
    const DecayBlocks b = decay_blocks(d.n, d.tokens, d.heads, d.dk, d.dv);
    P.block = b.block, P.blocks = b.blocks, P.slots = b.slots;
    P.block_states = b.split ? (float *)d_ws : nullptr;
    if (type == MMV_TYPE_F16) return d.dk <= 64 ? launch_prompts_of<2, f16_t>(P, s) : launch_prompts_of<4, f16_t>(P, s);
    return d.dk <= 64 ? launch_prompts_of<2, bf16_t>(P, s) : d.dk <= 96 ? launch_prompts_of<3, bf16_t>(P, s) : launch_prompts_of<4, bf16_t>(P, s);
}
template <typename T> mmv_status launch_step(DecayParams P, hipStream_t s) {
    const uint32_t rows = (uint32_t)ceil_div(P.dk, 256 / (P.dv / 4)), most = most_of_a_launch(256, P.heads);   // rows: of a thread
    for (; P.first < P.n; P.first += most) {
        const uint32_t blocks = (P.n - P.first < most ? P.n - P.first : most) * P.heads;
        if (rows <= 4) decay_step_kernel<T, 4><<<blocks, 256, 0, s>>>(P);
        else if (rows <= 8) decay_step_kernel<T, 8><<<blocks, 256, 0, s>>>(P);
        else decay_step_kernel<T, 16><<<blocks, 256, 0, s>>>(P);
        if (const mmv_status st = launched()) return st;
    }
    return MMV_OK;
}
mmv_status decay_step_call(const DecayParams &P, int type, hipStream_t s) { return type == MMV_TYPE_F16 ? launch_step<f16_t>(P, s) : launch_step<bf16_t>(P, s); }

}  // namespace
