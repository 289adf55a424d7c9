// libmmvseg, part of the translation unit serving.hip (included there, in order).
// Host side of a serving step's calls: argument checks, workspaces, launches (attention's are in attention_host.h).
#pragma once

namespace {

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

mmv_status attention_over(const AttentionParams &P, int type, int cache_type, void *d_ws, hipStream_t s) {
    if (type == MMV_TYPE_F16) return cache_type == MMV_TYPE_E4M3 ? attention_call<f16_t, kE4m3>(P, d_ws, s) : attention_call<f16_t, kSixteenBits>(P, d_ws, s);
    return cache_type == MMV_TYPE_E4M3 ? attention_call<bf16_t, kE4m3>(P, d_ws, s) : attention_call<bf16_t, kSixteenBits>(P, d_ws, s);
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
