// libmmvseg, part of the translation unit block.hip (included there, in order).
// Host side of the calls on a cache of 8-bit values in blocks: argument checks, launches.
#pragma once

namespace {

constexpr uint64_t kMostAppended = 1ull << 26;   // tokens of a call: the pieces of any run have numbers below 2^31

inline mmv_status check_block_cache(const mmv_block_cache *c) {
    if (!c) return MMV_ERR_NULL;
    if (c->type != MMV_TYPE_I8 && c->type != MMV_TYPE_E4M3) return MMV_ERR_INVALID_ARG;
    if (c->page < 8 || c->page > 65536 || c->heads < 1 || c->heads > kMostHeads || c->dim < 8 || c->dim > 256 || c->dim % 8) return MMV_ERR_INVALID_ARG;
    if (c->block < 8 || c->block % 8 || c->page % c->block) return MMV_ERR_INVALID_ARG;
    if (c->pages >= k2to31 || c->pages * c->page >= k2to31 || c->page_stride % 8 || c->head_stride % 8 || c->slot_stride % 8) return MMV_ERR_INVALID_ARG;
    // (kernels hold the strides of pages and slots in 32 bits, the bytes of seven slots too; heads may lie further apart)
    if (c->page_stride >= k2to31 || c->head_stride > (1ull << 40) || c->slot_stride >= (1ull << 28)) return MMV_ERR_INVALID_ARG;
    if (c->pages && (!c->d_k || !c->d_v || !c->d_k_scales || !c->d_v_scales)) return MMV_ERR_NULL;
    return aligned_to(c->d_k, 16) && aligned_to(c->d_v, 16) && aligned_to(c->d_k_scales, 4) && aligned_to(c->d_v_scales, 4) ? MMV_OK : MMV_ERR_INVALID_ARG;
}
inline BlockCacheParams block_cache_params(const mmv_block_cache &c) {
    BlockCacheParams C = {};
    C.k = c.d_k, C.v = c.d_v, C.k_scales = c.d_k_scales, C.v_scales = c.d_v_scales;
    C.page_stride = c.page_stride, C.head_stride = c.head_stride, C.slot_stride = c.slot_stride;
    C.heads = c.heads, C.page_blocks = c.page / c.block, C.block = c.block, C.num_slots = (uint32_t)(c.pages * c.page), C.pages = (uint32_t)c.pages;
    C.page_of_block = divider(C.page_blocks), C.slots = divider(c.block), C.pieces = divider(c.dim / 8);
    return C;
}

// Tokens whose runs one wave looks after: one where there are few waves' worth of them (every run in a wave of its own, at once), else as many as a
// block holds: most windows of a prompt then have one run to begin (windows of 16 and 8 tokens for blocks of 32 take 11 % and 40 % longer, by the waves that find nothing to do).  us, one / a block
// (16 tokens), 8 heads of 128: single tokens of 256 requests 4.3 / 18.3, of 1024 9.6 / 19.0, of 2048 17.0 / 22.9; prompts of 128 tokens, 8 of them 6.5 / 5.4, 16 10.2 / 6.8.  At 1024 tokens single
// tokens, which a program appends at every step, gain more than prompts lose.  At 2048 they would still (5.9 of 22.9 us, prompts lose 3.4); there the rule takes the prompts' side: a call of so many tokens is
// more often prompts than one token each of as many requests, which take a third longer for it.
constexpr uint64_t kFewWaves = 16384;
template <int kHeld> mmv_status launch_append(const BlockAppendParams &P, unsigned blocks, int type, bool int8, hipStream_t s) {
    if (type == MMV_TYPE_F16) int8 ? block_append_kernel<kHeld, f16_t, true><<<blocks, 256, 0, s>>>(P) : block_append_kernel<kHeld, f16_t, false><<<blocks, 256, 0, s>>>(P);
    else int8 ? block_append_kernel<kHeld, bf16_t, true><<<blocks, 256, 0, s>>>(P) : block_append_kernel<kHeld, bf16_t, false><<<blocks, 256, 0, s>>>(P);
    return launched();
}
// Registers for the runs that there can be, or for their first part where they are too long anyway: us with 2 / 4 / 8 times 64 pieces, 17600 tokens of 8 heads of 128 (16 pieces) in blocks of
// 8 24.1 / 27.7 / 32.8, of 16 24.3 / 22.9 / 24.0, of 32 28.9 / 27.7 / 25.1, of 64 30.9 / 31.8 / 33.8; single tokens 4.4 / 4.7 / 5.2.
mmv_status block_append_call(BlockAppendParams P, int type, bool int8, hipStream_t s) {
    const uint64_t each = 2ull * P.c.heads;
    P.window = P.tokens * each <= kFewWaves ? 1 : P.c.block < 32 ? P.c.block : 32;
    const uint32_t pieces = P.window == 1 ? 0 : P.c.block * P.c.pieces.divisor;
    const uint64_t windows = ceil_div(P.tokens, P.window), most = ((1ull << 32) - 256) / 64 / each;
    for (uint64_t first = 0; first < windows; first += most) {
        P.first_window = (uint32_t)first, P.windows = (uint32_t)(windows - first < most ? windows - first : most);
        const unsigned blocks = (unsigned)ceil_div(P.windows * each, 4);
        const mmv_status st = pieces <= 128 || pieces > 512 ? launch_append<2>(P, blocks, type, int8, s) : pieces <= 256 ? launch_append<4>(P, blocks, type, int8, s) : launch_append<8>(P, blocks, type, int8, s);
        if (st) return st;
    }
    return MMV_OK;
}
mmv_status block_read_call(BlockReadParams P, int type, bool int8, hipStream_t s) {
    while (P.lanes < 6 && 1u << P.lanes < P.token_pieces) ++P.lanes;
    const uint64_t each = 4u << (6 - P.lanes), most = ((1ull << 24) - 1) * each;   // tokens of a workgroup; of a launch: fewer than 2^32 threads
    for (uint64_t first = 0; first < P.tokens; first += most) {
        P.first_token = (uint32_t)first;
        const uint64_t tokens = P.tokens - first < most ? P.tokens - first : most;
        const unsigned blocks = (unsigned)ceil_div(tokens, each);
        if (type == MMV_TYPE_F16) int8 ? block_read_kernel<f16_t, true><<<blocks, 256, 0, s>>>(P) : block_read_kernel<f16_t, false><<<blocks, 256, 0, s>>>(P);
        else int8 ? block_read_kernel<bf16_t, true><<<blocks, 256, 0, s>>>(P) : block_read_kernel<bf16_t, false><<<blocks, 256, 0, s>>>(P);
        if (const mmv_status st = launched()) return st;
    }
    return MMV_OK;
}

mmv_status block_attention_over(const AttentionParams &P, int type, int cache_type, void *d_ws, hipStream_t s) {
    if (type == MMV_TYPE_F16) return cache_type == MMV_TYPE_I8 ? attention_call<f16_t, kBlocksInt8>(P, d_ws, s) : attention_call<f16_t, kBlocksE4m3>(P, d_ws, s);
    return cache_type == MMV_TYPE_I8 ? attention_call<bf16_t, kBlocksInt8>(P, d_ws, s) : attention_call<bf16_t, kBlocksE4m3>(P, d_ws, s);
}

}  // namespace
