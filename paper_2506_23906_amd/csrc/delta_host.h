// libmmvseg, part of the translation unit delta.hip (included there, in order).
// Host side of the gated delta rule: argument checks, workspaces, launches.
#pragma once

namespace {

inline bool delta_sizes(uint64_t n, uint64_t tokens, uint32_t heads, uint32_t k_heads, uint32_t dk, uint32_t dv) {
    return n < kMostRequests && tokens < k2to31 && heads >= 1 && heads <= kMostHeads && k_heads >= 1 && k_heads <= heads && heads % k_heads == 0 && dk >= 8 && dk <= kMostDk &&
           dk % 8 == 0 && dv >= 8 && dv <= kMostDv && dv % 8 == 0 && n * heads < k2to31;
}
mmv_status delta_params(DeltaParams &P, uint64_t n, uint64_t tokens, uint32_t heads, uint32_t k_heads, uint32_t dk, uint32_t dv, const void *q, uint64_t q_stride, const void *k,
                        uint64_t k_stride, const void *v, uint64_t v_stride, int type, const float *log_decay, const float *beta, float scale, const float *state_in,
                        float *state_out, uint64_t states, const int32_t *state_index, void *out) {
    if (!valid_value_type(type) || states >= k2to31 || q_stride % 8 || k_stride % 8 || v_stride % 8) return MMV_ERR_INVALID_ARG;
    if (tokens > 1 && (q_stride < (uint64_t)k_heads * dk || k_stride < (uint64_t)k_heads * dk || v_stride < (uint64_t)heads * dv)) return MMV_ERR_INVALID_ARG;
    if (q_stride > kMostStride || k_stride > kMostStride || v_stride > kMostStride) return MMV_ERR_INVALID_ARG;
    if (!state_index && (state_in || state_out) && states < n) return MMV_ERR_INVALID_ARG;
    if (tokens && n && (!q || !k || !v || !out || !log_decay || !beta)) return MMV_ERR_NULL;
    for (const void *p : {q, k, v, (const void *)out, (const void *)state_in, (const void *)state_out})
        if (!aligned_to(p, 16)) return MMV_ERR_INVALID_ARG;
    if (!aligned_to(log_decay, 4) || !aligned_to(beta, 4) || !aligned_to(state_index, 4)) return MMV_ERR_INVALID_ARG;
    const uint64_t bytes = states * heads * dk * dv * 4;
    if (state_in && state_out && state_in != state_out && (uintptr_t)state_in < (uintptr_t)state_out + bytes && (uintptr_t)state_out < (uintptr_t)state_in + bytes)
        return MMV_ERR_INVALID_ARG;
    P.q = q, P.k = k, P.v = v, P.q_stride = q_stride, P.k_stride = k_stride, P.v_stride = v_stride, P.tokens = tokens;
    if (tokens <= 1) P.q_stride = P.k_stride = (uint64_t)k_heads * dk, P.v_stride = (uint64_t)heads * dv;   // (not checked above: no second token)
    P.log_decay = log_decay, P.beta = beta, P.state_in = state_in, P.state_out = state_out, P.state_index = state_index, P.states = states, P.out = out;
    P.n = (uint32_t)n, P.heads = heads, P.group = heads / k_heads, P.dk = dk, P.dv = dv, P.scale = scale;
    return MMV_OK;
}

// Rows that the threads of a workgroup have at once (16 at most: their sums are joined one by one), and of a thread: as few registers as hold them, for more waves (128 requests of 32 heads of
// 64 x 64, four rows a thread: 32.3 us, with registers for sixteen 37.3; 200 of 16 heads of 64 x 160, eight: 60.0, 65.4).
template <typename T, int kThreads> mmv_status launch_step(DeltaParams P, hipStream_t s) {
    const uint32_t fit = kThreads / (P.dv / 4), step = fit < 16 ? fit : 16, rows = (uint32_t)ceil_div(P.dk, step), most = most_of_a_launch(kThreads, P.heads);
    for (; P.first < P.n; P.first += most) {
        const uint32_t blocks = (P.n - P.first < most ? P.n - P.first : most) * P.heads;
        if (rows <= 4) delta_step_kernel<T, 4, kThreads><<<blocks, kThreads, 0, s>>>(P, step);
        else if (rows <= 8) delta_step_kernel<T, 8, kThreads><<<blocks, kThreads, 0, s>>>(P, step);
        else delta_step_kernel<T, 16, kThreads><<<blocks, kThreads, 0, s>>>(P, step);
        if (const mmv_status st = launched()) return st;
    }
    return MMV_OK;
}
template <typename T> mmv_status launch_steps(const DeltaParams &P, hipStream_t s) { return step_threads(P.dv) == 512 ? launch_step<T, 512>(P, s) : launch_step<T, 256>(P, s); }
mmv_status delta_step_call(const DeltaParams &P, int type, hipStream_t s) { return type == MMV_TYPE_F16 ? launch_steps<f16_t>(P, s) : launch_steps<bf16_t>(P, s); }

// Chunks that the requests can have together, and blocks of a head that the device has at once (a workgroup on a compute unit).
inline uint64_t delta_chunks(uint64_t n, uint64_t tokens) { return tokens / kChunk + (n < tokens ? n : tokens); }
// States of blocks: a request of more than one block fills more than half of its own, and a block is as large as the plan on the device makes it, or kLeastBlock.  0: never taken apart.
inline uint32_t delta_round(uint32_t heads, uint32_t dv) { return kUnits / (heads * delta_slices(dv, 4)); }
inline uint64_t delta_slots(uint64_t n, uint64_t tokens, uint32_t heads, uint32_t dv) {
    const uint64_t chunks = delta_chunks(n, tokens), round = delta_round(heads, dv), most = 2 * round;
    const uint64_t longest = ceil_div(tokens, kChunk);
    if (!worth_taking_apart(longest, longest, (uint32_t)round)) return 0;   // (all tokens in one request: nothing is more uneven)
    return 2 * chunks / kLeastBlock < most ? 2 * chunks / kLeastBlock : most;
}
inline size_t delta_chunk_bytes(uint64_t n, uint64_t tokens, uint32_t heads) { return (size_t)delta_chunks(n, tokens) * heads * kChunkBytes; }
inline size_t delta_state_bytes(uint64_t slots, uint32_t heads, uint32_t dk, uint32_t dv) { return round256((size_t)slots * heads * dk * (dk + dv) * 4); }
inline bool delta_counted(uint64_t n, uint64_t tokens) { return n > kCountedByAll && tokens; }
inline size_t delta_count_bytes(uint64_t n, uint64_t tokens, uint64_t slots) { return delta_counted(n, tokens) ? round256(4 * (slots ? 3 * n + 2 : n)) : 0; }
inline size_t delta_workspace(uint64_t n, uint64_t tokens, uint32_t heads, uint32_t dk, uint32_t dv) {
    const uint64_t slots = delta_slots(n, tokens, heads, dv);
    return delta_chunk_bytes(n, tokens, heads) + delta_state_bytes(slots, heads, dk, dv) + delta_count_bytes(n, tokens, slots);
}
template <typename T> mmv_status launch_chunks(DeltaPromptParams P, hipStream_t s) {
    const uint32_t most = most_of_a_launch(256, P.d.heads);
    for (; P.first < P.most_chunks; P.first += most) {
        delta_chunks_kernel<T><<<(P.most_chunks - P.first < most ? P.most_chunks - P.first : most) * P.d.heads, 256, 0, s>>>(P);
        if (const mmv_status st = launched()) return st;
    }
    return MMV_OK;
}
// Workgroups go on to the next block by themselves: where nothing is taken apart, the launches for that are of as many as the device holds.
// Workgroups of 128 columns where they fill the device twice, of 64 and four more waves that bring chunks where a request's own time counts (and where 64 are all).  us, 64 / 128: requests from 64 to
// 4096 tokens, 240 workgroups (of 128) 266 / 412, 384 306 / 463 (fp16 474 / 597), 512 388 / 505; requests of one length, 512 393 / 376, 1024 765 / 722 (fp16 1082 / 868), 3200 (100 tokens) 486 / 386.  Lengths
// are not known here, so that uneven ones lose at 512 what even ones gain from there on.
constexpr uint32_t kFilledTwice = 2 * kUnits;
constexpr uint64_t kMostWorkgroups = 1u << 22;
template <int KD, typename T, int kCompute> mmv_status launch_delta_prompts(const DeltaPromptParams &P, hipStream_t s) {
    if (P.block_states) {
        // (64 columns to a workgroup here whatever the requests are: 45000 tokens 416 us, 128 columns 451)
        delta_prompt_kernel<KD, T, true, 4><<<4 * kUnits, 512, 0, s>>>(P);
        if (const mmv_status st = launched()) return st;
        delta_states_kernel<KD><<<4 * kUnits, 64 * KD, 0, s>>>(P);
        if (const mmv_status st = launched()) return st;
    }
    uint64_t blocks = (uint64_t)P.d.n * P.d.heads * delta_slices(P.d.dv, kCompute);
    if (P.block_states && blocks < 4 * kUnits) blocks = 4 * kUnits;
    delta_prompt_kernel<KD, T, false, kCompute><<<(unsigned)(blocks < kMostWorkgroups ? blocks : kMostWorkgroups), 512, 0, s>>>(P);
    return launched();
}
template <int KD, typename T> mmv_status launch_delta_prompts(const DeltaPromptParams &P, hipStream_t s) {
    return P.d.n * P.d.heads * delta_slices(P.d.dv, 8) >= kFilledTwice && P.d.dv > 64 ? launch_delta_prompts<KD, T, 8>(P, s) : launch_delta_prompts<KD, T, 4>(P, s);
}
template <typename T> mmv_status delta_prompts(const DeltaPromptParams &P, hipStream_t s) {
    if (P.ends) {
        delta_count_kernel<<<1, kCountThreads, 0, s>>>(P);
        if (const mmv_status st = launched()) return st;
    }
    if (const mmv_status st = launch_chunks<T>(P, s)) return st;
    if (P.d.dk <= 64) return launch_delta_prompts<2, T>(P, s);
    if constexpr (__is_same(T, bf16_t))
        if (P.d.dk <= 96) return launch_delta_prompts<3, T>(P, s);
    return launch_delta_prompts<4, T>(P, s);
}
mmv_status delta_call(const DeltaParams &d, int type, void *d_ws, hipStream_t s) {
    DeltaPromptParams P = {};
    P.d = d, P.chunks = (char *)d_ws, P.most_chunks = (uint32_t)delta_chunks(d.n, d.tokens);
    P.slots = (uint32_t)delta_slots(d.n, d.tokens, d.heads, d.dv), P.round = delta_round(d.heads, d.dv);
    char *const behind = (char *)d_ws + delta_chunk_bytes(d.n, d.tokens, d.heads);
    if (P.slots) P.block_states = (float *)behind;
    if (delta_counted(d.n, d.tokens)) {
        P.ends = (uint32_t *)(behind + delta_state_bytes(P.slots, d.heads, d.dk, d.dv));
        if (P.slots) P.block_ends = P.ends + d.n, P.slot_ends = P.block_ends + d.n, P.plan = P.slot_ends + d.n;
    }
    return type == MMV_TYPE_F16 ? delta_prompts<f16_t>(P, s) : delta_prompts<bf16_t>(P, s);
}

}  // namespace
