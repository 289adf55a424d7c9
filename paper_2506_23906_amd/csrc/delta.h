// libmmvseg, part of the translation unit delta.hip (included there, in order).
// The gated delta rule.
#pragma once

namespace {

struct DeltaParams {
    const void *q, *k, *v;
    uint64_t q_stride, k_stride, v_stride, tokens;   // strides in elements
    const int32_t *offsets;                          // (prompts)
    const float *log_decay, *beta;                   // [tokens][heads]
    const float *state_in;
    float *state_out;
    const int32_t *state_index;
    uint64_t states;
    void *out;
    uint32_t n, heads, group, dk, dv;
    uint32_t first;                                  // request of a launch
    float scale;
};
constexpr uint32_t kMostDk = 128, kMostDv = 256;
// e^g with an error of fp32's last bit: the exponent in two parts.  Below e^-200, 0 in fp32, the same as there (0 * -infinity is no exponent).
__device__ __forceinline__ float at_least_200(float g) { return g < -200.f ? -200.f : g; }
__device__ __forceinline__ float exp_of(float g) {
    constexpr float kLog2e = 1.44269504f, kRest = 1.92596299e-8f;
    g = at_least_200(g);
    const float x = g * kLog2e, rest = __builtin_fmaf(g, kLog2e, -x) + g * kRest, y = __builtin_amdgcn_exp2f(x);
    return x < 127.f ? __builtin_fmaf(y, rest * 0.693147181f, y) : y;
}

// The state that request r starts from and leaves, ~0 for none.
__device__ __forceinline__ uint64_t state_of(const DeltaParams &P, uint32_t r) {
    const int64_t i = P.state_index ? P.state_index[r] : r;
    return i >= 0 && (uint64_t)i < P.states ? (uint64_t)i : ~0ull;
}
struct Span {
    uint32_t begin, end;
};
__device__ __forceinline__ Span span_of(const DeltaParams &P, uint32_t r) {
    const int64_t most = (int64_t)P.tokens;
    int64_t a = P.offsets[r], b = P.offsets[r + 1];
    a = a < 0 ? 0 : a > most ? most : a;
    b = b < a ? a : b > most ? most : b;
    return {(uint32_t)a, (uint32_t)b};
}

// ---- single tokens -------------------------------------------------------------------------------------------------
//
//   S' = e^g S,   u = beta (v - k S'),   S = S' + k u^T,   out = scale q S = scale (q S' + (q . k) u)
// Bound by reading and writing the state: 8 dk dv bytes for 6 dk dv operations.  A workgroup has one state; a thread takes four columns (16 bytes) of every `step`-th row, so that a pass of the
// workgroup is one run of memory, and all its rows are loaded before the first is used and stay in registers.  k S' and q S' are added up in one pass and joined in LDS.  States are read and written
// past the caches: no other call needs them before the next step.  (Rows in neighbouring lanes, whose sums need no LDS, read less than whole lines where dv is no multiple of 32: 200 requests of 16
// heads of 64 x 160 118 us, so 60.)  128 requests of 32 heads, 128 x 128: 103 us, 5.2 TB/s; 4 of 8 heads of 64 x 64, all of it waiting for memory once, 4.8.
// 512 threads where 256 would have more than sixteen rows of four columns each (128 registers for the state).
constexpr uint32_t step_threads(uint32_t dv) { return dv > 128 ? 512 : 256; }
template <typename T, int kRows, int kThreads> __global__ __launch_bounds__(kThreads, kRows > 8 ? 4 : 6) void delta_step_kernel(DeltaParams P, uint32_t step) {
    __shared__ float query[kMostDk], key[kMostDk], qk[16];
    __shared__ __align__(16) float part[2][kThreads * 4];
    const uint32_t r = P.first + blockIdx.x / P.heads, h = blockIdx.x % P.heads, tid = threadIdx.x, shared = h / P.group;
    const uint64_t state = state_of(P, r);
    const bool have = state != ~0ull;
    const uint32_t quads = P.dv / 4, first = tid / quads, c = (tid - first * quads) * 4;
    const bool live = first < step;   // (threads beyond step * quads have no rows)
    const uint64_t at = (state * P.heads + h) * ((uint64_t)P.dk * P.dv) + c;
    f32x4 S[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const uint32_t d = first + i * step;
        S[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
        if (P.state_in && have && live && d < P.dk) S[i] = __builtin_nontemporal_load((const f32x4 *)(P.state_in + at + (uint64_t)d * P.dv));
    }
    if (tid < P.dk) {
        query[tid] = to_f32(((const T *)P.q)[r * P.q_stride + (uint64_t)shared * P.dk + tid]);
        key[tid] = to_f32(((const T *)P.k)[r * P.k_stride + (uint64_t)shared * P.dk + tid]);
    }
    const T *pv = (const T *)P.v + r * P.v_stride + (uint64_t)h * P.dv + c;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (live) v = (f32x4){to_f32(pv[0]), to_f32(pv[1]), to_f32(pv[2]), to_f32(pv[3])};
    const float decay = exp_of(P.log_decay[(uint64_t)r * P.heads + h]), beta = P.beta[(uint64_t)r * P.heads + h];
    __syncthreads();
    f32x4 by_key = {0.f, 0.f, 0.f, 0.f}, by_query = by_key;
    float both = 0.f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const uint32_t d = first + i * step;
        if (live && d < P.dk) {
            S[i] *= decay;
            by_key += key[d] * S[i], by_query += query[d] * S[i], both += query[d] * key[d];
        }
    }
    if (live) {
        *(f32x4 *)&part[0][first * P.dv + c] = by_key, *(f32x4 *)&part[1][first * P.dv + c] = by_query;
        if (c == 0) qk[first] = both;
    }
    __syncthreads();
    if (!live) return;
    by_key = by_query = (f32x4){0.f, 0.f, 0.f, 0.f}, both = 0.f;
    for (uint32_t i = 0; i < step; ++i) by_key += *(const f32x4 *)&part[0][i * P.dv + c], by_query += *(const f32x4 *)&part[1][i * P.dv + c], both += qk[i];
    const f32x4 u = beta * (v - by_key);
    if (first == 0) {
        const f32x4 o = P.scale * (by_query + both * u);
        *(u32x2 *)((T *)P.out + ((uint64_t)r * P.heads + h) * P.dv + c) = (u32x2){pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
    }
    if (!P.state_out || !have) return;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const uint32_t d = first + i * step;
        if (d < P.dk) {
            const f32x4 x = S[i] + key[d] * u;
            __builtin_nontemporal_store(x, (f32x4 *)(P.state_out + at + (uint64_t)d * P.dv));
        }
    }
}

// ---- prompts: chunks -----------------------------------------------------------------------------------------------
//
// Chunks of 64 tokens on the matrix cores.  With i, j counted from the chunk's beginning, G_i the sum of log_decay up to i, S the state before the chunk and u_i what token i writes,
//   u_i = beta_i (v_i - e^(G_i) k_i S - sum_(j < i) e^(G_i - G_j) (k_i . k_j) u_j)     or   (I + L) U = diag(beta) (V - diag(e^G) K S)
//   out_i = scale (e^(G_i) q_i S + sum_(j <= i) e^(G_i - G_j) (q_i . k_j) u_j),   S' = e^(G_63) S + sum_j e^(G_63 - G_j) k_j u_j^T
// What does not depend on the state is made for all chunks and heads at once (delta_chunks_kernel): T = (I + L)^-1 diag(beta) and, with the scores W_ij = scale e^(G_i - G_j) (q_i . k_j),
//   E = diag(e^(G_63 - G)) T,   M = W T.
// delta_prompt_kernel then goes through a request's chunks: R = V - diag(e^G) K S, out = scale diag(e^G) Q S + M R, S' = e^(G_63) S + K^T E R.
constexpr uint32_t kChunk = 64;
// Workgroups go to the eight dies in turn, and each has a cache of its own: of `each` (the heads of a chunk; of a request, with their slices of columns), neighbours, which read the same, to one (64 prompts of 1024 tokens, 16 heads: 735 to 748 us, so 731 to 741).
__device__ __forceinline__ uint32_t by_die(uint32_t i, uint32_t each) { return each % 8 ? i : (i & 7) * (each / 8) + i / 8; }

// What a chunk of a head leaves: E and M, three bf16 terms (fp32's 24 bits) of each, as operands of 16x16x32 products: rows 32 s + 8 (r / 4) + 4 t + r % 4 (s, t = 0, 1), columns
// 32 c + 8 g + 0..7 in lane 16 g + r, c <= s (above the diagonal there is nothing): the operands (s, t, c) = (0,0,0) (0,1,0) (1,0,0) (1,1,0) (1,0,1) (1,1,1).  One below the diagonal has 64
// pieces of 16 bytes, one on it 40, for the lanes with g <= r / 4, and one of zeros that the other lanes read: a term takes 5 KB instead of 6, and three terms of M the place of two.
constexpr uint32_t kOperands = 6, kTerms = 3, kCorner = 48, kZeros = 44, kPlane = 4 * kCorner + 2 * 64;   // (kCorner, kPlane: pieces of an operand on the diagonal, of a term)
__host__ __device__ constexpr bool on_diagonal(uint32_t f) { return f < 2 || f >= 4; }
__host__ __device__ constexpr uint32_t operand_at(uint32_t f) { return f < 2 ? f * kCorner : f < 4 ? 2 * kCorner + (f - 2) * 64 : 2 * kCorner + 2 * 64 + (f - 4) * kCorner; }
// (a piece's place, in fours: those that the lanes of a read bring at once, 0-3 12-15 20-23 24-27 and so on, lie in different banks; 11: the zeros)
__device__ __forceinline__ uint32_t corner_piece(uint32_t g, uint32_t r) { return g <= r >> 2 ? 4 * (uint32_t)(0xA861B935BB24BBB0ull >> 4 * ((r & 12) + g) & 15) + (r & 3) : kZeros; }
constexpr uint32_t kMatrixPieces = 2 * kTerms * kPlane;                                          // E's terms, then M's
constexpr uint32_t kChunkBytes = kMatrixPieces * 16 + 512;                                     // behind the matrices: e^(G_i), scale e^(G_i)

struct DeltaPromptParams {
    DeltaParams d;
    char *chunks;            // [chunks of all requests][heads] of kChunkBytes
    uint32_t most_chunks;    // as many as there is room for
    uint32_t first;          // chunk of a launch
    float *block_states;     // [slots][heads][dk][dv + dk]; null: requests are not taken apart
    uint32_t round, slots;   // blocks of a head that the device has at once; states of blocks that there is room for
    uint32_t *ends, *block_ends, *slot_ends, *plan;   // (more than kCountedByAll requests) chunks up to each request, its own too; where they may be taken apart, blocks and slots, and a BlockPlan
};

__device__ __forceinline__ uint32_t wave_sum32(uint32_t v) {
    v += dpp_or_zero<0x111, 0xF>(v);
    v += dpp_or_zero<0x112, 0xF>(v);
    v += dpp_or_zero<0x114, 0xF>(v);
    v += dpp_or_zero<0x118, 0xF>(v);
    v += dpp_or_zero<0x142, 0xA>(v);
    return lane_value(v + dpp_or_zero<0x143, 0xC>(v), 63);
}
constexpr uint32_t kMostOfLane = (1u << 26) - 1;   // more chunks than there are; where offsets go backwards a lane's sum is cut there, so that 64 of them do not wrap
__device__ __forceinline__ uint32_t chunks_of(Span s) { return (s.end - s.begin + kChunk - 1) / kChunk; }

// Which request chunk `number` is of, and its first token; chunks are numbered request after request.
struct ChunkPlace {
    uint32_t request, begin, end;   // the chunk's tokens
    bool found;
};
__device__ __forceinline__ uint32_t counted_before(const uint32_t *ends, uint32_t r) { return r ? ends[r - 1] : 0u; }
// The first request whose end is behind a number; n if there is none.  64 at a time.
__device__ __forceinline__ uint32_t first_behind(const uint32_t *ends, uint32_t n, uint32_t number) {
    const uint32_t lane = threadIdx.x & 63;
    uint32_t from = 0, size = n;
    while (size > 64) {
        const uint32_t step = (size + 63) / 64, last = min((lane + 1) * step, size) - 1;   // (a lane's share may lie beyond the others': the last request again)
        const uint64_t hit = __ballot(ends[from + last] > number);
        if (!hit) return n;
        const uint32_t l = __builtin_ctzll(hit);
        from += l * step, size = min(step, size - l * step);
    }
    const uint64_t hit = __ballot(lane < size && ends[from + min(lane, size - 1)] > number);
    return hit ? from + (uint32_t)__builtin_ctzll(hit) : n;
}
__device__ __forceinline__ ChunkPlace find_chunk(const DeltaPromptParams &PP, uint32_t number) {
    const DeltaParams &P = PP.d;
    const uint32_t lane = threadIdx.x & 63;
    if (PP.ends) {
        const uint32_t r = first_behind(PP.ends, P.n, number);
        if (r == P.n) return {0, 0, 0, false};
        const Span s = span_of(P, r);
        const uint32_t begin = s.begin + (number - counted_before(PP.ends, r)) * kChunk;
        return {r, begin, s.end - begin < kChunk ? s.end : begin + kChunk, true};
    }
    uint32_t before = 0;
    for (uint32_t first = 0; first < P.n; first += 64) {
        const uint32_t r = first + lane;
        const Span s = r < P.n ? span_of(P, r) : Span{0, 0};
        const uint32_t own = chunks_of(s);
        uint32_t upto = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(upto, d);
            upto += lane >= (uint32_t)d ? o : 0u;
        }
        const uint64_t hit = __ballot(before + upto > number);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            const uint32_t inside = number - (before + lane_value(upto - own, l));
            const uint32_t begin = lane_value(s.begin, l) + inside * kChunk, end = lane_value(s.end, l);
            return {first + l, begin, end - begin < kChunk ? end : begin + kChunk, true};
        }
        before += lane_value(upto, 63);
    }
    return {0, 0, 0, false};
}

// Requests in blocks.  Chunks of a request depend on each other through the state.  Where few long requests would leave the device idle they are taken apart into blocks of as many chunks: what a
// block makes of a state, S -> A S + B, is found for all blocks at once (A from the columns of the identity, B from a state of zeros), then the state before each block, then all blocks' outputs.
// That is 2.3 times the work and two more launches, so it is done where the longest request has more than three times an even share of the chunks and twelve more, 16 at least (a call that cannot
// have so many is not charged with the two launches): us of a call, whole / in blocks, where the longest of the requests has as many chunks and as many times an even share, and the others are up to a
// quarter as long (16 heads of 128 x 128):
//   16 chunks, 8 times 70 / 69;   24, 6 times 100 / 100, 12 times (4 heads) 96 / 86;   32, 4 times 129 / 104, 8 times 123 / 99;   64, 3 times 258 / 226, 4 times 246 / 159;   128, 3 times 494 / 412, 4 times 469 / 272
// Where sides change depends on the others' lengths too, which the rule leaves out; it takes the later places (24 chunks, 6 times: 4 heads of 128 x 128 101 / 123, 8 of 64 x 64 84 / 99, 4 of
// 128 x 256 96 / 107).
// Blocks have four chunks at least, and are as many as fill the device once (once, twice: one of 4096 tokens 133, 173 us, of 32768 685, 722; 45000 tokens of eight requests 938, 937; but
// of six, one with most of them, 953, 861).
constexpr uint32_t kLeastBlock = 4, kLeastApart = 16, kApartFixed = 12, kApartShare = 3;
__host__ __device__ constexpr bool worth_taking_apart(uint64_t most, uint64_t all, uint32_t round) { return most >= kLeastApart && (most - kApartFixed) * round > kApartShare * all; }
constexpr uint32_t kMostOrdered = 256;
struct BlockPlan {
    uint32_t chunks, blocks;   // chunks of a block (~0: all of a request), blocks in all
};
__host__ __device__ constexpr uint32_t delta_slices(uint32_t columns, uint32_t waves) { return (columns + 16 * waves - 1) / (16 * waves); }
__device__ __forceinline__ uint32_t blocks_in(uint32_t chunks, uint32_t block) { return block == ~0u ? 1u : max(1u, (chunks + block - 1) / block); }
__device__ __forceinline__ BlockPlan plan_blocks(const DeltaPromptParams &PP) {
    const DeltaParams &P = PP.d;
    if (!PP.block_states) return {~0u, P.n};
    if (PP.plan) return {uniform(PP.plan[0]), uniform(PP.plan[1])};
    const uint32_t lane = threadIdx.x & 63;
    uint32_t all = 0, most = 0;
    for (uint32_t r = lane; r < P.n; r += 64) {
        const uint32_t own = chunks_of(span_of(P, r));
        all += own, most = max(most, own);
    }
    all = wave_sum32(min(all, kMostOfLane));
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d));
    most = uniform(most);
    if (!worth_taking_apart(most, all, PP.round)) return {~0u, P.n};
    const uint32_t block = max(kLeastBlock, (all + PP.round - 1) / PP.round);
    uint32_t blocks = 0;
    for (uint32_t r = lane; r < P.n; r += 64) blocks += blocks_in(chunks_of(span_of(P, r)), block);
    return {block, wave_sum32(blocks)};
}

// Up to kCountedByAll requests every workgroup counts the chunks before its own by itself; for more, which would take time with the square of their number, one workgroup counts them for all first, in
// a launch more.  us a prompt of 8 tokens, 8 heads of 64, counted by all / first: 256 prompts 0.45 / 0.43, 512 0.41 / 0.33, 768 0.45 / 0.33, 1024 0.48 / 0.33; counted by all 4096 0.9, 16384 2.8, so 0.31
// for both.  (Where there are few heads the launch counts for more: short calls are left without it.)  Sums of requests that overlap, where offsets go backwards, are cut: behind all that there is room for.
constexpr uint32_t kCountedByAll = 768, kCountThreads = 1024;
__device__ __forceinline__ uint32_t cut31(uint64_t v) { return v > 0x7fffffffu ? 0x7fffffffu : (uint32_t)v; }
struct Counted {
    uint64_t upto, all;   // with the thread's own; of the workgroup
};
__device__ __forceinline__ Counted count(uint64_t own, uint64_t *waves) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t o = __shfl_up((unsigned long long)own, d);
        own += lane >= (uint32_t)d ? o : 0u;
    }
    if (lane == 63) waves[wave] = own;
    __syncthreads();
    uint64_t before = 0, all = 0;
    for (uint32_t w = 0; w < kCountThreads / 64; ++w) before += w < wave ? waves[w] : 0u, all += waves[w];
    __syncthreads();
    return {before + own, all};
}
__global__ __launch_bounds__(kCountThreads) void delta_count_kernel(DeltaPromptParams PP) {
    __shared__ uint64_t waves[kCountThreads / 64];
    __shared__ uint32_t longest;
    const DeltaParams &P = PP.d;
    const uint32_t tid = threadIdx.x;
    if (tid == 0) longest = 0;
    uint64_t all = 0;
    uint32_t most = 0;
    for (uint32_t first = 0; first < P.n; first += kCountThreads) {
        const uint32_t r = first + tid, own = r < P.n ? chunks_of(span_of(P, r)) : 0u;
        const Counted c = count(own, waves);
        if (r < P.n) PP.ends[r] = cut31(all + c.upto);
        all += c.all, most = max(most, own);
    }
    if (!PP.block_states) return;
    atomicMax(&longest, most);
    __syncthreads();
    if (!worth_taking_apart(longest, all, PP.round)) {
        if (tid == 0) PP.plan[0] = ~0u, PP.plan[1] = P.n;
        return;
    }
    const uint32_t block = max(kLeastBlock, cut31((all + PP.round - 1) / PP.round));
    uint64_t blocks = 0, slots = 0;
    for (uint32_t first = 0; first < P.n; first += kCountThreads) {
        const uint32_t r = first + tid, own = r < P.n ? blocks_in(chunks_of(span_of(P, r)), block) : 0u;
        const Counted b = count(own, waves), s = count(own > 1 ? own : 0u, waves);
        if (r < P.n) PP.block_ends[r] = cut31(blocks + b.upto), PP.slot_ends[r] = cut31(slots + s.upto);
        blocks += b.all, slots += s.all;
    }
    if (tid == 0) PP.plan[0] = block, PP.plan[1] = cut31(blocks);
}

// Which block of which request has a number, counted request after request.
struct BlockPlace {
    uint32_t request, block, blocks;   // the block's number in its request, and how many that has
    uint32_t slot, chunk;              // its state's place, if there are several; its first chunk
    bool found;
};
__device__ __forceinline__ bool room_for(const DeltaPromptParams &PP, uint32_t first_slot, uint32_t blocks) { return blocks == 1 || (first_slot <= PP.slots && blocks <= PP.slots - first_slot); }
__device__ __forceinline__ BlockPlace find_block(const DeltaPromptParams &PP, uint32_t block, uint32_t number) {
    const DeltaParams &P = PP.d;
    const uint32_t lane = threadIdx.x & 63;
    if (PP.ends) {
        const uint32_t r = uniform(first_behind(PP.block_ends, P.n, number));
        if (r == P.n) return {0, 0, 0, 0, 0, false};
        BlockPlace at;
        const uint32_t first = counted_before(PP.block_ends, r), first_slot = counted_before(PP.slot_ends, r);
        at.request = r, at.block = number - first, at.blocks = uniform(PP.block_ends[r] - first);
        at.slot = first_slot + at.block, at.chunk = counted_before(PP.ends, r) + (at.block ? at.block * block : 0u);
        at.found = uniform(room_for(PP, first_slot, at.blocks)) != 0;
        return at;
    }
    uint32_t before = 0, chunks_before = 0, slots_before = 0;
    for (uint32_t first = 0; first < P.n; first += 64) {
        const uint32_t r = first + lane, chunks = r < P.n ? chunks_of(span_of(P, r)) : 0u, own = r < P.n ? blocks_in(chunks, block) : 0u, slots = own > 1 ? own : 0u;
        uint32_t upto = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(upto, d);
            upto += lane >= (uint32_t)d ? o : 0u;
        }
        const uint64_t hit = __ballot(before + upto > number);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            BlockPlace at;
            at.request = first + l, at.blocks = lane_value(own, l), at.block = number - (before + lane_value(upto, l) - at.blocks);
            const uint32_t first_slot = slots_before + wave_sum32((int)lane < l ? slots : 0u);
            at.slot = first_slot + at.block, at.chunk = chunks_before + wave_sum32((int)lane < l ? chunks : 0u) + (at.block ? at.block * block : 0u);
            at.found = room_for(PP, first_slot, at.blocks);   // (there is room for all of them, unless offsets go backwards)
            return at;
        }
        before += lane_value(upto, 63), chunks_before += wave_sum32(chunks), slots_before += wave_sum32(slots);
    }
    return {0, 0, 0, 0, 0, false};
}

// The same where requests are whole.
__device__ __forceinline__ BlockPlace find_whole(const DeltaPromptParams &PP, uint32_t request) {
    const DeltaParams &P = PP.d;
    if (!PP.most_chunks) return {request, 0, 1, 0, 0, true};   // (no tokens)
    if (PP.ends) return {request, 0, 1, 0, uniform(counted_before(PP.ends, request)), true};
    uint32_t before = 0;
#pragma unroll 4
    for (uint32_t r = threadIdx.x & 63; r < request; r += 64) before += chunks_of(span_of(P, r));
    return {request, 0, 1, 0, wave_sum32(min(before, kMostOfLane)), true};
}
// Where they are more than the device takes at once: the longest first, so that none of them begins when the others are done (24 requests of 64 to 4096 tokens, the longest
// ones last: 369 us as they come, 298).  Up to 256 requests: a lane has four of them, and the length that a place in that order has is found by bisection.
__device__ __forceinline__ BlockPlace find_longest(const DeltaParams &P, uint32_t place) {
    const uint32_t lane = threadIdx.x & 63;
    uint32_t chunks[kMostOrdered / 64], most = 0;   // and one: 0 where there is no request
#pragma unroll
    for (uint32_t j = 0; j < kMostOrdered / 64; ++j) {
        const uint32_t r = j * 64 + lane;
        chunks[j] = r < P.n ? chunks_of(span_of(P, r)) + 1 : 0u;
        most = max(most, chunks[j]);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d));
    const auto as_long = [&](uint32_t least) __attribute__((always_inline)) {
        uint32_t n = 0;
#pragma unroll
        for (uint32_t j = 0; j < kMostOrdered / 64; ++j) n += __builtin_popcountll(__ballot(chunks[j] >= least));
        return n;
    };
    uint32_t own = 1, behind = uniform(most) + 1;   // more than `place` requests have as many as `own`, no more than `place` as many as `behind`
    while (behind - own > 1) {
        const uint32_t middle = own + (behind - own) / 2;
        (as_long(middle) > place ? own : behind) = middle;
    }
    uint32_t left = place - as_long(own + 1);
    BlockPlace at = {0, 0, 1, 0, 0, true};
    bool found = false;
#pragma unroll
    for (uint32_t j = 0; j < kMostOrdered / 64; ++j) {
        uint64_t same = __ballot(chunks[j] == own);
        const uint32_t here = __builtin_popcountll(same);
        if (!found && left < here) {
            for (uint32_t i = 0; i < left; ++i) same &= same - 1;
            at.request = j * 64 + __builtin_ctzll(same), found = true;
        }
        left -= found ? 0u : here;
    }
    uint32_t before = 0;
#pragma unroll
    for (uint32_t j = 0; j < kMostOrdered / 64; ++j) before += j * 64 + lane < at.request ? chunks[j] - 1 : 0u;
    at.chunk = wave_sum32(before);
    return at;
}

// The value itself, made anew where it is used (no instruction): what follows from it is not kept in registers all through a loop.
__device__ __forceinline__ uint32_t here(uint32_t v) {
    asm volatile("" : "+v"(v));
    return v;
}
// Four values of a lane as the three terms of half an operand, and eight.
template <int half> __device__ __forceinline__ void half_terms(f32x4 x, u32x4 (&to)[3]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t terms[3];
        take_apart<3>(x[2 * i], x[2 * i + 1], terms);
#pragma unroll
        for (int c = 0; c < 3; ++c) to[c][2 * half + i] = terms[c];
    }
}
__device__ __forceinline__ void three_terms(const f32x4 (&x)[2], u32x4 (&to)[3]) { half_terms<0>(x[0], to), half_terms<1>(x[1], to); }
template <int k> struct Number {
    static constexpr int value = k;
};
template <int first, int behind, typename Step> __device__ __forceinline__ void in_order(const Step &step) {
    if constexpr (first < behind) {
        step(Number<first>());
        in_order<first + 1, behind>(step);
    }
}
__device__ __forceinline__ f32x4 mfma_f32(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// E and M of one chunk and head.  Wave w makes the rows 16 w .. 16 w + 15 of K K^T and Q K^T, straight from memory; then the first one the inverses of the four 16x16 blocks on the diagonal of
// I + L, a column a lane, by substitution (which loses nothing where keys are alike, as powers of L would); then wave j the blocks below the diagonal of block column j, and those of M,
//   T_ij = -T_ii sum_(j <= m < i) L_im T_mj,   M_ij = sum_(j <= m <= i) W_im T_mj
// in fp32 products (16x16x4): the column of a step of the operand is 4 g + step, so that a result's registers are the next product's operand.
// fp32, not bf16 terms: with keys alike and beta 2, T's entries cancel in sums of 64.  Bound by the phases of a workgroup, which wait for each other (28 KB written for 16 KB of keys and queries
// read, 2.2 TB/s): 24 prompts of 24000 tokens in all, 16 heads, 89 us; six of 45000, 149 us.  Five workgroups on a compute unit, for which keys go through T's place in LDS and T's empty quarter
// is left out, for four 96 us in place of 90.
template <typename T> __global__ __launch_bounds__(256, 5) void delta_chunks_kernel(DeltaPromptParams PP) {
    constexpr uint32_t kWide = kChunk + 4, kHalf = kChunk / 2, kNarrow = kHalf + 4;
    // below the diagonal L, from it on W transposed; T, later M, the first 32 rows without columns 32 .. 63: five workgroups on a compute unit.  Before T is there, keys lie in its place.
    __shared__ __align__(16) float LW[kChunk][kWide], X_[kHalf * (kNarrow + kWide)];
    const auto X = [&](uint32_t row) __attribute__((always_inline)) { return X_ + (row < kHalf ? row * kNarrow : kHalf * kNarrow + (row - kHalf) * kWide); };
    __shared__ double upto[kChunk];
    __shared__ float betas[kChunk], left[kChunk];
    const DeltaParams &P = PP.d;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4, r = lane & 15;
    const uint32_t in_launch = uniform(blockIdx.x / P.heads), h = uniform(by_die(blockIdx.x - in_launch * P.heads, P.heads)), shared = uniform(h / P.group), number = PP.first + in_launch;
    const ChunkPlace at = find_chunk(PP, number);
    if (!at.found || number >= PP.most_chunks) return;
    const uint32_t t0 = uniform(at.begin), m = uniform(at.end - at.begin), pieces = P.dk / 8;
    char *const to = PP.chunks + ((uint64_t)number * P.heads + h) * kChunkBytes;
    float *const decays = (float *)(to + kMatrixPieces * 16);

    // keys and queries of a tile of 16 tokens, a row a lane: components 32 p + 8 g + 0..7 (rows and components that are not there read 0)
    const auto rows_of = [&](const void *base, uint64_t stride) __attribute__((always_inline)) {
        return make_rsrc((const void *)uniform64((uint64_t)((const T *)base + (uint64_t)shared * P.dk + t0 * stride)), uniform((m - 1) * 2 * (uint32_t)stride + 2 * P.dk));
    };
    const auto k_rows = rows_of(P.k, P.k_stride), q_rows = rows_of(P.q, P.q_stride);
    u32x4 own_k[4], own_q[4];
    u32x4 *const keys = (u32x4 *)X_ + lane;   // of the first three tiles, [tile][p][lane]
    const auto load = [&](u32x4 (&x)[4], auto rows, uint32_t tile, uint64_t stride) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint32_t off = (tile * 16 + r) * 2 * (uint32_t)stride + (p * 4 + g < pieces ? (p * 4 + g) * 16 : 1u << 31);
            x[p] = __builtin_amdgcn_raw_buffer_load_b128(rows, off, 0, 0);
        }
    };
    double sum = 0.0;
    float beta = 0.f;
    if (wave == 0 && lane < m) {
        const uint64_t at_token = (uint64_t)(t0 + lane) * P.heads + h;
        sum = (double)at_least_200(P.log_decay[at_token]), beta = P.beta[at_token];
    }
    load(own_k, k_rows, wave, P.k_stride);
    load(own_q, q_rows, wave, P.q_stride);
    if (wave < 3)
#pragma unroll
        for (int p = 0; p < 4; ++p) keys[(wave * 4 + p) * 64] = own_k[p];
    if (wave == 0) {
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const double o = __shfl_up(sum, d);
            if (lane >= (uint32_t)d) sum += o;
        }
        const double last = __shfl(sum, 63);
        const float by = exp_of((float)sum);
        upto[lane] = sum, betas[lane] = beta, left[lane] = exp_of((float)(last - sum));
        decays[lane] = by, decays[64 + lane] = P.scale * by;
    }
    __syncthreads();
#pragma unroll
    for (int tile = 0; tile < 4; ++tile)
        if ((uint32_t)tile <= wave) {
            f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                u32x4 x = own_k[p];
                if ((uint32_t)tile < wave) x = keys[(tile * 4 + p) * 64];
                a = mfma_16x16x32(T(), own_k[p], x, a), b = mfma_16x16x32(T(), own_q[p], x, b);
            }
            const uint32_t j = tile * 16 + r;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t i = wave * 16 + 4 * g + e;
                if (i >= j) {
                    const float decay = exp_of((float)(upto[i] - upto[j]));
                    LW[j][i] = b[e] * (P.scale * decay);
                    if (i > j) LW[i][j] = a[e] * (betas[i] * decay);
                }
            }
        }
    __syncthreads();
    if (wave == 0) {
        const float (*const block)[kWide] = (const float (*)[kWide])&LW[16 * g][16 * g];
        float column[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float x = (uint32_t)i == r ? 1.f : 0.f;
#pragma unroll
            for (int c = 0; c < i; ++c) x = __builtin_fmaf(-block[i][c], column[c], x);
            column[i] = x;
            X(16 * g + i)[16 * g + r] = x;
        }
    } else if (wave == 3) {   // (what operands have above the diagonal)
#pragma unroll
        for (int e = 0; e < 4; ++e) X(4 * g + e)[16 + r] = 0.f, X(32 + 4 * g + e)[48 + r] = 0.f;
    }
    __syncthreads();
    f32x4 T_[4], M[4];   // blocks (i, wave); before a block of T is there, the sum that it is made of.  (products of as many blocks as there are, in turn: none waits for the one before)
#pragma unroll
    for (int i = 0; i < 4; ++i) T_[i] = M[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if ((uint32_t)c >= wave) {
            if ((uint32_t)c == wave) {
#pragma unroll
                for (int e = 0; e < 4; ++e) T_[c][e] = X(c * 16 + 4 * g + e)[c * 16 + r];
            } else {
                const f32x4 d = *(const f32x4 *)&X(c * 16 + r)[c * 16 + 4 * g];
                f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 4; ++e) y = mfma_f32(d[e], -T_[c][e], y);
                T_[c] = y;
#pragma unroll
                for (int e = 0; e < 4; ++e) X(c * 16 + 4 * g + e)[wave * 16 + r] = y[e];
            }
            f32x4 l[4], w[4];
#pragma unroll
            for (int i = c; i < 4; ++i) {
                if (i > c) l[i] = *(const f32x4 *)&LW[i * 16 + r][c * 16 + 4 * g];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t column = c * 16 + 4 * g + e, row = i * 16 + r;
                    w[i][e] = c < i || column <= row ? LW[column][row] : 0.f;
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
#pragma unroll
                for (int i = c + 1; i < 4; ++i) T_[i] = mfma_f32(l[i][e], T_[c][e], T_[i]);
#pragma unroll
                for (int i = c; i < 4; ++i) M[i] = mfma_f32(w[i][e], T_[c][e], M[i]);
            }
        }
    __syncthreads();
    const auto write_operands = [&](uint32_t first, auto rows_by) __attribute__((always_inline)) {
        for (uint32_t f = wave; f < kOperands; f += 4) {
            const uint32_t row = (f >= 2 ? 32 : 0) + 8 * (r >> 2) + 4 * (f & 1) + (r & 3), column = (f >= 4 ? 32 : 0) + 8 * g;
            const float *const x = X(row) + column, *const by = &betas[column], row_by = rows_by(row);
            u32x4 out[kTerms];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t terms[kTerms];
                take_apart<kTerms>(x[2 * i] * by[2 * i] * row_by, x[2 * i + 1] * by[2 * i + 1] * row_by, terms);
#pragma unroll
                for (int c = 0; c < (int)kTerms; ++c) out[c][i] = terms[c];
            }
            const uint32_t piece = on_diagonal(f) ? corner_piece(g, r) : lane;
            const bool zeros = on_diagonal(f) && g > r >> 2;
            if (!zeros || lane == 48) {
#pragma unroll
                for (int c = 0; c < (int)kTerms; ++c) ((u32x4 *)to)[first + c * kPlane + operand_at(f) + piece] = zeros ? (u32x4){0, 0, 0, 0} : out[c];
            }
        }
    };
    write_operands(0, [&](uint32_t row) __attribute__((always_inline)) { return left[row]; });
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if ((uint32_t)i >= wave) {
#pragma unroll
            for (int e = 0; e < 4; ++e) X(i * 16 + 4 * g + e)[wave * 16 + r] = M[i][e];
        }
    __syncthreads();
    write_operands(kTerms * kPlane, [](uint32_t) __attribute__((always_inline)) { return 1.f; });
}

__device__ __forceinline__ uint32_t of_neighbour(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false); }   // lanes 2 i and 2 i + 1 swapped
// Two rows of 16-bit values, columns c and c + 1 in each word, for lanes of two columns: the even lane has rows 0 .. 3 of both, the odd one rows 4 .. 7; they
// exchange what is the other's.  Words (0, 1), (2, 3), ... of the lane's own column.
__device__ __forceinline__ u32x4 own_column(const uint32_t (&row)[4], bool odd) {
    const uint32_t sel = odd ? 0x07060302u : 0x05040100u, other = odd ? 0x05040100u : 0x07060302u;
    const uint32_t a = __builtin_amdgcn_perm(row[1], row[0], sel), b = __builtin_amdgcn_perm(row[3], row[2], sel);
    const uint32_t c = of_neighbour(__builtin_amdgcn_perm(row[1], row[0], other)), d = of_neighbour(__builtin_amdgcn_perm(row[3], row[2], other));
    return odd ? (u32x4){c, d, a, b} : (u32x4){a, b, c, d};
}

// A workgroup takes a request's chunks for one head and 16 columns for each of kCompute waves, whose state stays in the wave's registers (fp32).
// Layout (products 16x16x32, lane = 16 g + r): the lane has column r and, of a pair of result tiles, the rows 32 s + 8 g + 0..7 (operand rows are those of kOperands' comment): as B
// of the next product those are its own, so the state goes into K S and Q S, R into M R and E R, and that into K^T E R, each from the registers where it is.
// What is no 16-bit input meets the matrix cores as three bf16 terms (fp32's 24 bits), each the upper half of what the ones before left, the last one rounded: E, M, the state, R and E R.  For outputs
// too, though they are rounded to 16 bits: with two terms of the state, M and R there an output was off by up to 2^-17 of its largest summand, which is all of it where summands cancel, and it cost as much
// time (24 prompts of 24000 tokens 302 us, so 295; 6 of 45000 946 and 950; 3 of 1000, 8 heads of 64, 32.4 and 34.7).  Errors of fp16 outputs 2.074e-4, the rounding's own; of states 1.9e-7.  Inputs in fp16 are
// two terms each (exact).
// A chunk is brought into LDS while the one before is computed: matrices straight from memory, keys and queries through registers (a second copy of keys lies by component), one barrier a chunk;
// fp16 with more than 64 components has room for one chunk's keys only, and two barriers.  kCompute 4: four waves compute and four bring.  A chunk of 128 x 64 takes 3.2 us in bf16 (5.8 in fp16), 1.4
// of them the matrix instructions' (216 of 16 cycles), the rest vector instructions (terms) and waits between the chunk's three dependent products: bound by that chain, a request after the other's
// end.  kCompute 8: all do both, 128 columns, two waves to a vector unit fill each other's waits: 5.7 us for twice the columns, so more in all but later for each.  launch_delta_prompts has the rule and
// both sides.  24 prompts of 24000 tokens in all, 16 heads, 128 x 128, bf16: 224 us, where four waves that did everything in turn, two workgroups on a compute unit, took 386.  Two groups of 16 columns
// to a wave, which halve the reads of LDS, need twice the registers and were slower; so was an order of matrix and vector instructions by hand (7 % more).  What is not finite is
// done again token by token, 0.5 us each.
// kStates: what blocks make of a state (columns dv and on: of the identity), without outputs.
constexpr size_t kLdsBytes = 160 * 1024;
template <int KD, int kIn, bool kStates> struct DeltaStage {   // what a chunk needs in LDS; planes of terms
    static constexpr uint32_t kRow = KD == 2 ? 64 : 128, kMatrix = kStates ? kTerms * kPlane : kMatrixPieces;
    uint16_t k[kIn][kChunk][kRow], q[kStates ? 0 : kIn][kChunk][kRow], kt[kIn][KD * 32][kChunk];
};
// A barrier for what lies in LDS alone: output stores stay under way (loads into LDS are waited for where the next chunk is taken in).
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
template <int KD, typename T, bool kStates, int kCompute> __global__ __launch_bounds__(512, 2) void delta_prompt_kernel(DeltaPromptParams PP) {
    constexpr int NW = kCompute, kIn = __is_same(T, f16_t) ? 2 : 1, kPieces = KD * 4;
    typedef DeltaStage<KD, kIn, kStates> Stage;
    constexpr uint32_t kRow = Stage::kRow;
    constexpr bool kBringers = kCompute < 8;   // four waves compute, four bring the chunks
    struct Matrices {
        u32x4 m[Stage::kMatrix];
        float d[2 * kChunk];
    };
    constexpr int kStages = 2 * (sizeof(Stage) + sizeof(Matrices)) <= kLdsBytes ? 2 : 1;
    constexpr int kItemsK = 16 * kPieces, kItems = kStates ? kItemsK : 2 * kItemsK, kPer = (kItems + 64 * NW - 1) / (64 * NW);
    constexpr uint32_t kMatrix = Stage::kMatrix;
    __shared__ __align__(16) Stage stages[kStages];
    __shared__ __align__(16) Matrices made[2];
    const DeltaParams &P = PP.d;
    const BlockPlan plan = plan_blocks(PP);
    if (kStates && plan.chunks == ~0u) return;
    const uint32_t slices = delta_slices(kStates ? P.dv + P.dk : P.dv, kCompute), each = P.heads * slices;
    for (uint64_t item = blockIdx.x; item < (uint64_t)plan.blocks * each; item += gridDim.x) {
        const uint32_t tid = here(threadIdx.x) & (64 * NW - 1), lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4, r = lane & 15;
        const uint32_t ordinal = uniform((uint32_t)(item / each)), rest = uniform(by_die((uint32_t)(item - (uint64_t)ordinal * each), each)), h = uniform(rest / slices), slice = uniform(rest - h * slices);
        const uint32_t shared = uniform(h / P.group);
        const bool ordered = plan.chunks == ~0u && P.n <= kMostOrdered && (uint64_t)P.n * each > kUnits;
        const BlockPlace at = ordered ? find_longest(P, ordinal) : plan.chunks == ~0u ? find_whole(PP, ordinal) : find_block(PP, plan.chunks, ordinal);
        const Span span = span_of(P, at.request);
        const uint32_t block_tokens = plan.chunks == ~0u ? 0u : plan.chunks * kChunk;
        const uint32_t begin = uniform(span.begin + at.block * block_tokens), end = uniform(at.block + 1 == at.blocks ? span.end : begin + block_tokens);
        uint32_t number = uniform(at.chunk);
        if (!at.found || (kStates && at.block + 1 == at.blocks)) continue;
        if (begin < end && (number > PP.most_chunks || (end - begin + kChunk - 1) / kChunk > PP.most_chunks - number)) continue;   // (offsets that go backwards)
        const uint64_t state = state_of(P, at.request), state_at = (state * P.heads + h) * ((uint64_t)P.dk * P.dv);
        float *const block_state = PP.block_states + ((uint64_t)at.slot * P.heads + h) * ((uint64_t)P.dk * (P.dv + P.dk));
        const uint32_t column = (slice * kCompute + wave) * 16 + r, columns = kStates ? P.dv + P.dk : P.dv;
        const bool live_column = column < columns, live_wave = (slice * kCompute + wave) * 16 < columns;   // (columns that are not there compute what nobody reads)
        constexpr uint32_t kNowhere = 1u << 31;
        const uint32_t pieces = P.dk / 8;
        const bool odd_lane = lane & 1;
        const uint32_t column2 = (column & ~1u) < P.dv ? 2 * (column & ~1u) : kNowhere;   // of the lane's pair of columns, in bytes
        const auto chunk_rows = [&](const void *base, uint32_t m, uint32_t stride, uint32_t width) __attribute__((always_inline)) {
            return make_rsrc((const void *)uniform64((uint64_t)base), uniform((m - 1) * stride + width));
        };
        const auto anew = [&](uint32_t v) __attribute__((always_inline)) { return here(v); };   // (addresses that stay would fill the registers)
        // A lane brings 4 tokens x 8 components of K or of Q into LDS; a wave has either.
        struct Part {
            bool live, is_q;
            uint32_t row, piece;
        };
        const auto part_of = [&](int b) __attribute__((always_inline)) {
            const uint32_t first = (kItemsK % (64 * NW) ? wave * 64 : 0u) + b * 64 * NW, rest = kItemsK % (64 * NW) ? 0u : wave * 64;   // (known when compiled where they divide)
            Part p;
            p.live = first < kItems, p.is_q = !kStates && first >= kItemsK;
            const uint32_t id = first + rest - (p.is_q ? kItemsK : 0) + anew(lane);
            p.piece = id % kPieces, p.row = id / kPieces * 4;
            return p;
        };
        // LDS rows are pieces of 16 bytes, exchanged by the row's number so that the sixteen rows of an operand, 8 (r / 4) + r % 4 + ..., lie in different banks.  K by component as in
        // rows d: piece u, 8 tokens, at u ^ (2 (d / 8 mod 4) + (d / 2 mod 2)) ^ (d / 32 mod 2), its two halves exchanged where d / 64 is odd: the lanes of a read have d = 8 (r / 4) +
        // r % 4 + ..., those of a write d / 8 from 0 to 15.
        const auto row_piece = [&](uint32_t row, uint32_t u) __attribute__((always_inline)) {
            return kRow == 128 ? row * 256 + ((u ^ (row & 3) ^ (row >> 3 & 3) * 4) * 16) : row * 128 + ((u ^ (row >> 1 & 1) ^ (row >> 3 & 3) * 2) * 16);
        };
        const uint32_t own_kt = ((r >> 2) * 8 + (r & 3)) * 128 + (g ^ (r >> 1)) * 16;
        // Rows of tile (s, t) = (tile / 2, tile % 2), 32 s + 4 t behind the lane's own: pieces there are exchanged by the same bits.
        const uint32_t own_corner = corner_piece(g, r);
        const uint32_t own_rows = row_piece(8 * (r >> 2) + (r & 3), g);
        u32x4 staged[kPer][4];
        float decays = 0.f;
        const auto load_chunk = [&](uint32_t t0) __attribute__((always_inline)) {
            const uint32_t m = min(kChunk, end - t0);
#pragma unroll
            for (int b = 0; b < kPer; ++b) {
                const Part p = part_of(b);
                if (p.live) {
                    const uint32_t stride = 2 * (uint32_t)(p.is_q ? P.q_stride : P.k_stride), off = p.row * stride + (p.piece < pieces ? p.piece * 16 : kNowhere);
                    const auto rows = chunk_rows(p.is_q ? (const T *)P.q + (uint64_t)shared * P.dk + t0 * P.q_stride : (const T *)P.k + (uint64_t)shared * P.dk + t0 * P.k_stride, m, stride, 2 * P.dk);
#pragma unroll
                    for (int j = 0; j < 4; ++j) staged[b][j] = __builtin_amdgcn_raw_buffer_load_b128(rows, off + j * stride, 0, 0);
                }
            }
        };
        // Matrices go from memory straight into LDS, 1 KB a wave at a time.
        const auto bring_matrices = [&](uint32_t chunk, Matrices &to) __attribute__((always_inline)) {
            const char *const from = PP.chunks + ((uint64_t)chunk * P.heads + h) * kChunkBytes;
#pragma unroll
            for (uint32_t b = 0; b < kMatrix; b += 64 * NW)
                if (b + wave * 64 < kMatrix) __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(from + (b + tid) * 16), (__attribute__((address_space(3))) void *)&to.m[b + wave * 64], 16, 0, 0);
            if (tid < 2 * kChunk) decays = ((const float *)(from + kMatrixPieces * 16))[tid];
        };
        const auto have_matrices = [&](Matrices &to) __attribute__((always_inline)) {
            __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
            if (tid < 2 * kChunk) to.d[tid] = decays;
        };
        const auto write_chunk = [&](Stage &to_stage) __attribute__((always_inline)) {
#pragma unroll
            for (int b = 0; b < kPer; ++b) {
                const Part p = part_of(b);
                if (p.live) {
#pragma unroll
                    for (int a = 0; a < kIn; ++a) {
                        uint32_t w[4][4];
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                uint32_t terms[kIn];
                                input_terms<T, kIn>(staged[b][j][i], terms);
                                w[j][i] = terms[a];
                            }
                        char *const to = p.is_q ? (char *)to_stage.q[a] : (char *)to_stage.k[a];
#pragma unroll
                        for (int j = 0; j < 4; ++j) *(u32x4 *)(to + row_piece(p.row + j, p.piece)) = (u32x4){w[j][0], w[j][1], w[j][2], w[j][3]};
                        if (!p.is_q) {
                            const uint32_t place = p.row / 8 ^ (p.piece & 3) * 2 ^ (p.piece / 4 & 1), half = (p.row / 4 & 1) ^ (p.piece / 8 & 1);
                            char *const kt = (char *)to_stage.kt[a] + p.piece * 8 * 128 + half * 8;
#pragma unroll
                            for (int c = 0; c < 8; ++c) {   // component c of the four tokens
                                const uint32_t sel = c % 2 ? 0x07060302u : 0x05040100u;
                                *(u32x2 *)(kt + c * 128 + (place ^ (c / 2 & 1)) * 16) = (u32x2){__builtin_amdgcn_perm(w[1][c / 2], w[0][c / 2], sel), __builtin_amdgcn_perm(w[3][c / 2], w[2][c / 2], sel)};
                            }
                        }
                    }
                }
            }
        };
        // (whole waves take either branch, and come by as many barriers in both: one before the first chunk, kStages == 1 ? 2 : 1 for each)
        if (kBringers && threadIdx.x >= 64 * NW) {
            if (begin < end) {
                bring_matrices(number, made[0]);
                load_chunk(begin);
                write_chunk(stages[0]);
                if (begin + kChunk < end) load_chunk(begin + kChunk);
                have_matrices(made[0]);
            }
            lds_barrier();
            uint32_t next = 1;
            for (uint32_t t0 = begin; t0 < end; t0 += kChunk) {
                const bool more = end - t0 > kChunk;
                if (more) bring_matrices(++number, made[next]);
                if constexpr (kStages == 1) lds_barrier();
                if (more) {
                    write_chunk(stages[kStages == 1 ? 0 : next]);
                    if (end - t0 > 2 * kChunk) load_chunk(t0 + 2 * kChunk);
                    have_matrices(made[next]);
                }
                lds_barrier();
                next ^= 1;
            }
            continue;
        }
        f32x4 S[2 * KD];
        const float *const from = kStates ? nullptr : at.blocks > 1 ? block_state : P.state_in && state != ~0ull ? P.state_in + state_at : nullptr;
        // (through a buffer of the state's size: rows and columns that are not there read 0 and are not written, without a branch for each)
        const auto state_rows = [&](const float *base, uint32_t stride) __attribute__((always_inline)) {
            return make_rsrc((const void *)uniform64((uint64_t)base), uniform(base ? P.dk * stride * 4 : 0u));
        };
        const uint32_t from_stride = at.blocks > 1 ? P.dv + P.dk : P.dv;
        const auto from_rows = state_rows(from, from_stride);
        const uint32_t from_first = live_column ? (g * 8 * from_stride + column) * 4 : kNowhere;
#pragma unroll
        for (int i = 0; i < 2 * KD; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t d = (i / 2) * 32 + g * 8 + (i % 2) * 4 + e;
                if constexpr (kStates) S[i][e] = column == P.dv + d ? 1.f : 0.f;
                else S[i][e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(from_rows, from_first + ((i / 2) * 32 + (i % 2) * 4 + e) * from_stride * 4, 0, 0));
            }
        uint32_t values[2][4];
        const auto load_values = [&](uint32_t t0) __attribute__((always_inline)) {
            const uint32_t m = min(kChunk, end - t0);
            const uint32_t stride = 2 * (uint32_t)P.v_stride, off = (anew(g) * 8 + (odd_lane ? 4 : 0)) * stride;
            const auto rows = chunk_rows((const T *)P.v + (uint64_t)h * P.dv + t0 * P.v_stride, m, stride, 2 * P.dv);
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int j = 0; j < 4; ++j) values[s][j] = __builtin_amdgcn_raw_buffer_load_b32(rows, off + (s * 32 + j) * stride + column2, 0, 0);
        };
#pragma unroll
        for (int i = 0; i < 8; ++i) values[i / 4][i % 4] = 0;
        if (begin < end) {
            if constexpr (!kBringers) bring_matrices(number, made[0]), load_chunk(begin);
            load_values(begin);
            if constexpr (!kBringers) write_chunk(stages[0]), have_matrices(made[0]);
        }
        // The state and the first chunk's values are waited for here: with any of them under way at the loop's head, the compiler's wait there would be for all that the wave has
        // issued, the stores of the chunk before among them.
#pragma unroll
        for (int i = 0; i < 2 * KD; ++i) asm volatile("" : "+v"(S[i]));
#pragma unroll
        for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(values[i / 4][i % 4]));
        lds_barrier();
        uint32_t stage = 0;
        for (uint32_t t0 = begin; t0 < end; t0 += kChunk) {
            const uint32_t m = min(kChunk, end - t0);
            const Stage &now = stages[kStages == 1 ? 0 : stage];
            const Matrices &matrices = made[stage];
            const u32x4 *const whole = matrices.m + lane, *const corners = matrices.m + own_corner;
            const auto kt_tile = [&](int a, int t, int s) __attribute__((always_inline)) {   // components of tile t, tokens 32 s + 8 g .. + 7
                const u32x4 w = *(const u32x4 *)((const char *)now.kt[a] + (own_kt ^ (s * 64) ^ (t / 2 % 2 * 16)) + (t / 2) * 32 * 128 + (t % 2) * 4 * 128);
                return t / 4 % 2 ? (u32x4){w[2], w[3], w[0], w[1]} : w;
            };
            const auto operand = [&](const uint16_t *plane, int tile, int p) __attribute__((always_inline)) {
                return *(const u32x4 *)((const char *)plane + (own_rows ^ (p * 64)) + ((tile / 2) * 32 + (tile % 2) * 4) * 2 * kRow);
            };
            // values: tokens 32 s + 8 g + 2 i, + 1 of the lane's columns
            u32x4 V[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) V[s] = own_column(values[s], odd_lane);
            const bool more = t0 + kChunk < end;
            if (more) {
                if constexpr (!kBringers) bring_matrices(++number, made[stage ^ 1]), load_chunk(t0 + kChunk);
                load_values(t0 + kChunk);
            }
            const auto bring = [&] __attribute__((always_inline)) {   // the next chunk, where it does not take this one's place
                __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): loads that have been under way since the chunk's beginning, those into LDS too
                if (kBringers || !more) return;
                have_matrices(made[stage ^ 1]);
                if constexpr (kStages == 2) write_chunk(stages[stage ^ 1]);
            };
            if (!live_wave) bring();
            else {
                const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
                f32x4 O[4], R[4], U[4];
                u32x4 A[2][4], B[2][3];
                // The products of a chunk in steps of up to four rows of operands: K S and Q S by 32 components and term of the inputs; then E R by its terms and M R by its, for the tokens
                // 32 s .. 32 s + 31; then K^T E R.  A step's loads from LDS are under way while the step before is multiplied, and nothing is moved from step to step.
                constexpr int kOfS = kStates ? 1 : 2, kOfR = kStates ? kTerms : 2 * kTerms;   // (states alone: without queries and M)
                constexpr int kState = kOfS * kIn * KD, kSystem = kState + 2 * kOfR, kUpdate = 2 * ((2 * KD + 3) / 4) * kIn, kSteps = kSystem + kUpdate;
                const auto fetch = [&](auto number) __attribute__((always_inline)) {
                    constexpr int k = decltype(number)::value;
                    u32x4 (&to)[4] = A[k % 2];
                    if constexpr (k < kState) {
                        constexpr int p = k / (kOfS * kIn), a = k / kOfS % kIn;
#pragma unroll
                        for (int tile = 0; tile < 4; ++tile) to[tile] = operand(k % kOfS ? &now.q[a][0][0] : &now.k[a][0][0], tile, p);
                    } else if constexpr (k < kSystem) {
                        constexpr int s = (k - kState) / kOfR, a = (k - kState) % kOfR, first = s == 0 ? 0 : 4, last = s == 0 ? 4 : 6;
#pragma unroll
                        for (int f = first; f < last; ++f) to[f - first] = (on_diagonal(f) ? corners : whole)[a * kPlane + operand_at(f)];
                    } else if constexpr (k < kSteps) {
                        constexpr int a = (k - kSystem) % kIn, each = kUpdate / 2, s = (k - kSystem) / each, first = (k - kSystem) % each / kIn * 4;
#pragma unroll
                        for (int i = 0; i < 4 && first + i < 2 * KD; ++i) to[i] = kt_tile(a, first + i, s);
                    }
                };
                const auto decay_of = [&](int which, int tile) __attribute__((always_inline)) { return *(const f32x4 *)&matrices.d[which * kChunk + (tile / 2) * 32 + g * 8 + (tile % 2) * 4]; };
                const float decay = matrices.d[kChunk - 1];
                T *const out = (T *)P.out + ((uint64_t)t0 * P.heads + h) * P.dv;
                const uint32_t out_stride = 2 * P.heads * P.dv;
                const auto out_rows = chunk_rows(out, m, out_stride, 2 * P.dv);
                const auto store = [&](int tile) __attribute__((always_inline)) {   // tokens 0, 1 of a tile's four are the even lane's, 2, 3 the odd one's, both columns of each
                    const uint32_t a = pack2<T>(O[tile][0], O[tile][1]), b = pack2<T>(O[tile][2], O[tile][3]);   // own column
                    const uint32_t got = of_neighbour(odd_lane ? a : b), mine = odd_lane ? b : a;              // the lane's two tokens, the other column and this one
                    const uint32_t left = odd_lane ? got : mine, right = odd_lane ? mine : got;
                    const uint32_t off = (anew(g) * 8 + (odd_lane ? 2 : 0)) * out_stride + column2 + ((tile / 2) * 32 + (tile % 2) * 4) * out_stride;
                    __builtin_amdgcn_raw_buffer_store_b32(__builtin_amdgcn_perm(right, left, 0x05040100u), out_rows, off, 0, 0);
                    __builtin_amdgcn_raw_buffer_store_b32(__builtin_amdgcn_perm(right, left, 0x07060302u), out_rows, off + out_stride, 0, 0);
                };
                const auto step = [&](auto number) __attribute__((always_inline)) {
                    constexpr int k = decltype(number)::value;
                    fetch(Number<k + 1>());
                    const u32x4 (&from)[4] = A[k % 2];
                    if constexpr (k < kState) {
                        constexpr int p = k / (kOfS * kIn), a = k / kOfS % kIn, terms = 3 - a;
                        f32x4 (&to)[4] = k % kOfS ? O : R;
#pragma unroll
                        for (int c = 0; c < terms; ++c)
#pragma unroll
                            for (int tile = 0; tile < 4; ++tile) to[tile] = mfma_bf16(from[tile], B[p % 2][c], p == 0 && a == 0 && c == 0 ? zero : to[tile]);
                        if constexpr (p + 1 < KD) {   // the next components' state
                            if constexpr (k % (kOfS * kIn) == 0) half_terms<0>(S[2 * p + 2], B[(p + 1) % 2]);
                            if constexpr (k % (kOfS * kIn) == kOfS * kIn - 1) half_terms<1>(S[2 * p + 3], B[(p + 1) % 2]);
                        }
                    } else if constexpr (k < kSystem) {
                        constexpr int s = (k - kState) / kOfR, a = (k - kState) % kOfR, first = s == 0 ? 0 : 4, last = s == 0 ? 4 : 6;   // operands; the tile of one behind the fourth is two before it
                        constexpr int terms = kTerms - a % kTerms;
#pragma unroll
                        for (int c = 0; c < terms; ++c)
#pragma unroll
                            for (int f = first; f < last; ++f) {
                                const int tile = f < 4 ? f : f - 2;
                                if constexpr (a < (int)kTerms) U[tile] = mfma_bf16(from[f - first], B[s][c], f < 4 && a == 0 && c == 0 ? zero : U[tile]);
                                else O[tile] = mfma_bf16(from[f - first], B[s][c], O[tile]);
                            }
                        if constexpr (s == 0 && a == 0) three_terms({R[2], R[3]}, B[1]);
                        if constexpr (!kStates && s == 0 && a == 1) {
#pragma unroll
                            for (int tile = 0; tile < 4; ++tile) O[tile] *= decay_of(1, tile);
                        }
                    } else {
                        constexpr int a = (k - kSystem) % kIn, each = kUpdate / 2, s = (k - kSystem) / each, first = (k - kSystem) % each / kIn * 4;
#pragma unroll
                        for (int c = 0; c + a < 3; ++c)
#pragma unroll
                            for (int i = 0; i < 4 && first + i < 2 * KD; ++i) S[first + i] = mfma_bf16(from[i], B[s][c], S[first + i]);
                        if constexpr (s == 0 && first == 0 && a == 0) three_terms({U[2], U[3]}, B[1]);
                        if constexpr (s == 0 && a == 0) {   // the next four rows' state
#pragma unroll
                            for (int i = first + 4; i < first + 8 && i < 2 * KD; ++i) S[i] *= decay;
                        }
                        if constexpr (!kStates) {
#pragma unroll
                            for (int tile = 0; tile < 4; ++tile)
                                if (tile * kUpdate / 4 == k - kSystem) store(tile);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                };
                three_terms({S[0], S[1]}, B[0]);
                fetch(Number<0>());
                in_order<0, kState>(step);
                if constexpr (!kStates) {   // (products that nothing waits for are put off otherwise, past the barriers of the schedule, and their operands fill the registers)
#pragma unroll
                    for (int tile = 0; tile < 4; ++tile) asm volatile("" : "+v"(O[tile]));
                }
                // R, from the values
#pragma unroll
                for (int tile = 0; tile < 4; ++tile) {
                    const f32x4 by = decay_of(0, tile);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t w = V[tile / 2][tile % 2 * 2 + i];   // (of an element of a vector itself, a bit cast takes the first)
                        float x, y;
                        if constexpr (kIn == 1) {
                            x = low_half(w), y = high_half(w);
                        } else {
                            typedef f16_t pair __attribute__((ext_vector_type(2)));
                            const pair both = __builtin_bit_cast(pair, w);
                            x = (float)both[0], y = (float)both[1];
                        }
                        R[tile][2 * i] = x - by[2 * i] * R[tile][2 * i], R[tile][2 * i + 1] = y - by[2 * i + 1] * R[tile][2 * i + 1];
                    }
                }
                three_terms({R[0], R[1]}, B[0]);
                in_order<kState, kSystem>(step);
                bring();
                float odd = 0.f;   // NaN if anything that is written is not finite
#pragma unroll
                for (int tile = 0; tile < 4; ++tile)
#pragma unroll
                    for (int e = 0; e < 4; ++e) odd = __builtin_fmaf(U[tile][e], 0.f, odd);
                if (kStates || !__any(odd != 0.f)) {   // (what is not finite leaves no finite state)
#pragma unroll
                    for (int i = 0; i < 4 && i < 2 * KD; ++i) S[i] *= decay;
                    three_terms({U[0], U[1]}, B[0]);
                    in_order<kSystem, kSteps>(step);
                } else if constexpr (!kStates) {   // token by token: what is not finite must not meet the zeros of earlier ones
                    for (uint32_t j = 0; j < m; ++j) {
                        const uint64_t at_token = (uint64_t)(t0 + j) * P.heads + h;
                        const float by = exp_of(P.log_decay[at_token]), beta = P.beta[at_token];
                        const auto component = [&](const uint16_t (*plane)[kChunk][kRow], int p, int c) __attribute__((always_inline)) {   // 32 p + 8 g + c
                            float x = 0.f;
#pragma unroll
                            for (int a = 0; a < kIn; ++a) x += low_half(*(const uint16_t *)((const char *)plane[a] + row_piece(j, p * 4 + g) + 2 * c));
                            return x;
                        };
                        const float v = live_column ? to_f32(((const T *)P.v)[(t0 + j) * P.v_stride + (uint64_t)h * P.dv + column]) : 0.f;
                        float y = 0.f, o = 0.f;
#pragma unroll
                        for (int p = 0; p < KD; ++p)
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                float &x = ((float *)&S[2 * p + c / 4])[c % 4];
                                x *= by;
                                if (p * 32 + g * 8 < P.dk) y += component(now.k, p, c) * x;
                            }
                        y += __shfl_xor(y, 16);
                        y += __shfl_xor(y, 32);
                        const float u = beta * (v - y);
#pragma unroll
                        for (int p = 0; p < KD; ++p)
#pragma unroll
                            for (int c = 0; c < 8; ++c)
                                if (p * 32 + g * 8 < P.dk) {
                                    float &x = ((float *)&S[2 * p + c / 4])[c % 4];
                                    x += component(now.k, p, c) * u;
                                    o += component(now.q, p, c) * x;
                                }
                        o += __shfl_xor(o, 16);
                        o += __shfl_xor(o, 32);
                        if (live_column && g == 0) out[(uint64_t)j * P.heads * P.dv + column] = from_f32<T>(o * P.scale);
                    }
                }
            }
            lds_barrier();   // (keys, queries and matrices are free)
            if constexpr (kStages == 1) {
                if (!kBringers && more) write_chunk(stages[0]);
                lds_barrier();
            }
            stage ^= 1;
        }
        float *const to = kStates ? block_state : at.block + 1 == at.blocks && P.state_out && state != ~0ull ? P.state_out + state_at : nullptr;
        const uint32_t to_stride = kStates ? P.dv + P.dk : P.dv;
        const auto to_rows = state_rows(to, to_stride);
        // (places made anew: kept from the state's loads on they would go through memory, one wait each: 4 prompts of 4000 tokens 318 us, so 300)
        const uint32_t to_first = live_column ? (anew(g) * 8 * to_stride + column) * 4 : kNowhere;
#pragma unroll
        for (int i = 0; i < 2 * KD; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = S[i][e];   // (of an element of a vector itself, a bit cast takes the first)
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, x), to_rows, to_first + ((i / 2) * 32 + (i % 2) * 4 + e) * to_stride * 4, 0, 0);
            }
    }
}

// The state before each block of the requests that are taken apart, over the blocks' B: S_(b + 1) = A_b S_b + B_b.  A workgroup has 16 columns, wave w the rows 32 w .. 32 w + 31; the rows
// go from wave to wave through LDS.  Both operands are fp32: three terms each.  Bound by the way from one block's state to the next, once for each block: six requests of 45000 tokens, 16 heads of 128 x 128, 27 us.
template <int KD> __global__ __launch_bounds__(64 * KD) void delta_states_kernel(DeltaPromptParams PP) {
    __shared__ __align__(16) float state_rows[2][16][KD * 32 + 4];
    const DeltaParams &P = PP.d;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4, r = lane & 15;
    const BlockPlan plan = plan_blocks(PP);
    if (plan.chunks == ~0u) return;
    const uint32_t slices = (P.dv + 15) / 16, each = P.heads * slices, wide = P.dv + P.dk;
    for (uint64_t item = blockIdx.x; item < (uint64_t)P.n * each; item += gridDim.x) {
        const uint32_t request = uniform((uint32_t)(item / each)), rest = uniform((uint32_t)(item - (uint64_t)request * each)), h = uniform(rest / slices), slice = uniform(rest - h * slices);
        const uint32_t blocks = uniform(blocks_in(chunks_of(span_of(P, request)), plan.chunks));
        if (blocks == 1) continue;
        uint32_t slot = 0;   // of its first block
        if (PP.ends) slot = uniform(counted_before(PP.slot_ends, request));
        else {
            uint32_t mine = 0;
            for (uint32_t i = lane; i < request; i += 64) {
                const uint32_t b = blocks_in(chunks_of(span_of(P, i)), plan.chunks);
                mine += b > 1 ? b : 0u;
            }
            slot = wave_sum32(mine);
        }
        const uint32_t column = slice * 16 + r, first_row = wave * 32 + g * 8;
        if (slot > PP.slots || blocks > PP.slots - slot) continue;
        const uint64_t step = P.heads * (uint64_t)P.dk * wide, state = state_of(P, request);
        float *const matrices = PP.block_states + ((uint64_t)slot * P.heads + h) * ((uint64_t)P.dk * wide);
        const bool live = column < P.dv && first_row < P.dk;
        f32x4 x[2], A[2][KD][2], B[2];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i / 4][i % 4] = live && P.state_in && state != ~0ull ? P.state_in[(state * P.heads + h) * ((uint64_t)P.dk * P.dv) + (uint64_t)(first_row + i) * P.dv + column] : 0.f;
        const auto load = [&](uint32_t b) __attribute__((always_inline)) {
            const float *const from = matrices + b * step;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint32_t row = wave * 32 + 8 * (r >> 2) + 4 * t + (r & 3);
#pragma unroll
                for (int p = 0; p < KD; ++p)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        A[t][p][i] = (f32x4){0.f, 0.f, 0.f, 0.f};
                        if (row < P.dk && p * 32 + g * 8 < P.dk) A[t][p][i] = *(const f32x4 *)(from + (uint64_t)row * wide + P.dv + p * 32 + g * 8 + 4 * i);
                    }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) B[i / 4][i % 4] = live ? from[(uint64_t)(first_row + i) * wide + column] : 0.f;
        };
        load(0);
        for (uint32_t b = 0; b < blocks; ++b) {
            if (live)
#pragma unroll
                for (int i = 0; i < 8; ++i) matrices[b * step + (uint64_t)(first_row + i) * wide + column] = x[i / 4][i % 4];
            if (b + 1 == blocks) break;
            float (*const rows)[KD * 32 + 4] = state_rows[b & 1];
            *(f32x4 *)&rows[r][first_row] = x[0], *(f32x4 *)&rows[r][first_row + 4] = x[1];
            __syncthreads();   // (one barrier a block: the other rows are written behind it)
            u32x4 a[2][KD][3];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int p = 0; p < KD; ++p) three_terms(A[t][p], a[t][p]);
            x[0] = B[0], x[1] = B[1];
            if (b + 2 < blocks) load(b + 1);
#pragma unroll
            for (int p = 0; p < KD; ++p) {
                const f32x4 s[2] = {*(const f32x4 *)&rows[r][p * 32 + g * 8], *(const f32x4 *)&rows[r][p * 32 + g * 8 + 4]};
                u32x4 terms[3];
                three_terms(s, terms);
#pragma unroll
                for (int i = 0; i < 3; ++i)
#pragma unroll
                    for (int c = 0; c + i < 3; ++c)
#pragma unroll
                        for (int t = 0; t < 2; ++t) x[t] = mfma_bf16(a[t][p][i], terms[c], x[t]);
            }
        }
        __syncthreads();   // (the rows are free)
    }
}

}  // namespace
