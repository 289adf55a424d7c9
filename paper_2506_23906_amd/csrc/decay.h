// libmmvseg, part of the translation unit serving.hip (included there, in order).
// Linear attention with a decay for each head.
#pragma once

namespace {

struct DecayParams {
    const void *q, *k, *v;
    uint64_t q_stride, k_stride, v_stride, tokens;   // strides in elements
    const int32_t *offsets;                          // null: one token for each request
    const float *log_decay;
    const float *state_in;
    float *state_out;
    const int32_t *state_index;
    uint64_t states;
    void *out;
    uint32_t n, heads, group, dk, dv;
    uint32_t first;                                  // request of a step's launch
    float scale;
};
constexpr uint32_t kMostDk = 128, kMostDv = 256;

// The state that request r starts from and leaves, ~0 for none.
__device__ __forceinline__ uint64_t state_of(const DecayParams &P, uint32_t r) {
    const int64_t i = P.state_index ? P.state_index[r] : r;
    return i >= 0 && (uint64_t)i < P.states ? (uint64_t)i : ~0ull;
}
__device__ __forceinline__ float head_decay(const DecayParams &P, uint32_t h) {
    const float d = P.log_decay[h];
    return d < -1e30f ? -1e30f : d;   // (0 * -infinity is no exponent)
}
struct Span {
    uint32_t begin, end;
};
__device__ __forceinline__ Span span_of(const DecayParams &P, uint32_t r) {
    if (!P.offsets) return {r, r + 1};
    const int64_t most = (int64_t)P.tokens;
    int64_t a = P.offsets[r], b = P.offsets[r + 1];
    a = a < 0 ? 0 : a > most ? most : a;
    b = b < a ? a : b > most ? most : b;
    return {(uint32_t)a, (uint32_t)b};
}

// ---- single tokens -------------------------------------------------------------------------------------------------
//
// Bound by reading and writing the state: 8 dk dv bytes for 4 dk dv operations.  A workgroup has one state; a thread takes four
// columns (16 bytes) of every kth row, kRows of them loaded before the first is used, and the sums over the rows go through LDS.  States are read and
// written past the caches: no other call needs them before the next step.  128 requests of 32 heads, 128 x 128: 101 us (through the caches 108), 5.3 TB/s;
// 64 requests 51 (58).
template <typename T, int kRows> __global__ __launch_bounds__(256) void decay_step_kernel(DecayParams P) {
    __shared__ float query[kMostDk], key[kMostDk];
    __shared__ __align__(16) float part[256 * 4];
    const uint32_t r = P.first + blockIdx.x / P.heads, h = blockIdx.x % P.heads, tid = threadIdx.x, kv = h / P.group;
    const uint64_t state = state_of(P, r), at = (state * P.heads + h) * ((uint64_t)P.dk * P.dv);
    const bool have = state != ~0ull;
    const uint32_t quads = P.dv / 4, step = 256 / quads, first = tid / quads, c = (tid - first * quads) * 4;   // (threads beyond step * quads have no rows)
    const bool live = first < step;
    const float *in = P.state_in && have ? P.state_in + at + c : nullptr;
    float *to = P.state_out && have ? P.state_out + at + c : nullptr;
    f32x4 S[kRows];
    const auto load = [&](uint32_t row) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            S[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
            if (in && live && row + i * step < P.dk) S[i] = __builtin_nontemporal_load((const f32x4 *)(in + (uint64_t)(row + i * step) * P.dv));
        }
    };
    load(first);
    if (tid < P.dk) {
        query[tid] = to_f32(((const T *)P.q)[r * P.q_stride + (uint64_t)h * P.dk + tid]);
        key[tid] = to_f32(((const T *)P.k)[r * P.k_stride + (uint64_t)kv * P.dk + tid]);
    }
    const T *pv = (const T *)P.v + r * P.v_stride + (uint64_t)kv * P.dv + c;
    f32x4 v = {0.f, 0.f, 0.f, 0.f}, o = {0.f, 0.f, 0.f, 0.f};
    if (live) v = (f32x4){to_f32(pv[0]), to_f32(pv[1]), to_f32(pv[2]), to_f32(pv[3])};
    const float decay = __builtin_amdgcn_exp2f(head_decay(P, h) * kLog2e);
    __syncthreads();
    for (uint32_t row = first; live && row < P.dk; row += kRows * step) {
        if (row != first) load(row);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const uint32_t d = row + i * step;
            if (d < P.dk) {
                S[i] = S[i] * decay + key[d] * v;
                o += query[d] * S[i];
                if (to) __builtin_nontemporal_store(S[i], (f32x4 *)(to + (uint64_t)d * P.dv));
            }
        }
    }
    if (live) *(f32x4 *)&part[first * P.dv + c] = o;
    __syncthreads();
    if (tid < P.dv) {
        float sum = 0.f;
        for (uint32_t i = 0; i < step; ++i) sum += part[i * P.dv + tid];
        ((T *)P.out)[((uint64_t)r * P.heads + h) * P.dv + tid] = from_f32<T>(sum * P.scale);
    }
}

// ---- prompts ------------------------------------------------------------------------------------------------------
//
// Chunks of 64 tokens on the matrix cores.  With i, j counted from the chunk's beginning, m tokens in it and S the state before it,
//   out_i = scale (sum_(j <= i) e^(ld (i - j)) (q_i . k_j) v_j + e^(ld (i + 1)) q_i S),   S' = e^(ld m) S + sum_j e^(ld (m - 1 - j)) k_j v_j^T
// A workgroup takes a block of a request's tokens for one head, chunk after chunk, every wave 16 columns of v, out and S, which stays
// in its registers (fp32).  Blocks of one request depend on each other through the state alone: for requests of several, a first
// launch adds up what every block but the last adds to the state (kStates), a second one turns those into the state before each block, and
// the third does all blocks at once.
//
// Layout (products 16x16x32, lane = 16 g + r).  Row r of a state tile's K^T operand is key component 32 p + 8 (r / 4) + 4 t + r % 4, so that
// a lane's parts of the tiles (p, 0) and (p, 1) are the components 32 p + 8 g + 0..7: eight consecutive ones, the state's operand in q S without
// an exchange between lanes.  Scores are made as K Q^T: four consecutive keys of one query in a lane, one 8-byte write to LDS.
// Pairs of lanes load two columns, four consecutive tokens' values each (from memory into registers: waves share no values), and exchange what is the
// other's, so that each has eight tokens of its own column.
//
// What bounds it: vector instructions (56 % of the time of the blocks' launch; matrix ones 30 %) in phases between barriers, which two workgroups on a
// compute unit overlap in part.  12 prompts of 63000 tokens together, 16 heads, 128 columns: 458 to 473 us (states 141 to 148, blocks 22, prompts 287 to 315; floor 161),
// 3.6 TB/s; 3 prompts of 1000 tokens, 8 heads of 64: 17.8 us, three launches of 5 to 8.
//
// Rounding.  The matrix cores take 16-bit operands.  What is no 16-bit input is taken apart into bf16 terms, x = x0 + x1 + ...,
// each the upper half of what the ones before it left (8 bits), the last one rounded: values times their decay into three, which is fp32's
// 24 bits (their sums are the states, fp32 results: 1.4e-7 off), the state and the scores into two where they meet q and v, whose result is rounded to
// 16 bits: 2^-16 of a term, where one term alone (2^-9) would add as much error as that rounding, and a third would take
// 5 to 9 % (12 prompts of up to 32768 tokens 890 us -> 951) for a part of 2^-7 of that rounding's.  Inputs in fp16 are two bf16 terms each (11 bits,
// exact): with bf16's exponents no sum of products overflows that fp32 holds.
constexpr uint32_t kChunk = 64;

struct PromptParams {
    DecayParams d;
    float *block_states;    // [slots * heads][dk * dv]
    uint32_t block;         // tokens (a multiple of kChunk) at least
    uint32_t blocks;        // of one head: as many as there is room for, at least one for each request
    uint32_t slots;         // of the states of blocks: as many as the requests of several blocks can have together
    uint32_t first_block, first_request;   // of a launch
};

__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) { return mfma_16x16x32(bf16_t(), a, b, c); }
__device__ __forceinline__ float low_half(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }
// Two values into kTerms words of bf16 pairs: the upper halves of what is left each time, the last of it rounded.
template <int kTerms> __device__ __forceinline__ void take_apart(float a, float b, uint32_t (&to)[kTerms]) {
#pragma unroll
    for (int i = 0; i + 1 < kTerms; ++i) {
        to[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u);
        a -= high_half(__builtin_bit_cast(uint32_t, a)), b -= high_half(__builtin_bit_cast(uint32_t, b));
    }
    to[kTerms - 1] = pack2<bf16_t>(a, b);
}
// A word of two inputs as its bf16 terms.
template <typename T, int kTerms> __device__ __forceinline__ void input_terms(uint32_t w, uint32_t (&to)[kTerms]) {
    if constexpr (kTerms == 1) {
        to[0] = w;
    } else {
        typedef f16_t pair __attribute__((ext_vector_type(2)));
        const pair h = __builtin_bit_cast(pair, w);
        take_apart<kTerms>((float)h[0], (float)h[1], to);
    }
}

// Tokens of a block: the fewest that need no more than the blocks there are, so that the workgroups come in whole rounds of what the device holds.  (Up to 64
// requests the lengths decide; for more, what is enough for any lengths.  Every workgroup finds the same.)
__device__ __forceinline__ uint32_t wave_sum32(uint32_t v) {
    v += dpp_or_zero<0x111, 0xF>(v);
    v += dpp_or_zero<0x112, 0xF>(v);
    v += dpp_or_zero<0x114, 0xF>(v);
    v += dpp_or_zero<0x118, 0xF>(v);
    v += dpp_or_zero<0x142, 0xA>(v);
    return lane_value(v + dpp_or_zero<0x143, 0xC>(v), 63);
}
__device__ __forceinline__ uint32_t blocks_of(Span s, uint32_t block) { return max(1u, (s.end - s.begin + block - 1) / block); }
__device__ __forceinline__ uint32_t slots_of(uint32_t blocks) { return blocks > 1 ? blocks : 0u; }   // (a request of one block starts from its own state)
__device__ __forceinline__ uint32_t choose_block(const PromptParams &PP) {
    const DecayParams &P = PP.d;
    if (P.n > 64 || PP.block >= P.tokens) return PP.block;
    const uint32_t lane = threadIdx.x & 63;
    const Span s = lane < P.n ? span_of(P, lane) : Span{0, 0};
    const uint32_t length = s.end - s.begin;
    uint32_t block = max(PP.block, (wave_sum32(length) / PP.blocks + kChunk - 1) / kChunk * kChunk);
    for (;;) {   // (at the longest length there are n blocks and no slots)
        const uint32_t own = lane < P.n ? blocks_of(s, block) : 0u;
        if (wave_sum32(own) <= PP.blocks && wave_sum32(slots_of(own)) <= PP.slots) return uniform(block);
        block += max(1u, block / (16 * kChunk)) * kChunk;
    }
}

// Which block of which request a workgroup has; blocks are numbered request after request, at least one each.
struct BlockPlace {
    uint32_t request, block, blocks;   // the block's number in its request, and how many that has
    uint32_t slot;                     // its state's, if there are several
    bool found;
};
__device__ __forceinline__ BlockPlace find_block(const PromptParams &PP, uint32_t block, uint32_t number) {
    const DecayParams &P = PP.d;
    const uint32_t lane = threadIdx.x & 63;
    BlockPlace at = {0, 0, 0, 0, false};
    if (block >= P.tokens) return {number, 0, 1, 0, number < P.n};   // (one for each)
    uint32_t before = 0, slots_before = 0;
    for (uint32_t first = 0; first < P.n; first += 64) {
        const uint32_t r = first + lane, own = r < P.n ? blocks_of(span_of(P, r), block) : 0u;
        uint32_t upto = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(upto, d);
            upto += lane >= (uint32_t)d ? o : 0u;
        }
        const uint64_t hit = __ballot(before + upto > number);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            at.request = uniform(first + l);
            at.blocks = uniform(__shfl(own, l));
            at.block = number - (uniform(before + __shfl(upto, l)) - at.blocks);
            const uint32_t first_slot = slots_before + wave_sum32((int)lane < l ? slots_of(own) : 0u);
            at.slot = first_slot + at.block;
            at.found = at.blocks == 1 || first_slot + at.blocks <= PP.slots;   // (no more than there are, unless offsets go backwards)
            return at;
        }
        before += uniform(__shfl(upto, 63));
        slots_before += wave_sum32(slots_of(own));
    }
    return at;
}

// The value itself, made anew where it is used (no instruction): what follows from it is not kept in registers all through a loop.
__device__ __forceinline__ uint32_t here(uint32_t v) {
    asm volatile("" : "+v"(v));
    return v;
}
// Nothing is moved across: the compiler would load operands so far ahead that registers spill.  (3 do all the same in bf16 with more than 96 key
// components and 64 columns, 22 in fp16 with more than 64 and 160.)
__device__ __forceinline__ void phase() { __builtin_amdgcn_sched_barrier(0); }

// Two rows of 16-bit values, columns c and c + 1 in each word, for lanes of two columns: the even lane has rows 0 .. 3 of both, the odd one rows 4 .. 7; they
// exchange what is the other's.  Words (0, 1), (2, 3), ... of the lane's own column.
__device__ __forceinline__ uint32_t of_neighbour(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false); }   // lanes 2 i and 2 i + 1 swapped
__device__ __forceinline__ u32x4 own_column(const uint32_t (&row)[4], bool odd) {
    const uint32_t sel = odd ? 0x07060302u : 0x05040100u, other = odd ? 0x05040100u : 0x07060302u;
    const uint32_t a = __builtin_amdgcn_perm(row[1], row[0], sel), b = __builtin_amdgcn_perm(row[3], row[2], sel);
    const uint32_t c = of_neighbour(__builtin_amdgcn_perm(row[1], row[0], other)), d = of_neighbour(__builtin_amdgcn_perm(row[3], row[2], other));
    return odd ? (u32x4){c, d, a, b} : (u32x4){a, b, c, d};
}

// KD: key components / 32, rounded up; NW: waves, each of which has 16 columns.
// Waves on a SIMD that LDS leaves room for, at most four (128 registers each): the bound for the registers.
template <int KD, int NW, typename T, bool kStates> constexpr int prompt_occupancy() {
    constexpr int kIn = __is_same(T, f16_t) ? 2 : 1, kRow = KD == 2 ? 64 : 128;
    constexpr int kBytes = 2 * (kIn * KD * 32 * (int)kChunk + (kStates ? 0 : 2 * kIn * (int)kChunk * kRow + 2 * (int)(kChunk * kChunk))) + 1024;
    constexpr int kGroups = 160 * 1024 / kBytes, kWaves = kGroups * NW / 4;
    return kWaves > 4 ? 4 : kWaves < 1 ? 1 : kWaves;
}
template <int KD, int NW, typename T, bool kStates> __global__ __launch_bounds__(64 * NW, (prompt_occupancy<KD, NW, T, kStates>())) void decay_prompt_kernel(PromptParams PP) {
    constexpr int kIn = __is_same(T, f16_t) ? 2 : 1;                   // terms of an input
    constexpr int kMid = 2;                                            // of a score, of the state
    constexpr int kRow = KD == 2 ? 64 : 128;                           // of K and Q in LDS
    constexpr int kPieces = KD * 4;                                    // of 8 components
    // A lane brings 4 tokens x 8 components of K or of Q into LDS; a wave has either.
    constexpr int kItemsK = 16 * kPieces, kItems = kStates ? kItemsK : 2 * kItemsK, kPer = (kItems + 64 * NW - 1) / (64 * NW);
    __shared__ __align__(16) uint16_t lds_q[kStates ? 1 : kIn][kStates ? 1 : kChunk][kRow], lds_k[kStates ? 1 : kIn][kStates ? 1 : kChunk][kRow];
    __shared__ __align__(16) uint16_t lds_kt[kIn][KD * 32][kChunk], lds_p[kMid][kStates ? 1 : kChunk][kChunk];
    __shared__ __align__(16) float by_row[kChunk], by_token[kChunk];   // scale e^(ld (i + 1)); the tokens' decay up to the chunk's end (kStates: the block's)
    const DecayParams &P = PP.d;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4, r = lane & 15;
    const uint32_t in_launch = uniform(blockIdx.x / P.heads), h = uniform(blockIdx.x - in_launch * P.heads), kv = uniform(h / P.group), number = PP.first_block + in_launch;
    const uint32_t block = choose_block(PP);
    const BlockPlace at = find_block(PP, block, number);
    if (!at.found || (kStates && at.block + 1 == at.blocks)) return;
    const uint64_t slot = (uint64_t)at.slot * P.heads + h;
    const Span span = span_of(P, at.request);
    const uint32_t begin = uniform(span.begin + at.block * block);
    const uint32_t end = uniform(min(span.end, begin + block));
    const uint64_t state = state_of(P, at.request), matrix = (uint64_t)P.dk * P.dv;
    const float ld2 = head_decay(P, h) * kLog2e;
    const uint32_t column = wave * 16 + r;
    const bool live_column = column < P.dv;   // (the others compute what nobody reads)
    f32x4 S[2 * KD];
    // the state's rows of this lane: tile 2 p + t, register i
    const float *from = kStates ? nullptr : at.blocks > 1 ? PP.block_states + slot * matrix
                                          : P.state_in && state != ~0ull ? P.state_in + (state * P.heads + h) * matrix : nullptr;
#pragma unroll
    for (int m = 0; m < 2 * KD; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t d = (m / 2) * 32 + g * 8 + (m % 2) * 4 + i;
            S[m][i] = from && live_column && d < P.dk ? from[(uint64_t)d * P.dv + column] : 0.f;
        }

    // Rows are read and written through buffers that end behind the chunk's last token: rows beyond read 0 and are not written, and so do
    // components and columns that dk and dv do not have, whose offsets lie behind any end.
    constexpr uint32_t kNowhere = 1u << 31;
    const uint32_t pieces = P.dk / 8;
    // Lane numbers made anew for every phase: addresses that stay the same from chunk to chunk would fill the registers, and those that spill are loaded
    // behind the next chunk's rows, whose arrival they then wait for.
    struct At {
        uint32_t r, g;
        bool odd;
        uint32_t column2;   // of the lane's pair of columns, in bytes
    };
    const auto lane_at = [&]() __attribute__((always_inline)) {
        const uint32_t l = here(lane), c = wave * 16 + (l & 14);
        return At{l & 15, l >> 4, (l & 1) != 0, c < P.dv ? 2 * c : kNowhere};
    };
    // (three that every phase needs do stay)
    const uint32_t own_row = here(kRow == 128 ? r * 256 + (g ^ r) * 16 : r * 128 + (g ^ r >> 1) * 16), own_score = here(r * 128 + (g ^ r >> 1) * 16),
                   own_kt = here(((r >> 2) * 8 + (r & 3)) * 128 + (g ^ (r >> 1)) * 16);
    u32x4 staged[kPer][4];
    uint32_t values[2][4];
    struct Part {
        bool live, is_q;
        uint32_t rows, piece;
    };
    const auto part_of = [&](int b) __attribute__((always_inline)) {
        const uint32_t first = wave * 64 + b * 64 * NW;
        Part p;
        p.live = first < kItems, p.is_q = first >= kItemsK;
        const uint32_t id = first - (p.is_q ? kItemsK : 0) + here(lane);
        p.piece = id % kPieces, p.rows = id / kPieces * 4;
        return p;
    };
    const auto chunk_rows = [&](const void *base, uint32_t m, uint32_t stride, uint32_t width) __attribute__((always_inline)) {
        return make_rsrc((const void *)uniform64((uint64_t)base), uniform((m - 1) * stride + width));
    };
    const auto load_chunk = [&](uint32_t t0) __attribute__((always_inline)) {
        const uint32_t m = min(kChunk, end - t0);
#pragma unroll
        for (int b = 0; b < kPer; ++b) {
            const Part p = part_of(b);
            if (p.live) {
                const uint32_t stride = 2 * (uint32_t)(p.is_q ? P.q_stride : P.k_stride), off = p.rows * stride + (p.piece < pieces ? p.piece * 16 : kNowhere);
                const auto rows = chunk_rows(p.is_q ? (const T *)P.q + (uint64_t)h * P.dk + t0 * P.q_stride : (const T *)P.k + (uint64_t)kv * P.dk + t0 * P.k_stride, m, stride, 2 * P.dk);
#pragma unroll
                for (int j = 0; j < 4; ++j) staged[b][j] = __builtin_amdgcn_raw_buffer_load_b128(rows, off + j * stride, 0, 0);
            }
        }
        const At l = lane_at();
        const uint32_t stride = 2 * (uint32_t)P.v_stride, off = (l.g * 8 + (l.odd ? 4 : 0)) * stride + l.column2;
        const auto rows = chunk_rows((const T *)P.v + (uint64_t)kv * P.dv + t0 * P.v_stride, m, stride, 2 * P.dv);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) values[s][j] = __builtin_amdgcn_raw_buffer_load_b32(rows, off + (s * 32 + j) * stride, 0, 0);
    };
    // LDS rows are pieces of 16 bytes, exchanged by the row's number so that sixteen lanes with as many rows find them in different banks whatever lanes
    // of one product go together (at the rows' natural places a read of C took 4 cycles more of 8): row i of 256 bytes has piece u at u ^ (i mod 16), of
    // 128 bytes at u ^ (i / 2 mod 8).  K by component, row d: piece u, 8 tokens, at u ^ (2 (d / 8 mod 4) + (d / 2 mod 2)) ^ (d / 32 mod 2), its two halves
    // exchanged where d / 64 is odd: the lanes of a read have d = 8 (r / 4) + r % 4 + ..., those of a write d / 8 from 0 to 15.
    const auto row_piece = [&](uint32_t row, uint32_t u) __attribute__((always_inline)) { return kRow == 128 ? row * 256 + ((u ^ (row & 15)) * 16) : row * 128 + ((u ^ (row >> 1 & 7)) * 16); };
    const auto score_piece = [&](uint32_t row, uint32_t u) __attribute__((always_inline)) { return row * 128 + ((u ^ (row >> 1 & 7)) * 16); };
    const auto kt_tile = [&](int a, uint32_t own, int t, int s) __attribute__((always_inline)) {   // components of tile t, tokens 32 s + 8 g .. + 7
        const u32x4 w = *(const u32x4 *)((const char *)lds_kt[a] + (own ^ (s * 64) ^ (t / 2 % 2 * 16)) + (t / 2) * 32 * 128 + (t % 2) * 4 * 128);
        return t / 4 % 2 ? (u32x4){w[2], w[3], w[0], w[1]} : w;
    };

    if (!kStates && tid < kChunk) by_row[tid] = P.scale * __builtin_amdgcn_exp2f(ld2 * (float)(tid + 1));
    if (!kStates && tid < kChunk) by_token[tid] = __builtin_amdgcn_exp2f(ld2 * (float)(kChunk - 1 - tid));
    if (begin < end) load_chunk(begin);
    // The first chunk's loads are waited for here: with any of them under way at the loop's head, the compiler's wait there would be for all that the wave has
    // issued, the stores of the chunk before among them.
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    for (uint32_t t0 = begin; t0 < end; t0 += kChunk) {
        const uint32_t m = min(kChunk, end - t0);
        if (kStates && tid < kChunk) by_token[tid] = __builtin_amdgcn_exp2f(ld2 * (float)(end - 1 - t0 - tid));   // (blocks here are whole chunks)
        if (!kStates && m < kChunk && tid < kChunk) by_token[tid] = __builtin_amdgcn_exp2f(ld2 * (float)max((int)m - 1 - (int)tid, 0));
        // keys (by token and by component) and queries into LDS
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
                    if constexpr (!kStates) {
                        char *const to = p.is_q ? (char *)lds_q[a] : (char *)lds_k[a];
#pragma unroll
                        for (int j = 0; j < 4; ++j) *(u32x4 *)(to + row_piece(p.rows + j, p.piece)) = (u32x4){w[j][0], w[j][1], w[j][2], w[j][3]};
                    }
                    if (!p.is_q) {
                        const uint32_t unit = p.rows / 8 ^ (p.piece & 3) * 2 ^ (p.piece / 4 & 1), half = (p.rows / 4 & 1) ^ (p.piece / 8 & 1);
                        char *to = (char *)lds_kt[a] + p.piece * 8 * 128 + half * 8;
#pragma unroll
                        for (int c = 0; c < 8; ++c) {   // component c of the four tokens
                            const uint32_t sel = c % 2 ? 0x07060302u : 0x05040100u;
                            *(u32x2 *)(to + c * 128 + (unit ^ (c / 2 & 1)) * 16) = (u32x2){__builtin_amdgcn_perm(w[1][c / 2], w[0][c / 2], sel), __builtin_amdgcn_perm(w[3][c / 2], w[2][c / 2], sel)};
                        }
                    }
                }
            }
        }
        // values: tokens 32 s + 8 g + 2 i, + 1 of the lane's column in V[a][s][i]
        u32x4 V[kIn][2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            uint32_t y[4][kIn];
#pragma unroll
            for (int j = 0; j < 4; ++j) input_terms<T, kIn>(values[s][j], y[j]);
#pragma unroll
            for (int a = 0; a < kIn; ++a) {
                const uint32_t rows[4] = {y[0][a], y[1][a], y[2][a], y[3][a]};
                V[a][s] = own_column(rows, here(lane) & 1);
            }
        }
        __syncthreads();
        if (t0 + kChunk < end) load_chunk(t0 + kChunk);
        phase();

        f32x4 O[4];
        if constexpr (!kStates) {
            // scores: key tile by query tile up to the diagonal, and the two tiles of zeros beside it that a product reads
            constexpr uint32_t kQueryTiles = 0x8FFA94, kKeyTiles = 0xDE4910;   // two bits each: 0 1 1 2 2 2 3 3 3 3 0 2, 0 0 1 0 1 2 0 1 2 3 1 3
#pragma unroll
            for (int k = 0; k < (12 + NW - 1) / NW; ++k) {
                const uint32_t u = wave + k * NW;
                if (12 % NW == 0 || u < 12) {
                    const uint32_t qt = kQueryTiles >> (2 * u) & 3, kt = kKeyTiles >> (2 * u) & 3;
                    const At l = lane_at();
                    f32x4 x = {0.f, 0.f, 0.f, 0.f};
                    if (u < 10) {
#pragma unroll
                        for (int p = 0; p < KD; ++p)
#pragma unroll
                            for (int a = 0; a < kIn; ++a)
#pragma unroll
                                for (int b = 0; b + a < kIn; ++b)
                                    x = mfma_bf16(*(const u32x4 *)((const char *)lds_k[a] + kt * 32 * kRow + (own_row ^ (p * 64))), *(const u32x4 *)((const char *)lds_q[b] + qt * 32 * kRow + (own_row ^ (p * 64))), x);
                    }
                    const int apart = (int)(qt * 16 + l.r) - (int)(kt * 16 + l.g * 4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float by = P.scale * __builtin_amdgcn_exp2f(ld2 * (float)max(apart - i, 0));
                        x[i] = apart >= i ? x[i] * by : 0.f;
                    }
                    uint32_t lo[kMid], hi[kMid];
                    take_apart<kMid>(x[0], x[1], lo);
                    take_apart<kMid>(x[2], x[3], hi);
#pragma unroll
                    for (int a = 0; a < kMid; ++a) *(u32x2 *)((char *)lds_p[a] + score_piece(qt * 16 + l.r, kt * 2 + l.g / 2) + l.g % 2 * 8) = (u32x2){lo[a], hi[a]};
                    phase();
                }
            }
            // what the state before the chunk adds
#pragma unroll
            for (int p = 0; p < KD; ++p) {
                const uint32_t own = own_row ^ (p * 64);
                u32x4 B[kMid];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t x[kMid];
                    take_apart<kMid>(S[2 * p + i / 2][2 * (i % 2)], S[2 * p + i / 2][2 * (i % 2) + 1], x);
#pragma unroll
                    for (int a = 0; a < kMid; ++a) B[a][i] = x[a];
                }
#pragma unroll
                for (int a = 0; a < kIn; ++a) {
#pragma unroll
                    for (int t0_ = 0; t0_ < 4; t0_ += 2) {
                        u32x4 A[2];
#pragma unroll
                        for (int t = 0; t < 2; ++t) A[t] = *(const u32x4 *)((const char *)lds_q[a] + own + (t0_ + t) * 32 * kRow);
#pragma unroll
                        for (int b = 0; b + a < kMid; ++b)
#pragma unroll
                            for (int t = 0; t < 2; ++t) O[t0_ + t] = mfma_bf16(A[t], B[b], p == 0 && a == 0 && b == 0 ? (f32x4){0.f, 0.f, 0.f, 0.f} : O[t0_ + t]);
                    }
                }
                phase();
            }
            const At l = lane_at();
#pragma unroll
            for (int t = 0; t < 4; ++t) O[t] *= *(const f32x4 *)&by_row[t * 16 + l.g * 4];
            const float decay = __builtin_amdgcn_exp2f(ld2 * (float)m);
#pragma unroll
            for (int t = 0; t < 2 * KD; ++t) S[t] *= decay;
            phase();
        }
        // the state after it
        float odd = 0.f;   // NaN if one of the wave's values is not finite
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const At l = lane_at();
            u32x4 W[3];
            const f32x4 by[2] = {*(const f32x4 *)&by_token[32 * s + 8 * l.g], *(const f32x4 *)&by_token[32 * s + 8 * l.g + 4]};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x = low_half(V[0][s][i]), y = high_half(V[0][s][i]);
                if constexpr (kIn == 2) x += low_half(V[1][s][i]), y += high_half(V[1][s][i]);
                if constexpr (!kStates) odd = __builtin_fmaf(x, 0.f, __builtin_fmaf(y, 0.f, odd));
                uint32_t terms[3];
                take_apart<3>(x * by[i / 2][2 * (i % 2)], y * by[i / 2][2 * (i % 2) + 1], terms);
#pragma unroll
                for (int c = 0; c < 3; ++c) W[c][i] = terms[c];
            }
#pragma unroll
            for (int t0_ = 0; t0_ < 2 * KD; t0_ += 2) {
                constexpr int kTogether = 2;
#pragma unroll
                for (int a = 0; a < kIn; ++a) {
                    u32x4 A[kTogether];
#pragma unroll
                    for (int t = 0; t < kTogether; ++t) A[t] = kt_tile(a, own_kt, t0_ + t, s);
#pragma unroll
                    for (int c = 0; c + a < 3; ++c)
#pragma unroll
                        for (int t = 0; t < kTogether; ++t) S[t0_ + t] = mfma_bf16(A[t], W[c], S[t0_ + t]);
                }
                phase();
            }
        }
        if constexpr (!kStates) {
            __syncthreads();   // all scores are there
            const At l = lane_at();
            if (!__any(odd != 0.f)) {
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int a = 0; a < kMid; ++a) {
                        u32x4 A[4];
#pragma unroll
                        for (int t = 2 * s; t < 4; ++t) A[t] = *(const u32x4 *)((const char *)lds_p[a] + (own_score ^ (s * 64)) + t * 16 * 128);
#pragma unroll
                        for (int b = 0; b < kIn && b + a < kMid; ++b)
#pragma unroll
                            for (int t = 2 * s; t < 4; ++t) O[t] = mfma_bf16(A[t], V[b][s], O[t]);
                    }
            } else {   // the zeros of later tokens must not meet their infinities and NaN
                const uint32_t mine = wave * 16 + l.r;
                const T *base = (const T *)P.v + (uint64_t)kv * P.dv + (mine < P.dv ? mine : 0);
                for (uint32_t j = 0; j < m; ++j) {
                    const uint32_t rows = here(l.g * 4);
                    const float x = to_f32(base[(t0 + j) * P.v_stride]);
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t q = t * 16 + rows + i;
                            float w = 0.f;
#pragma unroll
                            for (int a = 0; a < kMid; ++a) w += low_half(*(const uint16_t *)((const char *)lds_p[a] + score_piece(q, j / 8) + j % 8 * 2));
                            O[t][i] = q >= j ? O[t][i] + w * x : O[t][i];
                            phase();
                        }
                }
            }
            // rows 0, 1 of a tile's four are the even lane's, 2, 3 the odd one's, both columns of each
            const uint32_t stride = 2 * P.heads * P.dv, off = (l.g * 4 + (l.odd ? 2 : 0)) * stride + l.column2;
            const auto rows = chunk_rows((T *)P.out + ((uint64_t)t0 * P.heads + h) * P.dv, m, stride, 2 * P.dv);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t a = pack2<T>(O[t][0], O[t][1]), b = pack2<T>(O[t][2], O[t][3]);   // own column
                const uint32_t got = of_neighbour(l.odd ? a : b), own = l.odd ? b : a;    // the lane's two rows, the other column and this one
                const uint32_t left = l.odd ? got : own, right = l.odd ? own : got;
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_amdgcn_perm(right, left, 0x05040100u), rows, off + t * 16 * stride, 0, 0);
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_amdgcn_perm(right, left, 0x07060302u), rows, off + (t * 16 + 1) * stride, 0, 0);
            }
        }
        // Keys and queries are free again.  (Without kStates that holds from the barrier above on; the scores, still read, are next written behind the next
        // chunk's first barrier.)
        if constexpr (kStates) __syncthreads();
    }
    float *to = kStates ? PP.block_states + slot * matrix
                        : at.block + 1 == at.blocks && P.state_out && state != ~0ull ? P.state_out + (state * P.heads + h) * matrix : nullptr;
    const uint32_t lane_rows = here(lane) / 16 * 8;
    if (to && live_column)
#pragma unroll
        for (int m = 0; m < 2 * KD; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t d = (m / 2) * 32 + lane_rows + (m % 2) * 4 + i;
                if (d < P.dk) to[(uint64_t)d * P.dv + column] = S[m][i];
            }
}

// What the blocks add, turned into the state before each of them (all but the last one's share is there): a thread has four elements of one state.
__global__ __launch_bounds__(256) void decay_blocks_kernel(PromptParams PP) {
    const DecayParams &P = PP.d;
    const uint64_t matrix = (uint64_t)P.dk * P.dv;
    const uint32_t slices = (uint32_t)((matrix + 1023) / 1024), slice = blockIdx.x % slices, h = blockIdx.x / slices % P.heads, request = PP.first_request + blockIdx.x / slices / P.heads;
    const uint32_t block = choose_block(PP), blocks = blocks_of(span_of(P, request), block);
    if (blocks == 1) return;
    uint32_t mine = 0;   // slots before this request's
    for (uint32_t i = threadIdx.x & 63; i < request; i += 64) mine += slots_of(blocks_of(span_of(P, i), block));
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) mine += __shfl_xor(mine, d);
    const uint64_t at = (uint64_t)slice * 1024 + threadIdx.x * 4;
    if (at >= matrix || mine + blocks > PP.slots) return;
    const uint64_t state = state_of(P, request);
    f32x4 S = {0.f, 0.f, 0.f, 0.f};
    if (P.state_in && state != ~0ull) S = *(const f32x4 *)(P.state_in + (state * P.heads + h) * matrix + at);
    const float decay = __builtin_amdgcn_exp2f(head_decay(P, h) * kLog2e * (float)block);
    float *slot = PP.block_states + ((uint64_t)mine * P.heads + h) * matrix + at;
    const uint64_t step = P.heads * matrix;
    uint32_t b = 0;
    for (; b + 4 < blocks; b += 4, slot += 4 * step) {   // (four blocks' loads under way)
        f32x4 add[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) add[i] = *(const f32x4 *)(slot + i * step);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            *(f32x4 *)(slot + i * step) = S;
            S = S * decay + add[i];
        }
    }
    for (; b < blocks; ++b, slot += step) {
        f32x4 add = {0.f, 0.f, 0.f, 0.f};
        if (b + 1 < blocks) add = *(const f32x4 *)slot;
        *(f32x4 *)slot = S;
        S = S * decay + add;
    }
}

}  // namespace
