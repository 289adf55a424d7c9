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
// columns (16 bytes) of every kth row, kRows of them loaded before the first is used, and the sums over the rows go through LDS.
template <typename T, int kRows> __global__ __launch_bounds__(256) void decay_step_kernel(DecayParams P) {
    __shared__ float query[kMostDk], key[kMostDk];
    __shared__ __align__(16) float part[256 * 4];
    const uint32_t r = blockIdx.x / P.heads, h = blockIdx.x % P.heads, tid = threadIdx.x, kv = h / P.group;
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
            if (in && live && row + i * step < P.dk) S[i] = *(const f32x4 *)(in + (uint64_t)(row + i * step) * P.dv);
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
                if (to) *(f32x4 *)(to + (uint64_t)d * P.dv) = S[i];
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
// A workgroup takes a block of a request's tokens for one head, chunk after chunk, every wave 32 columns of v, out and S, which stays
// in its registers (fp32).  Blocks of one request depend on each other through the state alone: for requests of several, a first
// launch adds up what every block but the last adds to the state (kStates), a second one turns those into the state before each block, and
// the third does all blocks at once.
//
// Layout (products 16x16x32, lane = 16 g + r).  Row r of a state tile's K^T operand is key component 32 p + 8 (r / 4) + 4 t + r % 4, so that
// a lane's parts of the tiles (p, 0) and (p, 1) are the components 32 p + 8 g + 0..7: eight consecutive ones, the state's operand in q S without
// an exchange between lanes.  Scores are made as K Q^T: four consecutive keys of one query in a lane, one 8-byte write to LDS.
// A lane loads two columns of eight consecutive tokens' values (from memory into registers: waves share no values) and exchanges halves: columns
// 2 r and 2 r + 1 are column r of the wave's two tiles.
//
// Rounding.  The matrix cores take 16-bit operands.  What is no 16-bit input is taken apart into bf16 terms, x = x0 + x1 + ...,
// each the rounding of what the ones before it left (8 bits each): values times their decay into three, which is fp32's
// 24 bits (their sums are the states, fp32 results), the state and the scores into two where they meet q and v, whose result is rounded to
// 16 bits: 2^-17 of a term, where one term alone (2^-9) would add as much error as that rounding.  Inputs in fp16 are two bf16 terms each (11 bits,
// exact): with bf16's exponents no sum of products overflows that fp32 holds.
constexpr uint32_t kChunk = 64;
constexpr uint32_t kDecayPad = 8;   // LDS rows end in 16 bytes more: sixteen rows' 16-byte pieces lie in other banks

struct PromptParams {
    DecayParams d;
    float *block_states;    // [blocks * heads][dk * dv]
    uint32_t block;         // tokens (a multiple of kChunk)
    uint32_t blocks;        // that there is room for (offsets that go backwards may ask for more)
};

__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) { return mfma_16x16x32(bf16_t(), a, b, c); }
__device__ __forceinline__ float low_half(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }
// Two values into kTerms words of bf16 pairs.
template <int kTerms> __device__ __forceinline__ void take_apart(float a, float b, uint32_t (&to)[kTerms]) {
#pragma unroll
    for (int i = 0; i < kTerms; ++i) {
        to[i] = pack2<bf16_t>(a, b);
        a -= low_half(to[i]), b -= high_half(to[i]);
    }
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

// Which block of which request a workgroup has; blocks are numbered request after request, at least one each.
struct BlockPlace {
    uint32_t request, block, blocks;   // the block's number in its request, and how many that has
    uint32_t first;                    // number of the request's first block
    bool found;
};
__device__ __forceinline__ uint32_t blocks_of(Span s, uint32_t block) { return max(1u, (s.end - s.begin + block - 1) / block); }
__device__ __forceinline__ BlockPlace find_block(const DecayParams &P, uint32_t block, uint32_t number) {
    const uint32_t lane = threadIdx.x & 63;
    BlockPlace at = {0, 0, 0, 0, false};
    uint32_t before = 0;
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
            at.first = uniform(before + __shfl(upto, l)) - at.blocks;
            at.block = number - at.first;
            at.found = true;
            return at;
        }
        before += uniform(__shfl(upto, 63));
    }
    return at;
}

// KD: key components / 32, rounded up; NW: waves, each of which has 32 columns.
template <int KD, int NW, typename T, bool kStates> __global__ __launch_bounds__(64 * NW, NW > 4 ? 2 : 2) void decay_prompt_kernel(PromptParams PP) {
    constexpr int kIn = sizeof(T) == 2 && __is_same(T, f16_t) ? 2 : 1;   // terms of an input
    constexpr int kMid = 2;                                            // of a score, of the state
    constexpr int kRow = KD * 32 + kDecayPad, kColumn = kChunk + kDecayPad;
    constexpr int kPieces = KD * 4;                                    // 8 components each
    constexpr int kBlocks8 = 8 * kPieces * (kStates ? 1 : 2);          // 8 x 8 pieces of K (and Q) of a chunk
    constexpr int kPer = (kBlocks8 + 64 * NW - 1) / (64 * NW);
    __shared__ __align__(16) uint16_t lds_q[kStates ? 1 : kIn][kStates ? 1 : kChunk][kRow], lds_k[kStates ? 1 : kIn][kStates ? 1 : kChunk][kRow];
    __shared__ __align__(16) uint16_t lds_kt[kIn][KD * 32][kColumn], lds_p[kMid][kStates ? 1 : kChunk][kColumn];
    const DecayParams &P = PP.d;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4, r = lane & 15;
    const uint32_t h = blockIdx.x % P.heads, kv = h / P.group;
    const BlockPlace at = find_block(P, PP.block, blockIdx.x / P.heads);
    if (!at.found || (kStates && at.block + 1 == at.blocks)) return;
    const Span span = span_of(P, at.request);
    uint32_t begin = uniform(span.begin) + at.block * PP.block;
    const uint32_t end = min(uniform(span.end), begin + PP.block);
    const uint64_t state = state_of(P, at.request), matrix = (uint64_t)P.dk * P.dv;
    const float ld2 = head_decay(P, h) * kLog2e;
    if (kStates && ld2 < 0.f) {   // tokens whose decay up to the block's end is zero in fp32 (below 2^-150) add nothing
        const float reach = 152.f / -ld2;
        if (reach + 1.f < (float)(end - begin)) begin += ((end - begin) - (uint32_t)reach - 1) / kChunk * kChunk;
    }
    const uint32_t column = wave * 32 + 2 * r;
    const bool live_column = column < P.dv;
    f32x4 S[2 * KD][2];
    // the state's rows of this lane: tile 2 p + t, register i
    const float *from = kStates ? nullptr : at.blocks > 1 ? PP.block_states + ((uint64_t)blockIdx.x) * matrix
                                          : P.state_in && state != ~0ull ? P.state_in + (state * P.heads + h) * matrix : nullptr;
#pragma unroll
    for (int m = 0; m < 2 * KD; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t d = (m / 2) * 32 + g * 8 + (m % 2) * 4 + i;
            float2 x = make_float2(0.f, 0.f);
            if (from && live_column && d < P.dk) x = *(const float2 *)(from + (uint64_t)d * P.dv + column);
            S[m][0][i] = x.x, S[m][1][i] = x.y;
        }

    u32x4 staged[kPer][8];
    uint32_t values[16];
    const uint32_t pieces = P.dk / 8;
    auto load_chunk = [&](uint32_t t0) __attribute__((always_inline)) {
        const uint32_t last = end - 1;
#pragma unroll
        for (int b = 0; b < kPer; ++b) {
            const uint32_t id = tid + b * 64 * NW;
            if (kPer * 64 * NW == kBlocks8 || id < kBlocks8) {
                const bool is_q = !kStates && id >= 8 * kPieces;
                const uint32_t in = is_q ? id - 8 * kPieces : id, piece = in % kPieces, rows = in / kPieces * 8;
                const T *base = (is_q ? (const T *)P.q + (uint64_t)h * P.dk : (const T *)P.k + (uint64_t)kv * P.dk) + (piece < pieces ? piece * 8 : 0);
                const uint64_t stride = is_q ? P.q_stride : P.k_stride;
#pragma unroll
                for (int j = 0; j < 8; ++j) staged[b][j] = *(const u32x4 *)(base + min(t0 + rows + j, last) * stride);
            }
        }
        const T *base = (const T *)P.v + (uint64_t)kv * P.dv + (live_column ? column : 0);
#pragma unroll
        for (int j = 0; j < 16; ++j) values[j] = *(const uint32_t *)(base + min(t0 + (j / 8) * 32 + g * 8 + j % 8, last) * P.v_stride);
    };
    auto put_piece = [&](uint16_t *to, const uint32_t (&w)[4]) __attribute__((always_inline)) { *(u32x4 *)to = (u32x4){w[0], w[1], w[2], w[3]}; };

    if (begin < end) load_chunk(begin);
    for (uint32_t t0 = begin; t0 < end; t0 += kChunk) {
        const uint32_t m = min(kChunk, end - t0);
        // keys (by token and by component) and queries into LDS
#pragma unroll
        for (int b = 0; b < kPer; ++b) {
            const uint32_t id = tid + b * 64 * NW;
            if (kPer * 64 * NW == kBlocks8 || id < kBlocks8) {
                const bool is_q = !kStates && id >= 8 * kPieces;
                const uint32_t in = is_q ? id - 8 * kPieces : id, piece = in % kPieces, rows = in / kPieces * 8;
                if (m < kChunk || piece >= pieces) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (rows + j >= m || piece >= pieces) staged[b][j] = (u32x4){0, 0, 0, 0};
                }
                uint32_t w[kIn][8][4];
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t terms[kIn];
                        input_terms<T, kIn>(staged[b][j][i], terms);
#pragma unroll
                        for (int a = 0; a < kIn; ++a) w[a][j][i] = terms[a];
                    }
#pragma unroll
                for (int a = 0; a < kIn; ++a) {
                    if constexpr (!kStates) {
                        uint16_t(*const to)[kRow] = is_q ? lds_q[a] : lds_k[a];
#pragma unroll
                        for (int j = 0; j < 8; ++j) put_piece(&to[rows + j][piece * 8], w[a][j]);
                    }
                    if (!is_q) {
#pragma unroll
                        for (int c = 0; c < 8; ++c) {   // component c of the eight tokens
                            uint32_t x[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_perm(w[a][2 * i + 1][c / 2], w[a][2 * i][c / 2], c % 2 ? 0x07060302u : 0x05040100u);
                            put_piece(&lds_kt[a][piece * 8 + c][rows], x);
                        }
                    }
                }
            }
        }
        // values: tokens 32 s + 8 g + 2 i, + 1 of column n in V[a][s][n][i]
        u32x4 V[kIn][2][2];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t x[2] = {values[8 * s + 2 * i], values[8 * s + 2 * i + 1]};
                if (m < kChunk || !live_column) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        if (!live_column || 32 * s + 8 * g + 2 * i + j >= m) x[j] = 0;
                }
                uint32_t y[2][kIn];
#pragma unroll
                for (int j = 0; j < 2; ++j) input_terms<T, kIn>(x[j], y[j]);
#pragma unroll
                for (int a = 0; a < kIn; ++a) {
                    V[a][s][0][i] = __builtin_amdgcn_perm(y[1][a], y[0][a], 0x05040100u);
                    V[a][s][1][i] = __builtin_amdgcn_perm(y[1][a], y[0][a], 0x07060302u);
                }
            }
        __syncthreads();
        if (t0 + kChunk < end) load_chunk(t0 + kChunk);

        f32x4 O[4][2];
        if constexpr (!kStates) {
            // scores: key tile by query tile, up to the diagonal and the zeros beside it that a product reads
            for (uint32_t u = wave; u < 12; u += NW) {
                const uint32_t qt = u < 2 ? 0 : u < 4 ? 1 : u < 8 ? 2 : 3, kt = u < 2 ? u : u < 4 ? u - 2 : u < 8 ? u - 4 : u - 8;
                f32x4 x = {0.f, 0.f, 0.f, 0.f};
                if (kt <= qt) {
#pragma unroll
                    for (int p = 0; p < KD; ++p)
#pragma unroll
                        for (int a = 0; a < kIn; ++a)
#pragma unroll
                            for (int b = 0; b + a < kIn; ++b)
                                x = mfma_bf16(*(const u32x4 *)&lds_k[a][kt * 16 + r][p * 32 + g * 8], *(const u32x4 *)&lds_q[b][qt * 16 + r][p * 32 + g * 8], x);
                }
                const int apart = (int)(qt * 16 + r) - (int)(kt * 16 + g * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = apart >= i ? x[i] * __builtin_amdgcn_exp2f(ld2 * (float)(apart - i)) : 0.f;
                uint32_t lo[kMid], hi[kMid];
                take_apart<kMid>(x[0], x[1], lo);
                take_apart<kMid>(x[2], x[3], hi);
#pragma unroll
                for (int a = 0; a < kMid; ++a) *(u32x2 *)&lds_p[a][qt * 16 + r][kt * 16 + g * 4] = (u32x2){lo[a], hi[a]};
            }
            // what the state before the chunk adds
#pragma unroll
            for (int t = 0; t < 4; ++t) O[t][0] = O[t][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < KD; ++p) {
                u32x4 B[2][kMid];
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t x[kMid];
                        take_apart<kMid>(S[2 * p + i / 2][n][2 * (i % 2)], S[2 * p + i / 2][n][2 * (i % 2) + 1], x);
#pragma unroll
                        for (int a = 0; a < kMid; ++a) B[n][a][i] = x[a];
                    }
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int a = 0; a < kIn; ++a) {
                        const u32x4 A = *(const u32x4 *)&lds_q[a][t * 16 + r][p * 32 + g * 8];
#pragma unroll
                        for (int n = 0; n < 2; ++n)
#pragma unroll
                            for (int b = 0; b + a < kMid; ++b) O[t][n] = mfma_bf16(A, B[n][b], O[t][n]);
                    }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float by = __builtin_amdgcn_exp2f(ld2 * (float)(t * 16 + g * 4 + i + 1));
                    O[t][0][i] *= by, O[t][1][i] *= by;
                }
        }
        // the state after it
        const float decay = __builtin_amdgcn_exp2f(ld2 * (float)m);
#pragma unroll
        for (int t = 0; t < 2 * KD; ++t) S[t][0] *= decay, S[t][1] *= decay;
        float odd = 0.f;   // NaN if one of the wave's values is not finite
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            u32x4 W[2][3];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = 32 * s + 8 * (int)g + 2 * i;
                const float a = __builtin_amdgcn_exp2f(ld2 * (float)max((int)m - 1 - j, 0)), b = __builtin_amdgcn_exp2f(ld2 * (float)max((int)m - 2 - j, 0));
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    float x = low_half(V[0][s][n][i]), y = high_half(V[0][s][n][i]);
                    if constexpr (kIn == 2) x += low_half(V[1][s][n][i]), y += high_half(V[1][s][n][i]);
                    odd = __builtin_fmaf(x, 0.f, __builtin_fmaf(y, 0.f, odd));
                    uint32_t terms[3];
                    take_apart<3>(x * a, y * b, terms);
#pragma unroll
                    for (int c = 0; c < 3; ++c) W[n][c][i] = terms[c];
                }
            }
#pragma unroll
            for (int t = 0; t < 2 * KD; ++t)
#pragma unroll
                for (int a = 0; a < kIn; ++a) {
                    const u32x4 A = *(const u32x4 *)&lds_kt[a][(t / 2) * 32 + (r >> 2) * 8 + (t % 2) * 4 + (r & 3)][s * 32 + g * 8];
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int c = 0; c + a < 3; ++c) S[t][n] = mfma_bf16(A, W[n][c], S[t][n]);
                }
        }
        if constexpr (!kStates) {
            __syncthreads();   // all scores are there
            if (!__any(odd != 0.f)) {
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int t = 2 * s; t < 4; ++t)
#pragma unroll
                        for (int a = 0; a < kMid; ++a) {
                            const u32x4 A = *(const u32x4 *)&lds_p[a][t * 16 + r][s * 32 + g * 8];
#pragma unroll
                            for (int n = 0; n < 2; ++n)
#pragma unroll
                                for (int b = 0; b < kIn && b + a < kMid; ++b) O[t][n] = mfma_bf16(A, V[b][s][n], O[t][n]);
                        }
            } else {   // the zeros of later tokens must not meet their infinities and NaN
                const T *base = (const T *)P.v + (uint64_t)kv * P.dv + (live_column ? column : 0);
                for (uint32_t j = 0; j < m; ++j) {
                    const float x = to_f32(base[(t0 + j) * P.v_stride]), y = to_f32(base[(t0 + j) * P.v_stride + 1]);
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t q = t * 16 + g * 4 + i;
                            if (q >= j) {
                                float w = 0.f;
#pragma unroll
                                for (int a = 0; a < kMid; ++a) w += low_half(lds_p[a][q][j]);
                                O[t][0][i] += w * x, O[t][1][i] += w * y;
                            }
                        }
                }
            }
            if (live_column)
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t q = t * 16 + g * 4 + i;
                        if (q < m) *(uint32_t *)((T *)P.out + ((uint64_t)(t0 + q) * P.heads + h) * P.dv + column) = pack2<T>(O[t][0][i] * P.scale, O[t][1][i] * P.scale);
                    }
        }
        __syncthreads();   // LDS is free again
    }
    float *to = kStates ? PP.block_states + (uint64_t)blockIdx.x * matrix
                        : at.block + 1 == at.blocks && P.state_out && state != ~0ull ? P.state_out + (state * P.heads + h) * matrix : nullptr;
    if (to && live_column)
#pragma unroll
        for (int m = 0; m < 2 * KD; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t d = (m / 2) * 32 + g * 8 + (m % 2) * 4 + i;
                if (d < P.dk) *(float2 *)(to + (uint64_t)d * P.dv + column) = make_float2(S[m][0][i], S[m][1][i]);
            }
}

// What the blocks add, turned into the state before each of them (all but the last one's share is there): a thread has four elements of one state.
__global__ __launch_bounds__(256) void decay_blocks_kernel(PromptParams PP) {
    const DecayParams &P = PP.d;
    const uint64_t matrix = (uint64_t)P.dk * P.dv;
    const uint32_t slices = (uint32_t)((matrix + 1023) / 1024), slice = blockIdx.x % slices, h = blockIdx.x / slices % P.heads, request = blockIdx.x / slices / P.heads;
    const uint32_t blocks = blocks_of(span_of(P, request), PP.block);
    if (blocks == 1) return;
    uint32_t mine = 0;   // blocks before this request's
    for (uint32_t i = threadIdx.x & 63; i < request; i += 64) mine += blocks_of(span_of(P, i), PP.block);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) mine += __shfl_xor(mine, d);
    const uint64_t at = (uint64_t)slice * 1024 + threadIdx.x * 4;
    if (at >= matrix || mine + blocks > PP.blocks) return;
    const uint64_t state = state_of(P, request);
    f32x4 S = {0.f, 0.f, 0.f, 0.f};
    if (P.state_in && state != ~0ull) S = *(const f32x4 *)(P.state_in + (state * P.heads + h) * matrix + at);
    const float decay = __builtin_amdgcn_exp2f(head_decay(P, h) * kLog2e * (float)PP.block);
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
