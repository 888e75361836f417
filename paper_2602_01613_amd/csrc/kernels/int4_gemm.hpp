// Products of many tokens with 4-bit weights: tokens in LDS, weights made in registers.
// Part of tn_int4.hip's translation unit, inside its anonymous namespace, after int4_stream.hpp.
#pragma once

// ---------------------------------------------------------------------------------------------
// A workgroup of four waves computes 16 * TM tokens x 256 features: each wave all of the tokens x 64 features, in TM x 4 accumulators of
// v_mfma_f32_16x16x32_f16. Side by side along the features, no two waves make the same weight: its codes go from memory to registers in the
// operand's order (1 KB a load) and become fp16 there, (code - zero) * (scale / 2^e) with one rounding of 2^-11; two weights are a shift, a mask, an or, an addition
// and a multiplication of packed halves, dealt out between the MFMAs of the step before. (In bf16 the rounding was 2^-8, as large as the output's, and the
// conversion half as long again.) The tokens, in fp16 under a power of two for each row, go from memory to LDS without passing through registers, in three stages
// of 64 k; a row is 128 bytes there, its 16-byte chunk c at position c ^ ((row / 2) % 8), so that the 16 rows a read touches at a time fall on 16
// different slots of the 64 banks.
//
// A step is 32 k: 4 * TM MFMAs, tokens outermost. Behind the four of token fragment i the fragment that the next step has in its place is
// read into the same registers. A stage is two steps; what the first one reads (its second half) are the last reads of the stage, so that after the
// barrier in the second step the stage after next but one goes where it is.
//
// Measured: 8192 x 5120 -> 25600 in 1745 us, 1.23 PFLOP/s (the vendor library's bf16 product of the same sizes 1775), matrix cores busy 56 % of the cycles at 2.1 GHz; 77 x
// 51200 -> 5120 (transposed) 62 us, busy 32 %. What bounds it is the one wave of each SIMD: its conversions (60 instructions of four cycles a step) hide only in part behind 4 * TM MFMAs of 16, so that
// a step takes longer than its MFMAs, by 160 ns with 32 tokens, 180 with 96 and 230 with 192, and large tiles are best wherever they fill the chip. More stages of tokens in LDS (four to six), and codes and
// scale words read a step ahead of their use, changed nothing (1 %).
// ---------------------------------------------------------------------------------------------
enum Int4Form : int { INT4_PLAIN = 0, INT4_GATED = 1, INT4_PARTIAL = 2 };

struct Int4GemmArgs {
    Int4Args l;
    int32_t n_row, n_col;            // output tiles
    int32_t band;                    // rows of tiles to a band
    int32_t blocks_per_split;        // blocks of k to a range
};

// LDS: two or three stages of tokens; a ring of CODES blocks of 128 k of the waves' codes, and one of their scale words. (Transposed, a block's words are
// read step by step, so that their ring has one block more.)
template <int TM>
constexpr int kInt4PerCU = TM <= 4 ? 2 : 1;
template <int TM, bool TRANSPOSED, int SUB>
struct Int4Shape {
    static constexpr int BM = 16 * TM, STAGE = BM * 128, NS = TM == 4 ? 2 : 3;
    static constexpr int CODES = TM >= 10 ? 4 : TM >= 6 ? 5 : 3;
    static constexpr int WORDS = TRANSPOSED ? CODES + 1 : CODES;
    static constexpr int WORD_LOADS = TRANSPOSED ? 2 * SUB : SUB, WAVE_WORDS = WORD_LOADS * 256;
    static constexpr int CODES_AT = NS * STAGE, WORDS_AT = CODES_AT + CODES * 16384, SMEM = WORDS_AT + WORDS * 4 * WAVE_WORDS;
    static_assert(kInt4PerCU<TM> * SMEM <= 160 * 1024, "LDS of a compute unit");
};

typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ floatx4 mfma16h(uintx4 w, halfx8 x, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(halfx8, w), x, c, 0, 0, 0); }

// Two weights from element pair `pair` of a word, in three parts: 1024 + code, which is a code in the low bits of an fp16 1024; code - zero; the
// product with the scale, which is the only one that rounds.
__device__ __forceinline__ halfx2 codes_as_half(unsigned w, int pair, unsigned thousands) {
    return __builtin_bit_cast(halfx2, ((w >> (4 * pair)) & 0x000F000Fu) | thousands);
}

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
    __builtin_amdgcn_s_waitcnt((N & 0xF) | (0x7 << 4) | (0xF << 8) | ((N >> 4) << 14));
}
template <typename F, int... Q>
__device__ __forceinline__ void for_constants(F&& f, std::integer_sequence<int, Q...>) {
    (f(std::integral_constant<int, Q>()), ...);
}

#ifdef __HIP_DEVICE_COMPILE__
// Keeps accumulators in the accumulation registers: without it they change places from step to step, by moves where those are nearly full.
template <int TM>
__device__ __forceinline__ void pin(floatx4 (&acc)[TM][4]) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            if constexpr (kInt4PerCU<TM> == 1) asm volatile("" : "+a"(acc[i][f]));
            else asm volatile("" : "+v"(acc[i][f]));
        }
}

template <int TM, int FORM, bool TRANSPOSED, int SUB>
__device__ __forceinline__ void int4_tile(const Int4GemmArgs& g) {
    using S = Int4Shape<TM, TRANSPOSED, SUB>;
    constexpr int LOADS = TM / 2;                 // of a stage, to a wave: 8 rows each
    constexpr int W = 4 + S::WORD_LOADS;          // of a block's codes and words
    static_assert(TM % 2 == 0, "whole loads for each wave");
    typedef __attribute__((address_space(3))) void lds_t;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const Int4Args& a = g.l;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // XCD x takes a contiguous eighth of the tiles, in bands of a few rows of them (rows fastest, ranges of k slowest): what runs there at a time shares
    // panels of both operands in its L2
    const int n_items = g.n_row * g.n_col * a.n_split, xcd = blockIdx.x & 7;
    const int item = int(int64_t(n_items) * xcd >> 3) + int(blockIdx.x >> 3);
    if (item >= int(int64_t(n_items) * (xcd + 1) >> 3)) return;
    const int split = __builtin_amdgcn_readfirstlane(item / (g.n_row * g.n_col)), tile = item - split * (g.n_row * g.n_col);
    const int band = tile / (g.band * g.n_col), in_band = tile - band * (g.band * g.n_col);
    const int band_rows = min(g.band, g.n_row - band * g.band);
    const int col_tile = __builtin_amdgcn_readfirstlane(in_band / band_rows);
    const int row_tile = __builtin_amdgcn_readfirstlane(band * g.band + in_band - col_tile * band_rows);
    const int kb0 = split * g.blocks_per_split, nk = min(a.k_blocks, kb0 + g.blocks_per_split) - kb0;

    // rows past the last token are out of the buffer's bounds: zeros, no memory is read
    constexpr int RSRC = 0x00020000;
    const int row_bytes = int(a.x_stride) * 2, rows = int(min(a.tokens - int64_t(row_tile) * S::BM, int64_t(S::BM)));
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<_Float16*>(static_cast<const _Float16*>(a.x) + int64_t(row_tile) * S::BM * a.x_stride), 0, (rows - 1) * row_bytes + a.k_blocks * (kBlock * 2), RSRC);
    const int vx = (wave * 8 + (lane >> 3)) * row_bytes + (((lane & 7) ^ ((wave & 1) * 4 + (lane >> 4))) * 16);
    const int last_stage = (kb0 + nk) * 2 - 1;
    auto load_x = [&](int n, int at, unsigned char* s) {              // n: load of the stage; at: stage in memory (past the last: that one, not read)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_t*)(s + (wave + 4 * n) * 1024), 16, vx + n * 32 * row_bytes, min(at, last_stage) * 128, 0, 0);
    };

    // the wave's four pieces: gated, two of gate's and the same two of up's; a wave that has none multiplies the first ones and stores nothing
    const int all_pieces = a.f_pieces * a.tensors;
    const int first = FORM == INT4_GATED ? col_tile * 8 + wave * 2 : col_tile * 16 + wave * 4;
    const bool there = FORM == INT4_GATED ? first < a.f_pieces : first < all_pieces;         // (pieces come in fours)
    auto piece_of = [&](int f) {
        const int p = there ? first : 0;
        return FORM == INT4_GATED ? (f < 2 ? p + f : a.f_pieces + p + f - 2) : p + f;
    };
    const int piece_bytes = a.k_blocks * 1024;
    const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned*>(a.packed + int64_t(piece_of(0)) * a.k_blocks * kPieceWords), 0,
                                                                        (FORM == INT4_GATED ? 2 : 4) * piece_bytes, RSRC);
    const __amdgpu_buffer_rsrc_t ru = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned*>(a.packed + int64_t(piece_of(2)) * a.k_blocks * kPieceWords), 0,
                                                                        2 * piece_bytes, RSRC);
    // Words of a block. As it is: of the four pieces at a time, [group within the block][piece][feature]. Transposed: 128 k of a group of features, of which
    // the wave has SUB (1 where groups are of 64 and more, 2 of 32).
    const unsigned* const words0 = TRANSPOSED ? a.halves + piece_of(0) / a.group_pieces * a.word_stride : a.halves + int64_t(piece_of(0)) * a.k_blocks * (SUB * kPiece);
    const int up_words = FORM == INT4_GATED ? (a.f_pieces - 2) * (a.k_blocks * SUB * kPiece * 4) : 0;       // from where a third piece would lie to where up's is
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<unsigned*>(words0), 0, TRANSPOSED ? int(SUB * a.word_stride * 4) : 4 * a.k_blocks * (SUB * kPiece * 4) + up_words, RSRC);
    const int vw = TRANSPOSED ? lane * 4 : (lane >> 4) * (a.k_blocks * SUB * kPiece * 4) + (lane & 15) * 4 + (lane >= 32 ? up_words : 0);
    unsigned char* const codes_lds = smem + S::CODES_AT + wave * 4096;
    unsigned char* const words_lds = smem + S::WORDS_AT + wave * S::WAVE_WORDS;
    auto load_weights = [&](int kb, int code_slot, int word_slot) {       // kb: block of the range (past the last: that one, not read)
        const int at = kb0 + min(kb, nk - 1);
        unsigned char *c = codes_lds + code_slot, *w = words_lds + word_slot;
#pragma unroll
        for (int f = 0; f < 4; ++f)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(FORM == INT4_GATED && f >= 2 ? ru : rc, (lds_t*)(c + f * 1024), 16, lane * 16,
                                                     (FORM == INT4_GATED ? f & 1 : f) * piece_bytes + at * 1024, 0, 0);
#pragma unroll
        for (int n = 0; n < S::WORD_LOADS; ++n)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_t*)(w + n * 256), 4, vw,
                                                     TRANSPOSED ? (n >> 1) * int(a.word_stride * 4) + at * 512 + (n & 1) * 256 : (at * SUB + n) * (kPiece * 4), 0, 0);
    };

    const int r = lane & 15, kq = lane >> 4;
    const int o0 = r * 128 + ((kq ^ (r >> 1)) * 16), o1 = r * 128 + (((4 + kq) ^ (r >> 1)) * 16);
    halfx8 fx[TM];
    uintx4 codes[4], fw[2][4];
    unsigned words[TRANSPOSED ? 1 : 4][TRANSPOSED ? 1 : SUB];
    uintx4 k_words[TRANSPOSED ? SUB : 1][2];
    floatx4 acc[TM][4];
    auto read_x = [&](int i, int half, const unsigned char* s) { fx[i] = *reinterpret_cast<const halfx8*>(s + (half ? o1 : o0) + i * 2048); };
    auto read_codes = [&](int code_slot, int word_slot) {
#pragma unroll
        for (int f = 0; f < 4; ++f) codes[f] = *reinterpret_cast<const uintx4*>(codes_lds + code_slot + f * 1024 + lane * 16);
        if constexpr (!TRANSPOSED) {
#pragma unroll
            for (int f = 0; f < 4; ++f)
#pragma unroll
                for (int s = 0; s < SUB; ++s) words[f][s] = *reinterpret_cast<const unsigned*>(words_lds + word_slot + s * 256 + f * 64 + r * 4);
        }
    };
    auto read_k_words = [&](int word_slot, int j) {                       // transposed: scales and offsets of the lane's 8 k of a step
        if constexpr (TRANSPOSED) {
#pragma unroll
            for (int n = 0; n < SUB; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) k_words[n][h] = *reinterpret_cast<const uintx4*>(words_lds + word_slot + n * 512 + j * 128 + kq * 32 + h * 16);
        }
    };
    unsigned thousands = 0x64006400u;             // 1024 twice, in a register: with the mask in another the two are one instruction
    asm volatile("" : "+v"(thousands));
    // part 0, 1 or 2 of word `at` of the 16 (pair p of fragment f) of step j
    halfx2 half_made[16];
    auto make = [&](uintx4 (&to)[4], int j, int at, int part) {
        const int f = at >> 2, p = at & 3;
        halfx2 scale, offset;
        if constexpr (TRANSPOSED) {
            const unsigned scales = k_words[f * SUB / 4][0][p], offsets = k_words[f * SUB / 4][1][p];          // (a cast of the element itself takes the vector's first)
            scale = __builtin_bit_cast(halfx2, scales);
            offset = __builtin_bit_cast(halfx2, offsets);
        } else {
            const halfx2 w2 = __builtin_bit_cast(halfx2, words[f][j * SUB / 4]);
            scale = halfx2{w2[0], w2[0]};
            offset = halfx2{w2[1], w2[1]};
        }
        if (part == 0) half_made[at] = codes_as_half(codes[f][j], p, thousands);
        else if (part == 1) half_made[at] = half_made[at] + offset;
        else to[f][p] = __builtin_bit_cast(unsigned, half_made[at] * scale);
    };

    // Loads are counted: every block brings LOADS of tokens, W of codes and words, and LOADS of tokens again, in this order. What is waited for in the middle of a stage
    // is the next one, and all that was requested before it.
    constexpr int NEWER_FIRST = S::NS == 3 ? W + LOADS : 0, NEWER_SECOND = S::NS == 3 ? W + LOADS : W;
    constexpr int WORD_STEP = 4 * S::WAVE_WORDS;
    load_weights(0, 0, 0);
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int n = 0; n < LOADS; ++n) load_x(n, kb0 * 2 + q, smem + q * S::STAGE);
    load_weights(1, 16384, WORD_STEP);
    if constexpr (S::NS == 3) {
#pragma unroll
        for (int n = 0; n < LOADS; ++n) load_x(n, kb0 * 2 + 2, smem + 2 * S::STAGE);
    }
#pragma unroll
    for (int q = 2; q < S::CODES; ++q) load_weights(q, q * 16384, q * WORD_STEP);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int f = 0; f < 4; ++f) acc[i][f] = floatx4{0.f, 0.f, 0.f, 0.f};
    pin(acc);
    __builtin_amdgcn_sched_barrier(0);
    wait_vmcnt<(S::NS - 1) * LOADS + (S::CODES - 1) * W>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    read_codes(0, 0);
    read_k_words(0, 0);
#pragma unroll
    for (int at = 0; at < 48; ++at) make(fw[0], 0, at / 3, at % 3);
    read_k_words(0, 1);
#pragma unroll
    for (int i = 0; i < TM; ++i) read_x(i, 0, smem);

    int stage = 0, code_slot = 0, word_slot = 0;  // of the current 64 k and block, in bytes
    for (int kb = 0; kb < nk; ++kb) {
        const int next_code_slot = code_slot == (S::CODES - 1) * 16384 ? 0 : code_slot + 16384;
        const int next_word_slot = word_slot == (S::WORDS - 1) * WORD_STEP ? 0 : word_slot + WORD_STEP;
        auto step = [&](auto j_c) {
            constexpr int j = decltype(j_c)::value, half = j & 1;
            unsigned char* s = smem + stage;
            const int after = stage == (S::NS - 1) * S::STAGE ? 0 : stage + S::STAGE;
            unsigned char* sn = smem + after;
            // second half: the barrier is in front of this fragment, and reads of the next stage (in the last step, of the next codes too) behind it
            constexpr int BAR = TM > 4 ? 2 : TM > 2 ? 1 : 0;
            // The 16 words of the next step, dealt over these fragments: a word's three parts need each other, so that each goes to a slot of its own,
            // beside others' (one after another in one slot, the next MFMA waits for all of them).
            constexpr int FROM = j == 3 ? BAR + 1 : 0, SLOTS = 4 * (TM - FROM);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                if (half && i == BAR) {
                    __builtin_amdgcn_s_waitcnt(0xC07F);                // lgkmcnt(0): this wave has read what it reads of the stage, and its codes
                    wait_vmcnt<j == 1 ? NEWER_FIRST : NEWER_SECOND>();  // the next stage, and the next block's codes, have landed
                    __builtin_amdgcn_s_barrier();
                    __builtin_amdgcn_sched_barrier(0);
                    if (j == 3) read_codes(next_code_slot, next_word_slot);
                }
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    acc[i][f] = mfma16h(fw[half][f], fx[i], acc[i][f]);
                    const int slot = (i - FROM) * 4 + f;
#pragma unroll
                    for (int at = 0; at < 16; ++at)
#pragma unroll
                        for (int part = 0; part < 3; ++part)
                            if (i >= FROM && at * (SLOTS - 2) / 16 + part == slot) make(fw[1 - half], (j + 1) & 3, at, part);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (!half) {
                    read_x(i, 1, s);
                } else if (i >= BAR) {
                    if (i == BAR) {
#pragma unroll
                        for (int q = 0; q < BAR; ++q) read_x(q, 0, sn);
                    }
                    read_x(i, 0, sn);
                    // the stage's loads, dealt over the rest of the step; in the first second half the codes' behind them
#pragma unroll
                    for (int n = 0; n < LOADS; ++n)
                        if (BAR + n * (TM - BAR) / LOADS == i) load_x(n, (kb0 + kb) * 2 + (j >> 1) + S::NS, s);
                    if (j == 1 && i == TM - 1) load_weights(kb + S::CODES, code_slot, TRANSPOSED ? (word_slot == 0 ? (S::WORDS - 1) * WORD_STEP : word_slot - WORD_STEP) : word_slot);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            read_k_words(j >= 2 ? next_word_slot : word_slot, (j + 2) & 3);
            if (half) stage = after;
            pin(acc);
        };
        step(std::integral_constant<int, 0>());
        step(std::integral_constant<int, 1>());
        step(std::integral_constant<int, 2>());
        step(std::integral_constant<int, 3>());
        code_slot = next_code_slot;
        word_slot = next_word_slot;
    }
    wait_vmcnt<0>();                              // no load into LDS outlives the workgroup
    if (!there) return;

    // lane: token l % 16 of fragment i, features 4 * (l / 16) .. + 3 of fragment f
    const int64_t row0 = int64_t(row_tile) * S::BM;
    int exponents[4][4];
#pragma unroll
    for (int f = 0; f < 4; ++f) __builtin_memcpy(exponents[f], a.exponents + int64_t(piece_of(f)) * kPiece + kq * 4, 16);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t token = row0 + i * 16 + r;
        if (token >= a.tokens) continue;
        const int e = a.x_exponents[FORM == INT4_PARTIAL ? int64_t(split) * a.tokens + token : token];
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[i][f][q] = ldexpf(acc[i][f][q], exponents[f][q] + e);
        if constexpr (FORM == INT4_PARTIAL) {
            float* p = a.partial + (int64_t(split) * a.tokens + token) * a.ld + first * kPiece + kq * 4;
#pragma unroll
            for (int f = 0; f < 4; ++f) *reinterpret_cast<floatx4*>(p + f * kPiece) = acc[i][f];
        } else {
            const int tensor = FORM == INT4_GATED ? 0 : first / a.f_pieces, f0 = (first - tensor * a.f_pieces) * kPiece + kq * 4;
            bf16_t* y = a.y + token * a.y_stride + int64_t(tensor) * a.features + f0;
#pragma unroll
            for (int f = 0; f < (FORM == INT4_GATED ? 2 : 4); ++f) {
                floatx4 v = acc[i][f];
                if constexpr (FORM == INT4_GATED) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[q] = gated_value(v[q], acc[i][f + 2][q]);
                }
                const int n = a.features - f0 - f * kPiece;
                if (n > 0) store4(y + f * kPiece, n, v);
            }
        }
    }
}
#endif

template <int TM, int FORM, bool TRANSPOSED, int SUB>
__global__ void __launch_bounds__(256, kInt4PerCU<TM>) int4_gemm_kernel(Int4GemmArgs g) {
#ifdef __HIP_DEVICE_COMPILE__
    int4_tile<TM, FORM, TRANSPOSED, SUB>(g);
#endif
}

// The ranges of K added up in order: a thread takes 4 neighbouring features of a token. Gated: of gate and of up, then silu(gate) * up.
template <bool GATED>
__global__ void __launch_bounds__(256) int4_reduce_kernel(Int4Args a) {
    const int64_t per_token = (GATED ? a.ld / 2 : a.ld) / 4, all = a.tokens * per_token, step = a.tokens * a.ld;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
        const int64_t token = i / per_token;
        const int f4 = int(i - token * per_token) * 4, tensor = f4 / (a.f_pieces * kPiece), f = f4 - tensor * a.f_pieces * kPiece;
        if (f >= a.features) continue;
        auto sum = [&](int at) {
            const float* p = a.partial + token * a.ld + at;
            floatx4 v = *reinterpret_cast<const floatx4*>(p);
            for (int s = 1; s < a.n_split; ++s) v += *reinterpret_cast<const floatx4*>(p + s * step);
            return v;
        };
        floatx4 v = sum(f4);
        if constexpr (GATED) {
            const floatx4 up = sum(f4 + int(a.ld / 2));
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = gated_value(v[q], up[q]);
        }
        store4(a.y + token * a.y_stride + int64_t(tensor) * a.features + f, a.features - f, v);
    }
}
