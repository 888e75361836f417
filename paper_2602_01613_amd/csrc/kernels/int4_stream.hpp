// Products of a few tokens with 4-bit weights: the weight streams from memory straight into the matrix cores' operands.
// Part of tn_int4.hip's translation unit, inside its anonymous namespace, after int4_weight.hpp.
#pragma once

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

struct Int4Args {
    const void* x;                             // rows 16-byte aligned, whole blocks of k, zeros where there is no input: bf16, for tiles fp16
    const int32_t* x_exponents;                // tiles: of the rows
    const unsigned *packed, *words, *halves;
    const int32_t* exponents;                  // of the features, for tiles
    bf16_t* y;
    float* partial;                            // fp32 sums [n_split][tokens][ld] of padded features
    int64_t tokens, x_stride, y_stride, ld;
    int64_t word_stride;                       // transposed: words of one group of features
    int32_t k_blocks, sub;                     // sub: groups in a block of k
    int32_t features, f_pieces, tensors;       // of one tensor: features, and pieces with the padding
    int32_t group_pieces;                      // transposed: pieces of features that share a scale
    int32_t transpose, n_split;
};

__device__ __forceinline__ floatx4 mfma16(bf16x8 w, bf16x8 x, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, c, 0, 0, 0); }
__device__ __forceinline__ bf16x8 operand(uintx4 v) { return __builtin_bit_cast(bf16x8, v); }

// The codes of a word as 16 + code in bf16, exactly: 16 .. 31 have the exponent of 16 and steps of 2^-3, so that a code goes to bits 3 to 6.
__device__ __forceinline__ bf16x8 codes_as_bf16(unsigned w) {
    uintx4 v;
    v[0] = ((w << 3) & 0x00780078u) | 0x41804180u;
    v[1] = ((w >> 1) & 0x00780078u) | 0x41804180u;
    v[2] = ((w >> 5) & 0x00780078u) | 0x41804180u;
    v[3] = ((w >> 9) & 0x00780078u) | 0x41804180u;
    return operand(v);
}
__device__ __forceinline__ float word_scale(unsigned s) { return __uint_as_float(s & ~15u); }
__device__ __forceinline__ float sixteen_and_zero(unsigned s) { return __uint_as_float(0x41800000u | ((s & 15u) << 19)); }       // 16 + zero
// One output by the definition, in fp32: for results that are not finite. (The sums of 16 + code lose an infinity's sign to inf - inf, and may overflow
// where the weights' do not.)
__device__ __forceinline__ float plain_sum(const unsigned* packed, const unsigned* words, const bf16_t* x, int k_blocks, int sub_shift, int block_step) {
    float sum = 0.f;
#pragma unroll 1
    for (int run = 0; run < k_blocks * 16; ++run) {          // 8 k: one word of codes, one scale
        const int kb = run >> 4, in = (run & 15) * 8;
        const unsigned w = packed[int64_t(kb) * kPieceWords + ((in >> 3) & 3) * 64 + (in >> 5)];
        const unsigned s = words[kb * int64_t(block_step) + (in >> sub_shift) * kPiece];
        const bf16x8 v = *reinterpret_cast<const bf16x8*>(x + int64_t(run) * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += float(int(w >> element_bit(e) & 15u) - int(s & 15u)) * word_scale(s) * float(v[e]);
    }
    return sum;
}

// silu(gate) * up: relative error 2^-20 down to gates of -87, below which the sigmoid is under fp32's least normal and comes out as 0; finite for every finite gate
__device__ __forceinline__ float gated_value(float gate, float up) { return gate * sigmoid(gate) * up; }

__device__ __forceinline__ bool is_finite(float v) { return (__float_as_uint(v) & 0x7fffffffu) < 0x7f800000u; }

// four neighbouring values of a row as bf16, of which n exist
__device__ __forceinline__ void store4(bf16_t* p, int n, floatx4 v) {
    bf16_t t[4] = {bf16_t(v[0]), bf16_t(v[1]), bf16_t(v[2]), bf16_t(v[3])};
    if (n >= 4) {
        __builtin_memcpy(p, t, 8);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = t[i];
    }
}

// ---------------------------------------------------------------------------------------------
// Y[t][f] = sum over groups g of scale[f][g] * (sum over k in g of (16 + code[f][k]) X[t][k] - (16 + zero[f][g]) * sum over k in g of X[t][k])
//
// on v_mfma_f32_16x16x32_bf16 with the tokens as the first operand, so that a lane of the result holds four tokens of one feature and needs one scale
// word a group. 16 + code is exact in bf16 and costs one shift, one mask and one or for two codes; the sums of X over a group come from the same
// instruction with ones for weights, once for all pieces. A workgroup takes GROUPS pieces (gated: half of them gate's, half up's) and TG x 16
// tokens, and all of k, which its waves deal out block by block and add up through LDS in a fixed order. Each wave has RING blocks requested ahead.
//
// Bound by HBM for one token: 5120 -> 2 x 25600 gated 31 us, 136 MB at 4.4 TB/s; 5120 -> 8192 7.1 us. With more tokens by their reads, which every workgroup makes anew and
// which come at 5 to 6 TB/s over all of them: 25600 -> 5120 with 8 tokens 24 us, 74 MB of weights and 65 of tokens.
// ---------------------------------------------------------------------------------------------
template <int GROUPS, int TG, int SUB>
struct StreamBlock {
    uintx4 codes[GROUPS];
    unsigned words[GROUPS][SUB];
    bf16x8 x[TG][4];
};
// Blocks in flight, as many as registers hold: of 32 tokens three, and two where a block has four groups' words (three kept 40 registers in scratch memory: 24 tokens, 5120 -> 25600 in groups
// of 32, 52 us, 30 with two; with groups of 128, 28).
template <int TG, int SUB>
constexpr int kRing = TG == 1 ? 4 : SUB == 4 ? 2 : 3;

template <int GROUPS, int TG, int SUB, bool GATED>
__global__ void __launch_bounds__(512) int4_stream_kernel(Int4Args a) {
    constexpr int RING = kRing<TG, SUB>;
    __shared__ floatx4 part[8][GROUPS][TG][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    // gated: the first half of the pieces are gate's, the others up's
    constexpr int OWN = GATED ? GROUPS / 2 : GROUPS;
    const int piece0 = blockIdx.x * OWN;
    auto piece_of = [&](int g) { return GATED && g >= OWN ? a.f_pieces + piece0 + g - OWN : piece0 + g; };
    const int64_t token0 = int64_t(blockIdx.y) * (16 * TG);
    const bf16_t* x[TG];
#pragma unroll
    for (int t = 0; t < TG; ++t) {
        const int64_t token = token0 + t * 16 + (lane & 15);           // rows past the end repeat the last one and are not stored
        x[t] = static_cast<const bf16_t*>(a.x) + (token < a.tokens ? token : a.tokens - 1) * a.x_stride + (lane >> 4) * 8;
    }
    const unsigned* codes[GROUPS];
    const unsigned* words[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        codes[g] = a.packed + int64_t(piece_of(g)) * a.k_blocks * kPieceWords + lane * 4;
        words[g] = a.words + int64_t(piece_of(g)) * a.k_blocks * (SUB * kPiece) + (lane & 15);
    }
    floatx4 out[GROUPS][TG];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int t = 0; t < TG; ++t) out[g][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    const bf16x8 ones = operand(uintx4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});

    typedef StreamBlock<GROUPS, TG, SUB> Block;
    auto load = [&](Block& b, int kb) {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) b.codes[g] = *reinterpret_cast<const uintx4*>(codes[g] + int64_t(kb) * kPieceWords);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g)
#pragma unroll
            for (int s = 0; s < SUB; ++s) b.words[g][s] = words[g][(int64_t(kb) * SUB + s) * kPiece];
#pragma unroll
        for (int t = 0; t < TG; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) b.x[t][j] = *reinterpret_cast<const bf16x8*>(x[t] + int64_t(kb) * kBlock + j * 32);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto multiply = [&](const Block& b) {
        constexpr int STEPS = 4 / SUB;
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            floatx4 sums[TG];
#pragma unroll
            for (int t = 0; t < TG; ++t) {
                sums[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < STEPS; ++j) sums[t] = mfma16(b.x[t][s * STEPS + j], ones, sums[t]);
            }
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                floatx4 acc[TG];
#pragma unroll
                for (int t = 0; t < TG; ++t) acc[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < STEPS; ++j) {
                    const bf16x8 w = codes_as_bf16(b.codes[g][s * STEPS + j]);
#pragma unroll
                    for (int t = 0; t < TG; ++t) acc[t] = mfma16(b.x[t][s * STEPS + j], w, acc[t]);
                }
                const float scale = word_scale(b.words[g][s]), centre = sixteen_and_zero(b.words[g][s]);
#pragma unroll
                for (int t = 0; t < TG; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) out[g][t][i] = fmaf(scale, fmaf(-centre, sums[t][i], acc[t][i]), out[g][t][i]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // A ring of blocks, each requested again as soon as it has been multiplied; past the last one that one again, which is in the caches (a branch
    // in the place of a load would make the waits for those before it wait for all).
    const int n = a.k_blocks > wave ? (a.k_blocks - wave + waves - 1) / waves : 0;          // of this wave: wave, wave + waves, ...
    if (n > 0) {
        const int last = wave + (n - 1) * waves;
        Block ring[RING];
#pragma unroll
        for (int q = 0; q < RING; ++q) load(ring[q], min(wave + q * waves, last));
        int i = 0;
        for (; i + RING < n; i += RING) {
#pragma unroll
            for (int q = 0; q < RING; ++q) {
                multiply(ring[q]);
                load(ring[q], min(wave + (i + q + RING) * waves, last));
            }
        }
#pragma unroll
        for (int q = 0; q < RING; ++q)
            if (i + q < n) multiply(ring[q]);
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int t = 0; t < TG; ++t) part[wave][g][t][lane] = out[g][t];
    __syncthreads();
    // lane: feature l % 16 of piece g, tokens 4 * (l / 16) .. + 3 of the 16
    auto total = [&](int g, int t, int64_t token) {
        floatx4 v = part[0][g][t][lane];
        for (int q = 1; q < waves; ++q) v += part[q][g][t][lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (is_finite(v[i]) || token + i >= a.tokens) continue;
            const int64_t piece = piece_of(g);
            const int f = lane & 15;
            const unsigned* p = a.packed + piece * a.k_blocks * kPieceWords + f * 4;
            const bf16_t* row = static_cast<const bf16_t*>(a.x) + (token + i) * a.x_stride;
            v[i] = plain_sum(p, a.words + piece * a.k_blocks * (SUB * kPiece) + f, row, a.k_blocks, SUB == 1 ? 7 : SUB == 2 ? 6 : 5, SUB * kPiece);
        }
        return v;
    };
    for (int u = wave; u < OWN * TG; u += waves) {
        const int g = u / TG, t = u - g * TG;
        const int64_t token = token0 + t * 16 + (lane >> 4) * 4;
        if (token >= a.tokens) continue;
        floatx4 v = total(g, t, token);
        if constexpr (GATED) {
            const floatx4 up = total(OWN + g, t, token);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = gated_value(v[i], up[i]);
        }
        const int piece = piece0 + g, tensor = piece / a.f_pieces, f = (piece - tensor * a.f_pieces) * kPiece + (lane & 15);
        if (f >= a.features) continue;
        bf16_t* y = a.y + token * a.y_stride + int64_t(tensor) * a.features + f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (token + i < a.tokens) y[i * a.y_stride] = bf16_t(v[i]);
    }
}
