// Products of a few tokens with 4-bit weights: the weight streams from memory straight into the matrix cores' operands.
// Part of tn_int4.hip's translation unit, inside its anonymous namespace, after int4_weight.hpp.
#pragma once

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

struct Int4Args {
    const bf16_t* x;                           // rows 16-byte aligned, whole blocks of k, zeros where there is no input
    const unsigned *packed, *words;
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
__device__ __forceinline__ float word_offset(unsigned s) { return -__uint_as_float(0x44800000u | ((s & 15u) << 13)) * word_scale(s); }  // -(1024 + zero) * scale, exact

// Two weights in bf16 from element pair `pair` of a word: with the code in the mantissa of an fp16 1024 the product with the scale and the
// offset -(1024 + zero) * scale are one fused operation that has nothing to round, (code - zero) * scale is at most 16 bits long.
__device__ __forceinline__ unsigned weights_as_bf16(unsigned w, int pair, float s0, float c0, float s1, float c1) {
    typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const halfx2 h = __builtin_bit_cast(halfx2, ((w >> (4 * pair)) & 0x000F000Fu) | 0x64006400u);
    bf16x2 r;
    r[0] = bf16_t(fmaf(float(h[0]), s0, c0));
    r[1] = bf16_t(fmaf(float(h[1]), s1, c1));
    return __builtin_bit_cast(unsigned, r);
}

// Four neighbouring outputs of a token by the definition, in fp32: for results that are not finite. (The sums of 16 + code lose an infinity's sign to
// inf - inf, and may overflow where the weights' do not.)
__device__ __noinline__ floatx4 plain_sums(const Int4Args& a, int64_t piece, int f0, int64_t token) {
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
    const bf16_t* x = a.x + token * a.x_stride;
    for (int kb = 0; kb < a.k_blocks; ++kb)
        for (int at = 0; at < 16; ++at) {                                   // runs of 8 k
            const int j = at >> 2, quarter = at & 3;
            const bf16_t* p = x + kb * kBlock + at * 8;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned w = a.packed[(piece * a.k_blocks + kb) * kPieceWords + (quarter * 16 + f0 + i) * 4 + j];
                for (int e = 0; e < 8; ++e) {
                    const unsigned s = a.transpose ? a.words[piece / a.group_pieces * a.word_stride + kb * kBlock + at * 8 + e]
                                                   : a.words[((piece * a.k_blocks + kb) * a.sub + (at * a.sub >> 4)) * kPiece + f0 + i];
                    const float q = float(int(w >> element_bit(e) & 15u) - int(s & 15u));
                    sum[i] += q * word_scale(s) * float(p[e]);
                }
            }
        }
    return sum;
}

// (up to the sign of the exponent's last values: relative error 2^-21, and finite for every finite gate)
__device__ __forceinline__ float gated_value(float gate, float up) { return gate * sigmoid(gate) * up; }

__device__ __forceinline__ bool all_finite(floatx4 v) {
    bool fine = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) fine = fine && (__float_as_uint(v[i]) & 0x7fffffffu) < 0x7f800000u;
    return fine;
}

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
// on v_mfma_f32_16x16x32_bf16 with the weight as the first operand, so that a lane of the result holds four consecutive features of one token. 16 + code is
// exact in bf16 and costs one shift, one mask and one or for two codes; the sums of X over a group come from the same instruction with ones for
// weights, once for all pieces. A workgroup takes GROUPS pieces (gated: half of them gate's, half up's) and TG x 16 tokens, and all of k, which its
// waves deal out BLOCKS blocks at a time and add up through LDS in a fixed order.
// Transposed, the scales run along k: weights are made in bf16 with their scale before they are multiplied.
// ---------------------------------------------------------------------------------------------
template <int GROUPS, int TG, int SUB, bool TRANSPOSED>
struct StreamBlock {
    uintx4 codes[GROUPS];
    uintx4 words[TRANSPOSED ? 8 : GROUPS * SUB];        // transposed: of the lane's 4 x 8 k
    bf16x8 x[TG][4];
};

template <int GROUPS, int TG, int SUB, bool TRANSPOSED, bool GATED>
__global__ void __launch_bounds__(512) int4_stream_kernel(Int4Args a) {
    constexpr int BLOCKS = TG == 1 ? 4 : TG == 2 ? 2 : 1;
    __shared__ floatx4 part[8][GROUPS][TG][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int64_t token0 = int64_t(blockIdx.y) * (16 * TG) + (lane & 15);
    // gated: the first half of the pieces are gate's, the others up's
    constexpr int OWN = GATED ? GROUPS / 2 : GROUPS;
    const int piece0 = blockIdx.x * OWN;
    auto piece_of = [&](int g) { return GATED && g >= OWN ? a.f_pieces + piece0 + g - OWN : piece0 + g; };
    const bf16_t* x[TG];
#pragma unroll
    for (int t = 0; t < TG; ++t) {
        const int64_t token = token0 + t * 16;           // rows past the end repeat the last one and are not stored
        x[t] = a.x + (token < a.tokens ? token : a.tokens - 1) * a.x_stride + (lane >> 4) * 8;
    }
    const unsigned* codes[GROUPS];
    const unsigned* words[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        codes[g] = a.packed + int64_t(piece_of(g)) * a.k_blocks * kPieceWords + lane * 4;
        words[g] = TRANSPOSED ? a.words + piece_of(g) / a.group_pieces * a.word_stride + (lane >> 4) * 8
                              : a.words + int64_t(piece_of(g)) * a.k_blocks * (SUB * kPiece) + (lane >> 4) * 4;
    }
    floatx4 out[GROUPS][TG];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int t = 0; t < TG; ++t) out[g][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    const bf16x8 ones = operand(uintx4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});

    typedef StreamBlock<GROUPS, TG, SUB, TRANSPOSED> Block;
    auto load = [&](Block& b, int kb) {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            b.codes[g] = *reinterpret_cast<const uintx4*>(codes[g] + int64_t(kb) * kPieceWords);
            if constexpr (!TRANSPOSED) {
#pragma unroll
                for (int s = 0; s < SUB; ++s) b.words[g * SUB + s] = *reinterpret_cast<const uintx4*>(words[g] + (int64_t(kb) * SUB + s) * kPiece);
            }
        }
        if constexpr (TRANSPOSED) {                      // (the host gives a workgroup pieces of one group)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) b.words[2 * j + h] = *reinterpret_cast<const uintx4*>(words[0] + int64_t(kb) * kBlock + j * 32 + h * 4);
        }
#pragma unroll
        for (int t = 0; t < TG; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) b.x[t][j] = *reinterpret_cast<const bf16x8*>(x[t] + int64_t(kb) * kBlock + j * 32);
    };
    auto multiply = [&](const Block& b) {
        if constexpr (TRANSPOSED) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float s[8], c[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const unsigned w = b.words[2 * j + (e >> 2)][e & 3];
                    s[e] = word_scale(w);
                    c[e] = word_offset(w);
                }
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    uintx4 v;
#pragma unroll
                    for (int p = 0; p < 4; ++p) v[p] = weights_as_bf16(b.codes[g][j], p, s[2 * p], c[2 * p], s[2 * p + 1], c[2 * p + 1]);
#pragma unroll
                    for (int t = 0; t < TG; ++t) out[g][t] = mfma16(operand(v), b.x[t][j], out[g][t]);
                }
            }
        } else {
            constexpr int STEPS = 4 / SUB;
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
                floatx4 sums[TG];
#pragma unroll
                for (int t = 0; t < TG; ++t) {
                    sums[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < STEPS; ++j) sums[t] = mfma16(ones, b.x[t][s * STEPS + j], sums[t]);
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
                        for (int t = 0; t < TG; ++t) acc[t] = mfma16(w, b.x[t][s * STEPS + j], acc[t]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const unsigned w = b.words[g * SUB + s][i];
                        const float scale = word_scale(w), centre = sixteen_and_zero(w);
#pragma unroll
                        for (int t = 0; t < TG; ++t) out[g][t][i] = fmaf(scale, fmaf(-centre, sums[t][i], acc[t][i]), out[g][t][i]);
                    }
                }
            }
        }
    };
    for (int kb = wave * BLOCKS; kb < a.k_blocks; kb += waves * BLOCKS) {
        if (kb + BLOCKS <= a.k_blocks) {
            Block b[BLOCKS];
#pragma unroll
            for (int q = 0; q < BLOCKS; ++q) load(b[q], kb + q);
#pragma unroll
            for (int q = 0; q < BLOCKS; ++q) multiply(b[q]);
        } else {
            for (int q = kb; q < a.k_blocks; ++q) {
                Block b;
                load(b, q);
                multiply(b);
            }
        }
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int t = 0; t < TG; ++t) part[wave][g][t][lane] = out[g][t];
    __syncthreads();
    auto total = [&](int g, int t, int64_t token) {
        floatx4 v = part[0][g][t][lane];
        for (int q = 1; q < waves; ++q) v += part[q][g][t][lane];
        if (!all_finite(v)) v = plain_sums(a, piece_of(g), (lane >> 4) * 4, token);
        return v;
    };
    for (int i = wave; i < OWN * TG; i += waves) {
        const int g = i / TG, t = i - g * TG;
        const int64_t token = token0 + t * 16;
        if (token >= a.tokens) continue;
        floatx4 v = total(g, t, token);
        if constexpr (GATED) {
            const floatx4 up = total(OWN + g, t, token);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = gated_value(v[q], up[q]);
        }
        const int piece = piece0 + g, tensor = piece / a.f_pieces, f = (piece - tensor * a.f_pieces) * kPiece + (lane >> 4) * 4;
        if (f < a.features) store4(a.y + token * a.y_stride + int64_t(tensor) * a.features + f, a.features - f, v);
    }
}
