// Products of a few tokens: the weight streams from memory straight into the matrix cores' operands.
// Part of tn_fp8.hip's translation unit, inside its anonymous namespace, after fp8_weight.hpp.
#pragma once

// ---------------------------------------------------------------------------------------------
// Y[t][f] = sum_k X[t][k] W[f][k] on v_mfma_scale_f32_16x16x128_f8f6f4: one instruction is 16 features x 16 tokens x one block of
// k, with the two scale bytes of its block applied by the instruction. The weight is the first operand, so a lane of the result
// holds four consecutive features of one token. A workgroup takes GROUPS pieces' worth of features (16 each) and all of k, which its
// waves deal out four blocks at a time (a word of scale bytes, of which the instruction picks one) and add up through LDS in a fixed order.
// Bound by memory: all of a quad's loads are requested before its first instruction, and with up to 16 waves to a workgroup a CU has 100 KB
// under way. One token 5120 -> 8192 in 8.0 us (42 MB, 5.2 TB/s), 25600 -> 5120 in 25.4; with blocks dealt out one by one and a scale byte to each, eight tokens
// of the latter took 36 us instead of 29.
// ---------------------------------------------------------------------------------------------
struct LinearArgs {
    const unsigned char *codes, *scales;       // X in 8 bits
    const unsigned char *packed, *w_scales;
    void* y;                                   // bf16 [tokens][y_stride]
    unsigned char *out_codes, *out_scales;     // gated form
    int64_t tokens, code_stride, scale_stride, y_stride;
    int64_t out_code_stride, out_scale_stride;
    int32_t k_blocks, w_scale_stride;
    int32_t features, f_pieces;                // of one tensor: features, and pieces of 16 with the padding
    int32_t tensors;
    int32_t spare;                             // gated form: scale bytes past the last block
    int32_t n_split;                           // ranges of K
    float* partial;                            // not null: fp32 sums [n_split][tokens][ld] of padded features instead of the output
    int64_t ld;
};

__device__ __forceinline__ intx8 load_piece(const unsigned char* p) {       // two loads of 16 bytes, 1 KB apart
    const intx4 a = *reinterpret_cast<const intx4*>(p), b = *reinterpret_cast<const intx4*>(p + 1024);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ intx8 load_row_chunks(const unsigned char* p) {          // of a row of tokens, 64 bytes apart
    const intx4 a = *reinterpret_cast<const intx4*>(p), b = *reinterpret_cast<const intx4*>(p + 64);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <int SEL_W = 0, int SEL_X = 0>
__device__ __forceinline__ floatx4 mfma_block(intx8 w, intx8 x, floatx4 c, unsigned sw, unsigned sx) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, 0, 0, SEL_W, int(sw), SEL_X, int(sx));
}

// (the hardware's exponential and reciprocal: relative error 2^-22 + |gate| * 2^-24, under that of the sums and far under a code's half
// step of 2^-4. With expf and a division tiles of 256 x 256 spent 12 us of 76 here.)
__device__ __forceinline__ floatx4 gate_value(floatx4 gate, floatx4 up) {
    floatx4 h;
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = gate[i] * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(gate[i] * -1.44269504f)) * up[i];
    return h;
}
__device__ __forceinline__ unsigned magnitude4(floatx4 v) {
    return max(max(finite_magnitude(v[0]), finite_magnitude(v[1])), max(finite_magnitude(v[2]), finite_magnitude(v[3])));
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

// Four blocks of k (a word of scale bytes) of GROUPS pieces and 16 tokens; `n` of the blocks are there
template <int GROUPS>
__device__ __forceinline__ void stream_quad(const unsigned char* w, int64_t group_bytes, const unsigned char* ws, const unsigned char* x,
                                            const unsigned char* xs, int kb, int n, floatx4 (&acc)[GROUPS]) {
    const unsigned sw = *reinterpret_cast<const unsigned*>(ws + kb), sx = *reinterpret_cast<const unsigned*>(xs + kb);
    intx8 fw[GROUPS][4], fx[4];
    auto load = [&](int b) {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) fw[g][b] = load_piece(w + g * group_bytes + int64_t(kb + b) * 2048);
        fx[b] = load_row_chunks(x + (kb + b) * kBlock);
    };
    auto multiply = [&](auto b_c) {
        constexpr int b = decltype(b_c)::value;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) acc[g] = mfma_block<b, b>(fw[g][b], fx[b], acc[g], sw, sx);
    };
    if (n >= 4) {
#pragma unroll
        for (int b = 0; b < 4; ++b) load(b);
        multiply(std::integral_constant<int, 0>());
        multiply(std::integral_constant<int, 1>());
        multiply(std::integral_constant<int, 2>());
        multiply(std::integral_constant<int, 3>());
    } else {
        load(0);
        multiply(std::integral_constant<int, 0>());
        if (n > 1) load(1), multiply(std::integral_constant<int, 1>());
        if (n > 2) load(2), multiply(std::integral_constant<int, 2>());
    }
}

// blockDim.x / 64 waves, 16 at the most: the host takes as many as leave each the same number of words of scales
template <int GROUPS>
__global__ void __launch_bounds__(1024) stream_kernel(LinearArgs a) {
    __shared__ floatx4 part[16][GROUPS][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int piece0 = blockIdx.x * GROUPS;                         // over all tensors; GROUPS divides 8
    const int64_t token = int64_t(blockIdx.y) * 16 + (lane & 15);
    const int64_t from = min(token, a.tokens - 1);                  // rows past the end repeat the last one and are not stored
    const unsigned char* w = a.packed + int64_t(piece0) * a.k_blocks * 2048 + lane * 16;
    const unsigned char* ws = a.w_scales + int64_t(piece0 >> 3) * a.w_scale_stride;
    const unsigned char* x = a.codes + from * a.code_stride + (lane >> 4) * 16;
    const unsigned char* xs = a.scales + from * a.scale_stride;
    floatx4 acc[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) acc[g] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int kb = wave * 4; kb < a.k_blocks; kb += waves * 4)
        stream_quad<GROUPS>(w, int64_t(a.k_blocks) * 2048, ws, x, xs, kb, a.k_blocks - kb, acc);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) part[wave][g][lane] = acc[g];
    __syncthreads();
    for (int g = wave; g < GROUPS; g += waves) {
        floatx4 v = part[0][g][lane];
        for (int q = 1; q < waves; ++q) v += part[q][g][lane];
        const int piece = piece0 + g, tensor = piece / a.f_pieces, f = (piece - tensor * a.f_pieces) * 16 + (lane >> 4) * 4;
        if (token >= a.tokens) continue;
        if (a.partial) *reinterpret_cast<floatx4*>(a.partial + token * a.ld + piece * 16 + (lane >> 4) * 4) = v;
        else store4(static_cast<bf16_t*>(a.y) + token * a.y_stride + int64_t(tensor) * a.features + f, a.features - f, v);
    }
}
