// Products of a few tokens: the weight streams from memory straight into the matrix cores' operands.
// Part of tn_fp8.hip's translation unit, inside its anonymous namespace, after fp8_weight.hpp.
#pragma once

// ---------------------------------------------------------------------------------------------
// Y[t][f] = sum_k X[t][k] W[f][k] on v_mfma_scale_f32_16x16x128_f8f6f4: one instruction is 16 features x 16 tokens x one block of
// k, with the two scale bytes of its block applied by the instruction. The weight is the first operand, so a lane of the result
// holds four consecutive features of one token. A workgroup takes GROUPS pieces' worth of features (16 each) and all of k, which its
// waves deal out block by block and add up through LDS in a fixed order.
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

template <int WAVES, int GROUPS, int NT>
__global__ void __launch_bounds__(WAVES * 64) stream_kernel(LinearArgs a) {
    __shared__ floatx4 part[WAVES][GROUPS * NT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int piece0 = blockIdx.x * GROUPS;                         // over all tensors; GROUPS divides 8
    const int64_t token0 = int64_t(blockIdx.y) * (16 * NT);
    const unsigned char* w = a.packed + int64_t(piece0) * a.k_blocks * 2048 + lane * 16;
    const unsigned char* ws = a.w_scales + int64_t(piece0 >> 3) * a.w_scale_stride;
    const unsigned char *x[NT], *xs[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {                                  // rows past the end repeat the last one and are not stored
        const int64_t token = min(token0 + t * 16 + (lane & 15), a.tokens - 1);
        x[t] = a.codes + token * a.code_stride + (lane >> 4) * 16;
        xs[t] = a.scales + token * a.scale_stride;
    }
    floatx4 acc[GROUPS][NT];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[g][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int kb = wave; kb < a.k_blocks; kb += WAVES) {
        intx8 fw[GROUPS];
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) fw[g] = load_piece(w + (int64_t(g) * a.k_blocks + kb) * 2048);
        const unsigned sw = ws[kb];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const intx8 fx = load_row_chunks(x[t] + kb * kBlock);
            const unsigned sx = xs[t][kb];
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) acc[g][t] = mfma_block(fw[g], fx, acc[g][t], sw, sx);
        }
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int t = 0; t < NT; ++t) part[wave][g * NT + t][lane] = acc[g][t];
    __syncthreads();
    for (int i = wave; i < GROUPS * NT; i += WAVES) {
        floatx4 v = part[0][i][lane];
#pragma unroll
        for (int q = 1; q < WAVES; ++q) v += part[q][i][lane];
        const int g = i / NT, t = i - g * NT, piece = piece0 + g;
        const int tensor = piece / a.f_pieces, f = (piece - tensor * a.f_pieces) * 16 + (lane >> 4) * 4;
        const int64_t token = token0 + t * 16 + (lane & 15);
        if (token < a.tokens)
            store4(static_cast<bf16_t*>(a.y) + token * a.y_stride + int64_t(tensor) * a.features + f, a.features - f, v);
    }
}

// ---------------------------------------------------------------------------------------------
// silu(gate) * up of a block of 128 features: wave w takes the pieces w % 8 of gate and of up, and every second block of k from
// w / 8 on. The maximum over the 128 features of a token meets in LDS.
// ---------------------------------------------------------------------------------------------
// (the hardware's exponential and reciprocal: relative error 2^-22 + |gate| * 2^-24, under that of the sums and far under a code's half
// step of 2^-4. With expf and a division the tiles of 256 x 256 below spent 12 us of 76 here.)
__device__ __forceinline__ floatx4 gate_value(floatx4 gate, floatx4 up) {
    floatx4 h;
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = gate[i] * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(gate[i] * -1.44269504f)) * up[i];
    return h;
}
__device__ __forceinline__ unsigned magnitude4(floatx4 v) {
    return max(max(finite_magnitude(v[0]), finite_magnitude(v[1])), max(finite_magnitude(v[2]), finite_magnitude(v[3])));
}

template <int NT>
__global__ void __launch_bounds__(1024) stream_gated_kernel(LinearArgs a) {
    __shared__ floatx4 part[8][2 * NT][64];
    __shared__ unsigned top[8][NT * 16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = wave & 7, half = wave >> 3;
    const int64_t token0 = int64_t(blockIdx.y) * (16 * NT);
    const unsigned char* w[2];
    const unsigned char* ws[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int piece = s * a.f_pieces + blockIdx.x * 8 + g;
        w[s] = a.packed + int64_t(piece) * a.k_blocks * 2048 + lane * 16;
        ws[s] = a.w_scales + int64_t(piece >> 3) * a.w_scale_stride;
    }
    const unsigned char *x[NT], *xs[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t token = min(token0 + t * 16 + (lane & 15), a.tokens - 1);
        x[t] = a.codes + token * a.code_stride + (lane >> 4) * 16;
        xs[t] = a.scales + token * a.scale_stride;
    }
    floatx4 acc[2][NT];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[s][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int kb = half; kb < a.k_blocks; kb += 2) {
        const intx8 fw[2] = {load_piece(w[0] + int64_t(kb) * 2048), load_piece(w[1] + int64_t(kb) * 2048)};
        const unsigned sw[2] = {ws[0][kb], ws[1][kb]};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const intx8 fx = load_row_chunks(x[t] + kb * kBlock);
            const unsigned sx = xs[t][kb];
#pragma unroll
            for (int s = 0; s < 2; ++s) acc[s][t] = mfma_block(fw[s], fx, acc[s][t], sw[s], sx);
        }
    }
    if (half) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int t = 0; t < NT; ++t) part[g][s * NT + t][lane] = acc[s][t];
    }
    __syncthreads();
    floatx4 h[NT];
    if (!half) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            h[t] = gate_value(acc[0][t] + part[g][t][lane], acc[1][t] + part[g][NT + t][lane]);
            unsigned m = magnitude4(h[t]);
            m = max(m, unsigned(__shfl_xor(int(m), 16)));
            m = max(m, unsigned(__shfl_xor(int(m), 32)));
            if (lane < 16) top[g][t * 16 + lane] = m;
        }
    }
    __syncthreads();
    if (half) return;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        unsigned m = 0;
#pragma unroll
        for (int q = 0; q < 8; ++q) m = max(m, top[q][t * 16 + (lane & 15)]);
        const unsigned byte = scale_byte(m);
        const int64_t token = token0 + t * 16 + (lane & 15);
        if (token >= a.tokens) continue;
        *reinterpret_cast<unsigned*>(a.out_codes + token * a.out_code_stride + blockIdx.x * kBlock + g * 16 + (lane >> 4) * 4) =
            codes4(h[t][0], h[t][1], h[t][2], h[t][3], inverse_scale(byte));
        unsigned char* s = a.out_scales + token * a.out_scale_stride;
        if (g == 0 && lane < 16) s[blockIdx.x] = static_cast<unsigned char>(byte);
        if (g == 1 && blockIdx.x == 0 && (lane >> 4) < a.spare) s[gridDim.x + (lane >> 4)] = 0;
    }
}
