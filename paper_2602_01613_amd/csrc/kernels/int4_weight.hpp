// 4-bit weights with group scales: quantisation, the order they are held in, and back; rows of activations laid out anew.
// Part of tn_int4.hip's translation unit, inside its anonymous namespace, after fp8_format.hpp.
#pragma once

// ---------------------------------------------------------------------------------------------
// The products multiply an operand W [features][k] (the tensor, or its transpose) held in pieces of 16 features x 128 k, 1 KB,
// [features / 16][k / 128]. Lane l of a wave that reads 16 bytes at 16 * l has feature l % 16; its word j holds k = 32 * j + 8 * (l / 16) .. + 7, which
// are that lane's operand of one v_mfma_f32_16x16x32_bf16. Within a word element e is at bit 4 * (e / 2) + 16 * (e % 2): one shift and one mask leave two
// neighbouring elements in the halves of a register.
//
// A group's scale and zero are one word: the scale as fp32, whose low 13 bits are clear (fp16 has 10 mantissa bits, bf16 7), with the zero in
// the low four. Of a tensor as it is, words lie [piece][k / 128][group within the 128][feature within the piece]; of a transposed one, whose
// groups run along the features, [feature / group][k]. Features are padded to a multiple of 64 per tensor and k to one of 128 per
// segment, with words of scale 0.
//
// Tiles multiply in fp16, for which there is a second word to a group: scale / 2^e in fp16 and -(1024 + zero), with e of the feature (transposed: of the group of
// features) such that the largest of its scales is in [2^10, 2^11). A weight is at most 15 of them. Scales down to 2^-24 of the largest keep all
// their bits; below, where fp16 is subnormal, they are off by 2^-35 of the largest at most, and the weight by 15 times that. They lie like the others, but transposed the scales and the zeros of 8 k beside each other: [feature / group][k / 8][2][8] halves.
// ---------------------------------------------------------------------------------------------
constexpr int kPiece = 16, kPieceWords = 256, kFeaturePad = 64;

struct OperandArgs {
    const unsigned char *codes, *zeros;            // the tensor: [m][(n + 1) / 2], [m][groups]
    const void* scales;
    unsigned *packed, *words, *halves;             // the operand
    int32_t* exponents;                            // of its features
    int64_t m, n, groups;
    int32_t group, scale_f16, transpose;
    int32_t k_blocks, sub;                         // of the operand: blocks of 128 k, groups in one
    int64_t piece0, k_block0, f_pieces;            // where this tensor starts in the operand, and pieces of its features
    int64_t own_k_blocks;                          // blocks of its k
    int64_t word_stride;                           // transposed: words of one group of features
};

__device__ __forceinline__ int element_bit(int e) { return 4 * (e >> 1) + 16 * (e & 1); }

// Codes in the operand's order: a thread makes a word, a workgroup a piece
__global__ void __launch_bounds__(256) int4_pack_kernel(OperandArgs a) {
    const int64_t piece = blockIdx.x, kb = blockIdx.y;
    const int lane = threadIdx.x >> 2, j = threadIdx.x & 3;
    const int64_t f = piece * kPiece + (lane & 15), k0 = kb * kBlock + j * 32 + (lane >> 4) * 8;
    const int64_t row_bytes = (a.n + 1) / 2;
    unsigned w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int64_t row = a.transpose ? k0 + e : f, col = a.transpose ? f : k0 + e;
        if (row < a.m && col < a.n) w |= (unsigned(a.codes[row * row_bytes + (col >> 1)]) >> (4 * (col & 1)) & 15u) << element_bit(e);
    }
    a.packed[((a.piece0 + piece) * a.k_blocks + a.k_block0 + kb) * kPieceWords + threadIdx.x] = w;
}

__device__ __forceinline__ unsigned scale_word(const OperandArgs& a, int64_t row, int64_t g) {
    if (row >= a.m || g >= a.groups) return 0u;
    const unsigned short s = static_cast<const unsigned short*>(a.scales)[row * a.groups + g];
    const unsigned zero = a.zeros ? a.zeros[row * a.groups + g] & 15u : 8u;
    unsigned bits = a.scale_f16 ? __float_as_uint(float(__builtin_bit_cast(_Float16, s))) : unsigned(s) << 16;
    return (bits & ~15u) | zero;
}

__global__ void __launch_bounds__(256) int4_words_kernel(OperandArgs a) {
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (a.transpose) {                              // [feature / group][k of this tensor]
        const int64_t k_all = a.own_k_blocks * kBlock, g = i / k_all, k = i - g * k_all;
        if (g < a.f_pieces * kPiece / a.group + 1 && g * a.group < a.f_pieces * kPiece) a.words[g * a.word_stride + a.k_block0 * kBlock + k] = scale_word(a, k, g);
    } else {                                        // [piece][k / 128][group within][feature within]
        const int64_t per_piece = a.own_k_blocks * a.sub * kPiece, piece = i / per_piece, in = i - piece * per_piece;
        if (piece < a.f_pieces) a.words[(a.piece0 + piece) * per_piece + in] = scale_word(a, piece * kPiece + (in & 15), in >> 4);
    }
}

// The least e for which |scale| < 2^(e + 11); 0 for no finite scale but zeros
__device__ __forceinline__ int scale_exponent(unsigned most) { return most ? int(most >> 23) - 127 - 10 : 0; }
__device__ __forceinline__ unsigned half_bits(float v) { return __builtin_bit_cast(unsigned short, _Float16(v)); }
__device__ __forceinline__ unsigned half_word(unsigned word, int e) {                   // scale in the low half, -(1024 + zero) in the high one
    return half_bits(ldexpf(__uint_as_float(word & ~15u), -e)) | half_bits(-1024.f - float(word & 15u)) << 16;
}

// The second words, from the first: a wave takes a feature of this tensor, or transposed (all tensors' k at once) a group of features
__global__ void __launch_bounds__(256) int4_halves_kernel(OperandArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t row = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= (a.transpose ? (a.f_pieces * kPiece + a.group - 1) / a.group : a.f_pieces * kPiece)) return;
    const int64_t count = a.transpose ? a.word_stride : a.own_k_blocks * a.sub;
    const int64_t first = a.transpose ? row * a.word_stride : (a.piece0 + (row >> 4)) * count * kPiece + (row & 15), step = a.transpose ? 1 : kPiece;
    unsigned most = 0;
    for (int64_t i = lane; i < count; i += 64) most = max(most, finite_magnitude(__uint_as_float(a.words[first + i * step] & ~15u)));
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) most = max(most, unsigned(__shfl_xor(int(most), d)));
    const int e = scale_exponent(most);
    for (int64_t i = lane; i < count; i += 64) {
        const unsigned w = half_word(a.words[first + i * step], e);
        if (a.transpose) {
            unsigned short* to = reinterpret_cast<unsigned short*>(a.halves) + row * a.word_stride * 2 + (i >> 3) * 16 + (i & 7);
            to[0] = static_cast<unsigned short>(w);
            to[8] = static_cast<unsigned short>(w >> 16);
        } else {
            a.halves[first + i * step] = w;
        }
    }
    if (a.transpose) {
        for (int64_t f = row * a.group + lane; f < min((row + 1) * a.group, a.f_pieces * kPiece); f += 64) a.exponents[f] = e;
    } else if (lane == 0) {
        a.exponents[a.piece0 * kPiece + row] = e;
    }
}

// Back: a thread takes a byte of codes; the first of a group its scale and zero
__global__ void __launch_bounds__(256) int4_unpack_kernel(OperandArgs a, unsigned char* codes, float* scales, unsigned char* zeros) {
    const int64_t row_bytes = (a.n + 1) / 2, row = blockIdx.y + int64_t(blockIdx.z) * 65535, at = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (row >= a.m || at >= row_bytes) return;
    unsigned byte = 0;
    for (int half = 0; half < 2; ++half) {
        const int64_t col = 2 * at + half;
        if (col >= a.n) break;
        const int64_t f = a.transpose ? col : row, k = a.transpose ? row : col;
        const int in = int(k & (kBlock - 1)), lane = int(f & 15) + 16 * ((in >> 3) & 3);
        const unsigned w = a.packed[((a.piece0 + (f >> 4)) * a.k_blocks + a.k_block0 + (k >> 7)) * kPieceWords + lane * 4 + (in >> 5)];
        byte |= (w >> element_bit(in & 7) & 15u) << (4 * half);
        if (col % a.group == 0) {
            const int64_t g = col / a.group;
            const unsigned s = a.transpose ? a.words[g * a.word_stride + a.k_block0 * kBlock + row]
                                           : a.words[(a.piece0 + (row >> 4)) * a.own_k_blocks * a.sub * kPiece + g * kPiece + (row & 15)];
            if (scales) scales[row * a.groups + g] = __uint_as_float(s & ~15u);
            if (zeros) zeros[row * a.groups + g] = static_cast<unsigned char>(s & 15u);
        }
    }
    if (codes) codes[row * row_bytes + at] = static_cast<unsigned char>(byte);
}

// Quantisation: a thread takes a group of a row and writes what the packing reads
template <typename T>
__global__ void __launch_bounds__(256) int4_quantise_kernel(const T* src, int64_t m, int64_t n, int64_t groups, int32_t group, unsigned char* codes,
                                                            bf16_t* scales, unsigned char* zeros) {
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= m * groups) return;
    const int64_t row = i / groups, k0 = (i - row * groups) * group, row_bytes = (n + 1) / 2;
    const int count = int(min(n - k0, int64_t(group)));
    const T* p = src + row * n + k0;
    float lo = 0.f, hi = 0.f;
    bool finite = true;
    for (int e = 0; e < count; ++e) {
        const float v = float(p[e]);
        finite = finite && (__float_as_uint(v) & 0x7fffffffu) < 0x7f800000u;
        lo = fminf(lo, v);
        hi = fmaxf(hi, v);
    }
    const bf16_t rounded = finite ? bf16_t(hi / 15.f - lo / 15.f) : __builtin_bit_cast(bf16_t, static_cast<unsigned short>(0x7fc0));
    const float s = float(rounded);
    const bool some = finite && s > 0.f;
    const float z = some ? fminf(fmaxf(rintf(-lo / s), 0.f), 15.f) : 8.f;
    scales[i] = rounded;
    zeros[i] = static_cast<unsigned char>(int(z));
    for (int e = 0; e < count; e += 2) {            // (groups are even, so no byte belongs to two of them)
        unsigned byte = 0;
        for (int half = 0; half < 2 && e + half < count; ++half) {
            const float q = some ? fminf(fmaxf(rintf(float(p[e + half]) / s) + z, 0.f), 15.f) : 8.f;
            byte |= unsigned(int(q)) << (4 * half);
        }
        codes[row * row_bytes + (k0 + e) / 2] = static_cast<unsigned char>(byte);
    }
}

// Rows of `segments` x cols with any stride and alignment to rows of segments x `padded`, zeros behind each segment's values
__global__ void __launch_bounds__(256) int4_rows_kernel(const bf16_t* x, int64_t x_stride, int64_t tokens, int32_t segments, int64_t cols, int64_t padded,
                                                        bf16_t* out) {
    const int64_t chunks = segments * padded / kChunk, all = tokens * chunks;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
        const int64_t token = i / chunks, at = (i - token * chunks) * kChunk, segment = at / padded, k = at - segment * padded;
        const int64_t left = cols - k;
        const int n = int(left < 0 ? 0 : left < kChunk ? left : kChunk);
        const Chunk<bf16_t> c = load_chunk(x + token * x_stride + segment * cols + (n ? k : 0), n);
        __builtin_memcpy(out + token * segments * padded + at, &c, sizeof(c));
    }
}

// The same rows in fp16 for the tiles, each divided by the power of two that puts its largest finite magnitude into [2^14, 2^15): exact but below 2^-29 of
// that, and there off by 2^-39 of it at most. A workgroup takes a row, or where the inputs are split a range of one, which has its own power of two (77 rows of 51200 are
// 12 ranges each: 20 us as whole rows, on 77 CUs, 6 so); NC chunks of it stay in a thread's registers between the maximum and
// the conversion, what is longer is read again from the caches.
template <int NC>
__global__ void __launch_bounds__(256) int4_half_rows_kernel(const bf16_t* x, int64_t x_stride, int32_t segments, int64_t cols, int64_t padded, int64_t range, _Float16* out,
                                                             int32_t* exponents, int64_t exponents_stride) {
    __shared__ unsigned part[4];
    const int64_t token = blockIdx.x, first = blockIdx.y * range, all = segments * padded / kChunk, chunks = first + range < all ? first + range : all;
    x += token * x_stride;
    out += token * segments * padded;
    auto load = [&](int64_t i) {
        const int64_t at = i * kChunk, segment = segments == 1 ? 0 : at / padded, k = at - segment * padded, left = cols - k;
        const int n = int(left < 0 ? 0 : left < kChunk ? left : kChunk);
        return load_chunk(x + segment * cols + (n ? k : 0), n);
    };
    unsigned most = 0;
    auto look = [&](const Chunk<bf16_t>& c) {
#pragma unroll
        for (int q = 0; q < kChunk; ++q) most = max(most, finite_magnitude(c[q]));
    };
    Chunk<bf16_t> held[NC];
#pragma unroll
    for (int h = 0; h < NC; ++h) {
        const int64_t i = first + h * 256 + int(threadIdx.x);
        if (i < chunks) held[h] = load(i);
    }
#pragma unroll
    for (int h = 0; h < NC; ++h)
        if (first + h * 256 + int(threadIdx.x) < chunks) look(held[h]);
    for (int64_t i = first + NC * 256 + threadIdx.x; i < chunks; i += 256) look(load(i));
    most = row16_max(most);
    most = max(most, unsigned(__shfl_xor(int(most), 16)));
    most = max(most, unsigned(__shfl_xor(int(most), 32)));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
    __syncthreads();
    most = max(max(part[0], part[1]), max(part[2], part[3]));
    // (bf16's subnormals have the exponent field 0: as if they were 2^-127, which keeps them in range)
    const int e = most ? int(most >> 23) - 127 - 14 : 0;
    auto store = [&](const Chunk<bf16_t>& c, int64_t i) {
        uint4 w;
        unsigned* p = &w.x;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
            const halfx2 h = {_Float16(ldexpf(c[2 * q], -e)), _Float16(ldexpf(c[2 * q + 1], -e))};
            p[q] = __builtin_bit_cast(unsigned, h);
        }
        *reinterpret_cast<uint4*>(out + i * kChunk) = w;
    };
#pragma unroll
    for (int h = 0; h < NC; ++h)
        if (first + h * 256 + int(threadIdx.x) < chunks) store(held[h], first + h * 256 + int(threadIdx.x));
    for (int64_t i = first + NC * 256 + threadIdx.x; i < chunks; i += 256) store(load(i), i);
    if (threadIdx.x == 0) exponents[blockIdx.y * exponents_stride + token] = e;
}
