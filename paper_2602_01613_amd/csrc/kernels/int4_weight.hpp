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
// ---------------------------------------------------------------------------------------------
constexpr int kPiece = 16, kPieceWords = 256, kFeaturePad = 64;

struct OperandArgs {
    const unsigned char *codes, *zeros;            // the tensor: [m][(n + 1) / 2], [m][groups]
    const void* scales;
    unsigned *packed, *words;                      // the operand
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
