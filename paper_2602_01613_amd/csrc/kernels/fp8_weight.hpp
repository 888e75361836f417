// 8-bit weights: quantisation at create, the order they are held in, and back.
// Part of tn_fp8.hip's translation unit, inside its anonymous namespace, after fp8_format.hpp.
#pragma once

// ---------------------------------------------------------------------------------------------
// The products multiply an operand W [features][k] (the tensor, or its transpose) held in pieces of 16 features x 128 k, 2 KB,
// [features / 16][k / 128]: byte (f, k) of a piece at 1024 * (k / 64) + 16 * (f + 16 * (k / 16 % 4)) + k % 16. Lane l of a wave that reads
// 16 bytes at 16 * l and at 1024 + 16 * l thus has feature l % 16 and the chunks l / 16 and 4 + l / 16 of 16 k each, in two contiguous 1 KB
// loads. (The order of k in the instruction's operands is free as long as both have the same: all 128 share a scale. This one lets the
// rows of tokens be read from LDS without conflicts.) Scale bytes lie [features / 128][k / 128], a row padded to a multiple of 4. Features
// are padded to whole blocks per tensor (zero codes), and so is k, as the rows of activations are.
// ---------------------------------------------------------------------------------------------
__host__ __device__ __forceinline__ int piece_offset(int f, int k) {
    return 1024 * (k >> 6) + 16 * (f + 16 * ((k >> 4) & 3)) + (k & 15);
}

struct WeightArgs {
    const void* src;               // [m][n]
    const unsigned char* src_scales;
    unsigned char *packed, *scales;
    int64_t m, n;
    int32_t transpose;
    int32_t f_block0, k_block0;    // where this tensor's blocks start in the operand
    int32_t k_blocks, scale_stride;
};

template <typename T>
struct CodesGiven { static constexpr bool value = false; };
template <>
struct CodesGiven<unsigned char> { static constexpr bool value = true; };

// One workgroup per block of 128 x 128 of the tensor: thread t holds rows t / 16 + 16 * i, columns 8 * (t % 16) .. + 7.
template <typename T>
__global__ void __launch_bounds__(256) weight_pack_kernel(WeightArgs a) {
    __shared__ unsigned top[4];
    __shared__ __attribute__((aligned(16))) unsigned char block[kBlock][kBlock];       // codes as the operand has them: [feature][k]
    const int tid = threadIdx.x, rb = blockIdx.y, cb = blockIdx.x;
    const int c0 = (tid & 15) * kChunk, r0 = tid >> 4;
    const int64_t row0 = int64_t(rb) * kBlock, col = int64_t(cb) * kBlock + c0;
    const int n = int(min(a.n - col, int64_t(kChunk)));
    uint2 codes[8];
    unsigned byte;
    if constexpr (CodesGiven<T>::value) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = row0 + r0 + 16 * i;
            unsigned char v[kChunk];
#pragma unroll
            for (int j = 0; j < kChunk; ++j) v[j] = r < a.m && j < n ? static_cast<const unsigned char*>(a.src)[r * a.n + col + j] : 0;
            __builtin_memcpy(&codes[i], v, 8);
        }
        byte = a.src_scales[int64_t(rb) * gridDim.x + cb];
    } else {
        float v[8][kChunk];
        unsigned most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = row0 + r0 + 16 * i;
            load8(static_cast<const T*>(a.src) + (r < a.m ? r * a.n + col : 0), r < a.m ? n : 0, v[i]);
#pragma unroll
            for (int j = 0; j < kChunk; ++j) most = max(most, finite_magnitude(v[i][j]));
        }
        most = row16_max(most);
        most = max(most, unsigned(__shfl_xor(int(most), 16)));
        most = max(most, unsigned(__shfl_xor(int(most), 32)));
        if ((tid & 63) == 0) top[tid >> 6] = most;
        __syncthreads();
        byte = scale_byte(max(max(top[0], top[1]), max(top[2], top[3])));
        const float inv = inverse_scale(byte);
#pragma unroll
        for (int i = 0; i < 8; ++i) codes[i] = make_uint2(codes4(v[i][0], v[i][1], v[i][2], v[i][3], inv), codes4(v[i][4], v[i][5], v[i][6], v[i][7], inv));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + 16 * i;
        if (a.transpose) {
            unsigned char v[kChunk];
            __builtin_memcpy(v, &codes[i], 8);
#pragma unroll
            for (int j = 0; j < kChunk; ++j) block[c0 + j][r] = v[j];
        } else {
            *reinterpret_cast<uint2*>(&block[r][c0]) = codes[i];
        }
    }
    __syncthreads();
    const int fb = a.f_block0 + (a.transpose ? cb : rb), kb = a.k_block0 + (a.transpose ? rb : cb);
    if (tid == 0) a.scales[int64_t(fb) * a.scale_stride + kb] = static_cast<unsigned char>(byte);
    // 8 pieces of 2 KB: 128 vectors of 16 bytes each
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int v = tid + 256 * i, piece = v >> 7, in = v & 127, l = in & 63;
        const int f = piece * 16 + (l & 15), k = 16 * (l >> 4) + 64 * (in >> 6);
        *reinterpret_cast<uint4*>(a.packed + ((int64_t(fb) * 8 + piece) * a.k_blocks + kb) * 2048 + in * 16) = *reinterpret_cast<const uint4*>(&block[f][k]);
    }
}

// The tensor's codes [m][n] and scales as its description has them
__global__ void __launch_bounds__(256) weight_unpack_kernel(WeightArgs a, unsigned char* codes, unsigned char* scales) {
    const int rb = blockIdx.y, cb = blockIdx.x;
    const int fb = a.f_block0 + (a.transpose ? cb : rb), kb = a.k_block0 + (a.transpose ? rb : cb);
    if (scales && threadIdx.x == 0) scales[int64_t(rb) * gridDim.x + cb] = a.scales[int64_t(fb) * a.scale_stride + kb];
    if (!codes) return;
    for (int i = threadIdx.x; i < kBlock * kBlock; i += 256) {
        const int r = i >> 7, c = i & 127, f = a.transpose ? c : r, k = a.transpose ? r : c;
        const int64_t row = int64_t(rb) * kBlock + r, col = int64_t(cb) * kBlock + c;
        if (row < a.m && col < a.n)
            codes[row * a.n + col] = a.packed[((int64_t(fb) * 8 + (f >> 4)) * a.k_blocks + kb) * 2048 + piece_offset(f & 15, k)];
    }
}
