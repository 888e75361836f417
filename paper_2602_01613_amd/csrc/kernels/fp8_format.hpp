// The 8-bit format (e4m3 codes, a power-of-two scale per block of 128) and what the row kernels share: loads and stores
// of 8 elements, reductions over lanes. Part of tn_fp8.hip's translation unit, inside its anonymous namespace.
#pragma once

typedef __bf16 bf16_t;
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = TN_FP8_BLOCK;
// Row kernels: a lane owns 8 consecutive elements (16 bytes in bf16, two such loads in fp32, 8 bytes of codes), so that a
// block of 128 is a row of 16 lanes.
constexpr int kChunk = 8;

// |v| as an ordered integer, 0 for an infinity or a NaN
__device__ __forceinline__ unsigned finite_magnitude(float v) {
    const unsigned a = __float_as_uint(v) & 0x7fffffffu;
    return a < 0x7f800000u ? a : 0u;
}

// E8M0 byte of a block whose largest finite magnitude is a (bits of an fp32): with a = m * 2^x, 1 <= m < 2, the least e with
// a <= 448 * 2^e = 1.75 * 2^(8 + e) is x - 8, or x - 7 where m > 1.75. Subnormal a and zero end at the least byte.
__device__ __forceinline__ unsigned scale_byte(unsigned a) {
    const int byte = int(a >> 23) - 8 + int((a & 0x7fffffu) > 0x600000u);
    return unsigned(byte > 0 ? byte : 0);
}

// 2^-e for that byte (at most 247): exact, and so is the product with it but for results below fp32's least
__device__ __forceinline__ float inverse_scale(unsigned byte) { return __uint_as_float((254u - byte) << 23); }

// Four codes in a word. The operands are at most 448 after scaling; what is not finite becomes NaN first, so that no mode bit
// of the conversion (saturation of infinities) matters.
__device__ __forceinline__ float nan_unless_finite(float v) {
    return (__float_as_uint(v) & 0x7fffffffu) < 0x7f800000u ? v : __uint_as_float(0x7fc00000u);
}
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d, float inv) {
    unsigned w = __builtin_amdgcn_cvt_pk_fp8_f32(nan_unless_finite(a) * inv, nan_unless_finite(b) * inv, 0u, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(nan_unless_finite(c) * inv, nan_unless_finite(d) * inv, w, true);
}

// Maximum over a row of 16 lanes, left in all of them: rotations by 8, 4, 2 and 1 within the row.
__device__ __forceinline__ unsigned row16_max(unsigned v) {
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x128, 0xf, 0xf, false)));
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x124, 0xf, 0xf, false)));
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x122, 0xf, 0xf, false)));
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x121, 0xf, 0xf, false)));
    return v;
}

// Sum over the wave, the same in all lanes
__device__ __forceinline__ float wave_sum(float v) {
#define TN_ROW_ADD(CTRL) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false))
    TN_ROW_ADD(0x128);
    TN_ROW_ADD(0x124);
    TN_ROW_ADD(0x122);
    TN_ROW_ADD(0x121);
#undef TN_ROW_ADD
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
    return v;
}

// 8 elements at p, of which the first n exist (the others are 0): rows of any alignment the type has
template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, float (&v)[kChunk]) {
    if (n >= kChunk) {
        T t[kChunk];
        __builtin_memcpy(t, p, sizeof(t));
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[i] = float(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[i] = i < n ? float(p[i]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, const float (&v)[kChunk]) {
    if (n >= kChunk) {
        T t[kChunk];
#pragma unroll
        for (int i = 0; i < kChunk; ++i) t[i] = T(v[i]);
        __builtin_memcpy(p, t, sizeof(t));
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
            if (i < n) p[i] = T(v[i]);
    }
}

// The 16 lanes of a block quantise it: 8 codes go to `codes`, one lane writes the scale byte. All 16 must be here.
__device__ __forceinline__ void quantise_block(const float (&v)[kChunk], unsigned char* codes, unsigned char* scale) {
    unsigned a = 0;
#pragma unroll
    for (int i = 0; i < kChunk; ++i) a = max(a, finite_magnitude(v[i]));
    const unsigned byte = scale_byte(row16_max(a));
    const float inv = inverse_scale(byte);
    *reinterpret_cast<uint2*>(codes) = make_uint2(codes4(v[0], v[1], v[2], v[3], inv), codes4(v[4], v[5], v[6], v[7], inv));
    if ((threadIdx.x & 15) == 0) *scale = static_cast<unsigned char>(byte);
}

struct RowLayout {          // rows in 8 bits
    int64_t code_stride, scale_stride;
    int32_t blocks;         // of one segment
    int32_t spare;          // scale bytes past the last block
};
