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

// Four codes in a word, of finite values that are at most 448 after scaling
__device__ __forceinline__ unsigned finite_codes4(float a, float b, float c, float d, float inv) {
    const unsigned w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0u, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
}
// The same of any values: what is not finite becomes NaN first, so that no mode bit of the conversion (saturation of infinities)
// matters.
__device__ __forceinline__ float nan_unless_finite(float v) {
    return (__float_as_uint(v) & 0x7fffffffu) < 0x7f800000u ? v : __uint_as_float(0x7fc00000u);
}
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d, float inv) {
    return finite_codes4(nan_unless_finite(a), nan_unless_finite(b), nan_unless_finite(c), nan_unless_finite(d), inv);
}

// 1 / (1 + exp(-v)) to 4 units of fp32's last place (below 2^-126: 0), in 8 instructions where expf and a division take 30: the exponent
// v * log2(e) in two parts, of which the hardware's 2^x takes the first. The second is a residue of either sign, applied as the positive factor
// 1 + rest * ln(2): below v = -88.72 the power is infinite, and so is its product with the factor, which makes the result 0. Past +-100 the
// result does not change (1 and 0). A NaN comes out as something finite, and makes a NaN where it is multiplied with v itself.
__device__ __forceinline__ float sigmoid(float v) {
    const float c = __builtin_amdgcn_fmed3f(v, -100.f, 100.f);
    const float t = c * -1.44269504f;
    const float rest = fmaf(c, -1.44269504f, -t) + c * -1.92596299e-8f;
    const float factor = fmaf(rest, 0.693147181f, 1.f);
    return __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_exp2f(t), factor, 1.f));
}

// Maximum over a row of 16 lanes, left in all of them: rotations by 8, 4, 2 and 1 within the row.
__device__ __forceinline__ unsigned row16_max(unsigned v) {
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x128, 0xf, 0xf, false)));
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x124, 0xf, 0xf, false)));
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x122, 0xf, 0xf, false)));
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x121, 0xf, 0xf, false)));
    return v;
}

// Sums over a row of 16 lanes and over the wave, the same in all lanes
__device__ __forceinline__ float row16_sum(float v) {
#define TN_ROW_ADD(CTRL) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false))
    TN_ROW_ADD(0x128);
    TN_ROW_ADD(0x124);
    TN_ROW_ADD(0x122);
    TN_ROW_ADD(0x121);
#undef TN_ROW_ADD
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
    v = row16_sum(v);
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
    return v;
}
// Sum of the up to 16 waves' parts: one read of LDS, where a loop over them waits for each
__device__ __forceinline__ float parts_sum(const float* part, int waves) {
    const int q = threadIdx.x & 15;
    return row16_sum(q < waves ? part[q] : 0.f);
}

// 8 elements at p, of which the first n exist (the others are 0), as they are in memory: rows of any alignment the type has.
// Two bf16 stay in a word (as an array of bf16 the compiler gives each a register of its own).
template <typename T>
struct Chunk;
template <>
struct Chunk<float> {
    float v[kChunk];
    __device__ __forceinline__ float operator[](int i) const { return v[i]; }
};
template <>
struct Chunk<bf16_t> {
    unsigned w[kChunk / 2];
    __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
};
template <typename T>
__device__ __forceinline__ Chunk<T> load_chunk(const T* p, int n) {
    Chunk<T> c;
    if (n >= kChunk) {
        __builtin_memcpy(&c, p, sizeof(c));
    } else {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < kChunk; ++i) c.v[i] = i < n ? p[i] : 0.f;
        } else {
            const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
            for (int i = 0; i < kChunk; i += 2) c.w[i >> 1] = (i < n ? unsigned(q[i]) : 0u) | (i + 1 < n ? unsigned(q[i + 1]) << 16 : 0u);
        }
    }
    return c;
}
template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, float (&v)[kChunk]) {
    const Chunk<T> c = load_chunk(p, n);
#pragma unroll
    for (int i = 0; i < kChunk; ++i) v[i] = c[i];
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

// The 16 lanes of a block quantise it: 8 codes go to `codes`, one lane writes the scale byte. All 16 must be here. The magnitudes
// are first taken as they are: an infinity or a NaN is larger than any finite one and shows in the maximum.
__device__ __forceinline__ void quantise_block(const float (&v)[kChunk], unsigned char* codes, unsigned char* scale) {
    unsigned a = 0;
#pragma unroll
    for (int i = 0; i < kChunk; ++i) a = max(a, __float_as_uint(v[i]) & 0x7fffffffu);
    a = row16_max(a);
    unsigned byte;
    uint2 c;
    if (a < 0x7f800000u) {
        byte = scale_byte(a);
        const float inv = inverse_scale(byte);
        c = make_uint2(finite_codes4(v[0], v[1], v[2], v[3], inv), finite_codes4(v[4], v[5], v[6], v[7], inv));
    } else {                                             // the same for the 16 lanes
        a = 0;
#pragma unroll
        for (int i = 0; i < kChunk; ++i) a = max(a, finite_magnitude(v[i]));
        byte = scale_byte(row16_max(a));
        const float inv = inverse_scale(byte);
        c = make_uint2(codes4(v[0], v[1], v[2], v[3], inv), codes4(v[4], v[5], v[6], v[7], inv));
    }
    *reinterpret_cast<uint2*>(codes) = c;
    if ((threadIdx.x & 15) == 0) *scale = static_cast<unsigned char>(byte);
}

struct RowLayout {          // rows in 8 bits
    int64_t code_stride, scale_stride;
    int32_t blocks;         // of one segment
    int32_t spare;          // scale bytes past the last block
};
