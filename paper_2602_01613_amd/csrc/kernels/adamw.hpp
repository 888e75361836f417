// The AdamW step over many tensors, and the norm of their gradients.
// Part of tn_adamw.hip's translation unit, inside its anonymous namespace, after fp8_format.hpp.
#pragma once

// ---------------------------------------------------------------------------------------------
// The tensors are cut into parts of 4096 values, two chunks of 8 for each thread; a table on the device says for each part which tensor it is
// of and which part of it, another what a tensor is. The gradients' addresses change from step to step and come with the launch, for up to 256 tensors
// at a time; more tensors take more launches.
//
// All of it is bound by HBM where tensors are large. 119 M values of 277 tensors: norm 95 us, 475 MB at 5.0 TB/s; step with states in 8 bits, fp32 gradients and bf16
// parameters 425 us, 2.1 GB at 5.0 TB/s (a copy has 5.1). 4.2 M values with states in 32 bits: 26 us, 127 MB at 4.9 TB/s. Below that by its launches: the norm of 0.9 M values 7.5 us in two
// of them.
// ---------------------------------------------------------------------------------------------
constexpr int kPartValues = 4096, kLaunchTensors = 256;

struct TensorEntry {
    void* param;
    int64_t size, place;             // values; where its state starts
    float decay;
    int32_t bf16;
};
struct PartEntry {
    int32_t tensor, part;
};
// what one thread makes for the step: all that is the same for every value
struct StepScalars {
    float clip, lr, step, root_bias2;     // step: lr / (1 - beta1^t); root_bias2: 1 / sqrt(1 - beta2^t)
    unsigned key;
    int32_t skip;
};
struct Gradients {
    const void* p[kLaunchTensors];
    unsigned bf16[kLaunchTensors / 32];
    int32_t tensor0;
    __device__ __forceinline__ const void* at(int t) const { return p[t - tensor0]; }
    __device__ __forceinline__ bool is_bf16(int t) const { return bf16[(t - tensor0) >> 5] >> ((t - tensor0) & 31) & 1; }
};
struct AdamwArgs {
    const TensorEntry* tensors;
    const PartEntry* parts;
    int64_t n_parts;                 // of this launch, from parts on
    void *first, *second;
    unsigned char *first_scales, *second_scales;
    float* master;
    const StepScalars* scalars;
    float beta1, rest1, beta2, rest2, eps;
    float least;                     // states in 8 bits: of |m|, what the root of v has at the least
};

// The part of a value of which a chunk of 8 is loaded as floats, whatever it is stored as
__device__ __forceinline__ void load_values(const void* p, bool bf16, int64_t at, int n, float (&v)[kChunk]) {
    if (bf16) load8(static_cast<const bf16_t*>(p) + at, n, v);
    else load8(static_cast<const float*>(p) + at, n, v);
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ double group_sum64(double v, double* part) {
    v = wave_sum64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < int(blockDim.x >> 6); ++w) v += part[w];
    return v;
}

// Sums of squares, one for each workgroup, in 64 bits: the clipping of all tensors hangs on the one value, and products of fp32 values are exact there. (All
// loads of a part requested together, by a branch for whole parts: a tenth longer, with fewer waves on a CU.)
__global__ void __launch_bounds__(256) gradient_norm_kernel(AdamwArgs a, Gradients g, double* sums) {
    __shared__ double part[4];
    double sum = 0;
    // (the next part's tables are read while this one's values are under way: without that, three loads wait for each other)
    PartEntry e{};
    TensorEntry t{};
    if (blockIdx.x < a.n_parts) {
        e = a.parts[blockIdx.x];
        t = a.tensors[e.tensor];
    }
    for (int64_t c = blockIdx.x; c < a.n_parts; c += gridDim.x) {
        const void* p = g.at(e.tensor);
        const bool bf16 = g.is_bf16(e.tensor);
        const int64_t at0 = int64_t(e.part) * kPartValues + int(threadIdx.x) * kChunk;
        float v[kPartValues / (256 * kChunk)][kChunk];
#pragma unroll
        for (int i = 0; i < kPartValues / (256 * kChunk); ++i) {
            const int64_t at = at0 + i * 256 * kChunk, left = t.size - at;
            load_values(p, bf16, left > 0 ? at : 0, int(left < 0 ? 0 : left < kChunk ? left : kChunk), v[i]);
        }
        if (c + gridDim.x < a.n_parts) {
            e = a.parts[c + gridDim.x];
            t = a.tensors[e.tensor];
        }
#pragma unroll
        for (int i = 0; i < kPartValues / (256 * kChunk); ++i)
#pragma unroll
            for (int q = 0; q < kChunk; ++q) sum += double(v[i][q]) * double(v[i][q]);
    }
    sum = group_sum64(sum, part);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__device__ __forceinline__ unsigned mix(unsigned x) {
    x = (x ^ (x >> 16)) * 0x9E3779B1u;
    x = (x ^ (x >> 15)) * 0xB7E15163u;
    return x ^ (x >> 16);
}

struct PrepareArgs {
    const double* sums;              // not null: the norm is theirs
    int32_t n_sums;
    float* norm;                     // written with sums, else read; null: neither
    StepScalars* scalars;            // null: the norm alone
    int64_t* count;
    double lr, max_norm, beta1, beta2;
    const float* lr_device;
    unsigned seed;
};

// One workgroup: the norm out of the workgroups' sums, then what the step needs once
__global__ void __launch_bounds__(1024) adamw_prepare_kernel(PrepareArgs a) {
    __shared__ double part[16];
    double n = 0;
    if (a.sums) {
        double sum = 0;
        for (int i = threadIdx.x; i < a.n_sums; i += blockDim.x) sum += a.sums[i];
        n = sqrt(group_sum64(sum, part));
    }
    if (threadIdx.x != 0) return;
    if (a.sums) {
        if (a.norm) *a.norm = float(n);
        n = double(float(n));
    } else if (a.norm) {
        n = double(*a.norm);
    }
    if (!a.scalars) return;
    StepScalars s{};
    const bool clip = a.max_norm > 0;
    s.skip = clip && !(n < __builtin_huge_val());            // (a NaN too; a norm is not negative)
    const int64_t t = *a.count + 1;
    if (!s.skip) *a.count = t;
    const double lr = a.lr_device ? *a.lr_device : float(a.lr);          // (in fp32 either way, so that both give the same)
    s.clip = clip && n > a.max_norm ? float(a.max_norm / n) : 1.f;
    s.lr = float(lr);
    s.step = float(lr / (1 - pow(a.beta1, double(t))));
    s.root_bias2 = float(1 / sqrt(1 - pow(a.beta2, double(t))));
    s.key = mix(mix(a.seed) ^ unsigned(t));
    *a.scalars = s;
}

// A code of 8 bits for v, |v| * inv at most 448, with 16 random bits: adding them below the code's last bit carries into it as often as
// the bits that are cut off say. 2^-6 is the least normal code; under it the steps stay those of 2^-6, which adding it gives them.
__device__ __forceinline__ unsigned random_code(float v, float inv, unsigned h16) {
    const unsigned bits = __float_as_uint(v * inv), size = bits & 0x7fffffffu;
    const bool low = size < 0x3c800000u;
    const unsigned moved = low ? __float_as_uint(__uint_as_float(size) + 0.015625f) : size;
    const unsigned code = ((moved + h16 * 16 + 8) >> 20) - (low ? 968u : 960u);
    return code | (bits >> 24 & 0x80u);
}

// The 16 lanes of a block put their 8 values each into 8 bits; all 16 must be here.
__device__ __forceinline__ void store_block(const float (&v)[kChunk], const unsigned (&h)[kChunk], int shift, unsigned char* codes, unsigned char* scale) {
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < kChunk; ++i) most = max(most, finite_magnitude(v[i]));
    const unsigned byte = scale_byte(row16_max(most));
    const float inv = inverse_scale(byte);
    unsigned w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
        const bool finite = (__float_as_uint(v[i]) & 0x7fffffffu) < 0x7f800000u;
        w[i >> 2] |= (finite ? random_code(v[i], inv, h[i] >> shift & 0xffffu) : 0x7fu) << (8 * (i & 3));
    }
    *reinterpret_cast<uint2*>(codes) = make_uint2(w[0], w[1]);
    if ((threadIdx.x & 15) == 0) *scale = static_cast<unsigned char>(byte);
}
__device__ __forceinline__ void load_block(const unsigned char* codes, const unsigned char* scale, float (&v)[kChunk]) {
    const uint2 c = *reinterpret_cast<const uint2*>(codes);
    const unsigned byte = *scale;
    const float s = byte ? __uint_as_float(byte << 23) : 5.877471754111438e-39f;          // 2^-127 is no normal number
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int w = int(h ? c.y : c.x);
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        v[4 * h] = lo[0] * s;
        v[4 * h + 1] = lo[1] * s;
        v[4 * h + 2] = hi[0] * s;
        v[4 * h + 3] = hi[1] * s;
    }
}

// a x + b y, every operation rounded. The point that decides between two codes is on fp32's grid, and a value less than half a unit below it is rounded onto it, so that one in two
// million codes is not the exact one. Which, depends on the arithmetic: of 119 M codes of m 54 to 86 so, as elementary operations have them, 43 to 78 with a fused sum, other ones; of r 65 to
// 86 so, 64 to 89 fused, and 50 to 66 by the difference to v, which has no rounding of beta2 in it (and would make a NaN of an infinite v, which 8 bits do not hold).
__device__ __forceinline__ float weighted(float a, float x, float b, float y) {
#pragma clang fp contract(off)
    const float ax = a * x, by = b * y;
    return ax + by;
}

template <int BITS>
__global__ void __launch_bounds__(256) adamw_step_kernel(AdamwArgs a, Gradients grads) {
    const PartEntry e = a.parts[blockIdx.x];
    const TensorEntry t = a.tensors[e.tensor];
    const StepScalars s = *a.scalars;
    if (s.skip) return;
    const void* gp = grads.at(e.tensor);
    const bool g16 = grads.is_bf16(e.tensor);
    const float decay = s.lr * t.decay;
#pragma unroll
    for (int i = 0; i < kPartValues / (256 * kChunk); ++i) {
        const int64_t at = int64_t(e.part) * kPartValues + (i * 256 + int(threadIdx.x)) * kChunk;
        // (the 16 lanes of a block that has values stay together: past the tensor's end theirs are zeros)
        if ((at & ~int64_t(TN_ADAMW_BLOCK - 1)) >= t.size) continue;
        const int64_t left = t.size - at, place = t.place + at;
        const int n = int(left < 0 ? 0 : left < kChunk ? left : kChunk);
        float g[kChunk], p[kChunk], m[kChunk], v[kChunk];
        load_values(gp, g16, n ? at : 0, n, g);
        if (t.bf16) load8(a.master + place, n, p);
        else load8(static_cast<const float*>(t.param) + (n ? at : 0), n, p);
        if constexpr (BITS == 32) {
            load8(static_cast<const float*>(a.first) + place, kChunk, m);
            load8(static_cast<const float*>(a.second) + place, kChunk, v);
        } else {
            load_block(static_cast<const unsigned char*>(a.first) + place, a.first_scales + place / TN_ADAMW_BLOCK, m);
            load_block(static_cast<const unsigned char*>(a.second) + place, a.second_scales + place / TN_ADAMW_BLOCK, v);
#pragma unroll
            for (int q = 0; q < kChunk; ++q) v[q] *= v[q];
        }
        float root[kChunk];
#pragma unroll
        for (int q = 0; q < kChunk; ++q) {
            const float c = g[q] * s.clip;
            m[q] = BITS == 32 ? fmaf(a.beta1, m[q], a.rest1 * c) : weighted(a.beta1, m[q], a.rest1, c);
            if (BITS == 8 && a.beta2 >= 0.5f) v[q] = fmaf(a.rest2, fmaf(c, c, -v[q]), v[q]);          // (with less of v left, its rounding would be larger than c^2)
            else v[q] = fmaf(a.beta2, v[q], a.rest2 * c * c);
            root[q] = sqrtf(v[q]);
            // A root that was rounded to zero beside an m that was not would move the parameter by m / eps: |m| <= sqrt(v) / least whatever the gradients were
            // (Cauchy and Schwarz over their past), and a smaller root is a rounding. (A comparison: a NaN stays one.)
            float under = root[q];
            if constexpr (BITS == 8) under = under < a.least * fabsf(m[q]) ? a.least * fabsf(m[q]) : under;
            // Decay and move are taken off together. (As a factor 1 - decay the decay would be a multiple of 2^-24 of the parameter: 1.19 times itself at 1e-7, nothing at
            // 1e-8. What is infinite stays so, as by the factor.)
            const float move = s.step * m[q] / fmaf(under, s.root_bias2, a.eps);
            p[q] -= fabsf(p[q]) < __builtin_inff() ? fmaf(decay, p[q], move) : move;
        }
        if (n) {
            if (t.bf16) {
                store8(a.master + place, n, p);
                store8(static_cast<bf16_t*>(t.param) + at, n, p);
            } else {
                store8(static_cast<float*>(t.param) + at, n, p);
            }
        }
        if constexpr (BITS == 32) {
            if (n) {
                store8(static_cast<float*>(a.first) + place, n, m);
                store8(static_cast<float*>(a.second) + place, n, v);
            }
        } else {
            unsigned h[kChunk];
            const unsigned key = mix(s.key ^ unsigned(uint64_t(place) >> 32));
#pragma unroll
            for (int q = 0; q < kChunk; ++q) {
                h[q] = mix((unsigned(place) + q) ^ key);
                if (q >= n) m[q] = root[q] = 0.f;
            }
            store_block(m, h, 0, static_cast<unsigned char*>(a.first) + place, a.first_scales + place / TN_ADAMW_BLOCK);
            store_block(root, h, 16, static_cast<unsigned char*>(a.second) + place, a.second_scales + place / TN_ADAMW_BLOCK);
        }
    }
}

// Masters of parameters in bf16
__global__ void __launch_bounds__(256) adamw_master_kernel(AdamwArgs a) {
    for (int64_t c = blockIdx.x; c < a.n_parts; c += gridDim.x) {
        const PartEntry e = a.parts[c];
        const TensorEntry t = a.tensors[e.tensor];
        if (!t.bf16) continue;
        for (int i = threadIdx.x; i < kPartValues; i += 256) {
            const int64_t at = int64_t(e.part) * kPartValues + i;
            if (at < t.size) a.master[t.place + at] = float(static_cast<const bf16_t*>(t.param)[at]);
        }
    }
}
