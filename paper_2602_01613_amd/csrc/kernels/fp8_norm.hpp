// Root-mean-square norm with the residual's addition and 8-bit output, and its gradients.
// Part of tn_fp8.hip's translation unit, inside its anonymous namespace, after fp8_format.hpp.
#pragma once

// ---------------------------------------------------------------------------------------------
// s = x + residual, y = s * r * weight with r = 1 / sqrt(mean(s^2) + eps). Bound by memory: every value is read once and
// written once, so a row stays in the registers of the waves that read it between the sum of squares and the output. WAVES
// waves share a row, lane l of them owning chunks l, l + 64 * WAVES, ... of 8 elements (NC of them); a single wave needs no
// barrier and its workgroup holds four rows.
// ---------------------------------------------------------------------------------------------
struct NormArgs {
    const void *x, *residual, *weight;
    void *sum, *y;
    unsigned char *codes, *scales;
    int64_t rows, x_stride, residual_stride, sum_stride, y_stride;
    RowLayout out;
    int32_t cols;
    float eps;
};

template <typename T, int WAVES, int NC>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) rms_norm_kernel(NormArgs a) {
    constexpr int THREADS = WAVES * 64;
    const int tid = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t row = WAVES == 1 ? int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (row >= a.rows) return;                       // whole waves, and with WAVES > 1 none
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* res = static_cast<const T*>(a.residual) + (a.residual ? row * a.residual_stride : 0);
    T* sum = static_cast<T*>(a.sum) + (a.sum ? row * a.sum_stride : 0);
    float s[NC][kChunk];
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int at = (c * THREADS + tid) * kChunk, n = a.cols - at;
        load8(x + at, n, s[c]);
        if (a.residual) {
            float v[kChunk];
            load8(res + at, n, v);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) s[c][i] = float(T(s[c][i] + v[i]));
        }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int at = (c * THREADS + tid) * kChunk, n = a.cols - at;
        if (a.sum) store8(sum + at, n, s[c]);
#pragma unroll
        for (int i = 0; i < kChunk; ++i) sq = fmaf(s[c][i], s[c][i], sq);
    }
    sq = wave_sum(sq);
    if constexpr (WAVES > 1) {
        __shared__ float part[WAVES];
        if ((tid & 63) == 0) part[tid >> 6] = sq;
        __syncthreads();
        sq = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sq += part[w];
    }
    if (!a.y && !a.codes) return;
    const float r = 1.f / sqrtf(sq / float(a.cols) + a.eps);
    const T* weight = static_cast<const T*>(a.weight);
    T* y = static_cast<T*>(a.y) + (a.y ? row * a.y_stride : 0);
    unsigned char* codes = a.codes + (a.codes ? row * a.out.code_stride : 0);
    unsigned char* scales = a.scales + (a.codes ? row * a.out.scale_stride : 0);
    const int padded = a.out.blocks * kBlock;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int at = (c * THREADS + tid) * kChunk, n = a.cols - at;
        float v[kChunk];
        if (a.weight) {
            load8(weight + at, n, v);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v[i] = s[c][i] * r * v[i];
        } else {
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v[i] = s[c][i] * r;
        }
        if (a.y) store8(y + at, n, v);
        if (a.codes && at < padded) {                // 16 lanes at a time: `padded` is whole blocks
            if (n < kChunk) {                        // past the row: zeros, whatever r is
#pragma unroll
                for (int i = 0; i < kChunk; ++i) v[i] = i < n ? v[i] : 0.f;
            }
            quantise_block(v, codes + at, scales + at / kBlock);
        }
    }
    if (a.codes && tid < a.out.spare) scales[a.out.blocks + tid] = 0;
}

// ---------------------------------------------------------------------------------------------
// dx = r * (g - u * mean(g * u)) + dsum with u = s * r, g = dy * weight; dweight = sum over rows of dy * u. One pass: a
// workgroup takes every gridDim.x-th row, holds s and dy of a row in registers between its two sums and its output, and adds up
// dweight for the columns its threads own; its partial sums go to the workspace and norm_grad_reduce_kernel adds them.
// ---------------------------------------------------------------------------------------------
struct NormGradArgs {
    const void *dy, *s, *weight, *dsum;
    void* dx;
    float* partial;          // [gridDim.x][cols], or null
    int64_t rows, dy_stride, s_stride, dsum_stride, dx_stride;
    int32_t cols;
    float eps;
};

template <typename T, int WAVES, int NC>
__global__ void __launch_bounds__(WAVES * 64) norm_grad_kernel(NormGradArgs a) {
    constexpr int THREADS = WAVES * 64;
    __shared__ float part[2][2 * WAVES];
    const int tid = threadIdx.x;
    float dw[NC][kChunk];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < kChunk; ++i) dw[c][i] = 0.f;
    int slot = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* ps = static_cast<const T*>(a.s) + row * a.s_stride;
        const T* pd = static_cast<const T*>(a.dy) + row * a.dy_stride;
        float s[NC][kChunk], d[NC][kChunk];
        float sq = 0.f, dot = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = (c * THREADS + tid) * kChunk, n = a.cols - at;
            load8(ps + at, n, s[c]);
            load8(pd + at, n, d[c]);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = (c * THREADS + tid) * kChunk, n = a.cols - at;
            float w[kChunk];
            if (a.weight) load8(static_cast<const T*>(a.weight) + at, n, w);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                sq = fmaf(s[c][i], s[c][i], sq);
                dot = fmaf(a.weight ? d[c][i] * w[i] : d[c][i], s[c][i], dot);
            }
        }
        sq = wave_sum(sq);
        dot = wave_sum(dot);
        if constexpr (WAVES > 1) {                   // one barrier a row: the next row writes the other slots
            if ((tid & 63) == 0) part[slot][tid >> 6] = sq, part[slot][WAVES + (tid >> 6)] = dot;
            __syncthreads();
            sq = dot = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) sq += part[slot][w], dot += part[slot][WAVES + w];
            slot ^= 1;
        }
        const float r = 1.f / sqrtf(sq / float(a.cols) + a.eps);
        const float along = dot * r * (r / float(a.cols));          // mean(g * u) * r
        T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
        const T* ds = static_cast<const T*>(a.dsum) + (a.dsum ? row * a.dsum_stride : 0);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = (c * THREADS + tid) * kChunk, n = a.cols - at;
            float w[kChunk], e[kChunk];
            if (a.weight) load8(static_cast<const T*>(a.weight) + at, n, w);
            if (a.dsum) load8(ds + at, n, e);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                const float u = s[c][i] * r;
                dw[c][i] = fmaf(d[c][i], u, dw[c][i]);
                const float v = r * (a.weight ? d[c][i] * w[i] : d[c][i]) - u * along;
                e[i] = a.dsum ? v + e[i] : v;
            }
            store8(dx + at, n, e);
        }
    }
    if (!a.partial) return;
    float* out = a.partial + int64_t(blockIdx.x) * a.cols;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int at = (c * THREADS + tid) * kChunk;
        store8(out + at, a.cols - at, dw[c]);
    }
}

// Column sums of partial [n][cols]: 64 columns to a workgroup, its 16 waves each take every 16th row.
__global__ void __launch_bounds__(1024) norm_grad_reduce_kernel(const float* partial, int n, int cols, float* dweight) {
    __shared__ float part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
    float v = 0.f;
    if (col < cols)
        for (int p = wave; p < n; p += 16) v += partial[int64_t(p) * cols + col];
    part[wave][lane] = v;
    __syncthreads();
    if (wave == 0 && col < cols) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) t += part[w][lane];
        dweight[col] = t;
    }
}
