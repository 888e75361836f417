// Root-mean-square norm with the residual's addition and 8-bit output, and its gradients.
// Part of tn_fp8.hip's translation unit, inside its anonymous namespace, after fp8_format.hpp.
#pragma once

// ---------------------------------------------------------------------------------------------
// s = x + residual, y = s * r * weight with r = 1 / sqrt(mean(s^2) + eps). Bound by memory: every value is read once and
// written once, so a row stays in the registers of the waves that read it between the sum of squares and the output: thread t
// of a workgroup owns its chunks t, t + blockDim.x, ... of 8 elements (NC of them). Rows of a single wave's chunks need no barrier, and
// a workgroup holds four of them. (8192 rows of 5120, bf16 and residual to bf16 sum, bf16 and 8 bits: 69 us, 5.5 TB/s, more than a
// copy reaches; in fp32 130 us, 5.5; 8192 rows of 5121 in bf16, which are not aligned to a lane's chunks, 94; one row: 3.0 us. Rows of 128, with 16 of
// a wave's lanes at work: 524288 of them to bf16 alone 150 us, 1.8 TB/s.)
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

template <typename T, int NC, bool ONE_WAVE>
__global__ void __launch_bounds__(ONE_WAVE ? 256 : 1024) rms_norm_kernel(NormArgs a) {
    const int threads = ONE_WAVE ? 64 : blockDim.x;
    const int tid = ONE_WAVE ? threadIdx.x & 63 : threadIdx.x;
    const int64_t row = ONE_WAVE ? int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (row >= a.rows) return;                       // whole waves, and none of a workgroup that shares a row
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* res = static_cast<const T*>(a.residual) + (a.residual ? row * a.residual_stride : 0);
    T* sum = static_cast<T*>(a.sum) + (a.sum ? row * a.sum_stride : 0);
    const T* weight = static_cast<const T*>(a.weight);
    const bool scaled = a.y || a.codes;
    Chunk<T> cx[NC], cr[NC], cw[NC];                 // all of a row's loads before the first use
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int at = (c * threads + tid) * kChunk, n = a.cols - at;
        cx[c] = load_chunk(x + at, n);
        if (a.residual) cr[c] = load_chunk(res + at, n);
        if (scaled && weight) cw[c] = load_chunk(weight + at, n);
    }
    float s[NC][kChunk];
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) {
            s[c][i] = cx[c][i];
            if (a.residual) s[c][i] = float(T(s[c][i] + cr[c][i]));
            sq = fmaf(s[c][i], s[c][i], sq);
        }
    }
    sq = wave_sum(sq);
    if constexpr (!ONE_WAVE) {
        __shared__ float part[16];
        if ((tid & 63) == 0) part[tid >> 6] = sq;
        __syncthreads();
        sq = parts_sum(part, threads >> 6);
    }
    if (a.sum) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = (c * threads + tid) * kChunk;
            store8(sum + at, a.cols - at, s[c]);
        }
    }
    if (!scaled) return;
    const float r = 1.f / sqrtf(sq / float(a.cols) + a.eps);
    T* y = static_cast<T*>(a.y) + (a.y ? row * a.y_stride : 0);
    unsigned char* codes = a.codes + (a.codes ? row * a.out.code_stride : 0);
    unsigned char* scales = a.scales + (a.codes ? row * a.out.scale_stride : 0);
    const int padded = a.out.blocks * kBlock;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int at = (c * threads + tid) * kChunk, n = a.cols - at;
        float v[kChunk];
#pragma unroll
        for (int i = 0; i < kChunk; ++i) v[i] = weight ? s[c][i] * r * cw[c][i] : s[c][i] * r;
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
// dweight for the columns its threads own; its partial sums go to the workspace and norm_grad_reduce_kernel adds them. (8192 rows of 5120 in bf16:
// 64 us, 5.2 TB/s; 4096 rows in fp32 67 with the sums of dweight, 5.0; 1024 rows in bf16 11.0 us, 256 workgroups with four rows each, one after another;
// 524288 rows of 128 228 us, 1.8 TB/s: 16 of a wave's lanes, and a barrier for each row.)
//
// WHOLE: rows of whole chunks. Their loads have no branches (threads past a row read its last chunk, and what they read counts as zeros; past the
// last row, that one once more), so that the compiler can wait for a row's loads and leave the next row's under way. With branches it waits
// for all of them (8192 rows: 84 us), and other widths are read so, a row at a time (8192 rows of 5121: 107 us with the sums of dweight, of 5120: 67).
// ---------------------------------------------------------------------------------------------
struct NormGradArgs {
    const void *dy, *s, *weight, *dsum;
    void* dx;
    float* partial;          // [gridDim.x][cols], or null
    int64_t rows, dy_stride, s_stride, dsum_stride, dx_stride;
    int32_t cols;
    float eps;
};

template <typename T, int NC, bool WHOLE, bool DSUM>
__global__ void __launch_bounds__(1024) norm_grad_kernel(NormGradArgs a) {
    __shared__ float part[2][2][16];
    const int threads = blockDim.x, tid = threadIdx.x, waves = threads >> 6;
    const T* weight = static_cast<const T*>(a.weight);
    float dw[NC][kChunk];
    Chunk<T> w[NC];
    struct Row {
        Chunk<T> s[NC], d[NC], e[NC];
    };
    auto load = [&](const void* p, int64_t at_row, int c) {
        const int at = (c * threads + tid) * kChunk;
        const T* row = static_cast<const T*>(p) + at_row;
        return WHOLE ? load_chunk(row + min(at, a.cols - kChunk), kChunk) : load_chunk(row + at, a.cols - at);
    };
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if (weight) w[c] = load(weight, 0, c);
#pragma unroll
        for (int i = 0; i < kChunk; ++i) dw[c][i] = 0.f;
    }
    auto load_row = [&](int row, Row& to) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            to.s[c] = load(a.s, int64_t(row) * a.s_stride, c);
            to.d[c] = load(a.dy, int64_t(row) * a.dy_stride, c);
            if (DSUM) to.e[c] = load(a.dsum, int64_t(row) * a.dsum_stride, c);
        }
    };
    auto store = [](auto* p, int n, const float (&v)[kChunk]) {
        if constexpr (WHOLE) {
            if (n > 0) store8(p, kChunk, v);
        } else {
            store8(p, n, v);
        }
    };
    // (dx may be an input: a row is read whole before it is stored, and only by the workgroup that stores it)
    auto one_row = [&](int row, const Row& now, int slot) {
        float sq = 0.f, dot = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            float q = 0.f, g = 0.f;
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                q = fmaf(now.s[c][i], now.s[c][i], q);
                g = fmaf(weight ? now.d[c][i] * w[c][i] : now.d[c][i], now.s[c][i], g);
            }
            const bool in = !WHOLE || (c * threads + tid) * kChunk < a.cols;
            sq += in ? q : 0.f;
            dot += in ? g : 0.f;
        }
        sq = wave_sum(sq);
        dot = wave_sum(dot);
        if ((tid & 63) == 0) part[slot][0][tid >> 6] = sq, part[slot][1][tid >> 6] = dot;
        __syncthreads();                             // one barrier a row: the next row writes the other slots
        sq = parts_sum(part[slot][0], waves);
        dot = parts_sum(part[slot][1], waves);
        const float r = 1.f / sqrtf(sq / float(a.cols) + a.eps);
        const float along = dot * r * (r / float(a.cols));          // mean(g * u) * r
        T* dx = static_cast<T*>(a.dx) + int64_t(row) * a.dx_stride;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = (c * threads + tid) * kChunk;
            float v[kChunk];
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                const float u = now.s[c][i] * r;
                dw[c][i] = fmaf(now.d[c][i], u, dw[c][i]);           // (past the row: not stored)
                v[i] = r * (weight ? now.d[c][i] * w[c][i] : now.d[c][i]) - u * along;
                if (DSUM) v[i] += now.e[c][i];
            }
            store(dx + at, a.cols - at, v);
        }
    };
    const int rows = int(a.rows), step = gridDim.x;  // (at most 2^30 rows)
    if constexpr (NC == 1 && WHOLE) {                // the next row is under way while this one is summed up
        Row r0, r1;
        load_row(blockIdx.x, r0);                    // the grid has no more workgroups than there are rows
        for (int row = blockIdx.x; row < rows; row += 2 * step) {
            load_row(min(row + step, rows - 1), r1);
            one_row(row, r0, 0);
            if (row + step >= rows) break;
            load_row(min(row + 2 * step, rows - 1), r0);
            one_row(row + step, r1, 1);
        }
    } else {
        int slot = 0;
        for (int row = blockIdx.x; row < rows; row += step, slot ^= 1) {
            Row r0;
            load_row(row, r0);
            one_row(row, r0, slot);
        }
    }
    if (!a.partial) return;
    float* out = a.partial + int64_t(blockIdx.x) * a.cols;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int at = (c * threads + tid) * kChunk;
        store(out + at, a.cols - at, dw[c]);
    }
}

// Column sums of partial [n][cols]: 32 columns to a workgroup, its 32 half waves each take every 32nd row.
__global__ void __launch_bounds__(1024) norm_grad_reduce_kernel(const float* partial, int n, int cols, float* dweight) {
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float v = 0.f;
    if (col < cols) {
        int p = group;
        for (; p + 96 < n; p += 128) {               // four loads in flight
            float q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = partial[int64_t(p + 32 * i) * cols + col];
#pragma unroll
            for (int i = 0; i < 4; ++i) v += q[i];
        }
        for (; p < n; p += 32) v += partial[int64_t(p) * cols + col];
    }
    part[group][lane] = v;
    __syncthreads();
    v = row16_sum(part[lane][group]);                // the other way round: a half wave adds up one column
    v += __shfl_xor(v, 16);
    if (lane == 0 && blockIdx.x * 32 + group < cols) dweight[blockIdx.x * 32 + group] = v;
}
