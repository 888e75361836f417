// Row kernels without a sum over the row: quantisation, silu(gate) * up and its gradients.
// Part of tn_fp8.hip's translation unit, inside its anonymous namespace, after fp8_format.hpp.
#pragma once

// ---------------------------------------------------------------------------------------------
// Bound by memory: one chunk of 8 elements to a lane, every value read and written once. Lanes count chunks of padded rows
// (whole blocks, so the 16 lanes of a block are in one row and all there); `per_row` of them to a row. (Gradients of 1024 x 2 x 25600 in bf16:
// 39 us, 5.4 TB/s; 59 with expf, divisions and a NaN check for every code. silu(gate) * up of as many to 8 bits 27 us, 4.9 TB/s. Quantisation of
// 8192 x 5120 in bf16 27 us, 4.6 TB/s, of 1001 x 5120 5.6 us: half of that is what a launch of few rows takes, 2.7 to 3.3 us for one.)
// ---------------------------------------------------------------------------------------------
struct RowArgs {
    const void *x, *dh;
    void* y;
    unsigned char *codes, *scales;
    int64_t x_stride, dh_stride, y_stride;
    int64_t items;             // rows of this launch * per_row
    RowLayout out;
    int32_t cols, per_row, segments;
};

enum RowOp : int { ROW_QUANTIZE = 0, ROW_GATE = 1, ROW_GATE_GRAD = 2 };

// the pieces of segment `seg` of a row that its lane writes: values if there is a y, codes if there are codes
template <typename T>
__device__ __forceinline__ void put_chunk(const RowArgs& a, int64_t row, int seg, int at, const float (&v)[kChunk]) {
    const int n = a.cols - at;
    if (a.y && n > 0) store8(static_cast<T*>(a.y) + row * a.y_stride + int64_t(seg) * a.cols + at, n, v);
    if (!a.codes) return;
    const int block = seg * a.out.blocks + at / kBlock;
    unsigned char* scales = a.scales + row * a.out.scale_stride;
    quantise_block(v, a.codes + row * a.out.code_stride + int64_t(seg) * a.out.blocks * kBlock + at, scales + block);
    if (block == 0 && int(threadIdx.x & 15) < a.out.spare) scales[a.segments * a.out.blocks + (threadIdx.x & 15)] = 0;
}

template <typename T, int OP>
__global__ void __launch_bounds__(256) row_kernel(RowArgs a) {
    // first item of the workgroup, in 64 bits once; the rest in 32
    const int64_t first = int64_t(blockIdx.x) * 256;
    const int64_t row0 = first / a.per_row;
    const unsigned rest = unsigned(first - row0 * a.per_row) + threadIdx.x;
    const unsigned over = rest / unsigned(a.per_row);
    const int64_t row = row0 + over;
    const int chunk = int(rest - over * unsigned(a.per_row));
    if (first + threadIdx.x >= a.items) return;       // `items` is a multiple of 16
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    if constexpr (OP == ROW_QUANTIZE) {
        const int per_segment = a.out.blocks * (kBlock / kChunk), seg = chunk / per_segment;
        const int at = (chunk - seg * per_segment) * kChunk;
        float v[kChunk];
        load8(x + int64_t(seg) * a.cols + at, a.cols - at, v);
        put_chunk<T>(a, row, seg, at, v);
    } else {
        const int at = chunk * kChunk, n = a.cols - at;
        float gate[kChunk], up[kChunk];
        load8(x + at, n, gate);
        load8(x + a.cols + at, n, up);
        if constexpr (OP == ROW_GATE) {
            float h[kChunk];
#pragma unroll
            for (int i = 0; i < kChunk; ++i) h[i] = gate[i] * sigmoid(gate[i]) * up[i];
            put_chunk<T>(a, row, 0, at, h);
        } else {
            float dh[kChunk], dg[kChunk], du[kChunk];
            load8(static_cast<const T*>(a.dh) + row * a.dh_stride + at, n, dh);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                const float sig = sigmoid(gate[i]);
                dg[i] = dh[i] * up[i] * sig * (1.f + gate[i] * (1.f - sig));
                du[i] = dh[i] * gate[i] * sig;
            }
            put_chunk<T>(a, row, 0, at, dg);
            put_chunk<T>(a, row, 1, at, du);
        }
    }
}
