// The operators around 8-bit projections (include/tn_fp8.h): host side and C ABI. Kernels: kernels/fp8_*.hpp.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <new>
#include <utility>

#include "../../include/tn_fp8.h"

namespace {

#include "kernels/fp8_format.hpp"
#include "kernels/fp8_norm.hpp"
#include "kernels/fp8_rows.hpp"
#include "kernels/fp8_weight.hpp"
#include "kernels/fp8_stream.hpp"
#include "kernels/fp8_gemm.hpp"

constexpr int64_t kMaxRows = int64_t(1) << 30;
constexpr int64_t kMaxCols = int64_t(1) << 24;
constexpr int64_t kOwnWorkspace = int64_t(64) << 20, kMostRanges = 16;

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void* p, unsigned n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int launched() { return hipGetLastError() == hipSuccess ? TN_OK : TN_ERR_HIP; }
int64_t element_bytes(int32_t dtype) { return dtype == TN_DTYPE_F32 ? 4 : 2; }

RowLayout row_layout(int64_t cols, int32_t segments) {
    RowLayout l;
    l.blocks = int32_t(div_up(cols, kBlock));
    l.code_stride = int64_t(segments) * l.blocks * kBlock;
    l.scale_stride = div_up(int64_t(segments) * l.blocks, 4) * 4;
    l.spare = int32_t(l.scale_stride - int64_t(segments) * l.blocks);
    return l;
}

// A launch has fewer than 2^32 threads: kernels that give every row threads of their own take longer inputs in runs of rows, of up to
// this many threads each.
constexpr int64_t kLaunchThreads = int64_t(1) << 31;
template <typename P>
void advance(P*& p, int64_t bytes) {
    if (p) p = reinterpret_cast<P*>(reinterpret_cast<uintptr_t>(p) + uintptr_t(bytes));
}

bool sizes_fit(int64_t rows, int64_t cols) { return rows <= kMaxRows && cols <= kMaxCols; }
// a matrix the caller gives: there, its rows apart, its elements aligned
bool matrix_ok(const void* p, int64_t stride, int64_t cols, int32_t dtype) { return p && stride >= cols && aligned(p, unsigned(element_bytes(dtype))); }
bool eight_bit_ok(const void* codes, const void* scales) {
    return (!codes && !scales) || (codes && scales && aligned(codes, 16) && aligned(scales, 4));
}
// no byte of [p, p + n) in [q, q + m)
bool apart(const void* p, int64_t n, const void* q, int64_t m) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return a + uintptr_t(n) <= b || b + uintptr_t(m) <= a;
}
bool float_type(int32_t dtype) { return dtype == TN_DTYPE_F32 || dtype == TN_DTYPE_BF16; }

// ---------------------------------------------------------------------------------------------
// norm
// ---------------------------------------------------------------------------------------------
// Threads of a workgroup that shares a row of `chunks` chunks, NC to a thread
unsigned row_threads(int64_t chunks, int nc) { return unsigned(div_up(chunks, 64 * nc) * 64); }

template <typename T, int NC>
int run_norm(const NormArgs& a, int64_t chunks, hipStream_t stream) {
    rms_norm_kernel<T, NC, false><<<dim3(unsigned(a.rows)), dim3(row_threads(chunks, NC)), 0, stream>>>(a);
    return launched();
}
template <typename T>
int norm_rows(const NormArgs& a, int64_t chunks, hipStream_t stream) {
    if (chunks <= 64) {
        rms_norm_kernel<T, 1, true><<<dim3(unsigned(div_up(a.rows, 4))), dim3(256), 0, stream>>>(a);
        return launched();
    }
    // one chunk to a thread as far as a workgroup goes: more waves with their loads under way (8192 rows of 5120: 72 us with 10 waves, 93
    // with 5 of two chunks each)
    return chunks <= 1024 ? run_norm<T, 1>(a, chunks, stream) : run_norm<T, 2>(a, chunks, stream);
}
template <typename T>
int dispatch_norm(NormArgs a, int64_t chunks, hipStream_t stream) {
    constexpr int64_t run = kLaunchThreads / 1024;
    int rc = TN_OK;
    for (int64_t left = a.rows; left > 0 && rc == TN_OK; left -= run) {
        a.rows = left < run ? left : run;
        rc = norm_rows<T>(a, chunks, stream);
        advance(a.x, run * a.x_stride * int64_t(sizeof(T)));
        advance(a.residual, run * a.residual_stride * int64_t(sizeof(T)));
        advance(a.sum, run * a.sum_stride * int64_t(sizeof(T)));
        advance(a.y, run * a.y_stride * int64_t(sizeof(T)));
        advance(a.codes, run * a.out.code_stride);
        advance(a.scales, run * a.out.scale_stride);
    }
    return rc;
}

// Workgroups of the gradient's one pass: about ten waves to a CU, and no more, since each adds a row of partial sums. (us with this many, and
// with twice as many: 8192 rows of 5120 63 + 5 / 66 + 5, 1024 rows 12 + 4 / 14 + 4, 4096 rows of 1024 10 + 5 / 11 + 9.)
int64_t norm_grad_groups(int64_t rows, int64_t cols) {
    const int64_t waves = div_up(div_up(cols, kChunk), 64), groups = 256 * (waves < 10 ? 10 / waves : 1);
    return rows < groups ? rows : groups;
}

template <typename T, int NC>
int run_norm_grad(const NormGradArgs& a, int64_t chunks, int64_t groups, hipStream_t stream) {
    const dim3 grid{unsigned(groups)}, block{row_threads(chunks, NC)};
    const bool whole = a.cols % kChunk == 0;
    if (whole && a.dsum) norm_grad_kernel<T, NC, true, true><<<grid, block, 0, stream>>>(a);
    else if (whole) norm_grad_kernel<T, NC, true, false><<<grid, block, 0, stream>>>(a);
    else if (a.dsum) norm_grad_kernel<T, NC, false, true><<<grid, block, 0, stream>>>(a);
    else norm_grad_kernel<T, NC, false, false><<<grid, block, 0, stream>>>(a);
    return launched();
}
template <typename T>
int dispatch_norm_grad(const NormGradArgs& a, int64_t chunks, int64_t groups, hipStream_t stream) {
    return chunks <= 1024 ? run_norm_grad<T, 1>(a, chunks, groups, stream) : run_norm_grad<T, 2>(a, chunks, groups, stream);
}

template <int OP>
int run_rows(int32_t dtype, int64_t rows, RowArgs a, hipStream_t stream) {
    const int64_t run = kLaunchThreads / a.per_row, size = element_bytes(dtype);      // (per_row is 2^29 at the most)
    int rc = TN_OK;
    for (int64_t left = rows; left > 0 && rc == TN_OK; left -= run) {
        a.items = (left < run ? left : run) * a.per_row;
        const dim3 grid(unsigned(div_up(a.items, 256)));
        if (dtype == TN_DTYPE_F32) row_kernel<float, OP><<<grid, dim3(256), 0, stream>>>(a);
        else row_kernel<bf16_t, OP><<<grid, dim3(256), 0, stream>>>(a);
        rc = launched();
        advance(a.x, run * a.x_stride * size);
        advance(a.dh, run * a.dh_stride * size);
        advance(a.y, run * a.y_stride * size);
        advance(a.codes, run * a.out.code_stride);
        advance(a.scales, run * a.out.scale_stride);
    }
    return rc;
}

}  // namespace

struct tn_fp8_linear_s {
    int32_t tensors = 1, transpose = 0;
    int64_t m = 0, n = 0;                 // of each tensor
    int32_t features = 0, f_blocks = 0;   // outputs of one of `out_segments` runs of features
    int32_t out_segments = 1;
    int32_t k_cols = 0, k_segments = 1;   // inputs: segments of k_cols
    int32_t k_blocks = 0, scale_stride = 0;
    unsigned char *packed = nullptr, *scales = nullptr;
    int64_t packed_bytes = 0, scale_bytes = 0;
    void* workspace = nullptr;            // partial sums
    int64_t workspace_bytes = 0;
    bool own_workspace = false;
    ~tn_fp8_linear_s() {
        if (own_workspace && workspace) (void)hipFree(workspace);
        if (packed) (void)hipFree(packed);
        if (scales) (void)hipFree(scales);
    }
};

namespace {

// What a description says by itself, tensors apart
int check_desc(const tn_fp8_linear_desc& d) {
    if (d.out_features < 1 || d.in_features < 1 || d.max_tokens < 1 || d.n_tensors < 1 || d.n_tensors > 2 || (d.flags & ~TN_FLAG_TRANSPOSE))
        return TN_ERR_INVALID_ARG;
    if (d.dtype != TN_DTYPE_FP8 && !float_type(d.dtype)) return TN_ERR_INVALID_ARG;
    if (d.workspace ? d.workspace_bytes < 1 || !aligned(d.workspace, 256) : d.workspace_bytes != 0) return TN_ERR_INVALID_ARG;
    return d.out_features > TN_FP8_MAX_FEATURES || d.in_features > TN_FP8_MAX_FEATURES || d.max_tokens > kMaxRows ? TN_ERR_UNSUPPORTED : TN_OK;
}

// sizes of the operand and of the workspace
void lay_out(const tn_fp8_linear_desc& d, tn_fp8_linear_s& h) {
    h.tensors = d.n_tensors;
    h.transpose = (d.flags & TN_FLAG_TRANSPOSE) ? 1 : 0;
    h.m = d.out_features;
    h.n = d.in_features;
    h.features = int32_t(h.transpose ? h.n : h.m);
    h.f_blocks = int32_t(div_up(h.features, kBlock));
    h.out_segments = h.transpose ? 1 : h.tensors;
    h.k_cols = int32_t(h.transpose ? h.m : h.n);
    h.k_segments = h.transpose ? h.tensors : 1;
    h.k_blocks = int32_t(h.k_segments * div_up(h.k_cols, kBlock));
    h.scale_stride = int32_t(div_up(h.k_blocks, 4) * 4);
    h.packed_bytes = int64_t(h.out_segments) * h.f_blocks * 8 * h.k_blocks * 2048;
    h.scale_bytes = int64_t(h.out_segments) * h.f_blocks * h.scale_stride;
    // the most ranges of K there are, at max_tokens: more than the products ask for, and no more than 64 MB
    const int64_t want = div_up(kMostRanges * d.max_tokens * h.out_segments * h.f_blocks * kBlock * 4, 256) * 256;
    h.workspace_bytes = d.workspace ? d.workspace_bytes : want < kOwnWorkspace ? want : kOwnWorkspace;
}

WeightArgs weight_args(const tn_fp8_linear_s& h, int slot) {
    WeightArgs a{};
    a.packed = h.packed;
    a.scales = h.scales;
    a.m = h.m;
    a.n = h.n;
    a.transpose = h.transpose;
    a.k_blocks = h.k_blocks;
    a.scale_stride = h.scale_stride;
    const int m_blocks = int(div_up(h.m, kBlock));
    a.f_block0 = h.transpose ? 0 : slot * m_blocks;
    a.k_block0 = h.transpose ? slot * m_blocks : 0;
    return a;
}

LinearArgs linear_args(const tn_fp8_linear_s& h, const void* codes, const void* scales, int64_t tokens) {
    LinearArgs a{};
    const RowLayout in = row_layout(h.k_cols, h.k_segments);
    a.codes = static_cast<const unsigned char*>(codes);
    a.scales = static_cast<const unsigned char*>(scales);
    a.packed = h.packed;
    a.w_scales = h.scales;
    a.tokens = tokens;
    a.code_stride = in.code_stride;
    a.scale_stride = in.scale_stride;
    a.k_blocks = h.k_blocks;
    a.w_scale_stride = h.scale_stride;
    a.features = h.features;
    a.f_pieces = h.f_blocks * 8;
    a.tensors = h.out_segments;
    a.n_split = 1;
    a.ld = int64_t(a.f_pieces) * 16 * a.tensors;
    return a;
}

// ---------------------------------------------------------------------------------------------
// which kernel a product runs on
// ---------------------------------------------------------------------------------------------
// Times in us, fitted to measurements on the MI355X (256 CUs) of products of 5120 to 25600 inputs and 1024 to 25600 outputs,
// 1 to 8192 tokens. Of 120 sizes tried (1 to 4096 tokens, outputs and inputs of 700 to 25600) the form chosen by them is within 2 % of the
// best at 86 and over 10 % longer at 14; 9 of these are 700 to 6000 outputs of up to 5120 inputs at 64 to 257 tokens, streamed with one or two runs
// of features to a workgroup where more, or tiles, would be better (1.47 times at the worst: 150 tokens 5120 -> 1024, 11.4 us for 7.8). Gated: over
// 10 % at 1 of 55.
struct TileCost {
    int tm, tn;
    double k_tile, rest;      // a workgroup's time for a K tile, and for a tile's beginning and end (with two on a CU: both of them)
};
// TN = 8 first: the gated form has only those
constexpr TileCost kTiles[] = {{2, 8, 0.50, 2.0}, {3, 8, 0.57, 5.0}, {4, 8, 0.72, 7.1}, {5, 8, 0.85, 7.5}, {6, 8, 0.97, 8.0}, {7, 8, 1.10, 8.8}, {8, 8, 1.24, 8.7},
                               {2, 4, 0.57, 3.1}, {3, 4, 0.69, 3.7}, {4, 4, 0.80, 4.7}, {6, 4, 0.57, 5.0}, {8, 4, 0.71, 6.7}};
constexpr int kTileCount = int(sizeof(kTiles) / sizeof(kTiles[0])), kGatedTiles = 7;
constexpr int kSplits[] = {1, 2, 3, 4, 6, 8, 10, 16};
constexpr int kCUs = 256;
// Rows of tiles to a band, at the most. (Gated 777 tokens on 5 rows: 179 us in one band, 185 in bands of 4 and 1, where the weight is read twice; 8192 x 5120 x
// 25600 on 32 rows: 764 us in bands of 5, 775 in bands of 4 or 8.)
constexpr int kBand = 5;
constexpr double kLaunch = 4.0, kReadRate = 5.3e6, kSumsRate = 8e6;      // bytes per us: memory, partial sums
constexpr double kTilesRate = 25e6, kStreamRate = 14e6, kStreamFarRate = 8e6;       // what is read again, from the caches
// Memory and computation overlap, but not wholly: of the shorter one this much is added.
double together(double a, double b) { return a > b ? a + 0.35 * b : b + 0.35 * a; }

struct Choice {
    int tile = -1;             // index into kTiles; -1: the stream kernel
    int split = 1, groups = 1;
    bool fused = false;        // gated: silu(gate) * up by the tile's own workgroup
    double us = 1e30;
};

constexpr int tiles_per_cu(const TileCost& t) {          // as GemmShape has it
    const int stage = 32 * (t.tm + t.tn) * kBlock, scales = ((32 * t.tm + 63) / 64 * 64 + 64) * 4;
    return 2 * (2 * stage + 2 * scales) <= 160 * 1024 ? 2 : 1;
}

Choice choose(const LinearArgs& a, bool gated, int64_t workspace_bytes) {
    const int64_t pieces = int64_t(a.f_pieces) * a.tensors, weight = pieces * a.k_blocks * 2048;
    const double outputs = double(a.tokens) * a.ld * 4;       // of one range's partial sums
    const auto sums = [&](int ranges) { return 3.0 + 2 * ranges * outputs / kSumsRate; };
    Choice best;
    // streamed, 16 tokens at a time: the weight comes from memory once, for every further 16 tokens from the caches, and each workgroup
    // reads its tokens. Pieces to a workgroup: one where there are few; two where one each would leave some CUs two workgroups and
    // others one (320 pieces of 25600 k, one token: 25.4 us with two to a workgroup, 30 with one); with more than four tokens, which a
    // workgroup reads once for all of its pieces, two up to 1023 pieces and four from 1024 on, where that leaves a workgroup or more to each CU (1600
    // pieces of 5120 k, 16 tokens: 28 us with four, 33 with one).
    if (a.tokens <= 16 * 65535 && (!gated || outputs <= double(workspace_bytes))) {
        Choice c;
        c.groups = pieces <= kCUs ? 1 : pieces < 2 * kCUs ? 2 : a.tokens <= 4 ? 1 : pieces < 4 * kCUs ? 2 : 4;
        const double passes = double(div_up(a.tokens, 16));
        const double cached = (passes * weight + double(pieces) / c.groups * a.tokens * a.k_blocks * kBlock) / (weight < (16 << 20) ? kStreamRate : kStreamFarRate);
        const double memory = weight / kReadRate;
        c.us = kLaunch + together(memory, cached) + (gated ? sums(1) : 0);
        best = c;
    }
    for (int t = 0; t < kTileCount; ++t) {
        const TileCost& cost = kTiles[t];
        const int per_cu = tiles_per_cu(cost);
        const int64_t n_row = div_up(a.tokens, 32 * cost.tm), n_col = div_up(pieces, 2 * cost.tn);
        for (const int split : kSplits) {
            const bool fused = gated && split == 1 && t < kGatedTiles;
            const int64_t items = n_row * (fused ? a.f_pieces / 8 : n_col) * split;
            if (split > 1 && (split * 4 > a.k_blocks || items > 4 * kCUs)) break;
            if ((split > 1 || (gated && !fused)) && split * outputs > double(workspace_bytes)) break;
            const int64_t nk = div_up(div_up(a.k_blocks, split), 4) * 4, rounds = div_up(items, int64_t(kCUs) * per_cu);
            // two workgroups share a CU only where there are enough of them
            const double alone = per_cu == 2 && items <= kCUs ? 0.6 : 1.0;
            const double compute = rounds * alone * (double(nk < a.k_blocks ? nk : a.k_blocks) * cost.k_tile + cost.rest);
            // the weight comes from memory for the first row of tiles; what is read again (and the tokens) from the caches
            const double memory = weight / kReadRate + double(n_row - 1) * weight / kTilesRate + (split > 1 ? 0 : outputs / 2) / kSumsRate;
            const double us = kLaunch + together(compute, memory) + (split > 1 || (gated && !fused) ? sums(split) : 0);
            if (us < best.us) {
                best.us = us;
                best.tile = t;
                best.split = split;
                best.fused = fused;
            }
        }
    }
    return best;
}

// Waves of a workgroup of the stream kernel, at most 16: the number that leaves the fewest of them without a word of scales (four blocks
// of k) in the last round, and the larger of such numbers.
int stream_waves(int k_blocks) {
    const int words = int(div_up(k_blocks, 4));
    int best = words < 16 ? words : 16;
    for (int w = best - 1; w >= 8; --w)
        if (div_up(words, w) * w < div_up(words, best) * best) best = w;
    return best;
}
template <int GROUPS>
int run_stream(const LinearArgs& a, hipStream_t stream) {
    const dim3 grid(unsigned(a.f_pieces * a.tensors / GROUPS), unsigned(div_up(a.tokens, 16)));
    stream_kernel<GROUPS><<<grid, dim3(64 * stream_waves(a.k_blocks)), 0, stream>>>(a);
    return launched();
}

template <int TM, int TN, int FORM>
int run_gemm(const LinearArgs& a, hipStream_t stream) {
    using S = GemmShape<TM, TN>;
    GemmArgs g{};
    g.l = a;
    g.ktiles_per_split = int(div_up(div_up(a.k_blocks, a.n_split), 4) * 4);
    g.l.n_split = int(div_up(a.k_blocks, g.ktiles_per_split));        // no range without a tile
    const int64_t n_row = div_up(a.tokens, S::BM), n_col = FORM == GEMM_GATED ? a.f_pieces / 8 : div_up(int64_t(a.f_pieces) * a.tensors, 2 * TN);
    const int64_t items = n_row * n_col * g.l.n_split;
    if (items > INT32_MAX / 8) return TN_ERR_UNSUPPORTED;
    g.n_row = int(n_row);
    g.n_col = int(n_col);
    g.band = int(div_up(n_row, div_up(n_row, kBand)));
    const int64_t held = kCUs * S::PER_CU, groups = div_up(items, 8) * 8;
    gemm_kernel<TM, TN, FORM><<<dim3(unsigned(groups < held ? groups : held)), dim3(256), S::SMEM, stream>>>(g);
    return launched();
}
template <int TM, int TN, int FORM>
bool allow_gemm() {          // more LDS than a launch gets by default
    return hipFuncSetAttribute(reinterpret_cast<const void*>(gemm_kernel<TM, TN, FORM>), hipFuncAttributeMaxDynamicSharedMemorySize,
                               GemmShape<TM, TN>::SMEM) == hipSuccess;
}
template <int FORM, int... T>
bool allow_gemms(std::integer_sequence<int, T...>) {
    return (allow_gemm<kTiles[T].tm, kTiles[T].tn, FORM>() && ...);
}
template <int FORM, int... T>
int run_tile(const LinearArgs& a, int tile, hipStream_t stream, std::integer_sequence<int, T...>) {
    int rc = TN_ERR_UNSUPPORTED;
    (void)((T == tile ? (rc = run_gemm<kTiles[T].tm, kTiles[T].tn, FORM>(a, stream), true) : false) || ...);
    return rc;
}

int run_product(const tn_fp8_linear_s& h, LinearArgs a, bool gated, hipStream_t stream) {
    const Choice c = choose(a, gated, h.workspace_bytes);
    const bool in_parts = c.split > 1 || (gated && !c.fused);
    if (in_parts) a.partial = static_cast<float*>(h.workspace);
    a.n_split = c.split;
    int rc;
    if (c.tile < 0) {
        rc = c.groups == 1 ? run_stream<1>(a, stream) : c.groups == 2 ? run_stream<2>(a, stream) : run_stream<4>(a, stream);
    } else if (c.fused) {
        rc = run_tile<GEMM_GATED>(a, c.tile, stream, std::make_integer_sequence<int, kGatedTiles>());
    } else {
        rc = in_parts ? run_tile<GEMM_PARTIAL>(a, c.tile, stream, std::make_integer_sequence<int, kTileCount>())
                      : run_tile<GEMM_PLAIN>(a, c.tile, stream, std::make_integer_sequence<int, kTileCount>());
    }
    if (rc != TN_OK || !in_parts) return rc;
    const int64_t ktiles = div_up(div_up(a.k_blocks, a.n_split), 4) * 4;
    a.n_split = int(div_up(a.k_blocks, ktiles));              // as the tiles took it
    const int64_t groups = div_up(a.tokens * a.ld / (gated ? 2 * kChunk : 4), 256);
    const dim3 grid(unsigned(groups < 8 * kCUs ? groups : 8 * kCUs));
    if (gated) gemm_reduce_gated_kernel<<<grid, dim3(256), 0, stream>>>(a);
    else gemm_reduce_kernel<<<grid, dim3(256), 0, stream>>>(a);
    return launched();
}

}  // namespace

extern "C" {

int tn_fp8_row_strides(int64_t cols, int32_t segments, int64_t* code_stride, int64_t* scale_stride) {
    if (cols < 1 || segments < 1) return TN_ERR_INVALID_ARG;
    if (cols > kMaxCols || segments > 256) return TN_ERR_UNSUPPORTED;
    const RowLayout l = row_layout(cols, segments);
    if (code_stride) *code_stride = l.code_stride;
    if (scale_stride) *scale_stride = l.scale_stride;
    return TN_OK;
}

int tn_fp8_quantize(int32_t dtype, int64_t rows, int64_t cols, int32_t segments, const void* x, int64_t x_stride,
                    void* codes, void* scales, void* stream) {
    if (!float_type(dtype) || rows < 0 || cols < 1 || segments < 1) return TN_ERR_INVALID_ARG;
    if (!sizes_fit(rows, cols) || segments > 256) return TN_ERR_UNSUPPORTED;
    if (rows == 0) return TN_OK;
    if (!matrix_ok(x, x_stride, cols * segments, dtype) || !codes || !eight_bit_ok(codes, scales)) return TN_ERR_INVALID_ARG;
    RowArgs a{};
    a.x = x;
    a.x_stride = x_stride;
    a.codes = static_cast<unsigned char*>(codes);
    a.scales = static_cast<unsigned char*>(scales);
    a.out = row_layout(cols, segments);
    a.cols = int32_t(cols);
    a.segments = segments;
    a.per_row = int32_t(a.out.code_stride / kChunk);
    return run_rows<ROW_QUANTIZE>(dtype, rows, a, static_cast<hipStream_t>(stream));
}

int tn_rms_norm(int32_t dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride, const void* residual,
                int64_t residual_stride, const void* weight, float eps, void* sum, int64_t sum_stride, void* y,
                int64_t y_stride, void* codes, void* scales, void* stream) {
    if (!float_type(dtype) || rows < 0 || cols < 1 || !(eps >= 0.f)) return TN_ERR_INVALID_ARG;
    if (rows > kMaxRows || cols > TN_FP8_MAX_NORM_COLS) return TN_ERR_UNSUPPORTED;
    if (rows == 0) return TN_OK;
    if (!sum && !y && !codes) return TN_ERR_INVALID_ARG;
    if (!matrix_ok(x, x_stride, cols, dtype) || (residual && !matrix_ok(residual, residual_stride, cols, dtype)) ||
        (sum && !matrix_ok(sum, sum_stride, cols, dtype)) || (y && !matrix_ok(y, y_stride, cols, dtype)) ||
        !aligned(weight, unsigned(element_bytes(dtype))) || !eight_bit_ok(codes, scales) || (sum && sum == y))
        return TN_ERR_INVALID_ARG;
    NormArgs a{};
    a.x = x;
    a.residual = residual;
    a.weight = weight;
    a.sum = sum;
    a.y = y;
    a.codes = static_cast<unsigned char*>(codes);
    a.scales = static_cast<unsigned char*>(scales);
    a.rows = rows;
    a.x_stride = x_stride;
    a.residual_stride = residual_stride;
    a.sum_stride = sum_stride;
    a.y_stride = y_stride;
    a.out = row_layout(cols, 1);
    a.cols = int32_t(cols);
    a.eps = eps;
    const int64_t chunks = codes ? a.out.code_stride / kChunk : div_up(cols, kChunk);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == TN_DTYPE_F32 ? dispatch_norm<float>(a, chunks, st) : dispatch_norm<bf16_t>(a, chunks, st);
}

int64_t tn_rms_norm_gradients_workspace(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1) return TN_ERR_INVALID_ARG;
    if (rows > kMaxRows || cols > TN_FP8_MAX_NORM_COLS) return TN_ERR_UNSUPPORTED;
    return norm_grad_groups(rows, cols) * cols * 4;
}

int tn_rms_norm_gradients(int32_t dtype, int64_t rows, int64_t cols, const void* dy, int64_t dy_stride, const void* s,
                          int64_t s_stride, const void* weight, float eps, const void* dsum, int64_t dsum_stride, void* dx,
                          int64_t dx_stride, float* dweight, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!float_type(dtype) || rows < 0 || cols < 1 || !(eps >= 0.f)) return TN_ERR_INVALID_ARG;
    const int64_t need = tn_rms_norm_gradients_workspace(rows, cols);
    if (need < 0) return int(need);
    if (!aligned(dweight, 4) || (dweight && need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16)))) return TN_ERR_INVALID_ARG;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t groups = norm_grad_groups(rows, cols);
    if (rows > 0) {
        if (!matrix_ok(dy, dy_stride, cols, dtype) || !matrix_ok(s, s_stride, cols, dtype) || !matrix_ok(dx, dx_stride, cols, dtype) ||
            (dsum && !matrix_ok(dsum, dsum_stride, cols, dtype)) || !aligned(weight, unsigned(element_bytes(dtype))))
            return TN_ERR_INVALID_ARG;
        NormGradArgs a{};
        a.dy = dy;
        a.s = s;
        a.weight = weight;
        a.dsum = dsum;
        a.dx = dx;
        a.partial = dweight ? static_cast<float*>(workspace) : nullptr;
        a.rows = rows;
        a.dy_stride = dy_stride;
        a.s_stride = s_stride;
        a.dsum_stride = dsum_stride;
        a.dx_stride = dx_stride;
        a.cols = int32_t(cols);
        a.eps = eps;
        const int64_t chunks = div_up(cols, kChunk);
        const int rc = dtype == TN_DTYPE_F32 ? dispatch_norm_grad<float>(a, chunks, groups, st) : dispatch_norm_grad<bf16_t>(a, chunks, groups, st);
        if (rc != TN_OK) return rc;
    }
    if (!dweight) return TN_OK;
    norm_grad_reduce_kernel<<<dim3(unsigned(div_up(cols, 32))), dim3(1024), 0, st>>>(static_cast<const float*>(workspace), int(groups), int(cols), dweight);
    return launched();
}

int tn_silu_gate(int32_t dtype, int64_t rows, int64_t cols, const void* gate_up, int64_t gate_up_stride, void* y,
                 int64_t y_stride, void* codes, void* scales, void* stream) {
    if (!float_type(dtype) || rows < 0 || cols < 1) return TN_ERR_INVALID_ARG;
    if (!sizes_fit(rows, cols)) return TN_ERR_UNSUPPORTED;
    if (rows == 0) return TN_OK;
    if ((!y && !codes) || !matrix_ok(gate_up, gate_up_stride, 2 * cols, dtype) || (y && !matrix_ok(y, y_stride, cols, dtype)) || !eight_bit_ok(codes, scales))
        return TN_ERR_INVALID_ARG;
    RowArgs a{};
    a.x = gate_up;
    a.x_stride = gate_up_stride;
    a.y = y;
    a.y_stride = y_stride;
    a.codes = static_cast<unsigned char*>(codes);
    a.scales = static_cast<unsigned char*>(scales);
    a.out = row_layout(cols, 1);
    a.cols = int32_t(cols);
    a.segments = 1;
    a.per_row = a.out.blocks * (kBlock / kChunk);
    return run_rows<ROW_GATE>(dtype, rows, a, static_cast<hipStream_t>(stream));
}

int tn_silu_gate_gradients(int32_t dtype, int64_t rows, int64_t cols, const void* gate_up, int64_t gate_up_stride,
                           const void* dh, int64_t dh_stride, void* d_gate_up, int64_t d_gate_up_stride, void* codes,
                           void* scales, void* stream) {
    if (!float_type(dtype) || rows < 0 || cols < 1) return TN_ERR_INVALID_ARG;
    if (!sizes_fit(rows, cols)) return TN_ERR_UNSUPPORTED;
    if (rows == 0) return TN_OK;
    if ((!d_gate_up && !codes) || !matrix_ok(gate_up, gate_up_stride, 2 * cols, dtype) || !matrix_ok(dh, dh_stride, cols, dtype) ||
        (d_gate_up && !matrix_ok(d_gate_up, d_gate_up_stride, 2 * cols, dtype)) || !eight_bit_ok(codes, scales))
        return TN_ERR_INVALID_ARG;
    RowArgs a{};
    a.x = gate_up;
    a.x_stride = gate_up_stride;
    a.dh = dh;
    a.dh_stride = dh_stride;
    a.y = d_gate_up;
    a.y_stride = d_gate_up_stride;
    a.codes = static_cast<unsigned char*>(codes);
    a.scales = static_cast<unsigned char*>(scales);
    a.out = row_layout(cols, 2);
    a.cols = int32_t(cols);
    a.segments = 2;
    a.per_row = a.out.blocks * (kBlock / kChunk);
    return run_rows<ROW_GATE_GRAD>(dtype, rows, a, static_cast<hipStream_t>(stream));
}

int tn_fp8_linear_create(tn_fp8_linear_t* out, const tn_fp8_linear_desc* d) {
    if (!out || !d || !d->tensors) return TN_ERR_INVALID_ARG;
    const bool given = d->dtype == TN_DTYPE_FP8;
    const int bad = check_desc(*d);
    if (bad != TN_OK) return bad;
    if (given && !d->scales) return TN_ERR_INVALID_ARG;
    for (int i = 0; i < d->n_tensors; ++i)
        if (!d->tensors[i] || (given && !d->scales[i]) || (!given && !aligned(d->tensors[i], unsigned(element_bytes(d->dtype))))) return TN_ERR_INVALID_ARG;
    tn_fp8_linear_s* h = new (std::nothrow) tn_fp8_linear_s;
    if (!h) return TN_ERR_ALLOC;
    lay_out(*d, *h);
    const hipStream_t st = static_cast<hipStream_t>(d->stream);
    int rc = allow_gemms<GEMM_PLAIN>(std::make_integer_sequence<int, kTileCount>()) && allow_gemms<GEMM_PARTIAL>(std::make_integer_sequence<int, kTileCount>()) && allow_gemms<GEMM_GATED>(std::make_integer_sequence<int, kGatedTiles>()) ? TN_OK : TN_ERR_HIP;
    if (rc == TN_OK && (hipMalloc(reinterpret_cast<void**>(&h->packed), size_t(h->packed_bytes)) != hipSuccess ||
        hipMalloc(reinterpret_cast<void**>(&h->scales), size_t(h->scale_bytes)) != hipSuccess)) {
        (void)hipGetLastError();
        rc = TN_ERR_ALLOC;
    }
    if (d->workspace) {
        h->workspace = d->workspace;
    } else if (rc == TN_OK) {
        h->own_workspace = true;
        if (hipMalloc(&h->workspace, size_t(h->workspace_bytes)) != hipSuccess) {
            (void)hipGetLastError();
            h->workspace = nullptr;
            rc = TN_ERR_ALLOC;
        }
    }
    for (int i = 0; rc == TN_OK && i < h->tensors; ++i) {
        WeightArgs a = weight_args(*h, i);
        a.src = d->tensors[i];
        a.src_scales = given ? static_cast<const unsigned char*>(d->scales[i]) : nullptr;
        const dim3 grid(unsigned(div_up(h->n, kBlock)), unsigned(div_up(h->m, kBlock)));
        if (given) weight_pack_kernel<unsigned char><<<grid, dim3(256), 0, st>>>(a);
        else if (d->dtype == TN_DTYPE_F32) weight_pack_kernel<float><<<grid, dim3(256), 0, st>>>(a);
        else weight_pack_kernel<bf16_t><<<grid, dim3(256), 0, st>>>(a);
        rc = launched();
    }
    if (rc == TN_OK && hipStreamSynchronize(st) != hipSuccess) rc = TN_ERR_HIP;
    if (rc != TN_OK) {
        delete h;
        return rc;
    }
    *out = h;
    return TN_OK;
}

int tn_fp8_linear_forward(tn_fp8_linear_t h, const void* codes, const void* scales, void* y, int64_t y_stride, int64_t tokens, void* stream) {
    if (!h || tokens < 0) return TN_ERR_INVALID_ARG;
    if (tokens > kMaxRows) return TN_ERR_UNSUPPORTED;
    if (tokens == 0) return TN_OK;
    if (!codes || !eight_bit_ok(codes, scales) || !matrix_ok(y, y_stride, int64_t(h->out_segments) * h->features, TN_DTYPE_BF16)) return TN_ERR_INVALID_ARG;
    LinearArgs a = linear_args(*h, codes, scales, tokens);
    a.y = y;
    a.y_stride = y_stride;
    return run_product(*h, a, false, static_cast<hipStream_t>(stream));
}

int tn_fp8_linear_gated(tn_fp8_linear_t h, const void* codes, const void* scales, void* out_codes, void* out_scales, int64_t tokens, void* stream) {
    if (!h || tokens < 0 || h->out_segments != 2) return TN_ERR_INVALID_ARG;
    if (tokens > kMaxRows) return TN_ERR_UNSUPPORTED;
    if (tokens == 0) return TN_OK;
    if (!codes || !out_codes || !eight_bit_ok(codes, scales) || !eight_bit_ok(out_codes, out_scales)) return TN_ERR_INVALID_ARG;
    LinearArgs a = linear_args(*h, codes, scales, tokens);
    const RowLayout o = row_layout(h->features, 1);
    a.out_codes = static_cast<unsigned char*>(out_codes);
    a.out_scales = static_cast<unsigned char*>(out_scales);
    a.out_code_stride = o.code_stride;
    a.out_scale_stride = o.scale_stride;
    a.spare = o.spare;
    // workgroups read rows of X while others write theirs of the output
    if (!apart(codes, tokens * a.code_stride, out_codes, tokens * o.code_stride) || !apart(scales, tokens * a.scale_stride, out_scales, tokens * o.scale_stride))
        return TN_ERR_INVALID_ARG;
    return run_product(*h, a, true, static_cast<hipStream_t>(stream));
}

int tn_fp8_linear_plan_query(const tn_fp8_linear_desc* d, int64_t tokens, int32_t gated, int32_t what, int64_t* value) {
    if (!d || !value || tokens < 1 || (gated && (d->n_tensors != 2 || (d->flags & TN_FLAG_TRANSPOSE)))) return TN_ERR_INVALID_ARG;
    const int bad = check_desc(*d);
    if (bad != TN_OK) return bad;
    if (tokens > kMaxRows) return TN_ERR_UNSUPPORTED;
    tn_fp8_linear_s h;
    lay_out(*d, h);
    const LinearArgs a = linear_args(h, nullptr, nullptr, tokens);
    const Choice c = choose(a, gated != 0, h.workspace_bytes);
    const TileCost tile = c.tile < 0 ? TileCost{} : kTiles[c.tile];
    switch (what) {
        case TN_FP8_PLAN_TILE_TOKENS: *value = 32 * tile.tm; return TN_OK;
        case TN_FP8_PLAN_TILE_FEATURES: *value = 32 * tile.tn; return TN_OK;
        case TN_FP8_PLAN_RANGES: *value = c.split; return TN_OK;
        case TN_FP8_PLAN_FUSED: *value = c.fused ? 1 : 0; return TN_OK;
        case TN_FP8_PLAN_STREAM_PIECES: *value = c.tile < 0 ? c.groups : 0; return TN_OK;
        default: return TN_ERR_INVALID_ARG;
    }
}

int tn_fp8_linear_tensor(tn_fp8_linear_t h, int32_t slot, void* codes, void* scales, void* stream) {
    if (!h || slot < 0 || slot >= h->tensors) return TN_ERR_INVALID_ARG;
    if (!codes && !scales) return TN_OK;
    const dim3 grid(unsigned(div_up(h->n, kBlock)), unsigned(div_up(h->m, kBlock)));
    weight_unpack_kernel<<<grid, dim3(256), 0, static_cast<hipStream_t>(stream)>>>(weight_args(*h, slot), static_cast<unsigned char*>(codes),
                                                                                   static_cast<unsigned char*>(scales));
    return launched();
}

int tn_fp8_linear_query(tn_fp8_linear_t h, int32_t what, int64_t* value) {
    if (!h || !value) return TN_ERR_INVALID_ARG;
    switch (what) {
        case TN_QUERY_OUT_FEATURES: *value = int64_t(h->out_segments) * h->features; return TN_OK;
        case TN_QUERY_IN_FEATURES: *value = int64_t(h->k_segments) * h->k_cols; return TN_OK;
        case TN_QUERY_PARAM_COUNT: *value = h->tensors * h->m * h->n; return TN_OK;
        case TN_QUERY_PACKED_BYTES: *value = h->packed_bytes + h->scale_bytes; return TN_OK;
        case TN_QUERY_WORKSPACE_BYTES: *value = h->workspace_bytes; return TN_OK;
        default: return TN_ERR_INVALID_ARG;
    }
}

int tn_fp8_linear_destroy(tn_fp8_linear_t h) {
    delete h;
    return TN_OK;
}

}  // extern "C"
