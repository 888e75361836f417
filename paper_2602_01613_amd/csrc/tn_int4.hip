// Projections with frozen 4-bit weights (include/tn_int4.h): host side and C ABI. Kernels: kernels/int4_*.hpp.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <new>
#include <utility>

#include "../../include/tn_fp8.h"
#include "../../include/tn_int4.h"

namespace {

#include "kernels/fp8_format.hpp"
#include "kernels/int4_weight.hpp"
#include "kernels/int4_stream.hpp"
#include "kernels/int4_gemm.hpp"

constexpr int64_t kMaxRows = int64_t(1) << 30, kMaxStride = int64_t(1) << 22;
constexpr int kCUs = 256, kBand = 5;

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void* p, unsigned n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int launched() { return hipGetLastError() == hipSuccess ? TN_OK : TN_ERR_HIP; }
int64_t whole(int64_t bytes) { return div_up(bytes, 256) * 256; }
// Whether some element of x [rows, x_cols] is one of y [rows, y_cols], both of 2 bytes. Columns of the same rows may lie beside each other: with y's first element at
// column d of x's rows, they are apart if d is past x's columns and y's end before the next row of x.
bool overlap(const void* x, int64_t x_stride, int64_t x_cols, const void* y, int64_t y_stride, int64_t y_cols, int64_t rows) {
    const intptr_t p = reinterpret_cast<intptr_t>(x), q = reinterpret_cast<intptr_t>(y);
    if (p >= q + ((rows - 1) * y_stride + y_cols) * 2 || q >= p + ((rows - 1) * x_stride + x_cols) * 2) return false;
    if (x_stride != y_stride || rows == 1) return true;
    const int64_t row = x_stride * 2, d = ((q - p) % row + row) % row;
    return d < x_cols * 2 || d + y_cols * 2 > row;
}

}  // namespace

struct tn_int4_linear_s {
    int32_t tensors = 1, transpose = 0, group = 128;
    int64_t m = 0, n = 0, groups = 0;     // of each tensor
    int32_t features = 0;                 // outputs of one of `out_segments` runs of features
    int32_t out_segments = 1, k_segments = 1;
    int64_t k_cols = 0;                   // inputs: segments of k_cols
    int64_t f_pieces = 0, own_k_blocks = 0, k_blocks = 0;
    unsigned *packed = nullptr, *words = nullptr, *halves = nullptr;
    int32_t* exponents = nullptr;
    int64_t packed_bytes = 0, word_bytes = 0, word_stride = 0, exponent_bytes = 0;
    ~tn_int4_linear_s() {
        if (packed) (void)hipFree(packed);
        if (words) (void)hipFree(words);
        if (halves) (void)hipFree(halves);
        if (exponents) (void)hipFree(exponents);
    }
};

namespace {

int check_desc(const tn_int4_linear_desc& d) {
    if (d.out_features < 1 || d.in_features < 1 || d.n_tensors < 1 || d.n_tensors > 2 || (d.flags & ~TN_FLAG_TRANSPOSE)) return TN_ERR_INVALID_ARG;
    if (d.group != 32 && d.group != 64 && d.group != 128) return TN_ERR_INVALID_ARG;
    if (d.dtype != TN_DTYPE_INT4 && d.dtype != TN_DTYPE_F32 && d.dtype != TN_DTYPE_BF16) return TN_ERR_INVALID_ARG;
    if (d.dtype == TN_DTYPE_INT4 && d.scale_dtype != TN_DTYPE_BF16 && d.scale_dtype != TN_DTYPE_F16) return TN_ERR_INVALID_ARG;
    if (d.out_features > TN_INT4_MAX_FEATURES || d.in_features > TN_INT4_MAX_FEATURES) return TN_ERR_UNSUPPORTED;
    // pieces of a tensor: offsets of its scale words within it are 32 bits, and launches that make it have fewer than 2^32 threads
    const int64_t f = (d.flags & TN_FLAG_TRANSPOSE) ? d.in_features : d.out_features, k = (d.flags & TN_FLAG_TRANSPOSE) ? d.out_features : d.in_features;
    return div_up(f, kFeaturePad) * (kFeaturePad / kPiece) * div_up(k, kBlock) > TN_INT4_MAX_WEIGHTS / (kPiece * kBlock) ? TN_ERR_UNSUPPORTED : TN_OK;
}

void lay_out(const tn_int4_linear_desc& d, tn_int4_linear_s& h) {
    h.tensors = d.n_tensors;
    h.transpose = (d.flags & TN_FLAG_TRANSPOSE) ? 1 : 0;
    h.group = d.group;
    h.m = d.out_features;
    h.n = d.in_features;
    h.groups = div_up(h.n, h.group);
    h.features = int32_t(h.transpose ? h.n : h.m);
    h.f_pieces = div_up(h.features, kFeaturePad) * (kFeaturePad / kPiece);
    h.out_segments = h.transpose ? 1 : h.tensors;
    h.k_cols = h.transpose ? h.m : h.n;
    h.k_segments = h.transpose ? h.tensors : 1;
    h.own_k_blocks = div_up(h.k_cols, kBlock);
    h.k_blocks = h.k_segments * h.own_k_blocks;
    h.packed_bytes = h.out_segments * h.f_pieces * h.k_blocks * kPieceWords * 4;
    h.exponent_bytes = h.out_segments * h.f_pieces * kPiece * 4;
    h.word_stride = h.k_blocks * kBlock;
    h.word_bytes = 4 * (h.transpose ? div_up(h.f_pieces * kPiece, h.group) * h.word_stride
                                    : h.out_segments * h.f_pieces * h.k_blocks * (kBlock / h.group) * kPiece);
}

OperandArgs operand_args(const tn_int4_linear_s& h, int slot) {
    OperandArgs a{};
    a.packed = h.packed;
    a.words = h.words;
    a.halves = h.halves;
    a.exponents = h.exponents;
    a.m = h.m;
    a.n = h.n;
    a.groups = h.groups;
    a.group = h.group;
    a.transpose = h.transpose;
    a.k_blocks = int32_t(h.k_blocks);
    a.sub = kBlock / h.group;
    a.piece0 = h.transpose ? 0 : slot * h.f_pieces;
    a.k_block0 = h.transpose ? slot * h.own_k_blocks : 0;
    a.f_pieces = h.f_pieces;
    a.own_k_blocks = h.own_k_blocks;
    a.word_stride = h.word_stride;
    return a;
}

Int4Args product_args(const tn_int4_linear_s& h, const void* x, int64_t x_stride, int64_t tokens) {
    Int4Args a{};
    a.x = x;
    a.x_stride = x_stride;
    a.packed = h.packed;
    a.words = h.words;
    a.halves = h.halves;
    a.exponents = h.exponents;
    a.tokens = tokens;
    a.word_stride = h.word_stride;
    a.k_blocks = int32_t(h.k_blocks);
    a.sub = kBlock / h.group;
    a.features = h.features;
    a.f_pieces = int32_t(h.f_pieces);
    a.tensors = h.out_segments;
    a.group_pieces = h.group / kPiece;
    a.transpose = h.transpose;
    a.n_split = 1;
    a.ld = h.out_segments * h.f_pieces * kPiece;
    return a;
}

// ---------------------------------------------------------------------------------------------
// which kernel a product runs on
// ---------------------------------------------------------------------------------------------
// Times in us, fitted to measurements on the MI355X (256 CUs) of products of 5120 to 51200 inputs and 1024 to 51200 outputs, 1 to 8192 tokens. Of the forms measured at such
// sizes the one chosen is mostly within 3 % of the best, and 1.1 times it at the worst.
constexpr int64_t kStreamTokens = 64;           // streamed up to here at the most
struct TileCost {
    int tm, per_cu;
    double alone, full;        // a block of 128 k: of one workgroup on a CU, and of as many as there is room for
};
constexpr TileCost kTiles[] = {{2, 2, 0.88, 1.5}, {4, 2, 1.15, 1.95}, {6, 1, 1.45, 1.5}, {8, 1, 1.75, 1.83}, {10, 1, 2.05, 2.12}, {12, 1, 2.4, 2.5}};
constexpr int kSplits[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24};
constexpr int64_t kMostSums = int64_t(128) << 20;
constexpr double kLaunch = 4.0, kTileRest = 3.0, kReadRate = 4.5e6, kCachedRate = 25e6, kSumsRate = 8e6, kRowsRate = 4e6;      // bytes per us
constexpr double kRowReadRate = 6e6, kRowPairReadRate = 7.5e6, kRowsAgainRate = 7e6, kOneCuRate = 32e3;      // of tokens by streaming workgroups; of the weight for their further tokens; of the weight by one CU
// Memory and computation overlap, but not wholly: of the shorter one this much is added.
double together(double a, double b) { return a > b ? a + 0.35 * b : b + 0.35 * a; }

struct Choice {
    int tm = 0;                // tile of 16 * tm tokens; 0: streamed
    int split = 1;
    int groups = 2, tg = 1;    // streamed: pieces and 16s of tokens to a workgroup
    int waves = 4;
    double us = 1e30;
};

// A streaming workgroup's pieces (GROUPS), tokens (16 * TG) and waves. Every workgroup reads its tokens anew, 64 bytes of 16 rows to a load, which come at 5 to 6 TB/s in
// all: with more tokens more pieces (25600 outputs of 5120 inputs, 16 tokens: 21 us with four, 31 with two, 46 with one), and 32 tokens at a time. Where there are few
// outputs, a workgroup's own time counts, the blocks of k that its waves take one after another: one piece (1024 outputs, 64 tokens: 11 us, 20 with 64 tokens to a workgroup), and
// eight waves instead of four (25600 -> 5120, one token: 19 us, 22 with four). Elsewhere four, so that a CU has several workgroups, one of them at its beginning or
// end while others stream (gated 25600 outputs, one token: 34 us in a graph, 46 with eight).
constexpr struct {
    int groups, tg;
} kStreams[] = {{1, 1}, {2, 1}, {4, 1}, {4, 2}};

Choice choose_stream(const Int4Args& a, bool gated, int64_t pieces) {
    Choice best;
    const double weight = double(pieces) * a.k_blocks * (1024 + 64 * a.sub);
    for (const auto& form : kStreams) {
        if (gated && form.groups == 1) continue;
        const int64_t tiles = div_up(a.tokens, 16 * form.tg), groups = pieces / form.groups * tiles;
        const double rows = double(groups) * (tiles > 1 || form.tg > 1 ? 16 * form.tg : a.tokens) * a.k_blocks * (kBlock * 2);
        const double one_cu = weight * double(tiles) / (double(groups < kCUs ? groups : kCUs) * kOneCuRate);
        const double read = weight / kReadRate + double(tiles - 1) * weight / kRowsAgainRate, memory = read > one_cu ? read : one_cu;
        for (const int waves : {4, 8}) {
            if (waves == 8 && (groups > kCUs || a.k_blocks < 100)) break;
            const double chain = (3.0 + double(div_up(a.k_blocks, waves)) * (0.13 + 0.1 * form.groups)) * (groups > 3 * kCUs ? double(groups) / (3 * kCUs) : 1.0);
            const double shared = together(memory, rows / (form.tg > 1 ? kRowPairReadRate : kRowReadRate)), us = kLaunch + 1.0 + (chain > shared ? chain : shared);
            if (us < 0.97 * best.us) {          // (of forms as good as each other the one with more workgroups)
                best.us = us;
                best.groups = form.groups;
                best.tg = form.tg;
                best.waves = waves;
            }
        }
    }
    return best;
}

Choice choose(const Int4Args& a, bool gated) {
    const int64_t pieces = int64_t(a.f_pieces) * a.tensors;
    Choice best;
    if (a.tokens <= kStreamTokens && !a.transpose) best = choose_stream(a, gated, pieces);
    const double weight = double(pieces) * a.k_blocks * (1024 + 64 * a.sub), rows = double(a.tokens) * a.k_blocks * (kBlock * 4), outputs = double(a.tokens) * a.ld * 4;
    const int64_t n_col = div_up(gated ? pieces / 2 : pieces, gated ? 8 : 16);
    for (const TileCost& t : kTiles) {
        const int64_t n_row = div_up(a.tokens, 16 * t.tm);
        for (const int split : kSplits) {
            if (split > 1 && (split * 4 > a.k_blocks || split * outputs > double(kMostSums))) break;
            const int64_t blocks = div_up(a.k_blocks, split), cols = gated && split > 1 ? div_up(pieces, 16) : n_col, items = n_row * cols * div_up(a.k_blocks, blocks);
            const int64_t held = items <= kCUs ? kCUs : int64_t(kCUs) * t.per_cu;
            const double compute = double(div_up(items, held)) * (double(blocks) * (items <= kCUs ? t.alone : t.full) + kTileRest);
            const double memory = weight / kReadRate + double(n_row - 1) * weight / kCachedRate;
            const double us = kLaunch + 3.0 + rows / kRowsRate + together(compute, memory) + (split > 1 ? 3.0 + 2 * split * outputs / kSumsRate : 0);
            if (us < best.us) {
                best = Choice();
                best.us = us;
                best.tm = t.tm;
                best.split = split;
            }
        }
    }
    return best;
}

template <int GROUPS, int TG, int SUB, bool GATED>
int run_stream(const Int4Args& a, int waves, hipStream_t stream) {
    constexpr int OWN = GATED ? GROUPS / 2 : GROUPS;
    const dim3 grid(unsigned((GATED ? a.f_pieces : int64_t(a.f_pieces) * a.tensors) / OWN), unsigned(div_up(a.tokens, 16 * TG)));
    int4_stream_kernel<GROUPS, TG, SUB, GATED><<<grid, dim3(unsigned(64 * (waves < a.k_blocks ? waves : a.k_blocks))), 0, stream>>>(a);
    return launched();
}
template <int GROUPS, int TG, int SUB>
int stream_form(const Int4Args& a, const Choice& c, bool gated, hipStream_t stream) {
    if constexpr (GROUPS > 1) {
        if (gated) return run_stream<GROUPS, TG, SUB, true>(a, c.waves, stream);
    }
    return run_stream<GROUPS, TG, SUB, false>(a, c.waves, stream);
}
template <int SUB>
int stream_sizes(const Int4Args& a, const Choice& c, bool gated, hipStream_t stream) {
    if (c.tg == 2) return stream_form<4, 2, SUB>(a, c, gated, stream);
    return c.groups == 1 ? stream_form<1, 1, SUB>(a, c, gated, stream) : c.groups == 2 ? stream_form<2, 1, SUB>(a, c, gated, stream) : stream_form<4, 1, SUB>(a, c, gated, stream);
}

template <int TM, int FORM, bool TRANSPOSED, int SUB>
int run_gemm(const Int4GemmArgs& g, hipStream_t stream) {
    const int64_t items = int64_t(g.n_row) * g.n_col * g.l.n_split;
    int4_gemm_kernel<TM, FORM, TRANSPOSED, SUB><<<dim3(unsigned(div_up(items, 8) * 8)), dim3(256), Int4Shape<TM, TRANSPOSED, SUB>::SMEM, stream>>>(g);
    return launched();
}
template <int TM, int FORM>
int gemm_form(const Int4GemmArgs& g, hipStream_t stream) {
    if constexpr (FORM != INT4_GATED) {
        if (g.l.transpose) return g.l.group_pieces >= 4 ? run_gemm<TM, FORM, true, 1>(g, stream) : run_gemm<TM, FORM, true, 2>(g, stream);
    }
    return g.l.sub == 1 ? run_gemm<TM, FORM, false, 1>(g, stream) : g.l.sub == 2 ? run_gemm<TM, FORM, false, 2>(g, stream) : run_gemm<TM, FORM, false, 4>(g, stream);
}
template <int TM>
int run_tiles(const Int4Args& a, int64_t range, bool gated, hipStream_t stream) {
    Int4GemmArgs g{};
    g.l = a;
    g.blocks_per_split = int(range);
    const bool fused = gated && !a.partial;
    const int64_t pieces = int64_t(a.f_pieces) * a.tensors;
    const int64_t n_row = div_up(a.tokens, 16 * TM), n_col = fused ? div_up(a.f_pieces, 8) : div_up(pieces, 16);
    if (n_row * n_col * g.l.n_split > INT32_MAX / 8) return TN_ERR_UNSUPPORTED;
    g.n_row = int(n_row);
    g.n_col = int(n_col);
    g.band = int(div_up(n_row, div_up(n_row, kBand)));
    int rc = fused ? gemm_form<TM, INT4_GATED>(g, stream) : a.partial ? gemm_form<TM, INT4_PARTIAL>(g, stream) : gemm_form<TM, INT4_PLAIN>(g, stream);
    if (rc != TN_OK || !a.partial) return rc;
    const int64_t blocks = div_up(a.tokens * (gated ? a.ld / 2 : a.ld) / 4, 256);
    const dim3 grid(unsigned(blocks < 8 * kCUs ? blocks : 8 * kCUs));
    if (gated) int4_reduce_kernel<true><<<grid, dim3(256), 0, stream>>>(g.l);
    else int4_reduce_kernel<false><<<grid, dim3(256), 0, stream>>>(g.l);
    return launched();
}

template <int TM, int FORM, bool TRANSPOSED, int SUB>
bool allow() {          // more LDS than a launch gets by default
    return hipFuncSetAttribute(reinterpret_cast<const void*>(int4_gemm_kernel<TM, FORM, TRANSPOSED, SUB>), hipFuncAttributeMaxDynamicSharedMemorySize,
                               Int4Shape<TM, TRANSPOSED, SUB>::SMEM) == hipSuccess;
}
template <int TM>
bool allow_tiles() {
    return allow<TM, INT4_PLAIN, false, 1>() && allow<TM, INT4_PLAIN, false, 2>() && allow<TM, INT4_PLAIN, false, 4>() && allow<TM, INT4_PLAIN, true, 1>() &&
           allow<TM, INT4_PLAIN, true, 2>() && allow<TM, INT4_PARTIAL, false, 1>() && allow<TM, INT4_PARTIAL, false, 2>() &&
           allow<TM, INT4_PARTIAL, false, 4>() && allow<TM, INT4_PARTIAL, true, 1>() && allow<TM, INT4_PARTIAL, true, 2>() &&
           allow<TM, INT4_GATED, false, 1>() && allow<TM, INT4_GATED, false, 2>() && allow<TM, INT4_GATED, false, 4>();
}

// Rows that the streaming kernel cannot read where they are
bool laid_out_anew(const tn_int4_linear_s& h, const void* x, int64_t x_stride) {
    return h.k_cols % kBlock != 0 || !aligned(x, 16) || x_stride % kChunk != 0 || x_stride >= kMaxStride;
}
struct Workspace {
    int64_t rows = 0, exponents = 0, sums = 0;
    int64_t all() const { return rows + exponents + sums; }
};
Workspace workspace_of(const tn_int4_linear_s& h, const Int4Args& a, const Choice& c) {
    Workspace w;
    if (c.tm || laid_out_anew(h, a.x, a.x_stride)) w.rows = whole(a.tokens * h.k_blocks * kBlock * 2);
    if (c.tm) w.exponents = whole(c.split * a.tokens * 4);
    if (c.tm && c.split > 1) w.sums = whole(c.split * a.tokens * a.ld * 4);
    return w;
}

int half_rows(const tn_int4_linear_s& h, const Int4Args& a, int ranges, int64_t blocks, _Float16* rows, int32_t* exponents, hipStream_t stream) {
    const bf16_t* x = static_cast<const bf16_t*>(a.x);
    const int64_t padded = h.own_k_blocks * kBlock, chunks = blocks * (kBlock / kChunk), run = int64_t(1) << 19;
    for (int64_t at = 0; at < a.tokens; at += run) {              // a launch has fewer than 2^32 threads
        const dim3 grid(unsigned(a.tokens - at < run ? a.tokens - at : run), unsigned(ranges));
        const bf16_t* from = x + at * a.x_stride;
        _Float16* to = rows + at * h.k_blocks * kBlock;
        if (chunks <= 512) int4_half_rows_kernel<2><<<grid, dim3(256), 0, stream>>>(from, a.x_stride, h.k_segments, h.k_cols, padded, chunks, to, exponents + at, a.tokens);
        else if (chunks <= 1024) int4_half_rows_kernel<4><<<grid, dim3(256), 0, stream>>>(from, a.x_stride, h.k_segments, h.k_cols, padded, chunks, to, exponents + at, a.tokens);
        else int4_half_rows_kernel<13><<<grid, dim3(256), 0, stream>>>(from, a.x_stride, h.k_segments, h.k_cols, padded, chunks, to, exponents + at, a.tokens);
        const int rc = launched();
        if (rc != TN_OK) return rc;
    }
    return TN_OK;
}

int run_product(const tn_int4_linear_s& h, const void* x, int64_t x_stride, void* y, int64_t y_stride, int64_t tokens, bool gated, void* workspace,
                int64_t workspace_bytes, hipStream_t stream) {
    if (tokens < 0) return TN_ERR_INVALID_ARG;
    if (tokens > kMaxRows) return TN_ERR_UNSUPPORTED;
    if (tokens == 0) return TN_OK;
    const int64_t x_cols = h.k_segments * h.k_cols, y_cols = gated ? h.features : int64_t(h.out_segments) * h.features;
    if (!x || !y || x_stride < x_cols || y_stride < y_cols || !aligned(x, 2) || !aligned(y, 2)) return TN_ERR_INVALID_ARG;
    // workgroups read rows of x while others write theirs of y
    if (overlap(x, x_stride, x_cols, y, y_stride, y_cols, tokens)) return TN_ERR_INVALID_ARG;
    Int4Args a = product_args(h, x, x_stride, tokens);
    const Choice c = choose(a, gated);
    const Workspace w = workspace_of(h, a, c);
    if (w.all() > 0 && (!workspace || workspace_bytes < w.all() || !aligned(workspace, 256))) return TN_ERR_INVALID_ARG;
    a.y = static_cast<bf16_t*>(y);
    a.y_stride = y_stride;
    const int64_t range = div_up(a.k_blocks, c.split);
    a.n_split = int32_t(div_up(a.k_blocks, range));         // no range without a block
    if (w.rows) {
        int rc;
        if (c.tm) {
            int32_t* exponents = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + w.rows);
            rc = half_rows(h, a, a.n_split, range, static_cast<_Float16*>(workspace), exponents, stream);
            a.x_exponents = exponents;
        } else {
            const int64_t blocks = div_up(tokens * h.k_blocks * (kBlock / kChunk), 256);
            int4_rows_kernel<<<dim3(unsigned(blocks < 32 * kCUs ? blocks : 32 * kCUs)), dim3(256), 0, stream>>>(
                static_cast<const bf16_t*>(x), x_stride, tokens, h.k_segments, h.k_cols, h.own_k_blocks * kBlock, static_cast<bf16_t*>(workspace));
            rc = launched();
        }
        if (rc != TN_OK) return rc;
        a.x = workspace;
        a.x_stride = h.k_blocks * kBlock;
    }
    if (c.tm == 0) return a.sub == 1 ? stream_sizes<1>(a, c, gated, stream) : a.sub == 2 ? stream_sizes<2>(a, c, gated, stream) : stream_sizes<4>(a, c, gated, stream);
    if (c.split > 1) a.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + w.rows + w.exponents);
    switch (c.tm) {
        case 2: return run_tiles<2>(a, range, gated, stream);
        case 4: return run_tiles<4>(a, range, gated, stream);
        case 6: return run_tiles<6>(a, range, gated, stream);
        case 8: return run_tiles<8>(a, range, gated, stream);
        case 10: return run_tiles<10>(a, range, gated, stream);
        default: return run_tiles<12>(a, range, gated, stream);
    }
}

}  // namespace

extern "C" {

int tn_int4_linear_create(tn_int4_linear_t* out, const tn_int4_linear_desc* d) {
    if (!out || !d || !d->tensors) return TN_ERR_INVALID_ARG;
    const int bad = check_desc(*d);
    if (bad != TN_OK) return bad;
    const bool given = d->dtype == TN_DTYPE_INT4;
    if (given && !d->scales) return TN_ERR_INVALID_ARG;
    for (int i = 0; i < d->n_tensors; ++i)
        if (!d->tensors[i] || (given && (!d->scales[i] || !aligned(d->scales[i], 2) || (d->zeros && !d->zeros[i]))) ||
            (!given && !aligned(d->tensors[i], d->dtype == TN_DTYPE_F32 ? 4 : 2)))
            return TN_ERR_INVALID_ARG;
    tn_int4_linear_s* h = new (std::nothrow) tn_int4_linear_s;
    if (!h) return TN_ERR_ALLOC;
    lay_out(*d, *h);
    const hipStream_t st = static_cast<hipStream_t>(d->stream);
    const int64_t row_bytes = div_up(h->n, 2);
    int rc = allow_tiles<2>() && allow_tiles<4>() && allow_tiles<6>() && allow_tiles<8>() && allow_tiles<10>() && allow_tiles<12>() ? TN_OK : TN_ERR_HIP;
    // (what is quantised here passes through the form that a caller gives)
    unsigned char* made = nullptr;
    const int64_t scales_at = whole(h->m * row_bytes), zeros_at = scales_at + whole(h->m * h->groups * 2);
    if (rc == TN_OK && (hipMalloc(reinterpret_cast<void**>(&h->packed), size_t(h->packed_bytes)) != hipSuccess ||
                        hipMalloc(reinterpret_cast<void**>(&h->words), size_t(h->word_bytes)) != hipSuccess ||
                        hipMalloc(reinterpret_cast<void**>(&h->halves), size_t(h->word_bytes)) != hipSuccess ||
                        hipMalloc(reinterpret_cast<void**>(&h->exponents), size_t(h->exponent_bytes)) != hipSuccess ||
                        (!given && hipMalloc(reinterpret_cast<void**>(&made), size_t(zeros_at + h->m * h->groups)) != hipSuccess))) {
        (void)hipGetLastError();
        rc = TN_ERR_ALLOC;
    }
    for (int i = 0; rc == TN_OK && i < h->tensors; ++i) {
        OperandArgs a = operand_args(*h, i);
        if (given) {
            a.codes = static_cast<const unsigned char*>(d->tensors[i]);
            a.scales = d->scales[i];
            a.zeros = d->zeros ? static_cast<const unsigned char*>(d->zeros[i]) : nullptr;
            a.scale_f16 = d->scale_dtype == TN_DTYPE_F16;
        } else {
            const dim3 grid(unsigned(div_up(h->m * h->groups, 256)));
            bf16_t* scales = reinterpret_cast<bf16_t*>(made + scales_at);
            if (d->dtype == TN_DTYPE_F32)
                int4_quantise_kernel<float><<<grid, dim3(256), 0, st>>>(static_cast<const float*>(d->tensors[i]), h->m, h->n, h->groups, h->group, made, scales, made + zeros_at);
            else
                int4_quantise_kernel<bf16_t><<<grid, dim3(256), 0, st>>>(static_cast<const bf16_t*>(d->tensors[i]), h->m, h->n, h->groups, h->group, made, scales, made + zeros_at);
            a.codes = made;
            a.scales = scales;
            a.zeros = made + zeros_at;
        }
        int4_pack_kernel<<<dim3(unsigned(h->f_pieces), unsigned(h->own_k_blocks)), dim3(256), 0, st>>>(a);
        const int64_t words = h->transpose ? div_up(h->f_pieces * kPiece, h->group) * h->own_k_blocks * kBlock
                                           : h->f_pieces * h->own_k_blocks * a.sub * kPiece;
        int4_words_kernel<<<dim3(unsigned(div_up(words, 256))), dim3(256), 0, st>>>(a);
        if (!h->transpose || i + 1 == h->tensors) {          // (transposed, a group of features has the scales of all tensors)
            const int64_t waves = h->transpose ? div_up(h->f_pieces * kPiece, h->group) : h->f_pieces * kPiece;
            int4_halves_kernel<<<dim3(unsigned(div_up(waves, 4))), dim3(256), 0, st>>>(a);
        }
        rc = launched();
    }
    if (rc == TN_OK && hipStreamSynchronize(st) != hipSuccess) rc = TN_ERR_HIP;
    if (made) {
        if (rc != TN_OK) (void)hipStreamSynchronize(st);
        (void)hipFree(made);
    }
    if (rc != TN_OK) {
        delete h;
        return rc;
    }
    *out = h;
    return TN_OK;
}

int64_t tn_int4_linear_workspace(tn_int4_linear_t h, const void* x, int64_t x_stride, int64_t tokens, int32_t gated) {
    if (!h || tokens < 0 || (gated && h->out_segments != 2)) return TN_ERR_INVALID_ARG;
    if (tokens > kMaxRows) return TN_ERR_UNSUPPORTED;
    if (tokens == 0) return 0;
    const Int4Args a = product_args(*h, x, x_stride, tokens);
    return workspace_of(*h, a, choose(a, gated != 0)).all();
}

int tn_int4_linear_forward(tn_int4_linear_t h, const void* x, int64_t x_stride, void* y, int64_t y_stride, int64_t tokens, void* workspace,
                           int64_t workspace_bytes, void* stream) {
    if (!h) return TN_ERR_INVALID_ARG;
    return run_product(*h, x, x_stride, y, y_stride, tokens, false, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

int tn_int4_linear_gated(tn_int4_linear_t h, const void* x, int64_t x_stride, void* y, int64_t y_stride, int64_t tokens, void* workspace,
                         int64_t workspace_bytes, void* stream) {
    if (!h || h->out_segments != 2) return TN_ERR_INVALID_ARG;
    return run_product(*h, x, x_stride, y, y_stride, tokens, true, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

int tn_int4_linear_plan_query(const tn_int4_linear_desc* d, int64_t tokens, int32_t gated, int32_t what, int64_t* value) {
    if (!d || !value || tokens < 1 || (gated && (d->n_tensors != 2 || (d->flags & TN_FLAG_TRANSPOSE)))) return TN_ERR_INVALID_ARG;
    const int bad = check_desc(*d);
    if (bad != TN_OK) return bad;
    if (tokens > kMaxRows) return TN_ERR_UNSUPPORTED;
    tn_int4_linear_s h;
    lay_out(*d, h);
    const Choice c = choose(product_args(h, nullptr, 0, tokens), gated != 0);
    switch (what) {
        case TN_INT4_PLAN_TILE_TOKENS: *value = 16 * c.tm; return TN_OK;
        case TN_INT4_PLAN_RANGES: *value = c.split; return TN_OK;
        case TN_INT4_PLAN_STREAM_TOKENS: *value = c.tm ? 0 : 16 * c.tg; return TN_OK;
        case TN_INT4_PLAN_STREAM_PIECES: *value = c.tm ? 0 : c.groups; return TN_OK;
        default: return TN_ERR_INVALID_ARG;
    }
}

int tn_int4_linear_tensor(tn_int4_linear_t h, int32_t slot, void* codes, void* scales, void* zeros, void* stream) {
    if (!h || slot < 0 || slot >= h->tensors || !aligned(scales, 4)) return TN_ERR_INVALID_ARG;
    if (!codes && !scales && !zeros) return TN_OK;
    const dim3 grid(unsigned(div_up(div_up(h->n, 2), 256)), unsigned(h->m < 65535 ? h->m : 65535), unsigned(div_up(h->m, 65535)));
    int4_unpack_kernel<<<grid, dim3(256), 0, static_cast<hipStream_t>(stream)>>>(operand_args(*h, slot), static_cast<unsigned char*>(codes),
                                                                                 static_cast<float*>(scales), static_cast<unsigned char*>(zeros));
    return launched();
}

int tn_int4_linear_query(tn_int4_linear_t h, int32_t what, int64_t* value) {
    if (!h || !value) return TN_ERR_INVALID_ARG;
    switch (what) {
        case TN_QUERY_OUT_FEATURES: *value = int64_t(h->out_segments) * h->features; return TN_OK;
        case TN_QUERY_IN_FEATURES: *value = h->k_segments * h->k_cols; return TN_OK;
        case TN_QUERY_PARAM_COUNT: *value = h->tensors * h->m * h->n; return TN_OK;
        case TN_QUERY_PACKED_BYTES: *value = h->packed_bytes + 2 * h->word_bytes + h->exponent_bytes; return TN_OK;
        default: return TN_ERR_INVALID_ARG;
    }
}

int tn_int4_linear_destroy(tn_int4_linear_t h) {
    delete h;
    return TN_OK;
}

}  // extern "C"
