// Products of many tokens: tiles of both operands in LDS.
// Part of tn_fp8.hip's translation unit, inside its anonymous namespace, after fp8_stream.hpp.
#pragma once

// ---------------------------------------------------------------------------------------------
// A workgroup of four waves (2 x 2) computes 32 * TM tokens x 32 * TN features: a wave 16 * TM x 16 * TN in TM x TN accumulators of
// v_mfma_scale_f32_16x16x128_f8f6f4. A K tile is one block of 128. Both operands go from memory to LDS without passing through
// registers, two or three stages of a K tile each; a row of tokens is 128 bytes there, its 16-byte chunk c at position c ^ ((row / 2) % 8), so that
// the 16 rows a read touches at a time fall on 16 different slots of the 64 banks; a piece of the weight is as it is in memory.
//
// The wave holds one set of fragments and walks its tile in quadrants of half its tokens (lo, hi) x half its features (x, y):
//     first half step:   lo * x (reading y),  lo * y (reading hi)
//     second half step:  hi * y (reading the next tile's lo),  hi * x (reading the next tile's x, into the registers of this one's y)
// so that each fragment is read one quadrant before its first use into registers whose last use has passed, and x and y change places
// from tile to tile. What a half step reads ((y, hi), then the next (lo, x)) is free in LDS when it ends: the loads of the tile that has this
// stage next go there in the half step after it, and have a whole K tile's time (with three stages almost two) to land before the barrier that
// lets them be read. One barrier a half step.
// Scale bytes: four K tiles of a row in a word, which the instruction picks its byte from; the words of the next four tiles go to LDS
// while these four are computed.
//
// What bounds it: the matrix cores at the clock that the power limit leaves (busy 78 % of the cycles at 1.75 to 1.9 GHz; where in the loop reads,
// loads and barriers stand no longer matters). 8192 x 8192 x 8192 in 361 us = 3.04 PFLOP/s, 8192 x 5120 x 25600 in 760 us = 2.82; 256 x 256 tiles take
// 1.26 us for a K tile, 64 x 256 ones 0.50. Reads with bank conflicts, descriptors in vector registers (every load a
// loop) and a mask for each load cost 0.4 us of a K tile together.
// ---------------------------------------------------------------------------------------------
struct GemmArgs {
    LinearArgs l;
    int32_t n_row, n_col;            // output tiles
    int32_t band;                    // rows of tiles to a band
    int32_t ktiles_per_split;        // a multiple of 4; at least one tile in every range
};

template <int TM, int TN>
struct GemmShape {
    static constexpr int BM = 32 * TM, BN = 32 * TN;
    static constexpr int A_BYTES = BM * kBlock, STAGE = (BM + BN) * kBlock;
    static constexpr int SCALE_ROWS = (BM + 63) / 64 * 64, SCALES = (SCALE_ROWS + 64) * 4;       // words of the rows, then of the feature blocks
    // stages: three where LDS holds them (for as many workgroups on a CU), else two
    static constexpr int LDS = 160 * 1024;
    static constexpr int PER_CU = 2 * (2 * STAGE + 2 * SCALES) <= LDS ? 2 : 1;
    static constexpr int NS = PER_CU * (3 * STAGE + 2 * SCALES + (TN == 8 ? 2 * BM * 4 : 0)) <= LDS ? 3 : 2;
    static constexpr int SMEM = NS * STAGE + 2 * SCALES + (TN == 8 ? 2 * BM * 4 : 0);            // and the gated form's maxima
};

// what becomes of the sums: y in bf16, silu(gate) * up in 8 bits, or fp32 to the workspace
enum GemmForm : int { GEMM_PLAIN = 0, GEMM_GATED = 1, GEMM_PARTIAL = 2 };

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
    __builtin_amdgcn_s_waitcnt((N & 0xF) | (0x7 << 4) | (0xF << 8) | ((N >> 4) << 14));
}

template <typename F, int... Q>
__device__ __forceinline__ void for_constants(F&& f, std::integer_sequence<int, Q...>) {
    (f(std::integral_constant<int, Q>()), ...);
}

#ifdef __HIP_DEVICE_COMPILE__
template <int TM, int TN, int FORM>
__device__ __forceinline__ void gemm_tile(const GemmArgs& g) {
    using S = GemmShape<TM, TN>;
    constexpr int LO = (TM + 1) / 2, HI = TM - LO, TH = TN / 2, NS = S::NS;
    static_assert(TM >= 2 && TN % 2 == 0 && (FORM != GEMM_GATED || TN == 8), "halves of both sides");
    typedef __attribute__((address_space(3))) void lds_t;
    typedef unsigned int uintx4 __attribute__((ext_vector_type(4)));
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const LinearArgs& a = g.l;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;

    // XCD x takes a contiguous eighth of the tiles in bands of up to five token tiles (tokens fastest): the 32 tiles that it runs at
    // a time share 5 + 7 operand panels in its L2, and the weight is read from behind it once a band. A launch has no more workgroups than the chip holds: each takes every so many of its
    // XCD's tiles, and brings the first stages of the next one while it stores this one.
    const int n_items = g.n_row * g.n_col * a.n_split, xcd = blockIdx.x & 7;
    const int end_item = int(int64_t(n_items) * (xcd + 1) >> 3), step_item = gridDim.x >> 3;
    int item = int(int64_t(n_items) * xcd >> 3) + int(blockIdx.x >> 3);
    if (item >= end_item) return;
    struct Place {
        int row_tile, col_tile, split;
    };
    auto place_of = [&](int at) {
        Place p;
        const int tile = at / a.n_split;
        p.split = __builtin_amdgcn_readfirstlane(at - tile * a.n_split);
        const int band = tile / (g.band * g.n_col), in_band = tile - band * (g.band * g.n_col);
        const int band_rows = min(g.band, g.n_row - band * g.band);
        p.col_tile = __builtin_amdgcn_readfirstlane(in_band / band_rows);
        p.row_tile = __builtin_amdgcn_readfirstlane(band * g.band + in_band - p.col_tile * band_rows);
        return p;
    };

    // tokens past the end, and pieces past theirs, are out of the buffers' bounds by the lane's own offset: no memory is read
    constexpr int RSRC = 0x00020000;
    const int code_stride = int(a.code_stride), scale_stride = int(a.scale_stride);
    const int piece_bytes = a.k_blocks * 2048;
    const int all_pieces = a.f_pieces * a.tensors;
    auto rows_of = [&](const Place& p) { return int(min(a.tokens - int64_t(p.row_tile) * S::BM, int64_t(S::BM))); };
    auto tokens_rsrc = [&](const Place& p) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(a.codes + int64_t(p.row_tile) * S::BM * a.code_stride), 0, rows_of(p) * code_stride, RSRC);
    };
    auto scales_rsrc = [&](const Place& p) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(a.scales + int64_t(p.row_tile) * S::BM * a.scale_stride), 0, rows_of(p) * scale_stride, RSRC);
    };
    // pieces of the two feature halves: wave column w, fragment j of half 0 or 1 is piece first(half) + w * W_STEP + j
    constexpr int W_STEP = FORM == GEMM_GATED ? TH : TN;
    auto first = [&](const Place& p, int half) { return p.col_tile * (FORM == GEMM_GATED ? TN : 2 * TN) + (half ? (FORM == GEMM_GATED ? a.f_pieces : TH) : 0); };
    auto weight_rsrc = [&](const Place& p, int half) {
        // (a clamp is a vector instruction, and a descriptor from vector registers makes every load a loop)
        const int there = __builtin_amdgcn_readfirstlane(max(0, min(all_pieces - first(p, half), W_STEP + TH)));
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(a.packed + int64_t(first(p, half)) * piece_bytes), 0, there * piece_bytes, RSRC);
    };
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(a.w_scales), 0, (all_pieces >> 3) * a.w_scale_stride, RSRC);

    // a load of tokens covers 8 rows x 128 bytes (lane l fills position l % 8 of row l / 8), one of features half a piece. The waves share a
    // fragment's worth of both wave rows (columns): wave w brings rows 8 * (w / 2) .. of wave row w % 2, half w / 2 of wave column w % 2's piece.
    const int pair = wave & 1, part = wave >> 1;
    const int va = (pair * TM * 16 + part * 8 + (lane >> 3)) * code_stride + (((lane & 7) ^ (part * 4 + (lane >> 4))) * 16);
    const int vb = pair * W_STEP * piece_bytes + part * 1024 + lane * 16;
    const int lds_a = (pair * TM * 16 + part * 8) * kBlock, lds_b = S::A_BYTES + pair * TN * 2048 + part * 1024;
    // (tiles past the range: the last one once more, into a stage that is not read again)
    auto load_a = [&](__amdgpu_buffer_rsrc_t r, int i, int at, unsigned char* s) {                        // at: K tile in memory
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_t*)(s + lds_a + i * 2048), 16, va + i * 16 * code_stride, at * kBlock, 0, 0);
    };
    auto load_b = [&](__amdgpu_buffer_rsrc_t r, int j, int at, unsigned char* s) {                        // j: fragment 0 .. TN - 1, r of its half
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_t*)(s + lds_b + j * 2048), 16, vb + (j < TH ? j : j - TH) * piece_bytes, at * 2048, 0, 0);
    };
    // scale words of four tiles: 64 rows to a load, then the two feature blocks (even and odd lanes). Every wave issues as many.
    constexpr int ROW_LOADS = S::SCALE_ROWS / 64, SCALE_LOADS = (ROW_LOADS + 1 + 3) / 4;
    auto load_scales = [&](__amdgpu_buffer_rsrc_t r, const Place& p, int word, unsigned char* s) {
        const int fb0 = first(p, 0) >> 3, fb1 = FORM == GEMM_GATED ? first(p, 1) >> 3 : fb0 + 1;          // the tile's blocks of features
#pragma unroll
        for (int q = 0; q < SCALE_LOADS; ++q) {
            const int n = min(wave + 4 * q, ROW_LOADS);
            if (n < ROW_LOADS)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_t*)(s + n * 256), 4, (n * 64 + lane) * scale_stride, word * 4, 0, 0);
            else
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_t*)(s + n * 256), 4, (lane & 1 ? fb1 : fb0) * a.w_scale_stride, word * 4, 0, 0);
        }
    };
    constexpr int LA = LO + TH, LB = HI + TH;
    unsigned char* const scale_lds = smem + NS * S::STAGE;
    // the first group's scales, then the stages in the order in which they are waited for
    auto begin = [&](const Place& p) {
        const __amdgpu_buffer_rsrc_t ra = tokens_rsrc(p), rb0 = weight_rsrc(p, 0), rb1 = weight_rsrc(p, 1);
        const int kt0 = p.split * g.ktiles_per_split, last = min(a.k_blocks, kt0 + g.ktiles_per_split) - 1;
        load_scales(scales_rsrc(p), p, kt0 >> 2, scale_lds);
#pragma unroll
        for (int q = 0; q < NS; ++q) {
            unsigned char* s = smem + q * S::STAGE;
            const int at = min(kt0 + q, last);
#pragma unroll
            for (int i = 0; i < LO; ++i) load_a(ra, i, at, s);
#pragma unroll
            for (int j = 0; j < TH; ++j) load_b(q & 1 ? rb1 : rb0, q & 1 ? TH + j : j, at, s);
#pragma unroll
            for (int i = LO; i < TM; ++i) load_a(ra, i, at, s);
#pragma unroll
            for (int j = 0; j < TH; ++j) load_b(q & 1 ? rb0 : rb1, q & 1 ? j : TH + j, at, s);
        }
    };

    // fragments: lane l has row (token, or feature) l % 16, its 16-byte chunks l / 16 and 4 + l / 16
    const int r = lane & 15, kq = lane >> 4;
    const int oa0 = (wm * TM * 16 + r) * kBlock + ((kq ^ (r >> 1)) * 16), oa1 = (wm * TM * 16 + r) * kBlock + (((4 + kq) ^ (r >> 1)) * 16);
    const int ob = S::A_BYTES + wn * TN * 2048 + lane * 16;
    intx4 fa[TM][2], fb[TN][2];
    floatx4 acc[TM][TN];
    unsigned sx[TM], sw[2], sw_next[2];
    auto read_a = [&](int i, int h, const unsigned char* s) { fa[i][h] = *reinterpret_cast<const intx4*>(s + (h ? oa1 : oa0) + i * 2048); };
    auto read_b = [&](int j, int h, const unsigned char* s) { fb[j][h] = *reinterpret_cast<const intx4*>(s + ob + h * 1024 + j * 2048); };
    auto read_sx = [&](int i, const unsigned char* s) { sx[i] = *reinterpret_cast<const unsigned*>(s + (wm * TM * 16 + i * 16 + r) * 4); };
    // the scale word of fragment j: gate and up are different blocks; otherwise a wave's features are within one, the tile's first or second
    auto read_sw = [&](int q, const unsigned char* s, unsigned (&to)[2]) {
        const int which = FORM == GEMM_GATED ? q : (wn * TN) >> 3;
        to[q] = *reinterpret_cast<const unsigned*>(s + S::SCALE_ROWS * 4 + which * 4);
    };

    Place place = place_of(item);
    begin(place);
    for (;;) {
    const int kt0 = place.split * g.ktiles_per_split, nk = min(a.k_blocks, kt0 + g.ktiles_per_split) - kt0, last = kt0 + nk - 1;
    const __amdgpu_buffer_rsrc_t ra = tokens_rsrc(place), rs = scales_rsrc(place), rb0 = weight_rsrc(place, 0), rb1 = weight_rsrc(place, 1);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[i][j][v] = 0.f;
            asm volatile("" : "+a"(acc[i][j]));
        }
    // The first K tile and the scales have landed. (Behind them the tile before stored its results: vector memory operations are counted in
    // order, so this and the next waits are for those stores too. A count that left them out would have to differ in a workgroup's first K
    // tiles, and a branch there lets the compiler move MFMAs out of the places they are dealt to: 1.38 us a K tile instead of 1.26.)
    wait_vmcnt<(NS - 1) * (LA + LB)>();
    __builtin_amdgcn_s_barrier();
#pragma unroll
    for (int i = 0; i < LO; ++i) {
        read_a(i, 0, smem);
        read_a(i, 1, smem);
        read_sx(i, scale_lds);
    }
#pragma unroll
    for (int j = 0; j < TH; ++j) {
        read_b(j, 0, smem);
        read_b(j, 1, smem);
    }
    read_sw(0, scale_lds, sw);
    if (FORM == GEMM_GATED) read_sw(1, scale_lds, sw);
    __builtin_amdgcn_s_waitcnt(0xC07F);          // lgkmcnt(0): the first half step's loads go where these reads were
    __builtin_amdgcn_s_barrier();

    // The slots of a half step: an MFMA, then what is dealt out there. BAR: where the barrier stands.
    auto half_step = [&](auto idx_c, auto half_c, int kt, unsigned char* s, unsigned char* sn, unsigned char* sc, unsigned char* sc_next) {
        constexpr int IDX = decltype(idx_c)::value, HALF = decltype(half_c)::value;
        constexpr int X = (IDX & 1) ? TH : 0, Y = TH - X;                        // first fragments of x and y
        constexpr int I0 = HALF ? LO : 0, NI = HALF ? HI : LO;
        constexpr int NQ = NI * TH, NM = 2 * NQ;                                 // MFMAs of a quadrant, of the half step
        constexpr int L = HALF ? LB : LA, NA = HALF ? HI : LO;
        constexpr int R0 = HALF ? 2 * LO : TN, R1 = HALF ? TN : 2 * HI;          // reads of the two quadrants
        constexpr int BAR = NM - (NQ >= 8 ? 4 : 1);
        const int at = min(kt0 + kt + NS, last);
        auto slot = [&](auto slot_c) {
            constexpr int q = decltype(slot_c)::value, quad = q / NQ, m = q % NQ;
            // first half: features outermost (y arrives one by one); second: tokens outermost (hi does)
            constexpr int i = I0 + (HALF ? m / TH : m % NI), jj = HALF ? m % TH : m / NI;
            constexpr int j = ((quad == 0) == (HALF == 0) ? X : Y) + jj;
            if constexpr (q == BAR) {
                __builtin_amdgcn_s_waitcnt(0xC07F);                              // lgkmcnt(0): this wave has read what the half step reads
                // its loads for the next half step's reads have landed: with two stages those of half a tile each time, with three, where
                // x and y have changed places in a stage when it is filled again, those of a whole tile in time for the first half
                wait_vmcnt<(NS == 2 || HALF) ? (NS - 1) * (LA + LB) : 2 * LA + LB>();
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_sched_barrier(0);
            }
            const intx8 b = __builtin_shufflevector(fb[j][0], fb[j][1], 0, 1, 2, 3, 4, 5, 6, 7);
            const intx8 t = __builtin_shufflevector(fa[i][0], fa[i][1], 0, 1, 2, 3, 4, 5, 6, 7);
            acc[i][j] = mfma_block<IDX, IDX>(b, t, acc[i][j], sw[FORM == GEMM_GATED && j >= TH ? 1 : 0], sx[i]);
            __builtin_amdgcn_sched_barrier(0);
            // reads, one after each MFMA of the quadrant's first ones, or as many as it takes: all are issued before the barrier, behind which
            // loads go where they read
            constexpr int NR = quad ? R1 : R0, SLOTS = quad ? BAR - NQ : NQ, PER = (NR + SLOTS - 1) / SLOTS;
            static_assert(SLOTS >= 1 && SLOTS * PER >= NR, "reads before the barrier");
            constexpr int FROM = m * PER < NR ? m * PER : NR, TO = (m + 1) * PER < NR ? (m + 1) * PER : NR;
#pragma unroll
            for (int n = FROM; n < TO; ++n) {
                if constexpr (HALF == 0 && quad == 0) read_b(Y + (n >> 1), n & 1, s);
                if constexpr (HALF == 0 && quad == 1) read_a(LO + (n >> 1), n & 1, s);
                if constexpr (HALF == 1 && quad == 0) read_a(n >> 1, n & 1, sn);
                if constexpr (HALF == 1 && quad == 1) read_b(Y + (n >> 1), n & 1, sn);
            }
            // scale words: hi's of this group in its first half step, the next group's others in its last one
            if constexpr (HALF == 0 && IDX == 0 && q == NQ) {
#pragma unroll
                for (int n = LO; n < TM; ++n) read_sx(n, sc);
            }
            if constexpr (HALF == 1 && IDX == 3 && q == 0) {
#pragma unroll
                for (int n = 0; n < LO; ++n) read_sx(n, sc_next);
                read_sw(0, sc_next, sw_next);
                if (FORM == GEMM_GATED) read_sw(1, sc_next, sw_next);
            }
#pragma unroll
            for (int l = 0; l < L; ++l)
                if (l * BAR / L == q) {
                    if (l < NA) load_a(ra, I0 + l, at, s);
                    else load_b((HALF ? Y : X) ? rb1 : rb0, (HALF ? Y : X) + l - NA, at, s);
                }
            if constexpr (HALF == 0 && IDX == 0 && q == 0) load_scales(rs, place, min((kt0 + kt + 4) >> 2, last >> 2), sc_next);
            __builtin_amdgcn_sched_barrier(0);
        };
        for_constants(slot, std::make_integer_sequence<int, NM>());
    };
    int stage = 0;                               // of the current tile, in bytes
    auto tile = [&](auto idx_c, int kt, unsigned char* sc, unsigned char* sc_next) {
        constexpr int IDX = decltype(idx_c)::value;
        unsigned char* s = smem + (NS == 2 ? (IDX & 1) * S::STAGE : stage);
        stage = stage == (NS - 1) * S::STAGE ? 0 : stage + S::STAGE;
        unsigned char* sn = smem + (NS == 2 ? (1 - (IDX & 1)) * S::STAGE : stage);
        half_step(idx_c, std::integral_constant<int, 0>(), kt, s, sn, sc, sc_next);
        half_step(idx_c, std::integral_constant<int, 1>(), kt, s, sn, sc, sc_next);
    };
    int flip = 0;
    for (int kt = 0; kt < nk; kt += 4) {
        unsigned char *sc = scale_lds + flip, *sc_next = scale_lds + (S::SCALES - flip);
        flip = S::SCALES - flip;
        __builtin_amdgcn_sched_barrier(0);
        tile(std::integral_constant<int, 0>(), kt, sc, sc_next);
        if (kt + 1 >= nk) break;
        tile(std::integral_constant<int, 1>(), kt + 1, sc, sc_next);
        if (kt + 2 >= nk) break;
        tile(std::integral_constant<int, 2>(), kt + 2, sc, sc_next);
        if (kt + 3 >= nk) break;
        tile(std::integral_constant<int, 3>(), kt + 3, sc, sc_next);
        sw[0] = sw_next[0];
        if (FORM == GEMM_GATED) sw[1] = sw_next[1];
#pragma unroll
        for (int i = 0; i < TM; ++i)                 // keep the accumulators in the accumulation registers across the back edge
#pragma unroll
            for (int j = 0; j < TN; ++j) asm volatile("" : "+a"(acc[i][j]));
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);              // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();                    // all waves have read what they read of LDS
    const Place done = place;
    item += step_item;
    const bool more = item < end_item;
    if (more) {
        place = place_of(item);
        begin(place);
    }
    __builtin_amdgcn_sched_barrier(0);

    // lane: token l % 16 of fragment i, features 4 * (l / 16) .. + 3 of fragment j. (The offsets of the stores are the same for each of a
    // workgroup's tiles; made from what the compiler cannot know to be, they take no registers while the next one is computed.)
    int lane_now = lane;
    asm volatile("" : "+v"(lane_now));
    const int row16 = lane_now & 15, quarter = lane_now >> 4;
    const int64_t row0 = int64_t(done.row_tile) * S::BM;
    const int tile_rows = rows_of(done), col_tile = done.col_tile;
    const int64_t token0 = row0 + wm * TM * 16 + row16;
    if constexpr (FORM == GEMM_GATED) {
        constexpr unsigned OUT = 0x80000000u;        // out of bounds: not stored
        unsigned* top = reinterpret_cast<unsigned*>(smem + NS * S::STAGE + 2 * S::SCALES);               // [wave column][token]
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int j = 0; j < TN; ++j) asm volatile("" : "+a"(acc[i][j]));
            __builtin_amdgcn_sched_barrier(0);
            unsigned m = 0;
#pragma unroll
            for (int j = 0; j < TH; ++j) {
                acc[i][j] = gate_value(acc[i][j], acc[i][TH + j]);
                m = max(m, magnitude4(acc[i][j]));
            }
            m = max(m, unsigned(__shfl_xor(int(m), 16)));
            m = max(m, unsigned(__shfl_xor(int(m), 32)));
            if (lane_now < 16) top[wn * S::BM + wm * TM * 16 + i * 16 + lane_now] = m;
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xC07F);          // (no __syncthreads(): it would wait for the next tile's loads)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc(a.out_codes + row0 * a.out_code_stride + col_tile * kBlock, 0, 0x7fffffff, RSRC);
        const __amdgpu_buffer_rsrc_t re = __builtin_amdgcn_make_buffer_rsrc(a.out_scales + row0 * a.out_scale_stride, 0, 0x7fffffff, RSRC);
        const int out_stride = int(a.out_code_stride), out_scale_stride = int(a.out_scale_stride);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int row = wm * TM * 16 + i * 16 + row16;
            const unsigned byte = scale_byte(max(top[row], top[S::BM + row]));
            const float inv = inverse_scale(byte);
            unsigned d[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) d[j] = codes4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3], inv);
            // 4 x 4 words between the four rows of lanes: row q ends up with the 16 features of fragment q
            const auto u = __builtin_amdgcn_permlane32_swap(d[0], d[2], false, false), v = __builtin_amdgcn_permlane32_swap(d[1], d[3], false, false);
            const auto lo = __builtin_amdgcn_permlane16_swap(u[0], v[0], false, false), hi = __builtin_amdgcn_permlane16_swap(u[1], v[1], false, false);
            const bool there = row < tile_rows;
            const uintx4 o = {lo[0], lo[1], hi[0], hi[1]};
            __builtin_amdgcn_raw_buffer_store_b128(o, rc, int(there ? unsigned(row * out_stride + wn * 64 + quarter * 16) : OUT), 0, 0);
            __builtin_amdgcn_raw_buffer_store_b8(static_cast<unsigned char>(byte), re, int(there && wn == 0 && quarter == 0 ? unsigned(row * out_scale_stride + col_tile) : OUT), 0, 0);
            if (col_tile == 0 && a.spare)
                __builtin_amdgcn_raw_buffer_store_b8(0, re, int(there && wn == 0 && quarter < a.spare ? unsigned(row * out_scale_stride + (a.f_pieces >> 3) + quarter) : OUT), 0, 0);
        }
    } else if constexpr (FORM == GEMM_PARTIAL) {
        const int piece0 = first(done, 0) + wn * TN;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t token = token0 + i * 16;
            float* p = a.partial + (int64_t(done.split) * a.tokens + token) * a.ld + piece0 * 16 + quarter * 4;
#pragma unroll
            for (int j = 0; j < TN; ++j) asm volatile("" : "+a"(acc[i][j]));
            __builtin_amdgcn_sched_barrier(0);
            if (token < a.tokens) {
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    if (piece0 + j < all_pieces) *reinterpret_cast<floatx4*>(p + j * 16) = acc[i][j];
            }
        }
    } else {
        const int piece0 = first(done, 0) + wn * TN;
        // two neighbouring fragments: two lane swaps make 8 consecutive features of a token, 64 bytes of each row at a time
        auto pack = [](float u, float v) {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            bf16x2 h;
            h[0] = bf16_t(u);
            h[1] = bf16_t(v);
            return __builtin_bit_cast(unsigned, h);
        };
        const int in32 = 16 * (lane_now >> 5) + 8 * ((lane_now >> 4) & 1);
        // a run of 32 features is within one tensor: where it goes, and how many of its features there are, is the same for the wave
        int col[TH], left[TH];
#pragma unroll
        for (int j = 0; j < TH; ++j) {
            const int piece = piece0 + 2 * j, tensor = piece / a.f_pieces, feature = (piece - tensor * a.f_pieces) * 16;
            col[j] = __builtin_amdgcn_readfirstlane(tensor * a.features + feature);
            left[j] = __builtin_amdgcn_readfirstlane(tensor < a.tensors ? a.features - feature : 0);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t token = token0 + i * 16;
            const int row = wm * TM * 16 + i * 16 + row16;
            bf16_t* y = static_cast<bf16_t*>(a.y) + token * a.y_stride + in32;
#pragma unroll
            for (int j = 0; j < TN; ++j) asm volatile("" : "+a"(acc[i][j]));
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < TH; ++j) {
                const floatx4 &p = acc[i][2 * j], &q = acc[i][2 * j + 1];
                const auto s0 = __builtin_amdgcn_permlane32_swap(pack(p[0], p[1]), pack(q[0], q[1]), false, false);
                const auto s1 = __builtin_amdgcn_permlane32_swap(pack(p[2], p[3]), pack(q[2], q[3]), false, false);
                const auto t0 = __builtin_amdgcn_permlane16_swap(s0[0], s0[1], false, false), t1 = __builtin_amdgcn_permlane16_swap(s1[0], s1[1], false, false);
                const uintx4 o = {t0[0], t1[0], t0[1], t1[1]};
                const int n = left[j] - in32;
                if (row >= tile_rows || n <= 0) continue;
                bf16_t* to = y + col[j];
                if (n >= 8) {
                    __builtin_memcpy(to, &o, 16);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < n) reinterpret_cast<unsigned short*>(to)[e] = static_cast<unsigned short>(o[e >> 1] >> (16 * (e & 1)));
                }
            }
        }
    }
    if (!more) break;
    }
    wait_vmcnt<0>();                                 // no load into LDS outlives the workgroup
}
#endif

template <int TM, int TN, int FORM>
__global__ void __launch_bounds__(256, 1) gemm_kernel(GemmArgs g) {
#ifdef __HIP_DEVICE_COMPILE__
    gemm_tile<TM, TN, FORM>(g);
#endif
}

// The ranges of K added up in order: a thread takes 4 neighbouring features of a token.
__global__ void __launch_bounds__(256) gemm_reduce_kernel(LinearArgs a) {
    const int64_t per_token = a.ld / 4, all = a.tokens * per_token, step = a.tokens * a.ld;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
        const int64_t token = i / per_token;
        const int f4 = int(i - token * per_token) * 4, tensor = f4 / (a.f_pieces * 16), f = f4 - tensor * a.f_pieces * 16;
        const float* p = a.partial + token * a.ld + f4;
        floatx4 v = *reinterpret_cast<const floatx4*>(p);
        for (int s = 1; s < a.n_split; ++s) v += *reinterpret_cast<const floatx4*>(p + s * step);
        store4(static_cast<bf16_t*>(a.y) + token * a.y_stride + int64_t(tensor) * a.features + f, a.features - f, v);
    }
}

// The same for gate and up, then silu(gate) * up in 8 bits: 16 lanes to a block of 128 features, all of them there.
__global__ void __launch_bounds__(256) gemm_reduce_gated_kernel(LinearArgs a) {
    const int64_t per_token = a.ld / 2 / kChunk, all = a.tokens * per_token, step = a.tokens * a.ld;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
        const int64_t token = i / per_token;
        const int f = int(i - token * per_token) * kChunk;
        const float* p = a.partial + token * a.ld + f;
        floatx4 v[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const float* from = p + h * (a.ld / 2) + q * 4;
                v[h][q] = *reinterpret_cast<const floatx4*>(from);
                for (int s = 1; s < a.n_split; ++s) v[h][q] += *reinterpret_cast<const floatx4*>(from + s * step);
            }
        const floatx4 h0 = gate_value(v[0][0], v[1][0]), h1 = gate_value(v[0][1], v[1][1]);
        const float h[kChunk] = {h0[0], h0[1], h0[2], h0[3], h1[0], h1[1], h1[2], h1[3]};
        unsigned char* scales = a.out_scales + token * a.out_scale_stride;
        quantise_block(h, a.out_codes + token * a.out_code_stride + f, scales + f / kBlock);
        if (f < 4 * kChunk && f / kChunk < a.spare) scales[(a.f_pieces >> 3) + f / kChunk] = 0;
    }
}
