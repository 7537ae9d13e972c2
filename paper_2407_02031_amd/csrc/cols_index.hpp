// What a tile of gemm_cols.hpp loads into which place of LDS, and where its wavefronts find it again, as functions of whole numbers alone: the kernels call them, and so does a program on the CPU that goes through
// all lanes, loads and steps of every tile.
#pragma once
#include "swizzle.hpp"

namespace sd {

// Which row of 16 B rows is row i of block b: every B-th
template <int B>
SD_INDEX_FN constexpr int spread(int b, int i) { return b / B * (16 * B) + B * i + b % B; }

template <bool FP8, int BM_, int BN_, int WGM_, int WGN_, int KS_, int STAGES_, bool GATED, bool OUT8>
struct ColsTileIndex {
    static constexpr int BM = BM_, BN = BN_, WGM = WGM_, WGN = WGN_, KS = KS_, STAGES = STAGES_;
    static constexpr int NW = WGM * WGN * KS, WM = BM / WGM, WN = BN / WGN, MI = WM / 16, NI = WN / 16;
    static constexpr int ROWS8 = (BM + BN) / 8, LPT = (ROWS8 + NW - 1) / NW;      // loads of a step, and of a wavefront
    static constexpr bool EVEN = BM / 8 % NW == 0 && BN / 8 % NW == 0;            // (where not, some are made twice, and a wavefront's are of P or of Q as its number says)
    static constexpr int NV = GATED ? NI / 2 : NI;                                // blocks of columns of the result
    static constexpr int BP = MI % 4 == 0 ? 4 : 2, BQ = OUT8 ? 4 : 2;
    static constexpr int BN_OUT = GATED ? BN / 2 : BN, WN_OUT = GATED ? WN / 2 : WN;
    static constexpr int PIECES = FP8 ? (BM + BN + 255) / 256 : 0;                // of a step's scales: a word a lane
    static constexpr int STAGE = (BM + BN) * 8 + PIECES * 16;                     // 16-byte chunks

    // Load j of a wavefront fills rows 8 eight .. + 8 of a stage, lane l the chunk at position l % 8 of row l / 8
    SD_INDEX_FN static constexpr int eight(int j, int wave) { return EVEN || j * NW + wave < ROWS8 - 1 ? j * NW + wave : ROWS8 - 1; }
    SD_INDEX_FN static constexpr bool of_p(int j, int first) { return EVEN ? j < BM / 8 / NW : first < BM; }
    // ... which of a row's chunks that is
    SD_INDEX_FN static constexpr int chunk(int eight, int lane) { return swz<8>(eight * 8 + (lane >> 3), lane & 7); }
    // ... and which row, counted from the tile's first of P, or of Q's values or gates; those of the tile behind the matrix's last are that one
    SD_INDEX_FN static constexpr int p_row(int first, int row, int m0, int M) {
        const int r = m0 + first / WM * WM + spread<BP>(first % WM / 16, row % 16);
        return (r < M ? r : M - 1) - m0;
    }
    SD_INDEX_FN static constexpr bool q_gate(int first) { return GATED && (first - BM) % WN / 16 >= NV; }
    SD_INDEX_FN static constexpr int q_row(int first, int row, int n0, int N) {
        const int b = (first - BM) % WN / 16, r = n0 + (first - BM) / WN * WN_OUT + spread<BQ>(q_gate(first) ? b - NV : b, row % 16);
        return (r < N ? r : N - 1) - n0;
    }
    // Scales: word a of a stage has those of rows 4 a .. 4 a + 3 of P's, then of Q's (values, gates); past the last row, the last word that there is.  Whether it is P's; the first row of the word.
    SD_INDEX_FN static constexpr bool scale_of_p(int a) { return a * 4 < BM || a * 4 >= BM + BN; }
    SD_INDEX_FN static constexpr int p_scale(int a, int m0, int M) {
        const int r = m0 + (a * 4 < BM ? a * 4 : 0), last = (M - 1) & ~3;
        return r < last ? r : last;
    }
    SD_INDEX_FN static constexpr int q_scale(int a, int n0, int N) {
        const int j = a * 4 - BM, r = n0 + (GATED && j >= BN_OUT ? N + j - BN_OUT : j), last = ((GATED ? 2 * N : N) - 1) & ~3;
        return r < last ? r : last;
    }
    // Whether a chunk of the step that begins at byte kb of a row is there (a row is a multiple of 16 bytes)
    SD_INDEX_FN static constexpr bool there(int kb, int chunk, int Kb) { return kb + chunk * 16 < Kb; }

    // Where a lane finds what it multiplies: chunk c of row l16 of P's block mi, or Q's block ni, is in the stage's chunk l16 * 8 + p_block + part, or q_block
    SD_INDEX_FN static constexpr int p_block(int wm, int mi) { return (wm + mi * 16) * 8; }
    SD_INDEX_FN static constexpr int q_block(int wn, int ni) { return (BM + wn + ni * 16) * 8; }
    SD_INDEX_FN static constexpr int part(int l16, int c) { return c ^ swz<8>(l16, 0); }
    // ... and the byte of a stage's scales at which those of its rows of BP blocks of P from BP i on, or BQ of Q, begin
    SD_INDEX_FN static constexpr int p_scales_at(int wm, int i, int l16) { return wm + i * 16 * BP + BP * l16; }
    SD_INDEX_FN static constexpr int q_scales_at(int wn_out, int i, int l16) {
        const bool gate = GATED && i >= NV / BQ;
        return BM + wn_out + (gate ? BN_OUT : 0) + (gate ? i - NV / BQ : i) * 16 * BQ + BQ * l16;
    }
    // Halves of steps (KS = 2): the place, among the stages, of sum i of those that half `of` finishes and wavefront w of the other half has
    SD_INDEX_FN static constexpr int meet(int w, int of, int i, int lane) { return w * (MI * NI * 64) + (of * (MI / KS) * NI + i) * 64 + lane; }
    // Rows and columns of the result that a lane has: of P's block mi, and of a group of 16 BQ columns the 4 BQ from here on
    SD_INDEX_FN static constexpr int result_row(int wm, int mi, int l16) { return wm + spread<BP>(mi, l16); }
    SD_INDEX_FN static constexpr int result_column(int wn_out, int group, int quad) { return wn_out + (group * 4 + quad) * 4 * BQ; }
};

}  // namespace sd
