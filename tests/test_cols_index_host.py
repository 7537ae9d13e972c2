"""Tiles of products with several columns a lane (csrc/cols_index.hpp) on the CPU: the functions that the kernels call, for every tile in the library as built, through all wavefronts, loads and lanes."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2407_02031_amd", "libswiftdiff.so")

MAIN = r"""
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "cols_index.hpp"
using namespace sd;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s; tile %dx%d, %dx%d wavefronts, %d halves, M %d N %d Kb %d m0 %d n0 %d kb %d\n", __LINE__, #x, I::BM, I::BN, I::WGM, I::WGN, I::KS, M, N, Kb, m0, n0, kb); std::exit(1); } } while (0)
static long accesses = 0;

// A 16-byte chunk of an operand: which (0 P, 1 Q's values, 2 its gates), its row, its number in the row; -1: zeros
struct Chunk { int which, row, chunk; bool operator==(const Chunk& o) const { return which == o.which && row == o.row && chunk == o.chunk; } };

template <class I, bool FP8, bool GATED, bool OUT8>
static void step(int M, int N, int Kb, int m0, int n0, int kb) {
    // ---- loads
    std::vector<Chunk> lds((I::BM + I::BN) * 8, Chunk{-2, 0, 0});
    for (int wave = 0; wave < I::NW; ++wave)
        for (int j = 0; j < I::LPT; ++j)
            for (int lane = 0; lane < 64; ++lane) {
                const int eight = I::eight(j, wave), first = eight * 8, row = first + (lane >> 3), chunk = I::chunk(eight, lane);
                CHECK(eight >= 0 && eight < I::ROWS8 && chunk >= 0 && chunk < 8);
                Chunk c;
                if (I::of_p(j, first)) {
                    CHECK(first < I::BM);
                    c = Chunk{0, m0 + I::p_row(first, row, m0, M), chunk};
                    CHECK(c.row >= m0 && c.row < M);
                } else {
                    CHECK(first >= I::BM);
                    const int r = n0 + I::q_row(first, row, n0, N);
                    CHECK(r >= n0 && r < N && (GATED || !I::q_gate(first)));
                    c = Chunk{I::q_gate(first) ? 2 : 1, r, chunk};
                }
                // the offset from the tile's first row has 32 bits; whole steps do not ask whether a chunk is there
                CHECK((int64_t)(c.row - (c.which ? n0 : m0)) * ((1 << 23) - 16) + chunk * 16 < (int64_t)1 << 32);
                if (kb + 128 <= Kb) CHECK(I::there(kb, chunk, Kb));
                if (!I::there(kb, chunk, Kb)) c = Chunk{-1, 0, chunk};
                else CHECK(kb + chunk * 16 + 16 <= Kb);
                Chunk& to = lds.at(first * 8 + lane);
                CHECK(to.which == -2 || to == c);
                to = c;
                ++accesses;
            }
    for (const Chunk& c : lds) CHECK(c.which != -2);
    // ---- scales, a byte each: -1 behind the last
    std::vector<int> sp, sq;
    if (FP8) {
        sp.assign(I::BM, -2);
        sq.assign(I::BN, -2);
        for (int a = 0; a < I::PIECES * 64; ++a) {
            const bool of_p = I::scale_of_p(a);
            const int rows = of_p ? M : GATED ? 2 * N : N, at = of_p ? I::p_scale(a, m0, M) : I::q_scale(a, n0, N);
            CHECK(at >= 0 && at % 4 == 0 && at < rows);      // (four bytes from a word's start: up to the last row's word)
            for (int e = 0; e < 4; ++e) {
                if (a * 4 < I::BM) sp[a * 4 + e] = at + e;
                else if (a * 4 < I::BM + I::BN) sq[a * 4 - I::BM + e] = at + e;
            }
        }
    }
    // ---- what the lanes multiply
    std::vector<int> rows(I::BM, 0), cols(I::BN_OUT, 0);
    const Chunk zero{-1, 0, 0};
    auto same = [&](int at, int which, int row, int chunk) {
        const Chunk& got = lds.at(at);
        return I::there(kb, chunk, Kb) ? got == Chunk{which, row, chunk} : got.which == zero.which;
    };
    for (int w = 0; w < I::WGM * I::WGN; ++w) {
        const int wm = w / I::WGN * I::WM, wn = w % I::WGN * I::WN, wn_out = w % I::WGN * I::WN_OUT;
        for (int l16 = 0; l16 < 16; ++l16)
            for (int mi = 0; mi < I::MI; ++mi) {
                const int r = I::result_row(wm, mi, l16);
                CHECK(r >= 0 && r < I::BM);
                ++rows[r];
                for (int c = 0; c < 8; ++c) CHECK(same(l16 * 8 + I::p_block(wm, mi) + I::part(l16, c), 0, m0 + r < M ? m0 + r : M - 1, c));
                if (FP8 && m0 + r < M) CHECK(sp.at(I::p_scales_at(wm, mi / I::BP, l16) + mi % I::BP) == m0 + r);
            }
        // element x of a lane's 4 BQ of a group is element x / BQ of its four of block x % BQ
        for (int quad = 0; quad < 4; ++quad)
            for (int g = 0; g < I::NV / I::BQ; ++g)
                for (int x = 0; x < 4 * I::BQ; ++x)
                    for (int gate = 0; gate <= (GATED ? 1 : 0); ++gate) {
                        const int ni = (gate ? I::NV : 0) + g * I::BQ + x % I::BQ, l16 = 4 * quad + x / I::BQ, col = I::result_column(wn_out, g, quad) + x;
                        CHECK(col >= 0 && col < I::BN_OUT);
                        if (!gate) ++cols[col];
                        for (int c = 0; c < 8; ++c) CHECK(same(l16 * 8 + I::q_block(wn, ni) + I::part(l16, c), 1 + gate, n0 + col < N ? n0 + col : N - 1, c));
                        if (FP8 && n0 + col < N) CHECK(sq.at(I::q_scales_at(wn_out, ni / I::BQ, l16) - I::BM + ni % I::BQ) == n0 + col + gate * N);
                    }
    }
    for (int n : rows) CHECK(n == I::WGN);
    for (int n : cols) CHECK(n == I::WGM);
}

template <bool FP8, int BM, int BN, int WGM, int WGN, int KS, int STAGES, bool GATED, bool OUT8>
static void tile() {
    using I = ColsTileIndex<FP8, BM, BN, WGM, WGN, KS, STAGES, GATED, OUT8>;
    // N of a gated layer of 8-bit rows is a multiple of 16
    const int ns[] = {FP8 && GATED ? 16 : 1, FP8 && GATED ? 48 : 3, I::BN_OUT, I::BN_OUT + 16, 3 * I::BN_OUT - (FP8 && GATED ? 16 : 1)};
    for (int M : {1, 2, 4, 5, BM - 1, BM, BM + 3, 3 * BM - 4})
        for (int N : ns)
            for (int Kb : {16, 112, 128, 144, 240, 256})
                for (int m0 = 0; m0 < M; m0 += BM)
                    for (int n0 = 0; n0 < N; n0 += I::BN_OUT)
                        for (int kb = 0; kb < Kb; kb += 128) step<I, FP8, GATED, OUT8>(M, N, Kb, m0, n0, kb);
    if (KS == 2) {      // the halves' sums: nobody's place is another's, all inside the stages, and each is read by who finishes it
        const int M = 0, N = 0, Kb = 0, m0 = 0, n0 = 0, kb = 0, sums = I::MI / 2 * I::NI;
        std::vector<int> from(STAGES * I::STAGE, -1);
        auto id = [](int w, int half, int i, int lane) { return ((w * 2 + half) * 1000 + i) * 64 + lane; };
        for (int w = 0; w < WGM * WGN; ++w)
            for (int half = 0; half < 2; ++half)
                for (int i = 0; i < sums; ++i)
                    for (int lane = 0; lane < 64; ++lane) {
                        int& to = from.at(I::meet(w, 0, 0, lane) + I::meet(0, 1 - half, i, 0));
                        CHECK(to == -1);
                        to = id(w, half, i, lane);
                    }
        for (int w = 0; w < WGM * WGN; ++w)
            for (int half = 0; half < 2; ++half)
                for (int i = 0; i < sums; ++i)
                    for (int lane = 0; lane < 64; ++lane) CHECK(from.at(I::meet(w, 0, 0, lane) + I::meet(0, half, i, 0)) == id(w, 1 - half, i, lane));
    }
}

int main() {
    TILES
    std::printf("%ld accesses\n", accesses);
    return 0;
}
"""


def tiles():
    """Template arguments of every tile in the library as built: mode, rows, columns, wavefronts, halves, stages, gated, to 8 bits"""
    if not os.path.exists(LIB):
        from paper_2407_02031_amd import build
        build.build(verbose=False)
    found = re.findall(rb"_ZN2sd11cols_kernelILi(\d)ELi(\d+)ELi(\d+)ELi(\d)ELi(\d)ELi(\d)ELi(\d)ELb(\d)ELb(\d)ELb\dEE", open(LIB, "rb").read())
    return sorted({tuple(map(int, t)) for t in found})


def test_every_chunk_and_scale_is_loaded_from_inside_and_found_again(tmp_path):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no g++")
    all_ = tiles()
    assert len(all_) >= 30 and {t[5] for t in all_} == {1, 2} and {t[0] for t in all_} == {0, 1, 2}
    calls = sorted({f"tile<{str(m > 0).lower()}, {bm}, {bn}, {wm}, {wn}, {ks}, {st}, {str(bool(g)).lower()}, {str(bool(o)).lower()}>();" for m, bm, bn, wm, wn, ks, st, g, o in all_})
    src, exe = tmp_path / "cols.cpp", tmp_path / "cols"
    src.write_text(MAIN.replace("    TILES", "\n".join("    " + c for c in calls)))
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "paper_2407_02031_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout
    assert int(r.stdout.split()[0]) > 10 ** 6
