"""CPU-only: what the transfers of attention's tiles fetch (csrc/pac_attn_tile.h), lane by lane, for every width of a head and every number of
rows: pieces of the matrix's own rows alone, each into its place."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "pac_attn_tile.h"
#include <stdio.h>
#include <string.h>
using namespace pac;

static int bad = 0;

template <int D, int ROWS, int WAVES> void go(int d, int have)
{
    using F = AttnFetch<D, ROWS, WAVES>;
    using T = AttnTile<D>;
    static char there[ROWS * T::RB / 16]; // places that are fetched
    memset(there, 0, sizeof there);
    const uint32_t row_bytes = 2 * d; // one head, dense: what follows its last row is not the matrix's
    const bool whole = F::whole(d, have);
    for (int wave = 0; wave < 4; ++wave)
        for (int lane = 0; lane < 64; ++lane)
            for (int i = 0; i < F::N; ++i) {
                const int first = F::first(wave), row = F::row(first, lane);
                int at = row + i * F::RPI;
                const int piece = F::piece(lane, at);
                if (!(whole ? F::part_of_whole(lane, row) : F::part(piece, d))) continue;
                const int place = first * 64 + i * 64 + lane;
                if (at >= ROWS || place * 16 != T::at(at, piece)) ++bad;
                else there[place] = 1;
                if (!whole && at >= have) at = have - 1;
                const uint64_t from = F::offset(at, piece, row_bytes);
                if (from < (uint64_t)at * row_bytes || from + 16 > (uint64_t)(at + 1) * row_bytes || from + 16 > (uint64_t)have * row_bytes) {
                    if (bad++ < 4) printf("D %d, %d rows, %d wavefronts, d %d, have %d: row %d, byte %lld of %d\n", D, ROWS, WAVES, d, have, at,
                                          (long long)(from - (uint64_t)at * row_bytes), (int)row_bytes);
                }
            }
    for (int row = 0; row < ROWS; ++row)
        for (int piece = 0; piece * 8 < d; ++piece)
            if (!there[T::at(row, piece) / 16]) ++bad;
}
template <int D> void width(int from)
{
    for (int d = from; d <= D; d += 8)
        for (int have = 1; have <= 200; ++have) {
            go<D, 64, 4>(d, have);
            go<D, 32, 4>(d, have);
            go<D, 32, 1>(d, have);
            go<D, 128, 4>(d, have);
        }
}
int main()
{
    width<32>(8);
    width<64>(40);
    width<96>(72);
    width<128>(104);
    printf("%d\n", bad);
    return bad != 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no C++ compiler")
def test_transfers_stay_in_their_rows(tmp_path):
    src, exe = tmp_path / "tiles.cpp", tmp_path / "tiles"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_2408_10746_amd", "csrc"), "-o", str(exe), str(src)], check=True)
    got = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True, timeout=120)
    assert got.returncode == 0, got.stdout
