// Attention's tiles in LDS, and which bytes of memory the transfers that fill them fetch: numbers alone, for host and device, so that the
// transfers' reach can be gone through without a GPU.
#pragma once
#include <stdint.h>

namespace pac {

// ---------------------------------------------------------------------------
// Tiles of keys, values, queries or their gradients in LDS: rows of D values (padded with zeros), read in two ways.
//   along the row   16 bytes a lane, 16 rows at the same place at a time
//   turned round    ds_read_b64_tr_b16: 8 bytes a lane, four rows of 64 bytes at a time
// Both are free of bank conflicts (64 banks of 4 bytes) where 16 neighbouring rows have their 16-byte pieces in 16 different
// places of the 256-byte line, and any four rows that begin at a multiple of four have theirs in different quarters of it:
// piece c of row x lies at c ^ swz(x).
// ---------------------------------------------------------------------------
template <int D> struct AttnTile {
    static constexpr int RB = D == 96 ? 256 : 2 * D; // bytes from row to row
    static constexpr int swz(int row)
    {
        if constexpr (RB == 256) return (row & 3) << 2 | (row >> 2 & 3);
        else if constexpr (RB == 128) return (row >> 1 & 1) << 2 | (row >> 2 & 3);
        else return row >> 2 & 3;
    }
    static constexpr int at(int row, int piece) { return row * RB + ((piece ^ swz(row)) << 4); }
};

// A tile of ROWS rows in transfers of 16 bytes a lane, a wavefront's 1 KB in a row, dealt to WAVES wavefronts.  Transfer i of a lane whose first
// row is `row` fetches piece(lane, row + i RPI) of that row into the place that AttnTile gives it; heads of d values have d / 8 pieces.
template <int D, int ROWS, int WAVES> struct AttnFetch {
    using T = AttnTile<D>;
    static constexpr int P = T::RB / 16, RPI = 64 / P;                                  // pieces of a row's place, rows of a transfer
    static constexpr int TOTAL = ROWS / RPI, N = TOTAL / WAVES > 0 ? TOTAL / WAVES : 1; // (few rows: wavefronts repeat one another's transfers)
    static constexpr int first(int wave) { return wave % WAVES * N % TOTAL; }           // a wavefront's first transfer of the tile's TOTAL
    static constexpr int row(int first, int lane) { return first * RPI + lane / P; }
    static constexpr int piece(int lane, int row) { return lane % P ^ T::swz(row); }
    static constexpr uint32_t offset(int row, int piece, uint32_t row_bytes) { return (uint32_t)row * row_bytes + (uint32_t)piece * 16u; }
    // Does a lane fetch its piece: has the head as many?  (What lies behind it is the next head's, or nobody's behind the last.)
    static constexpr bool part(int piece, int d) { return piece * 8 < d; }
    // Tiles without missing rows of heads of all D values, whose lanes take part in all of their transfers or in none, as in their first
    static constexpr bool whole(int d, int have) { return d == D && have >= ROWS; }
    static constexpr bool part_of_whole(int lane, int row) { return T::RB == 2 * D || part(piece(lane, row), D); }
    static constexpr bool steady()
    {
        for (int wave = 0; wave < WAVES; ++wave)
            for (int lane = 0; lane < 64; ++lane)
                for (int i = 1; i < N; ++i) {
                    const int r = row(first(wave), lane);
                    if (part(piece(lane, r + i * RPI), D) != part(piece(lane, r), D)) return false;
                }
        return true;
    }
};

} // namespace pac
