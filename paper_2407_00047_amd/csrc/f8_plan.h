// f8_plan.h -- which form a product in 8-bit floating point takes (host only).
#pragma once

#include <algorithm>
#include <cstdint>

namespace qlm_f8_host {

constexpr int kBlock = 128, kTile = 16, kCus = 256;

// side: 0 for 16 outputs to a workgroup that reads the rows itself (k_f8_thin), else the outputs and
// rows of a workgroup's tile (k_f8_wide).  The blocks of inputs go in `splits` runs of per_split.
struct Plan {
    int side, splits, per_split;
    double us;                   // the estimate
};

// The form of the least estimated time.  Measured on an MI355X (us; memory 5.1 TB/s, launches of
// 6 us and a second one of 4 as a caller of single products sees them):
//   thin    the weights' bytes, or both operands' from the second-level caches at 25 TB/s: 4096 x
//           4096 at 64 rows 7.4 and at 128 9.7, 16384 x 4096 at 64 rows 18.5
//   tiles   a block of inputs takes a compute unit 0.19 for a tile of 64 x 64, 0.53 of 128 x 128
//           and 1.87 of 256 x 256; alone there a tile waits for its loads, 0.23 and 0.56
// so (rows x outputs x inputs, thin / 64 / 128 / 256):
//     128 x  4096 x 4096     9.7 /  13.3 /  16.2 /  49
//     256 x  4096 x 4096    16.4 /  13.4 /  18   /  49
//     256 x 16384 x 4096     -   /  31.6 /  24.0 /  50
//    1500 x  4096 x 4096     -   /  42   /  33.2 /  51
//    2000 x 16384 x 4096     -   /  -    / 152   / 119
//    4096 x  4096 x 4096     -   /  -    /  72   /  61
// and in runs, 96 x 4096 x 16384 36 as it is and 22 in 4 (tiles of 64).
inline Plan form_of(int n_out, int n_in, int n_rows, int most_splits = 16)
{
    const int blocks = (n_in + kBlock - 1) / kBlock;
    const int64_t n_tiles = ((int64_t)n_out + kTile - 1) / kTile;
    const int64_t m_tiles = ((int64_t)n_rows + kTile - 1) / kTile;
    const double tile = (double)kBlock * kTile * blocks;        // bytes of a tile of 16 rows
    const double groups = (double)((m_tiles + 3) / 4);
    Plan best{0, 1, blocks, 5.0 + std::max(n_tiles * tile / 5.1e6,
                                           n_tiles * tile * (m_tiles + groups) / 25e6)};
    const struct {
        int side;
        double cost, alone;
    } forms[] = {{64, 0.19, 0.23}, {128, 0.53, 0.56}, {256, 1.87, 1.87}};
    for (auto f : forms) {
        // (offsets of 32 bits into a workgroup's tiles)
        if (tile * (f.side / kTile) >= 2147483648.0) continue;
        const double tiles = (double)((n_out + (int64_t)f.side - 1) / f.side) *
                             (double)((n_rows + (int64_t)f.side - 1) / f.side);
        for (int s = 1; s <= most_splits; s *= 2) {
            const int per = (blocks + s - 1) / s;
            if (s > 1 && per < 4) break;
            const int runs = (blocks + per - 1) / per;
            const double turns = (double)(int64_t)((tiles * runs + kCus - 1) / kCus);
            double t = 6.0 + std::max(per * std::max(f.alone, f.cost * turns),
                                      (n_tiles + m_tiles) * tile / 5.1e6);
            if (runs > 1) t += 4.0 + (runs + 0.5) * 4.0 * n_out * (double)n_rows / 5.1e6;
            if (t < best.us) best = {f.side, runs, per, t};
        }
    }
    return best;
}

// The rows in two parts where that is less, the first of whole tiles of 256: a last tile of a few
// rows takes as long as a whole one.  777 x 20001 x 5000 as a whole 113 us, as 768 rows and 9
// 97.
struct Parts {
    int n_first;                 // rows of the first part
    Plan first, rest;            // (rest: of no rows where n_first is all of them)
};

inline Parts parts_of(int n_out, int n_in, int n_rows)
{
    const Plan whole = form_of(n_out, n_in, n_rows);
    const int n_first = n_rows / 256 * 256;
    if (n_first > 0 && n_first < n_rows) {
        const Plan first = form_of(n_out, n_in, n_first, 1);
        const Plan rest = form_of(n_out, n_in, n_rows - n_first, 1);
        // (a second launch follows the first without a caller's share of either)
        if (first.us + rest.us - 3.0 < whole.us)
            return {n_first, first, rest};
    }
    return {n_rows, whole, whole};
}

}  // namespace qlm_f8_host
