// f8_plan.h -- which form a product in 8-bit floating point takes, and what a workgroup may load then.
#pragma once

#include <algorithm>
#include <cstdint>

namespace qlm_f8_host {

constexpr int kBlock = 128, kTile = 16, kCus = 256;
constexpr int kThinRows = 640;   // the most rows that k_f8_thin takes
// Blocks of inputs from which weights are long: between the 32 of 96 x 16384 x 4096, of which tiles of 4 x 2 are
// best, and the 128 of 96 x 4096 x 16384, of which they are not (sizes below).  What a cache still holds of
// them goes by the number of outputs as well, which this leaves out.
constexpr int kLong = 40;

// Tiles of outputs and of rows to a workgroup of k_f8_thin: as many as leave every compute unit a
// workgroup, as each tile of outputs reads the rows, and each group of rows the weights, from the
// second-level caches.  Of long weights a second group would find little there: few groups then.
// us, outputs x rows:
//                        1 x 1   1 x 2   2 x 2   4 x 2   2 x 3   2 x 4
//     20 x   300 x 16384   6.9     8.9    12.9              14
//    100 x  1000 x 8000    8.5     7.2     8.2               9.5
//     64 x  4096 x 4096    8.7     7.8     6.6     8.2       7.2     8.8
//     48 x 16384 x 4096                   14.4    14.4      13.5    14.2
//     64 x 16384 x 4096   20      18      15.2    14.7      16.7    14.8
//     96 x 16384 x 4096           25      19.5    17.1      18.5    20.7
//     96 x  4096 x 16384          26.8    24.7    21.6      18.5    20.8
struct Thin {
    int outs, rows;
};

inline Thin thin_of(int64_t n_tiles, int64_t m_tiles, int blocks)
{
    auto groups = [&](int outs, int64_t rows) {
        return (n_tiles + outs - 1) / outs * ((m_tiles + rows - 1) / rows);
    };
    if (m_tiles == 1) return {1, 1};
    const int64_t few = (m_tiles + 3) / 4, rows = (m_tiles + few - 1) / few;   // 2, 3 or 4
    if (m_tiles > 4 && blocks <= kLong && groups(4, 2) >= kCus) return {4, 2};
    if (groups(2, rows) >= kCus) return {2, (int)rows};
    if (groups(2, 2) >= kCus) return {2, 2};
    return groups(1, 2) >= kCus / 2 ? Thin{1, 2} : Thin{1, 1};
}

// side: 0 for a workgroup that reads weights and rows past shared memory (k_f8_thin), else the outputs and
// rows of a workgroup's tile (k_f8_wide).  The blocks of inputs go in `splits` runs of per_split.
struct Plan {
    int side, splits, per_split;
    double us;                   // the estimate
    bool one_more;               // tiles of 256 take a last tile of 16 rows with them
};

// The form of the least estimated time.  Measured on an MI355X (us; memory 5.1 TB/s, launches of
// 6 us and a second one of 4 as a caller of single products sees them):
//   thin    the weights' bytes, or both operands' from the second-level caches at 25 TB/s; half of the
//           weights' bytes for each further group of rows where they are long; 3.9 for every 512
//           workgroups
//   tiles   a block of inputs takes a compute unit 0.19 for a tile of 64 x 64 (0.3 for one alone),
//           0.48 of 128 x 128 (0.56 alone, 0.40 for one of two), 1.5 of 256 x 256, a tile of which
//           takes 3 to begin and end; 1.65 and 6 of 256 with a last tile of 16 rows beside it
//           (one_more); then the outputs are written
// so (rows x outputs x inputs, thin / 64 / 128 / 256):
//     128 x  4096 x 4096     8.6 /  13.3 /  16.2 /  49
//     256 x  4096 x 4096    12.3 /  13.4 /  18   /  49
//     128 x 16384 x 4096    20.2 /  18.4 /  -    /  -
//     256 x 16384 x 4096     -   /  31.6 /  24.0 /  50
//    1500 x  4096 x 4096     -   /  42   /  33.2 /  51
//     779 x  6531 x 8056     -   /  -    /  57   /  -
//     347 x  9961 x 805     17.8 /  13.9 /  10.8 /  -
//    1178 x 19884 x 896      -   /  60   /  39.8 /  48.5
//    3672 x   638 x 1080    21   /  11.6 /  10.9 /  -
//    2000 x 16384 x 4096     -   /  -    / 152   / 119
//    4096 x  4096 x 4096     -   /  -    /  72   /  61
// and in four runs of the inputs: 96 x 4096 x 16384 by tiles of 64 36 and 22 us, 3414 x 300 x 13578
// by tiles of 128 56 and 33.
inline Plan form_of(int n_out, int n_in, int n_rows, int most_splits = 16)
{
    const int blocks = (n_in + kBlock - 1) / kBlock;
    const int64_t n_tiles = ((int64_t)n_out + kTile - 1) / kTile;
    const int64_t m_tiles = ((int64_t)n_rows + kTile - 1) / kTile;
    const double tile = (double)kBlock * kTile * blocks;        // bytes of a tile of 16 rows
    Plan best{0, 1, blocks, 1e30, false};
    if (n_rows <= kThinRows) {
        const Thin thin = thin_of(n_tiles, m_tiles, blocks);
        const double groups = (double)((m_tiles + thin.rows - 1) / thin.rows);
        const double reads = n_tiles * groups +
                             (double)m_tiles * ((n_tiles + thin.outs - 1) / thin.outs);
        const double again = blocks > kLong ? 1 + 0.5 * (groups - 1) : 1;
        const double begun = groups * (double)((n_tiles + thin.outs - 1) / thin.outs) / (2 * kCus);
        best.us = 4.5 + std::max({n_tiles * tile / 5.1e6 * again, reads * tile / 25e6, 3.9 * begun});
    }
    const double out = 2.0 * n_out * (double)n_rows / 5.1e6;
    const struct {
        int side;
        double one, two, more;        // us of a block with so many tiles to a compute unit, for each
    } forms[] = {{64, 0.30, 0.19, 0.19}, {128, 0.56, 0.40, 0.48}, {256, 1.5, 1.5, 1.5}};
    for (auto f : forms) {
        // (offsets of 32 bits into a workgroup's tiles)
        if (tile * (f.side / kTile) >= 2147483648.0) continue;
        const bool one_more = f.side == 256 && m_tiles > 16 && m_tiles % 16 == 1;
        const double tiles = (double)((n_out + (int64_t)f.side - 1) / f.side) *
                             (double)((n_rows + (int64_t)f.side - 1) / f.side - one_more);
        for (int s = 1; s <= most_splits; s *= 2) {
            const int per = (blocks + s - 1) / s;
            if (s > 1 && per < 4) break;
            const int runs = (blocks + per - 1) / per;
            const double turns = (double)(int64_t)((tiles * runs + kCus - 1) / kCus);
            const double cost =
                turns * (one_more ? 1.65 : turns <= 1 ? f.one : turns <= 2 ? f.two : f.more);
            const double ends = f.side < 256 ? 0.0 : one_more ? 6.0 : 3.0;
            double t = 6.0 + std::max(per * cost + ends * turns + out,
                                      (n_tiles + m_tiles) * tile / 5.1e6);
            if (runs > 1) t += 4.0 + (runs + 0.5) * 4.0 * n_out * (double)n_rows / 5.1e6;
            if (t < best.us) best = {f.side, runs, per, t, one_more};
        }
    }
    return best;
}

// Bytes that a workgroup of `own` tiles of outputs (or rows) may load from its first tile's block b0 on,
// where `left` tiles are left.  (Of its own tiles and no others: form_of holds those under 2 GiB, which 16
// of the longest inputs pass.)
constexpr int load_bytes(int left, int own, int blocks, int b0)
{
    return ((left < own ? left : own) * blocks - b0) * (kBlock * kTile);
}

// The rows in two parts where that is less, the first of whole tiles of 256: a last tile of a few
// rows takes as long as a whole one.  800 x 20000 x 5000 as a whole 110 us, as 768 rows and 32
// 91.
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

// Workgroups of k_f8_thin, and of the launch that joins runs' sums, four outputs a thread.
inline int64_t thin_groups(int64_t n_tiles, int64_t m_tiles, int blocks)
{
    const Thin t = thin_of(n_tiles, m_tiles, blocks);
    return ((n_tiles + t.outs - 1) / t.outs + 7) / 8 * 8 * ((m_tiles + t.rows - 1) / t.rows);
}

inline int64_t join_groups(int n_out, int n_rows)
{
    return (n_rows * (((int64_t)n_out + 3) / 4) + 255) / 256;
}

// Whether a form's launches can be made: fewer than 2^32 threads in each, tiles counted in 32 bits.
inline bool fits(int n_out, int n_in, int n_rows, const Plan &p)
{
    auto can_launch = [](int64_t groups, int threads) { return groups < (1ll << 32) / threads; };
    if (!p.side)
        return can_launch(thin_groups(((int64_t)n_out + kTile - 1) / kTile,
                                      ((int64_t)n_rows + kTile - 1) / kTile,
                                      (n_in + kBlock - 1) / kBlock), 512);
    const int64_t tiles = ((int64_t)n_out + p.side - 1) / p.side *
                          (((int64_t)n_rows + p.side - 1) / p.side) * p.splits;
    return tiles <= INT32_MAX / 2 &&
           (p.splits == 1 || can_launch(join_groups(n_out, n_rows), 256));
}

}  // namespace qlm_f8_host
