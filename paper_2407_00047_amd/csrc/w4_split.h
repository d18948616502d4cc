// w4_split.h -- how the products of many rows (w4.hip, k_w4_wide) share the inputs
// among workgroups.  Plain host code, so that the rule can be walked without a GPU.
#pragma once

#include <algorithm>
#include <cstdint>

namespace qlm_w4_host {

constexpr int kStep = 128;           // inputs of a step

// Splits of n_in inputs: split s takes the steps s * per .. (s + 1) * per.  per is even:
// steps are taken in pairs and both of a pair are read, so only the last split may end
// inside one, and that only where the steps are odd in number, whose rows are padded with
// zeros to a whole pair.
inline void split_of(int32_t n_out, int32_t n_in, int32_t rows, int *splits, int *per)
{
    const int steps = (n_in + kStep - 1) / kStep;
    // two workgroups to a CU, eight steps each at least (48 rows, 20001 x 8192: half and
    // twice as many splits were no faster)
    const int64_t wg = ((int64_t)n_out + 63) / 64 * ((rows + 63) / 64);
    const int64_t want = std::min<int64_t>((512 + wg - 1) / wg, std::max(1, steps / 8));
    *per = (int)((steps + 2 * want - 1) / (2 * want)) * 2;
    *splits = (steps + *per - 1) / *per;
}

}  // namespace qlm_w4_host
