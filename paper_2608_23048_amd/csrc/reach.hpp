// reach.hpp -- offsets of loads that may run past the end of an operand, in
// plain C++, so that a host program can go through them all.
#pragma once

#include <stdint.h>

namespace roi {

// A byte offset that no buffer of the products reaches: a load from there gives
// zeros.
constexpr uint32_t kNowhere = 0x80000000u;

// What a buffer load takes beside its buffer: an offset for each lane and one for
// the wave, both unsigned.
struct LoadAt {
    uint32_t lane, wave;
};

// Byte `byte` of row `item` of a step, the rows of `row_bytes` bytes lying from the
// buffer's start on.  `rows_left` of the sum's rows are left there: past them the
// last again; past the end of the sum, where none are left (0 or fewer), nowhere.
// There the wave's offset is 0: a negative one would be a large unsigned one.
constexpr LoadAt row_load(int item, int rows_left, uint32_t byte, bool in_row, uint32_t row_bytes)
{
    if (rows_left <= 0) return LoadAt{kNowhere, 0};
    const int row = item < rows_left ? item : rows_left - 1;
    return LoadAt{in_row ? byte : kNowhere, (uint32_t)row * row_bytes};
}

} // namespace roi
