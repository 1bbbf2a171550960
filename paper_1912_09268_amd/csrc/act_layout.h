// Columns of an 8-bit checkpoint: what of its memory belongs to it.  Plain C++, for the host and the device.
#ifndef MGWFBP_ACT_LAYOUT_H
#define MGWFBP_ACT_LAYOUT_H

#include <cstdint>

namespace ops {

// Columns of q and scale that are a checkpoint's own: channels up to the next multiple of 16.  Those behind them, up to ld, may be
// another's.
constexpr int64_t own_columns(int64_t channels) { return (channels + 15) / 16 * 16; }

// Where a piece of `width` columns (8 or 16) is read that a tile wants at `col`: there, or the last one among the own columns, since
// behind the last row's there may be no memory.  Without columns there is nothing to read.
constexpr int64_t piece_at(int64_t col, int64_t columns, int width) { return col < columns - width ? col : columns - width; }

}  // namespace ops

#endif
