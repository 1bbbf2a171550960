// Columns of an 8-bit checkpoint: what of its memory belongs to it.  Plain C++, for the host and the device.
#ifndef MGWFBP_ACT_LAYOUT_H
#define MGWFBP_ACT_LAYOUT_H

#include <cstdint>

namespace ops {

// Columns of q and scale that are a checkpoint's own: channels up to the next multiple of 16.  Those behind them, up to ld, may be
// another's.
constexpr int64_t own_columns(int64_t channels) { return (channels + 15) / 16 * 16; }

}  // namespace ops

#endif
