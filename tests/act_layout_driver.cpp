// Checks where csrc/act_layout.h lets the pieces of a checkpoint's rows be read, for every number of channels up to 2000.  Built and run
// by tests/test_act_layout.py.
#include <cstdio>
#include <initializer_list>

#include "act_layout.h"

int main() {
    for (int64_t channels = 1; channels <= 2000; ++channels) {
        const int64_t columns = ops::own_columns(channels);
        if (columns < channels || columns % 16 != 0 || columns - channels >= 16) return std::printf("own_columns(%d)\n", int(channels)), 1;
        for (int width : {8, 16})
            for (int64_t col = 0; col < channels + 512; col += width) {          // what tiles of up to 256 channels ask for
                const int64_t at = ops::piece_at(col, columns, width);
                if (at < 0 || at + width > columns || (col < channels && at != col))
                    return std::printf("%d channels: %d at %d is read at %d\n", int(channels), width, int(col), int(at)), 1;
            }
    }
    if (ops::own_columns(0) != 0) return std::puts("own_columns(0)"), 1;
    std::puts("ok");
}
