// Whether matrices share memory, of their addresses alone.  Plain C++, for the host.
#ifndef MGWFBP_SPANS_H
#define MGWFBP_SPANS_H

#include <algorithm>
#include <cstdint>

namespace ops {

// A matrix in memory: `rows` rows of `width` bytes that begin `stride` bytes apart (any value for a single row).  Null or without bytes: nothing.
// rows * stride has to fit 62 bits, and stride to be the width or more.
struct Span {
    const void* p;
    int64_t rows, width, stride;
    bool none() const { return p == nullptr || rows <= 0 || width <= 0; }
    int64_t bytes() const { return rows > 1 ? (rows - 1) * stride + width : width; }
};
inline Span vector_span(const void* p, int64_t n, int64_t elem_bytes) { return {p, 1, n * elem_bytes, 0}; }
// In elements; of a matrix that is left out the stride may be any number.
inline Span matrix_span(const void* p, int64_t rows, int64_t width, int64_t stride, int64_t elem_bytes) {
    return {p, rows, width * elem_bytes, p != nullptr && width > 0 && rows > 1 ? stride * elem_bytes : 0};
}

// Whether a byte is in a row of both.  Matrices whose rows are at one distance may lie beside each other in the same rows (parts of one product);
// where the distances differ, their ranges have to be apart.
inline bool share(const Span& a, const Span& b) {
    if (a.none() || b.none()) return false;
    const int64_t behind = static_cast<int64_t>(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p));
    if (behind >= a.bytes() || behind <= -b.bytes()) return false;
    if (a.rows > 1 && b.rows > 1 && a.stride != b.stride) return true;
    // A row of b begins behind + m * step bytes behind one of a, -a.rows < m < b.rows; they share a byte if that is within -b.width .. a.width,
    // both excluded.
    const int64_t step = a.rows > 1 ? a.stride : b.rows > 1 ? b.stride : 1;
    const auto floor_div = [step](int64_t x) { return x >= 0 ? x / step : -((-x + step - 1) / step); };
    const int64_t least = std::max(1 - a.rows, floor_div(-b.width - behind) + 1), most = std::min(b.rows - 1, -floor_div(behind - a.width) - 1);
    return least <= most;
}
// The same elements in the same places.
inline bool same(const Span& a, const Span& b) { return a.p == b.p && a.rows == b.rows && a.width == b.width && (a.rows <= 1 || a.stride == b.stride); }

// What a call reads; bit i of `under`: its i-th output may lie over it, as a whole.
struct Read {
    Span span;
    uint32_t under;
};
// Whether outputs share memory with each other, or with what is read in other ways than those.  Nearly always all ranges are apart, and that is seen from
// their ends: some 20 ns a call.
template <int W, int R> bool tangled(const Span (&writes)[W], const Read (&reads)[R]) {
    uintptr_t begin[W + R], end[W + R];
    const auto range = [&](const Span& s, int i) {
        begin[i] = reinterpret_cast<uintptr_t>(s.p);
        end[i] = s.none() ? 0 : begin[i] + static_cast<uintptr_t>(s.bytes());
    };
    for (int w = 0; w < W; ++w) range(writes[w], w);
    for (int r = 0; r < R; ++r) range(reads[r].span, W + r);
    for (int w = 0; w < W; ++w)
        for (int o = w + 1; o < W + R; ++o) {
            if (begin[o] >= end[w] || begin[w] >= end[o]) continue;
            const Span& other = o < W ? writes[o] : reads[o - W].span;
            if (o >= W && (reads[o - W].under >> w & 1) != 0 && same(writes[w], other)) continue;
            if (share(writes[w], other)) return true;
        }
    return false;
}

}  // namespace ops

#endif
