// Checks csrc/spans.h against a map of the bytes, for small matrices in every position to each other.  Built and run by tests/test_spans.py.
#include <cstdio>
#include <cstring>

#include "spans.h"

using ops::Span;

static bool by_bytes(const Span& a, const Span& b, const char* base) {
    static bool held[4096];
    std::memset(held, 0, sizeof held);
    const auto at = [base](const Span& s, int64_t row, int64_t i) { return static_cast<const char*>(s.p) - base + row * s.stride + i; };
    for (int64_t r = 0; r < a.rows; ++r)
        for (int64_t i = 0; i < a.width; ++i) held[at(a, r, i)] = true;
    for (int64_t r = 0; r < b.rows; ++r)
        for (int64_t i = 0; i < b.width; ++i)
            if (held[at(b, r, i)]) return true;
    return false;
}

int main() {
    static char memory[4096];
    long shared = 0, apart = 0;
    for (int stride = 1; stride <= 7; ++stride)
        for (int rows_a = 1; rows_a <= 4; ++rows_a)
            for (int rows_b = 1; rows_b <= 4; ++rows_b)
                for (int width_a = 1; width_a <= (rows_a == 1 ? 9 : stride); ++width_a)
                    for (int width_b = 1; width_b <= (rows_b == 1 ? 9 : stride); ++width_b)
                        for (int shift = -40; shift <= 40; ++shift) {
                            const Span a{memory + 1000, rows_a, width_a, rows_a == 1 ? -12345 : stride}, b{memory + 1000 + shift, rows_b, width_b, rows_b == 1 ? 99999 : stride};
                            Span a1 = a, b1 = b;
                            if (rows_a == 1) a1.stride = width_a;
                            if (rows_b == 1) b1.stride = width_b;
                            const bool want = by_bytes(a1, b1, memory);
                            if (ops::share(a, b) != want || ops::share(b, a) != want)
                                return std::printf("stride %d rows %d %d widths %d %d shift %d: %d\n", stride, rows_a, rows_b, width_a, width_b, shift, want), 1;
                            ++(want ? shared : apart);
                        }
    // rows at two distances: apart only if their ranges are
    for (int shift = -60; shift <= 60; ++shift) {
        const Span a{memory + 1000, 3, 2, 10}, b{memory + 1000 + shift, 4, 2, 7};
        if (ops::share(a, b) != (shift < 22 && shift > -23) || (!ops::share(a, b) && by_bytes(a, b, memory))) return std::printf("two distances, %d\n", shift), 1;
    }
    const Span whole{memory, 3, 8, 16}, half{memory, 3, 4, 16}, other{memory + 4, 3, 4, 16}, none{nullptr, 3, 8, 16}, empty{memory, 0, 8, 16};
    const bool lies[] = {ops::tangled({whole}, {{whole, 1}}),         ops::tangled({none, whole}, {{whole, 2}}), ops::tangled({half, other}, {{half, 1}, {other, 2}}),
                         ops::tangled({none, empty}, {{whole, 0}}),   ops::tangled({half}, {{other, 0}, {none, 0}})};
    const bool tangles[] = {ops::tangled({whole}, {{whole, 0}}),      ops::tangled({none, whole}, {{whole, 1}}), ops::tangled({half}, {{whole, 1}}),
                            ops::tangled({whole, other}, {{none, 0}}),       ops::tangled({half, half}, {{none, 0}}),            ops::tangled({half, other}, {{half, 2}})};
    for (bool t : lies)
        if (t) return std::puts("what lies well is refused"), 1;
    for (bool t : tangles)
        if (!t) return std::puts("what is tangled is taken"), 1;
    // far apart and far wide: nothing overflows
    const Span low{reinterpret_cast<const void*>(uintptr_t(1) << 12), int64_t(1) << 20, 4, int64_t(1) << 41}, high{reinterpret_cast<const void*>((uintptr_t(1) << 12) + 4), int64_t(1) << 20, 4, int64_t(1) << 41};
    if (ops::share(low, high) || !ops::share(low, low)) return std::puts("wide"), 1;
    // what is left out may come with any stride
    const Span out = ops::matrix_span(nullptr, 5, 4, INT64_MAX, 4), no_width = ops::matrix_span(memory, 5, 0, INT64_MAX, 8), one = ops::matrix_span(memory, 1, 4, INT64_MAX, 4);
    if (ops::share(out, whole) || ops::share(no_width, whole) || !ops::share(one, whole) || one.bytes() != 16) return std::puts("left out"), 1;
    if (shared < 1000 || apart < 1000) return std::puts("too few of one kind"), 1;
    std::puts("ok");
}
