// Whether what a call writes shares values with what it reads: host only, for the calls' checks of their arguments.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>
#include <initializer_list>

namespace pxr {

// A view of a device buffer: `width` adjacent values of `element` bytes, in up to three dimensions of `count`, `stride` values apart.
struct View {
    const void* data;
    uint64_t element, width;
    struct {
        uint64_t count;
        int64_t stride;
    } dims[3];
};

namespace views {

typedef __int128 wide;  // (strides are any numbers)

inline wide size(wide v) { return v < 0 ? -v : v; }

struct Strides {
    wide least, most, bytes;
};

// Whether |apart + sum of i_d bytes_d| < values for some least_d <= i_d <= most_d, strides from `s` on, the largest first.
inline bool meet(wide apart, wide values, const Strides* s, int n) {
    if (n == 0) return size(apart) < values;
    // where each stride is as large as all that the smaller ones reach over, as in views that do not overlap themselves, only the nearest multiples come into question
    const wide at = s->bytes ? -apart / s->bytes : 0;
    wide tried = s->most + 1;  // (none)
    for (int k = -2; k <= 2; ++k) {
        const wide i = std::max(s->least, std::min(s->most, at + k));
        if (i == tried) continue;
        tried = i;
        if (meet(apart + i * s->bytes, values, s + 1, n - 1)) return true;
    }
    return false;
}

}  // namespace views

inline bool same_strides(const View& a, const View& b) {
    for (int d = 0; d < 3; ++d)
        if (a.dims[d].count > 1 && b.dims[d].count > 1 && a.dims[d].stride != b.dims[d].stride) return false;
    return true;
}

// Exact where the strides of what both have several of are the same and neither overlaps itself; of others that reach over the same addresses only the first values are compared.
inline bool share(const View& a, const View& b) {
    using namespace views;
    const wide apart = (wide) reinterpret_cast<uintptr_t>(b.data) - (wide) reinterpret_cast<uintptr_t>(a.data), values = (wide)a.element * a.width, other = (wide)b.element * b.width;
    wide a_low = 0, a_high = values, b_low = 0, b_high = other;
    Strides s[3];
    for (int d = 0; d < 3; ++d) {
        const wide a_more = (wide)a.dims[d].count - 1, b_more = (wide)b.dims[d].count - 1;
        if (a_more < 0 || b_more < 0) return false;
        const wide x = a_more ? (wide)a.element * a.dims[d].stride : 0, y = b_more ? (wide)b.element * b.dims[d].stride : 0;
        (x < 0 ? a_low : a_high) += a_more * x;
        (y < 0 ? b_low : b_high) += b_more * y;
        s[d] = {-a_more, b_more, a_more ? x : y};
    }
    if (apart + b_low >= a_high || a_low >= apart + b_high) return false;
    if (!same_strides(a, b) || values != other) return apart < 0 ? -apart < other : apart < values;
    std::sort(s, s + 3, [](const Strides& p, const Strides& q) { return size(p.bytes) > size(q.bytes); });
    return meet(apart, values, s, 3);
}

inline bool share(const View& written, std::initializer_list<View> read) {
    for (const View& v : read)
        if (share(written, v)) return true;
    return false;
}

// The same values in the same places.
inline bool itself(const View& a, const View& b) {
    for (int d = 0; d < 3; ++d)
        if (a.dims[d].count != b.dims[d].count) return false;
    return a.data == b.data && a.element == b.element && a.width == b.width && same_strides(a, b);
}

}  // namespace pxr
