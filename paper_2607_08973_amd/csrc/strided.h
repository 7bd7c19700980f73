// Which strided rows overlap: host-side checks of the row operators. Plain C++
// (bytes and addresses only).
#pragma once
#include <cstdint>

namespace sifar {

// `rows` rows of `size` bytes, `stride` bytes apart. Stride 0: one row for all.
struct Rows {
    uint64_t at = 0;
    uint64_t rows = 0, stride = 0, size = 0;
};

inline bool empty(const Rows &r) { return r.at == 0 || r.rows == 0 || r.size == 0; }

inline uint64_t rows_end(const Rows &r) { return r.at + (r.rows - 1) * r.stride + r.size; }

// May a byte belong to both? Exact for rows at one stride (interleaved views of
// one buffer) and for spans that are apart; rows at different strides count as
// overlapping where their spans do.
inline bool may_overlap(const Rows &a, const Rows &b) {
    if (empty(a) || empty(b)) return false;
    if (rows_end(a) <= b.at || rows_end(b) <= a.at) return false;
    if (a.stride != b.stride || a.rows == 1 || b.rows == 1 || a.size > a.stride ||
        b.size > b.stride)
        return true;
    // b's rows start d bytes behind the start of one of a's (extended) rows
    const uint64_t d = b.at >= a.at ? (b.at - a.at) % a.stride
                                    : (a.stride - (a.at - b.at) % a.stride) % a.stride;
    return d < a.size || a.stride - d < b.size;
}

// Row for row the same bytes: what a workgroup overwrites, only it has read.
inline bool same_rows(const Rows &a, const Rows &b) {
    return a.at == b.at && a.size == b.size && (a.stride == b.stride || a.rows == 1);
}

}  // namespace sifar
