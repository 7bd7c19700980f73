// The paged key-value cache that sifar_cache_append writes and sifar_paged_attention
// reads: its strides, and which elements two caches share. Plain C++ (host only).
#pragma once

#include <stdint.h>

#include "operands.h"

namespace sifar {

// Elements of a cache in units of the element type: three loops over rows of `dim`.
struct Paged {
    int64_t count[3];   // pages, slots, heads, by ascending stride once sorted
    int64_t stride[3];
    int64_t dim;
};

// Loops of one turn have no stride; the others by ascending stride.
inline Paged paged(int64_t pages, int64_t slots, int64_t heads, int64_t page_stride,
                   int64_t slot_stride, int64_t head_stride, int64_t dim) {
    Paged p{{pages, slots, heads}, {page_stride, slot_stride, head_stride}, dim};
    for (int i = 0; i < 3; ++i)
        if (p.count[i] == 1) p.stride[i] = 0;
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (p.stride[j] > p.stride[j + 1]) {
                int64_t t = p.stride[j];
                p.stride[j] = p.stride[j + 1], p.stride[j + 1] = t;
                t = p.count[j];
                p.count[j] = p.count[j + 1], p.count[j + 1] = t;
            }
    return p;
}

// From the first element to behind the last, or 0 where the strides do not keep the
// elements apart, are not multiples of 8, or lead beyond
// SIFAR_CACHE_MAX_ELEMENTS.
inline int64_t extent(const Paged &p) {
    int64_t e = p.dim;
    for (int i = 0; i < 3; ++i) {
        if (p.count[i] == 1) continue;
        if (p.stride[i] < e || p.stride[i] % 8 || p.stride[i] > kMaxStride) return 0;
        const unsigned __int128 more =
            static_cast<unsigned __int128>(p.count[i] - 1) * static_cast<uint64_t>(p.stride[i]);
        if (more > SIFAR_CACHE_MAX_ELEMENTS) return 0;
        e += static_cast<int64_t>(more);
    }
    return e <= SIFAR_CACHE_MAX_ELEMENTS ? e : 0;
}

// A table of `rows` rows of pages, `stride` apart, whose bytes can be counted.
inline bool good_table(int64_t rows, int64_t stride) {
    return stride >= 0 && (rows <= 1 || stride <= kMaxStride / rows);
}
inline Rows table_of(const void *p, int64_t rows, int64_t stride, int64_t width) {
    return span_of(p, 4ull * static_cast<uint64_t>((rows <= 1 ? 0 : (rows - 1) * stride) + width));
}

// Does a cache share an element with one of the same strides whose first element lies
// `d` elements away? Exact for strides that extent() accepts: rows of one loop reach at
// most into the next turn of the loop around it.
inline bool shares(const Paged &p, int64_t d, int loop = 2) {
    if (d < 0) d = -d;  // the same pair, seen from the other
    if (loop < 0) return d < p.dim;
    if (p.count[loop] == 1) return shares(p, d, loop - 1);
    const int64_t turn = d / p.stride[loop], rest = d % p.stride[loop];
    return (turn < p.count[loop] && shares(p, rest, loop - 1)) ||
           (turn + 1 < p.count[loop] && shares(p, rest - p.stride[loop], loop - 1));
}

}  // namespace sifar
