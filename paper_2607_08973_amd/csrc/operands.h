// Host-side checks that the operators on strided rows share. Plain C++ (bytes and
// addresses only).
#pragma once

#include <stdint.h>

#include "sifar.h"
#include "strided.h"

namespace sifar {

constexpr int64_t kMaxStride = int64_t{1} << 40;

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

inline bool good_dtype(int32_t dtype) { return dtype >= SIFAR_BF16 && dtype <= SIFAR_FP32; }

inline uint64_t size_of(int32_t dtype) { return dtype == SIFAR_FP32 ? 4 : 2; }

inline Rows rows_of(const void *p, int32_t dtype, int64_t tokens, int64_t stride,
                    int64_t hidden) {
    Rows r;
    r.at = reinterpret_cast<uintptr_t>(p);
    r.rows = static_cast<uint64_t>(stride == 0 ? 1 : tokens);
    r.stride = static_cast<uint64_t>(stride) * size_of(dtype);
    r.size = static_cast<uint64_t>(hidden) * size_of(dtype);
    return r;
}

// `bytes` adjacent bytes.
inline Rows span_of(const void *p, uint64_t bytes) {
    Rows r;
    r.at = reinterpret_cast<uintptr_t>(p);
    r.rows = 1;
    r.size = bytes;
    return r;
}

// A row stride, which only several tokens use: a multiple of 8 that keeps them apart.
inline bool good_stride(int64_t stride, int64_t tokens, int64_t hidden) {
    return tokens <= 1 || (stride % 8 == 0 && stride >= hidden && stride <= kMaxStride);
}

}  // namespace sifar
