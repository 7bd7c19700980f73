// Matrix tiles of the blocks of a decode layer (attention.hip, experts.hip): 16 x 16
// tiles of fp32 sums over 64 bytes of each row, one matrix instruction of 16-bit
// elements or four of 32-bit ones. gfx950 (MI355X) only.
#pragma once

#include <hip/hip_runtime.h>

#include "rows.h"

namespace sifar {

typedef float F4 __attribute__((ext_vector_type(4)));

// Lane l of a wave holds row (l & 15) of its operand: 16 bytes, those of quarter l >> 4
// of 64 bytes (both operands share the order of the summands, which is all that has to
// agree). In the sums lane l holds column l & 15, rows 4 (l >> 4) to 4 (l >> 4) + 3: the
// rows are the first operand's, the columns the second's.
template <int D>
__device__ __forceinline__ F4 mma(const U4 &a, const U4 &b, F4 c) {
    if constexpr (D == SIFAR_BF16) {
        typedef __bf16 B8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, a),
                                                       __builtin_bit_cast(B8, b), c, 0, 0, 0);
    } else if constexpr (D == SIFAR_FP16) {
        typedef _Float16 H8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(H8, a),
                                                      __builtin_bit_cast(H8, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]),
                                                     c, 0, 0, 0);
        return c;
    }
}

// 16-bit elements of a row, two a word: 8 a lane (4 words) as above, or 4 a lane of 32
// bytes of each row.
template <int WORDS>
struct Half {
    uint32_t w[WORDS];
};
template <int D, int WORDS>
__device__ __forceinline__ F4 mma_half(const Half<WORDS> &a, const Half<WORDS> &b, F4 c) {
    static_assert(WORDS == 4 || WORDS == 2, "8 or 4 elements");
    if constexpr (WORDS == 4) {
        return mma<D>(__builtin_bit_cast(U4, a), __builtin_bit_cast(U4, b), c);
    } else if constexpr (D == SIFAR_BF16) {
        typedef short S4 __attribute__((ext_vector_type(4)));
        return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(S4, a),
                                                         __builtin_bit_cast(S4, b), c, 0, 0, 0);
    } else {
        typedef _Float16 H4 __attribute__((ext_vector_type(4)));
        return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(H4, a),
                                                     __builtin_bit_cast(H4, b), c, 0, 0, 0);
    }
}

// 16-bit elements in a word's halves, widened.
template <int D>
__device__ __forceinline__ float low_half(uint32_t w) {
    if constexpr (D == SIFAR_BF16) return __uint_as_float(w << 16);
    else return widen<D>(w & 0xFFFFu);
}
template <int D>
__device__ __forceinline__ float high_half(uint32_t w) {
    if constexpr (D == SIFAR_BF16) return __uint_as_float(w & 0xFFFF0000u);
    else return widen<D>(w >> 16);
}

// Two values as the sum of two 16-bit elements each: the second holds what the rounding
// to the first leaves, so the pair is good to 2^-17 of the value (bf16; fp16 2^-22,
// where neither is subnormal).
struct Split {
    uint32_t high, low;
};
template <int D>
__device__ __forceinline__ Split split(float a, float b) {
    Split s;
    s.high = pack16<D>(a, b);
    s.low = pack16<D>(a - low_half<D>(s.high), b - high_half<D>(s.high));
    return s;
}

}  // namespace sifar
