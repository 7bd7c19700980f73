// 2^t in 64 bits, for the row operators that rank scores or add up weights where
// 32 bits would let a neighbour win. Plain C++ for host and device.
//
// t = i + f with i the nearest integer: 2^t = 2^i (1 + f q(f)), |f| <= 1/2. q
// interpolates (2^f - 1) / f at Chebyshev nodes; its degree sets the error
// (tests/test_exp2.py measures both against 80-bit arithmetic). f = 0 gives 1
// exactly. One fma per degree: on gfx950 a 64-bit fma issues at the rate of an
// unpacked 32-bit one. Rounding to i and scaling by 2^i are additions to the bits.
// Outside the stated ranges the result is garbage, but nothing traps.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#define SIFAR_HD __host__ __device__ __forceinline__
#else
#define SIFAR_HD inline
#endif

namespace sifar {

// i in the low bits, for |t| below 2^31.
SIFAR_HD double exp2_magic(double t) { return t + 0x1.8p52; }

SIFAR_HD uint32_t exp2_whole(double magic) {
    uint64_t bits;
    __builtin_memcpy(&bits, &magic, 8);
    return static_cast<uint32_t>(bits);
}

// q * 2^i, where exponents stay in range.
SIFAR_HD double exp2_scale(double q, uint32_t i) {
    uint64_t bits;
    __builtin_memcpy(&bits, &q, 8);
    uint32_t high = static_cast<uint32_t>(bits >> 32);
#if defined(__HIP_DEVICE_COMPILE__)
    // (left to itself the compiler makes two to five instructions on 64 bits of it)
    asm("v_lshl_add_u32 %0, %1, 20, %0" : "+v"(high) : "v"(i));
#else
    high += i << 20;
#endif
    bits = (static_cast<uint64_t>(high) << 32) | static_cast<uint32_t>(bits);
    __builtin_memcpy(&q, &bits, 8);
    return q;
}

// 2^t for |t| <= 1020, relative error below 3e-16.
SIFAR_HD double exp2_64(double t) {
    const double m = exp2_magic(t);
    const double f = t - (m - 0x1.8p52);
    double q = 0x1.e9d4d5f786506p-32;
    q = __builtin_fma(q, f, 0x1.e606425df1ca8p-28);
    q = __builtin_fma(q, f, 0x1.b524fa5b1918cp-24);
    q = __builtin_fma(q, f, 0x1.62bfd475ca6bdp-20);
    q = __builtin_fma(q, f, 0x1.ffcbfc674abbep-17);
    q = __builtin_fma(q, f, 0x1.43091309706fcp-13);
    q = __builtin_fma(q, f, 0x1.5d87fe78a51d0p-10);
    q = __builtin_fma(q, f, 0x1.3b2ab6fba1dd8p-7);
    q = __builtin_fma(q, f, 0x1.c6b08d704a0c2p-5);
    q = __builtin_fma(q, f, 0x1.ebfbdff82c598p-3);
    q = __builtin_fma(q, f, 0x1.62e42fefa39efp-1);
    return exp2_scale(__builtin_fma(q, f, 1.0), exp2_whole(m));
}

// 2^(y c + BITS) for y c in [-1000, 0], relative error below 4e-14: for sums in
// units of 2^-42. Below 2^-900 where it is not kept: one select, of the exponent, does
// for both words.
template <int BITS>
SIFAR_HD double exp2_quick(double y, double c, bool keep = true) {
    constexpr double s = static_cast<double>(1ull << BITS);
    const double m = __builtin_fma(y, c, 0x1.8p52);
    const double f = __builtin_fma(y, c, 0x1.8p52 - m);
    double q = 0x1.b638808675ca6p-24 * s;
    q = __builtin_fma(q, f, 0x1.63d136355f669p-20 * s);
    q = __builtin_fma(q, f, 0x1.ffcb9515c8f1ap-17 * s);
    q = __builtin_fma(q, f, 0x1.4308ac85abb17p-13 * s);
    q = __builtin_fma(q, f, 0x1.5d87fe86fe7ccp-10 * s);
    q = __builtin_fma(q, f, 0x1.3b2ab7181b74ap-7 * s);
    q = __builtin_fma(q, f, 0x1.c6b08d7047e52p-5 * s);
    q = __builtin_fma(q, f, 0x1.ebfbdff823cedp-3 * s);
    q = __builtin_fma(q, f, 0x1.62e42fefa39efp-1 * s);
    return exp2_scale(__builtin_fma(q, f, s), keep ? exp2_whole(m) : 0u - 1000u);
}

}  // namespace sifar
