// Shared by the row operators of a decode step (block_norm.hip, route.hip,
// sample.hip): element types, reductions over a wave, and the host-side checks
// of strided rows. gfx950 (MI355X) only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sifar.h"
#include "strided.h"

namespace sifar {

constexpr int kRowWave = 64;

// The storage type of an element type: bf16 and fp16 as raw 16 bits.
template <int D>
using Stored = std::conditional_t<D == SIFAR_FP32, uint32_t, uint16_t>;

template <int D>
__device__ __forceinline__ float widen(uint32_t bits) {
    if constexpr (D == SIFAR_BF16) return __uint_as_float(bits << 16);
    else if constexpr (D == SIFAR_FP16)
        return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(bits)));
    else return __uint_as_float(bits);
}

// Two values to two 16-bit elements, round to nearest even (bf16: one
// V_CVT_PK_BF16_F32).
template <int D>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    static_assert(D == SIFAR_BF16 || D == SIFAR_FP16, "16-bit types");
    typedef float F2 __attribute__((ext_vector_type(2)));
    const F2 f = {lo, hi};
    if constexpr (D == SIFAR_BF16) {
        typedef __bf16 B2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, B2));
    } else {
        typedef _Float16 H2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, H2));
    }
}

typedef uint32_t U4 __attribute__((ext_vector_type(4)));

// Eight adjacent elements of a 16-byte aligned row, as they are stored.
template <int D>
struct Eight {
    U4 v[D == SIFAR_FP32 ? 2 : 1];
};

template <int D>
__device__ __forceinline__ Eight<D> load8(const void *row, int64_t at) {
    Eight<D> e;
    const U4 *p = reinterpret_cast<const U4 *>(static_cast<const Stored<D> *>(row) + at);
    e.v[0] = p[0];
    if constexpr (D == SIFAR_FP32) e.v[1] = p[1];
    return e;
}

template <int D>
__device__ __forceinline__ float element(const Eight<D> &e, int i) {
    if constexpr (D == SIFAR_FP32) return __uint_as_float(e.v[i >> 2][i & 3]);
    else if constexpr (D == SIFAR_BF16)
        return __uint_as_float(i & 1 ? e.v[0][i >> 1] & 0xFFFF0000u : e.v[0][i >> 1] << 16);
    else
        return widen<D>(i & 1 ? e.v[0][i >> 1] >> 16 : e.v[0][i >> 1] & 0xFFFFu);
}

// Rounded once, and stored without displacing cached lines: nothing in the
// launch reads an output row again.
template <int D>
__device__ __forceinline__ void store8(void *row, int64_t at, const float (&f)[8]) {
    U4 *p = reinterpret_cast<U4 *>(static_cast<Stored<D> *>(row) + at);
    if constexpr (D == SIFAR_FP32) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            U4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(f[4 * h + i]);
            __builtin_nontemporal_store(w, p + h);
        }
    } else {
        U4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack16<D>(f[2 * i], f[2 * i + 1]);
        __builtin_nontemporal_store(w, p);
    }
}

// Butterflies over segments of 2, 4 .. 64 adjacent lanes, in ascending steps.
// pair<STEP>(x) holds this lane's x and one from the other half of its segment
// of 2 * STEP lanes, in either order, so what joins the two has to be
// commutative. Within a row of 16 the step is a DPP move: 1 and 2 exchange
// lanes of a quad, 4 and 8 mirror 8 and 16 lanes, which reaches a lane with the
// partner's value because the steps below have made the quads, then the
// halves, uniform. 16 and 32 are gfx950's lane swaps. All of it stays in vector
// registers.
template <class T>
struct Pair {
    T a, b;
};

template <int STEP>
__device__ __forceinline__ Pair<uint32_t> pair32(uint32_t x) {
    if constexpr (STEP == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return {r[0], r[1]};
    } else if constexpr (STEP == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return {r[0], r[1]};
    } else {
        static_assert(STEP == 1 || STEP == 2 || STEP == 4 || STEP == 8, "a power of two");
        // quad_perm [1,0,3,2], quad_perm [2,3,0,1], row_half_mirror, row_mirror
        constexpr int ctrl = STEP == 1 ? 0xB1 : STEP == 2 ? 0x4E : STEP == 4 ? 0x141 : 0x140;
        const int v = static_cast<int>(x);
        return {x, static_cast<uint32_t>(
                       __builtin_amdgcn_update_dpp(v, v, ctrl, 0xF, 0xF, true))};
    }
}

template <int STEP, class T>
__device__ __forceinline__ Pair<T> pair(T x) {
    if constexpr (sizeof(T) == 4) {
        const Pair<uint32_t> p = pair32<STEP>(__builtin_bit_cast(uint32_t, x));
        return {__builtin_bit_cast(T, p.a), __builtin_bit_cast(T, p.b)};
    } else {
        static_assert(sizeof(T) == 8, "32 or 64 bits");
        const uint64_t b = __builtin_bit_cast(uint64_t, x);
        const Pair<uint32_t> lo = pair32<STEP>(static_cast<uint32_t>(b));
        const Pair<uint32_t> hi = pair32<STEP>(static_cast<uint32_t>(b >> 32));
        return {__builtin_bit_cast(T, (static_cast<uint64_t>(hi.a) << 32) | lo.a),
                __builtin_bit_cast(T, (static_cast<uint64_t>(hi.b) << 32) | lo.b)};
    }
}

// op over each segment of LANES lanes, the same bits in every lane of it.
template <int LANES = 64, class T, class Op>
__device__ __forceinline__ T wave_reduce(T v, Op op) {
    const auto join = [&](Pair<T> p) { return op(p.a, p.b); };
    if constexpr (LANES > 1) v = join(pair<1>(v));
    if constexpr (LANES > 2) v = join(pair<2>(v));
    if constexpr (LANES > 4) v = join(pair<4>(v));
    if constexpr (LANES > 8) v = join(pair<8>(v));
    if constexpr (LANES > 16) v = join(pair<16>(v));
    if constexpr (LANES > 32) v = join(pair<32>(v));
    return v;
}

// Lane `from`'s value (the same lane for the whole wave), in scalar registers.
template <class T>
__device__ __forceinline__ T lane_value(T x, int from) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(
            T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), from));
    } else {
        const uint64_t b = __builtin_bit_cast(uint64_t, x);
        const uint32_t lo = static_cast<uint32_t>(
            __builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(b)), from));
        const uint32_t hi = static_cast<uint32_t>(
            __builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(b >> 32)), from));
        return __builtin_bit_cast(T, (static_cast<uint64_t>(hi) << 32) | lo);
    }
}

// c ? a : b of values. (Written with elements of an array in registers, the operator
// selects between their addresses, and the array is indexed at run time.)
template <class T>
__device__ __forceinline__ T choose(bool c, T a, T b) {
    return c ? static_cast<T>(a) : static_cast<T>(b);
}

// Keeps the branch that it stands in from becoming selects. On gfx950 a comparison and
// the v_cndmasks that read its vcc take a SIMD 9 cycles a wave for one, 14 for two and
// 138 for eight (39 in the 64-bit encoding, or with the mask in other scalar
// registers), so several values under one condition are moved in a branch.
__device__ __forceinline__ void stay_branch() { asm volatile(""); }

struct Add {
    template <class T>
    __device__ __forceinline__ T operator()(T a, T b) const { return a + b; }
};
struct Max {
    template <class T>
    __device__ __forceinline__ T operator()(T a, T b) const { return choose(a > b, a, b); }
};

}  // namespace sifar
