// Routing to experts: sifar_route. gfx950 (MI355X) only.
//
// One wave a token. Lane l holds EPL adjacent experts, groups of experts lie in
// segments of lanes, so an expert's index grows with its place in the wave. A
// token's logits become keys that sort as (score + bias, lowest index first) and
// differ; each lane sorts its own, and top-k takes k times the largest of the 64
// heads, whose key names its expert.
//
// Where a bias or groups decide, keys are 64-bit scores whose ten lowest bits hold
// the index, so that scores next to each other rank as they should: 32-bit scores, off
// by 2^-24, would swap neighbours for a token in some thousands. Without them the
// logits' own order is the answer, and 16-bit logits fit a 32-bit key together with
// the index.
//
// Bound: for many tokens the vector instructions of the sort and of the k steps (486 a
// token for 512 experts of 16 bits, 782 for 256 with bias and groups; at four cycles
// each they fill the SIMDs for all of the kernel's time); for one token their latency.
// Measured, in a graph: 16384 x 512 bf16 softmax, top 10, 12.1 us (3.7 at a copy's
// rate; in fp32, by 64-bit keys, 15.6), 8192 x 256 with bias and groups, top 8, 11.5
// (1.7), one token of it 4.4.
#include <hip/hip_runtime.h>

#include "exp2.h"
#include "rows.h"

namespace sifar {
namespace {

constexpr int kIndexBits = 10;  // experts of a token: at most 1024
constexpr uint32_t kIndexMask = (1u << kIndexBits) - 1;
constexpr int kWaves = 4;       // tokens of a workgroup
constexpr double kLog2e = 1.4426950408889634;
constexpr double kLargest = 1.7976931348623157e308;
static_assert(SIFAR_ROUTE_MAX_EXPERTS <= 1 << kIndexBits, "an index fits a key");

struct RouteArgs {
    sifar_route_args a;
    int32_t per;    // experts of a group
    int32_t lanes;  // lanes of a group: a power of two
};

__device__ __forceinline__ double max64(double a, double b) {
    double r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ double min64(double a, double b) {
    double r;
    asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

// Over the wave, in a scalar register: DPP moves up within rows of 16, then from row
// to row; the last lane holds the result. 0 where no lane offers more.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    const auto step = [&](auto ctrl, auto rows) {
        const uint32_t y = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(
            0, static_cast<int>(x), decltype(ctrl)::value, decltype(rows)::value, 0xF, false));
        x = x > y ? x : y;
    };
    using std::integral_constant;
    step(integral_constant<int, 0x111>{}, integral_constant<int, 0xF>{});  // row_shr:1
    step(integral_constant<int, 0x112>{}, integral_constant<int, 0xF>{});
    step(integral_constant<int, 0x114>{}, integral_constant<int, 0xF>{});
    step(integral_constant<int, 0x118>{}, integral_constant<int, 0xF>{});
    step(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});  // row_bcast:15
    step(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});  // row_bcast:31
    return lane_value(x, 63);
}

// ---- keys ------------------------------------------------------------------------

// All ones for a negative number, by its high word.
__device__ __forceinline__ uint32_t sign_mask(uint32_t high) {
    return static_cast<uint32_t>(static_cast<int32_t>(high) >> 31);
}

// A value and an expert as one finite double that sorts by value, without its ten
// lowest bits (in steps of 2^-42 of it or less), then by the lower index. -inf, of what
// is not there, sorts behind every score.
__device__ __forceinline__ double wide_key(double value, int expert) {
    value = min64(max64(value + 0.0, -kLargest), kLargest);  // -0 counts as 0
    const uint64_t bits = __builtin_bit_cast(uint64_t, value);
    const uint32_t high = static_cast<uint32_t>(bits >> 32);
    // more mantissa is a larger positive and a smaller negative number
    // (past the last expert, where nothing is, an index may not fit)
    const uint32_t code = (kIndexMask - static_cast<uint32_t>(expert)) ^ sign_mask(high);
    const uint32_t low = (static_cast<uint32_t>(bits) & ~kIndexMask) | (code & kIndexMask);
    return __builtin_bit_cast(double, (static_cast<uint64_t>(high) << 32) | low);
}

// The same as an integer that sorts alike, in two words.
__device__ __forceinline__ void ordered(double key, uint32_t &hi, uint32_t &lo) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, key);
    const uint32_t high = static_cast<uint32_t>(bits >> 32), sign = sign_mask(high);
    hi = high ^ (sign | 0x80000000u);
    lo = static_cast<uint32_t>(bits) ^ sign;
}
constexpr uint32_t kNoneHigh = 0x00100000u;  // ordered()'s high word of what is not there

__device__ __forceinline__ int wide_expert(uint32_t low) {  // of ordered()'s low word
    return static_cast<int>(kIndexMask - (low & kIndexMask));
}

// A logit that was stored in 16 bits, whose ten lowest bits as fp32 are 0, and an
// expert as 32 bits that sort alike. -inf gives no more than kNoneKey.
__device__ __forceinline__ uint32_t short_key(float x, int expert) {
    const uint32_t bits = __float_as_uint(x + 0.0f);  // -0 counts as 0
    const uint32_t order = bits ^ (sign_mask(bits) | 0x80000000u);
    return (order & ~kIndexMask) | (kIndexMask - static_cast<uint32_t>(expert));
}
constexpr uint32_t kNoneKey = 0x007FFFFFu;

__device__ __forceinline__ float short_logit(uint32_t key) {
    return __uint_as_float((key ^ (~sign_mask(key) | 0x80000000u)) & ~kIndexMask);
}

__device__ __forceinline__ void exchange(double &hi, double &lo) {
    const double m = max64(hi, lo);
    lo = min64(hi, lo);
    hi = m;
}
__device__ __forceinline__ void exchange(uint32_t &hi, uint32_t &lo) {
    const uint32_t m = hi > lo ? hi : lo;
    lo = hi > lo ? lo : hi;
    hi = m;
}

// Descending odd-even merge sort (Batcher) of a lane's keys.
template <int N, class K>
__device__ __forceinline__ void sort_descending(K (&k)[N]) {
#pragma unroll
    for (int p = 1; p < N; p *= 2)
#pragma unroll
        for (int q = p; q >= 1; q /= 2)
#pragma unroll
            for (int j = q % p; j + q < N; j += 2 * q)
#pragma unroll
                for (int i = 0; i < q; ++i)
                    if (i + j + q < N && (i + j) / (2 * p) == (i + j + q) / (2 * p))
                        exchange(k[i + j], k[i + j + q]);
}

// ---- scores ----------------------------------------------------------------------

// 1 / d for d in [1, 2^1000]: the hardware's estimate and two Newton steps.
__device__ __forceinline__ double inverse(double d) {
    double y = __builtin_amdgcn_rcp(d);
    y = __builtin_fma(__builtin_fma(-d, y, 1.0), y, y);
    return __builtin_fma(__builtin_fma(-d, y, 1.0), y, y);
}

// Scores below 2^-1000 are 0, which keeps every exponent in range.
__device__ __forceinline__ double sigmoid(float x) {
    const double t = max64(-kLog2e * static_cast<double>(x), -1000.0);
    const double s = inverse(1.0 + exp2_64(t));
    return t > 1000.0 ? 0.0 : s;
}

// exp(x - m); 1 at the largest logit, which may be infinite.
__device__ __forceinline__ double softmax_weight(float x, float m) {
    const double t = (static_cast<double>(x) - static_cast<double>(m)) * kLog2e;
    const double w = exp2_64(t);
    return x == m ? 1.0 : t > -1000.0 ? w : 0.0;
}

// The two best of a group, joined with another's.
__device__ __forceinline__ void join_best(double &b1, double &b2, Pair<double> p1,
                                          Pair<double> p2) {
    b1 = max64(p1.a, p1.b);
    b2 = max64(min64(p1.a, p1.b), max64(p2.a, p2.b));
}

// The lane's EPL stored logits: 16 bytes or more at a time where all of them are
// there (global loads need no alignment beyond an element's).
template <int D, int EPL>
__device__ __forceinline__ void load_logits(const Stored<D> *p, int mine, uint32_t (&x)[EPL],
                                            uint32_t none) {
    struct __attribute__((packed, aligned(sizeof(Stored<D>)))) All {
        Stored<D> v[EPL];
    };
    if (mine >= EPL) {
        const All all = *reinterpret_cast<const All *>(p);
#pragma unroll
        for (int j = 0; j < EPL; ++j) x[j] = all.v[j];
    } else {
#pragma unroll
        for (int j = 0; j < EPL; ++j) x[j] = j < mine ? p[j] : none;
    }
}

// RANKED: a bias or groups decide. Otherwise the order of the logits does.
template <int D, int EPL, bool RANKED>
__global__ void __launch_bounds__(kRowWave *kWaves) route_kernel(const RouteArgs n) {
    // 16-bit logits in 32-bit keys
    constexpr bool SHORT = !RANKED && D != SIFAR_FP32;
    __shared__ float logits[RANKED ? kWaves : 1][RANKED ? kRowWave * EPL : 1];
    const sifar_route_args &a = n.a;
    const int lane = threadIdx.x, wave = threadIdx.y;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
    if (t >= a.tokens) return;
    const int group = lane / n.lanes;
    const int inside = (lane & (n.lanes - 1)) * EPL;         // of the group
    const int first = group * n.per + inside;
    const int mine = group < a.groups ? n.per - inside : 0;  // experts from `first` on
    const float none = -__builtin_inff();
    constexpr uint32_t none_bits = D == SIFAR_FP32 ? 0xFF800000u : D == SIFAR_BF16 ? 0xFF80u : 0xFC00u;

    uint32_t raw[EPL];
    load_logits<D, EPL>(static_cast<const Stored<D> *>(a.logits) + t * a.logits_stride + first,
                        mine, raw, none_bits);
    float x[EPL], m = none;
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
        x[j] = widen<D>(raw[j]);
        if (!(x[j] > none)) x[j] = none;  // NaN
        m = choose(x[j] > m, x[j], m);
    }
    const bool softmax = a.score == SIFAR_ROUTE_SOFTMAX;
    double scale = 1.0;  // 1 / the sum of the weights, where it matters
    if (softmax) {
        m = wave_reduce(m, Max{});
        if (RANKED || !a.renorm) {
            double total = 0.0;
#pragma unroll
            for (int j = 0; j < EPL; ++j) {
                const double w = softmax_weight(x[j], m);
                total += x[j] > none ? w : 0.0;
            }
            total = wave_reduce(total, Add{});
            scale = total > 0.0 ? inverse(total) : 0.0;
        }
    }

    int id = -1;         // of lane i: the i-th best expert
    float chosen = 0.f;  // and its logit
    if constexpr (SHORT) {
        uint32_t key[EPL];
#pragma unroll
        for (int j = 0; j < EPL; ++j) key[j] = short_key(x[j], first + j);
        sort_descending(key);
        uint32_t found = 0;
        for (int i = 0; i < a.topk; ++i) {
            const uint32_t best = wave_max(key[0]);
            found = lane == i ? best : found;
            if (key[0] == best) {
                stay_branch();
#pragma unroll
                for (int j = 0; j + 1 < EPL; ++j) key[j] = key[j + 1];
                key[EPL - 1] = 0;
            }
        }
        if (found > kNoneKey) {
            id = static_cast<int>(kIndexMask - (found & kIndexMask));
            chosen = short_logit(found);
        }
    } else {
        double value[EPL];
        if constexpr (RANKED) {
            double b1 = none, b2 = none;
#pragma unroll
            for (int j = 0; j < EPL; ++j) {
                logits[wave][lane * EPL + j] = x[j];
                const double s = softmax ? softmax_weight(x[j], m) * scale : sigmoid(x[j]);
                const double c =
                    a.bias ? s + static_cast<double>(a.bias[j < mine ? first + j : 0]) : s;
                // c is not there with its logit, nor at -inf or NaN
                value[j] = x[j] > none && c > none ? c : none;
                b2 = max64(b2, min64(b1, value[j]));
                b1 = max64(b1, value[j]);
            }
            if (a.groups > 1) {
                if (n.lanes > 1) join_best(b1, b2, pair<1>(b1), pair<1>(b2));
                if (n.lanes > 2) join_best(b1, b2, pair<2>(b1), pair<2>(b2));
                if (n.lanes > 4) join_best(b1, b2, pair<4>(b1), pair<4>(b2));
                if (n.lanes > 8) join_best(b1, b2, pair<8>(b1), pair<8>(b2));
                if (n.lanes > 16) join_best(b1, b2, pair<16>(b1), pair<16>(b2));
                const double worth = a.group_top == 2 && b2 > none ? b1 + b2 : b1;
                int better = 0;
                for (int g = 0; g < a.groups; ++g) {
                    const double other = lane_value(worth, g * n.lanes);
                    better += other > worth || (other == worth && g < group);
                }
                if (better >= a.top_groups) {
                    stay_branch();
#pragma unroll
                    for (int j = 0; j < EPL; ++j) x[j] = value[j] = none;
                }
            }
        }
        if (!RANKED || !a.bias) {  // the same order, also where scores saturate
#pragma unroll
            for (int j = 0; j < EPL; ++j) value[j] = static_cast<double>(x[j]);
        }
        double key[EPL];
#pragma unroll
        for (int j = 0; j < EPL; ++j) key[j] = wide_key(value[j], first + j);
        sort_descending(key);
        uint32_t hi[EPL], lo[EPL];
#pragma unroll
        for (int j = 0; j < EPL; ++j) ordered(key[j], hi[j], lo[j]);
        uint32_t found_hi = 0, found_lo = 0;
        for (int i = 0; i < a.topk; ++i) {
            // the high words decide, or now and then the low words among equal ones
            const uint32_t best = wave_max(hi[0]);
            bool taken = hi[0] == best;
            uint64_t who = __ballot(taken);
            if (__builtin_popcountll(who) != 1) {
                const uint32_t low = wave_max(taken ? lo[0] : 0u);
                taken = taken && lo[0] == low;
                who = __ballot(taken);
            }
            const uint32_t low = lane_value(lo[0], __builtin_ctzll(who));
            found_hi = lane == i ? best : found_hi;
            found_lo = lane == i ? low : found_lo;
            if (taken) {
                stay_branch();
#pragma unroll
                for (int j = 0; j + 1 < EPL; ++j) {
                    hi[j] = hi[j + 1];
                    lo[j] = lo[j + 1];
                }
                hi[EPL - 1] = 0;
            }
        }
        if constexpr (RANKED) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (found_hi > kNoneHigh) {
            id = wide_expert(found_lo);
            if constexpr (RANKED) {
                const int g = id / n.per, in = id - g * n.per;
                chosen = logits[wave][g * n.lanes * EPL + in];
            } else {
                // the key holds all of an fp32 logit
                const uint64_t o = (static_cast<uint64_t>(found_hi) << 32) | found_lo;
                const uint64_t bits = o >> 63 ? o & ~(uint64_t{1} << 63) : ~o;
                const double v = __builtin_bit_cast(double, bits & ~uint64_t{kIndexMask});
                chosen = static_cast<float>(v);
            }
        }
    }
    double w = 0.0;
    if (id >= 0) w = softmax ? softmax_weight(chosen, m) * scale : sigmoid(chosen);
    if (a.renorm) {
        const double sum = wave_reduce(w, Add{});
        w = sum > 0.0 ? w / sum : 0.0;
    }
    if (lane < a.topk) {
        a.ids[t * a.topk + lane] = id;
        a.weights[t * a.topk + lane] = static_cast<float>(w * static_cast<double>(a.scale));
    }
}

template <int D, int EPL>
hipError_t launch_epl(const RouteArgs &n, hipStream_t s) {
    const dim3 grid((n.a.tokens + kWaves - 1) / kWaves), block(kRowWave, kWaves);
    if constexpr (EPL <= SIFAR_ROUTE_MAX_EXPERTS / kRowWave) {  // more only with groups
        if (!n.a.bias && n.a.groups == 1) {
            route_kernel<D, EPL, false><<<grid, block, 0, s>>>(n);
            return hipGetLastError();
        }
    }
    route_kernel<D, EPL, true><<<grid, block, 0, s>>>(n);
    return hipGetLastError();
}

template <int D>
hipError_t launch_route(const RouteArgs &n, hipStream_t s) {
    const int need = (n.per + n.lanes - 1) / n.lanes;
    return need <= 1    ? launch_epl<D, 1>(n, s)
           : need <= 2  ? launch_epl<D, 2>(n, s)
           : need <= 4  ? launch_epl<D, 4>(n, s)
           : need <= 8  ? launch_epl<D, 8>(n, s)
           : need <= 16 ? launch_epl<D, 16>(n, s)
                        : launch_epl<D, 32>(n, s);
}

bool good(const sifar_route_args &a) {
    if (a.dtype < SIFAR_BF16 || a.dtype > SIFAR_FP32) return false;
    if (a.tokens < 0 || a.tokens > SIFAR_ROWS_MAX_TOKENS) return false;
    if (a.experts < 1 || a.experts > SIFAR_ROUTE_MAX_EXPERTS) return false;
    if (a.topk < 1 || a.topk > SIFAR_ROUTE_MAX_TOPK || a.topk > a.experts) return false;
    if (a.score != SIFAR_ROUTE_SOFTMAX && a.score != SIFAR_ROUTE_SIGMOID) return false;
    if (a.groups < 1 || a.groups > SIFAR_ROUTE_MAX_GROUPS || a.experts % a.groups) return false;
    if (a.top_groups < 1 || a.top_groups > a.groups) return false;
    if (a.group_top != 1 && a.group_top != 2) return false;
    if (a.renorm != 0 && a.renorm != 1) return false;
    if (a.tokens == 0) return true;
    if (!a.logits || !a.ids || !a.weights) return false;
    const uint64_t size = a.dtype == SIFAR_FP32 ? 4 : 2;
    const auto at = [](const void *p) { return reinterpret_cast<uintptr_t>(p); };
    if (at(a.logits) % size || at(a.bias) % 4 || at(a.ids) % 4 || at(a.weights) % 4) return false;
    if (a.tokens > 1 && (a.logits_stride < a.experts || a.logits_stride > (int64_t{1} << 40)))
        return false;
    // Waves take tokens in any order: what one writes, no other may read or write.
    const uint64_t tokens = static_cast<uint64_t>(a.tokens);
    const uint64_t out = tokens * static_cast<uint64_t>(a.topk) * 4;
    const Rows ids{at(a.ids), 1, 0, out}, weights{at(a.weights), 1, 0, out};
    const Rows bias{at(a.bias), 1, 0, static_cast<uint64_t>(a.experts) * 4};
    const Rows logits{at(a.logits), tokens, static_cast<uint64_t>(a.logits_stride) * size,
                      static_cast<uint64_t>(a.experts) * size};
    return !may_overlap(ids, weights) && !may_overlap(ids, logits) &&
           !may_overlap(weights, logits) && !may_overlap(ids, bias) &&
           !may_overlap(weights, bias);
}

}  // namespace
}  // namespace sifar

extern "C" int sifar_route(const sifar_route_args *args, void *stream) {
    using namespace sifar;
    if (!args || !good(*args)) return SIFAR_EINVAL;
    if (args->tokens == 0) return SIFAR_OK;
    RouteArgs n{};
    n.a = *args;
    n.per = args->experts / args->groups;
    int segments = 1;
    while (segments < args->groups) segments *= 2;
    n.lanes = kRowWave / segments;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = args->dtype == SIFAR_BF16   ? launch_route<SIFAR_BF16>(n, s)
                         : args->dtype == SIFAR_FP16 ? launch_route<SIFAR_FP16>(n, s)
                                                     : launch_route<SIFAR_FP32>(n, s);
    return e == hipSuccess ? SIFAR_OK : SIFAR_EHIP;
}
