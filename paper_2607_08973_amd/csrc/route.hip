// Routing to experts: sifar_route. gfx950 (MI355X) only.
//
// One wave a token. Lane l holds EPL adjacent experts, groups of experts lie in
// segments of lanes, so an expert's index grows with its place in the wave. The
// order of the experts is exact: a token's logits become 64-bit keys that sort
// as (score + bias, lowest index first), each lane sorts its own, and top-k takes
// k times the largest of the 64 heads. A key is a double whose ten lowest bits
// hold the index, so keys differ, one v_max_f64 compares value and index, and the
// largest names its expert. Bound: for many tokens the instructions of the sort
// and of the k steps; for one token their latency.
#include <hip/hip_runtime.h>

#include "exp2.h"
#include "rows.h"

namespace sifar {
namespace {

constexpr int kIndexBits = 10;  // experts of a token: at most 1024
constexpr uint64_t kIndexMask = (1u << kIndexBits) - 1;
constexpr int kWaves = 4;       // tokens of a workgroup
constexpr double kLog2e = 1.4426950408889634;
constexpr double kLargest = 1.7976931348623157e308;

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
struct Max64 {
    __device__ __forceinline__ double operator()(double a, double b) const { return max64(a, b); }
};

// A finite value and an expert as one double that sorts by value (to 2^-42 of it),
// then by the lower index.
__device__ __forceinline__ double key_of(double value, int expert) {
    value = min64(max64(value + 0.0, -kLargest), kLargest);  // -0 counts as 0
    const uint64_t bits = __builtin_bit_cast(uint64_t, value);
    // more mantissa is a larger positive and a smaller negative number
    const uint64_t code = bits >> 63 ? expert : kIndexMask - expert;
    return __builtin_bit_cast(double, (bits & ~kIndexMask) | code);
}

__device__ __forceinline__ int expert_of(double key) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, key);
    const uint32_t code = static_cast<uint32_t>(bits & kIndexMask);
    return static_cast<int>(bits >> 63 ? code : kIndexMask - code);
}

// 1 / d for d in [1, 2^1000]: the hardware's estimate and two Newton steps.
__device__ __forceinline__ double inverse(double d) {
    double y = __builtin_amdgcn_rcp(d);
    y = __builtin_fma(__builtin_fma(-d, y, 1.0), y, y);
    return __builtin_fma(__builtin_fma(-d, y, 1.0), y, y);
}

// Scores below 2^-1000 are 0, which keeps every exponent in range.
__device__ __forceinline__ double sigmoid(float x) {
    const double t = max64(-kLog2e * static_cast<double>(x), -1000.0);
    return t > 1000.0 ? 0.0 : inverse(1.0 + exp2_64(t));
}

// exp(x - m); 1 at the largest logit, which may be infinite.
__device__ __forceinline__ double softmax_weight(float x, float m) {
    if (x == m) return 1.0;
    const double t = (static_cast<double>(x) - static_cast<double>(m)) * kLog2e;
    return t < -1000.0 ? 0.0 : exp2_64(t);
}

// Descending odd-even merge sort (Batcher) of a lane's keys.
template <int N>
__device__ __forceinline__ void sort_descending(double (&k)[N]) {
#pragma unroll
    for (int p = 1; p < N; p *= 2)
#pragma unroll
        for (int q = p; q >= 1; q /= 2)
#pragma unroll
            for (int j = q % p; j + q < N; j += 2 * q)
#pragma unroll
                for (int i = 0; i < q; ++i)
                    if (i + j + q < N && (i + j) / (2 * p) == (i + j + q) / (2 * p)) {
                        const double hi = max64(k[i + j], k[i + j + q]);
                        k[i + j + q] = min64(k[i + j], k[i + j + q]);
                        k[i + j] = hi;
                    }
}

// The two best of a group, joined with another's.
__device__ __forceinline__ void join_best(double &b1, double &b2, Pair<double> p1,
                                          Pair<double> p2) {
    b1 = max64(p1.a, p1.b);
    b2 = max64(min64(p1.a, p1.b), max64(p2.a, p2.b));
}

template <int D, int EPL>
__global__ void __launch_bounds__(kRowWave *kWaves) route_kernel(const RouteArgs n) {
    const sifar_route_args &a = n.a;
    const int lane = threadIdx.x;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kWaves + threadIdx.y;
    if (t >= a.tokens) return;
    const Stored<D> *row = static_cast<const Stored<D> *>(a.logits) + t * a.logits_stride;
    const int group = lane / n.lanes;
    const int inside = (lane & (n.lanes - 1)) * EPL;   // of the group
    const int first = group * n.per + inside;
    int mine = group < a.groups ? n.per - inside : 0;  // experts of this lane
    const float none = -__builtin_inff();

    float x[EPL];
    float m = none;
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
        x[j] = none;
        if (j < mine) x[j] = widen<D>(row[first + j]);
        if (!(x[j] > none)) x[j] = none;  // NaN
        m = fmaxf(m, x[j]);
    }
    const bool softmax = a.score == SIFAR_ROUTE_SOFTMAX;
    double total = 1.0;
    if (softmax) {
        m = wave_reduce(m, Max{});
        if (a.bias || a.groups > 1 || !a.renorm) {
            total = 0.0;
#pragma unroll
            for (int j = 0; j < EPL; ++j) total += x[j] > none ? softmax_weight(x[j], m) : 0.0;
            total = wave_reduce(total, Add{});
        }
    }
    const double scale = total > 0.0 ? inverse(total) : 0.0;

    double key[EPL];
    if (a.bias || a.groups > 1) {
        double choice[EPL];
#pragma unroll
        for (int j = 0; j < EPL; ++j) {
            choice[j] = none;
            if (!(x[j] > none)) continue;
            const double s = softmax ? softmax_weight(x[j], m) * scale : sigmoid(x[j]);
            const double c = a.bias ? s + static_cast<double>(a.bias[first + j]) : s;
            if (c > none) choice[j] = c;
        }
        bool stay = true;
        if (a.groups > 1) {
            double b1 = none, b2 = none;
#pragma unroll
            for (int j = 0; j < EPL; ++j) {
                b2 = max64(b2, min64(b1, choice[j]));
                b1 = max64(b1, choice[j]);
            }
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
            stay = better < a.top_groups;
        }
#pragma unroll
        for (int j = 0; j < EPL; ++j)
            key[j] = stay && choice[j] > none
                         ? key_of(a.bias ? choice[j] : static_cast<double>(x[j]), first + j)
                         : none;
    } else {
#pragma unroll
        for (int j = 0; j < EPL; ++j)
            key[j] = x[j] > none ? key_of(static_cast<double>(x[j]), first + j) : none;
    }
    sort_descending(key);

    int id = -1;  // of lane i: the i-th best
    for (int i = 0; i < a.topk; ++i) {
        const double best = wave_reduce(key[0], Max64{});
        if (!(best > none)) break;  // the same in every lane
        if (lane == i) id = expert_of(best);
        const bool taken = key[0] == best;
#pragma unroll
        for (int j = 0; j + 1 < EPL; ++j) key[j] = taken ? key[j + 1] : key[j];
        key[EPL - 1] = taken ? none : key[EPL - 1];
    }
    double w = 0.0;
    if (id >= 0) {
        const float xi = widen<D>(row[id]);
        w = softmax ? softmax_weight(xi, m) * scale : sigmoid(xi);
    }
    if (a.renorm) {
        const double sum = wave_reduce(w, Add{});
        w = sum > 0.0 ? w / sum : 0.0;
    }
    if (lane < a.topk) {
        a.ids[t * a.topk + lane] = id;
        a.weights[t * a.topk + lane] = static_cast<float>(w * static_cast<double>(a.scale));
    }
}

template <int D>
hipError_t launch_route(const RouteArgs &n, hipStream_t s) {
    const int need = (n.per + n.lanes - 1) / n.lanes;
    const dim3 grid((n.a.tokens + kWaves - 1) / kWaves), block(kRowWave, kWaves);
    if (need <= 1) route_kernel<D, 1><<<grid, block, 0, s>>>(n);
    else if (need <= 2) route_kernel<D, 2><<<grid, block, 0, s>>>(n);
    else if (need <= 4) route_kernel<D, 4><<<grid, block, 0, s>>>(n);
    else if (need <= 8) route_kernel<D, 8><<<grid, block, 0, s>>>(n);
    else if (need <= 16) route_kernel<D, 16><<<grid, block, 0, s>>>(n);
    else route_kernel<D, 32><<<grid, block, 0, s>>>(n);
    return hipGetLastError();
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
