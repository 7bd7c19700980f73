// Norms before and after a block, fused with its gate, its scale and the
// residual stream: sifar_block_norm. gfx950 (MI355X) only.
//
// A row's two mean squares need the row twice: a = the block's output (or the
// sum of its partials) for the post-norm, r' = the new residual for the next
// block's norm. Both passes run on registers: a workgroup holds one row, eight
// adjacent elements a lane and vector, so each input is read and each output
// written once. Bound: HBM bytes for many rows; for a few rows the launch, two
// workgroup reductions and dependent memory round trips: the row, each further
// partial, and the norm's weights behind the second reduction. Measured: 4096 x 5120
// bf16 with an fp32 residual 47.8 us a call, 5.3 TB/s, the rate of a copy; in a graph
// 64 x 8192 over 8 partials 5.6 us and 1 x 4096 3.0.
#include <hip/hip_runtime.h>

#include "rows.h"

namespace sifar {
namespace {

constexpr int kMaxThreads = 1024;
constexpr int kMaxParts = 8;

struct NormArgs {
    sifar_block_norm_args a;
    float inv_hidden;
};

// The sum of v over the row's waves, in the same order in every wave: a
// butterfly in each wave, then the waves' sums in ascending order. `part` is
// one array per reduction, so a single barrier separates its writes and reads.
__device__ __forceinline__ float row_sum(float v, float *part, int wave, int waves) {
    v = wave_reduce(v, Add{});
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) part[wave] = v;
    __syncthreads();
    float s = part[0];
    for (int w = 1; w < waves; ++w) s += part[w];
    return s;
}

// D, R: element types of x and of the residual. V: vectors of 8 elements a lane.
template <int D, int R, int V>
__global__ void __launch_bounds__(kMaxThreads) block_norm_kernel(const NormArgs n) {
    __shared__ float part[2][kMaxThreads / kRowWave];
    const sifar_block_norm_args &a = n.a;
    const int waves = blockDim.x / kRowWave;
    const int wave = threadIdx.x / kRowWave;
    const int64_t t = blockIdx.x;
    const bool gated = a.gate != nullptr;
    const bool posted = a.post_weight != nullptr;
    const bool added = a.residual != nullptr;

    // Up to two vectors a lane, the post-norm's weights, gate and residual are loaded
    // before the first reduction; longer rows load them a vector at a time, where they
    // are used. (The next norm's weights are loaded where they are used in any row.)
    constexpr bool AHEAD = V <= 2;
    int h[V];
    bool on[V];
    Eight<D> x[V], gate[V], post[V];
    Eight<R> res[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        h[v] = (v * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * 8;
        on[v] = h[v] < a.hidden;
        if (on[v]) x[v] = load8<D>(a.x, t * a.x_stride + h[v]);
    }
    float f[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[v][i] = on[v] ? element<D>(x[v], i) : 0.f;
        if (!AHEAD || !on[v]) continue;
        if (posted) post[v] = load8<D>(a.post_weight, h[v]);
        if (gated) gate[v] = load8<D>(a.gate, t * a.gate_stride + h[v]);
        if (added) res[v] = load8<R>(a.residual, t * a.residual_stride + h[v]);
    }
    // The other partials. Each load stands under a condition of its own, and the
    // compiler waits for one before it issues the next: a memory round trip each,
    // whatever FLIGHT says (1 x 8192 in a graph 4.0 us of one partial, 5.4 of eight).
    constexpr int FLIGHT = V == 1 ? kMaxParts - 1 : V == 2 ? 2 : 1;
    for (int p = 1; p < a.parts; p += FLIGHT) {
        if constexpr (AHEAD) {
            Eight<D> e[FLIGHT][V];
#pragma unroll
            for (int q = 0; q < FLIGHT; ++q)
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (p + q < a.parts && on[v])
                        e[q][v] = load8<D>(a.x, (p + q) * a.part_stride + t * a.x_stride + h[v]);
#pragma unroll
            for (int q = 0; q < FLIGHT; ++q)
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (p + q < a.parts && on[v])
#pragma unroll
                        for (int i = 0; i < 8; ++i) f[v][i] += element<D>(e[q][v], i);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!on[v]) continue;
                const Eight<D> e = load8<D>(a.x, p * a.part_stride + t * a.x_stride + h[v]);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[v][i] += element<D>(e, i);
            }
        }
    }
    float inv = 1.f;
    if (posted) {
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) s = __builtin_fmaf(f[v][i], f[v][i], s);
        s = row_sum(s, part[0], wave, waves);
        inv = 1.f / __builtin_sqrtf(__builtin_fmaf(s, n.inv_hidden, a.eps));
    }
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (!on[v]) continue;
        if (!AHEAD) {
            if (posted) post[v] = load8<D>(a.post_weight, h[v]);
            if (gated) gate[v] = load8<D>(a.gate, t * a.gate_stride + h[v]);
            if (added) res[v] = load8<R>(a.residual, t * a.residual_stride + h[v]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float b = f[v][i];
            if (posted) b = b * inv * (a.weight_offset + element<D>(post[v], i));
            if (gated) b *= element<D>(gate[v], i);
            b *= a.branch_scale;
            if (added) b = __builtin_fmaf(a.residual_scale, element<R>(res[v], i), b);
            f[v][i] = b;
            s = __builtin_fmaf(b, b, s);
        }
        store8<R>(a.residual_out, t * a.residual_out_stride + h[v], f[v]);
    }
    if (!a.y) return;  // the same in every lane
    s = row_sum(s, part[1], wave, waves);
    inv = 1.f / __builtin_sqrtf(__builtin_fmaf(s, n.inv_hidden, a.eps));
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (!on[v]) continue;
        const Eight<D> w = load8<D>(a.norm_weight, h[v]);
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            o[i] = f[v][i] * inv * (a.weight_offset + element<D>(w, i));
        store8<D>(a.y, t * a.y_stride + h[v], o);
    }
}

template <int D, int R>
hipError_t launch_norm(const sifar_block_norm_args &a, hipStream_t s) {
    // Vectors of 8 a lane: as few as 1024 lanes allow. A row of one partial that would take
    // 768 lanes or more takes half of them with twice the vectors, so that another row's
    // workgroup loads while its waves wait for each other. us a call in a graph, bf16, with
    // the fewest vectors and with twice as many, for 1, 512 and 4096 rows:
    //    5632 (704 lanes)   3.1 3.5   5.0  5.1    32  28     not by the rule
    //    6144 (768)         3.2 3.5   5.0  5.2    32  30
    //    7168 (896)         3.7 3.6   6.1  5.5    43  35
    //    8192 (1024)        3.8 3.7   6.2  5.7    44  40
    //   12288 (768 x 2)     4.0 5.4   7.3  7.9    57  58
    //   16384 (1024 x 2)    5.0 5.6  12.4 10.1   104  79
    // (4096 x 5120 with an fp32 residual 39.4 and 42.4.) So the longest rows of each kind
    // gain where there are many, and the edge itself costs a few rows a tenth. Over
    // several partials more lanes keep more loads in flight (64 x 8192 over 8 partials
    // 5.5 and 6.1). The batch has no say: a row's sums do not depend on it.
    const int vecs = a.hidden / 8;
    int V = vecs <= kMaxThreads ? 1 : vecs <= 2 * kMaxThreads ? 2 : vecs <= 4 * kMaxThreads ? 4 : 8;
    if (a.parts == 1 && V <= 2 && vecs >= 768 * V) V *= 2;
    const int lanes = (vecs + V - 1) / V;
    const int threads = (lanes + kRowWave - 1) / kRowWave * kRowWave;
    NormArgs n{};
    n.a = a;
    n.inv_hidden = static_cast<float>(1.0 / a.hidden);
    const dim3 grid(a.tokens), block(threads);
    switch (V) {
        case 1: block_norm_kernel<D, R, 1><<<grid, block, 0, s>>>(n); break;
        case 2: block_norm_kernel<D, R, 2><<<grid, block, 0, s>>>(n); break;
        case 4: block_norm_kernel<D, R, 4><<<grid, block, 0, s>>>(n); break;
        default: block_norm_kernel<D, R, 8><<<grid, block, 0, s>>>(n); break;
    }
    return hipGetLastError();
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

uint64_t size_of(int32_t dtype) { return dtype == SIFAR_FP32 ? 4 : 2; }

Rows rows_of(const void *p, int32_t dtype, int64_t tokens, int64_t stride, int64_t hidden) {
    Rows r;
    r.at = reinterpret_cast<uintptr_t>(p);
    r.rows = static_cast<uint64_t>(stride == 0 ? 1 : tokens);
    r.stride = static_cast<uint64_t>(stride) * size_of(dtype);
    r.size = static_cast<uint64_t>(hidden) * size_of(dtype);
    return r;
}

// A row stride, which only several tokens use: a multiple of 8 that keeps them apart.
bool good_stride(int64_t stride, int32_t tokens, int32_t hidden) {
    return tokens <= 1 ||
           (stride % 8 == 0 && stride >= hidden && stride <= (int64_t{1} << 40));
}

bool good(const sifar_block_norm_args &a) {
    if (a.dtype < SIFAR_BF16 || a.dtype > SIFAR_FP32) return false;
    if (a.residual_dtype != a.dtype && a.residual_dtype != SIFAR_FP32) return false;
    if (a.tokens < 0 || a.tokens > SIFAR_ROWS_MAX_TOKENS) return false;
    if (a.hidden < 8 || a.hidden > 65536 || a.hidden % 8) return false;
    if (a.parts < 1 || a.parts > kMaxParts) return false;
    if (!(a.eps >= 0.0f)) return false;
    if (a.tokens == 0) return true;
    if (!a.x || !a.residual_out || !a.norm_weight != !a.y) return false;
    for (const void *p : {a.x, a.post_weight, a.gate, a.residual, static_cast<const void *>(a.residual_out),
                          a.norm_weight, static_cast<const void *>(a.y)})
        if (!aligned16(p)) return false;
    if (!good_stride(a.x_stride, a.tokens, a.hidden) ||
        !good_stride(a.residual_out_stride, a.tokens, a.hidden) ||
        (a.residual && !good_stride(a.residual_stride, a.tokens, a.hidden)) ||
        (a.y && !good_stride(a.y_stride, a.tokens, a.hidden)) ||
        (a.gate && a.gate_stride != 0 && !good_stride(a.gate_stride, a.tokens, a.hidden)))
        return false;
    if (a.parts > 1 && (a.part_stride % 8 || a.part_stride < 0 ||
                        a.part_stride > (int64_t{1} << 40)))
        return false;

    // What a row's workgroup writes, no other row's may read or write.
    const Rows x = rows_of(a.x, a.dtype, a.tokens, a.x_stride, a.hidden);
    const Rows res = rows_of(a.residual, a.residual_dtype, a.tokens, a.residual_stride, a.hidden);
    const Rows gate = rows_of(a.gate, a.dtype, a.tokens, a.gate_stride, a.hidden);
    const Rows out[2] = {
        rows_of(a.residual_out, a.residual_dtype, a.tokens, a.residual_out_stride, a.hidden),
        rows_of(a.y, a.dtype, a.tokens, a.y_stride, a.hidden)};
    if (may_overlap(out[0], out[1])) return false;
    for (const Rows &o : out) {
        if (empty(o)) continue;
        for (const Rows &in : {x, res, gate}) {
            const bool per_token = in.stride != 0 || a.tokens == 1;
            if (may_overlap(o, in) && !(per_token && same_rows(o, in))) return false;
        }
        for (int p = 1; p < a.parts; ++p) {
            Rows later = x;
            later.at += static_cast<uint64_t>(p) * static_cast<uint64_t>(a.part_stride) *
                        size_of(a.dtype);
            if (may_overlap(o, later)) return false;
        }
        for (const void *w : {a.post_weight, a.norm_weight})
            if (may_overlap(o, rows_of(w, a.dtype, 1, 0, a.hidden))) return false;
    }
    return true;
}

}  // namespace
}  // namespace sifar

extern "C" int sifar_block_norm(const sifar_block_norm_args *args, void *stream) {
    using namespace sifar;
    if (!args || !good(*args)) return SIFAR_EINVAL;
    const sifar_block_norm_args &a = *args;
    if (a.tokens == 0) return SIFAR_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (a.dtype == SIFAR_FP32) e = launch_norm<SIFAR_FP32, SIFAR_FP32>(a, s);
    else if (a.dtype == SIFAR_BF16)
        e = a.residual_dtype == SIFAR_FP32 ? launch_norm<SIFAR_BF16, SIFAR_FP32>(a, s)
                                           : launch_norm<SIFAR_BF16, SIFAR_BF16>(a, s);
    else
        e = a.residual_dtype == SIFAR_FP32 ? launch_norm<SIFAR_FP16, SIFAR_FP32>(a, s)
                                           : launch_norm<SIFAR_FP16, SIFAR_FP16>(a, s);
    return e == hipSuccess ? SIFAR_OK : SIFAR_EHIP;
}
