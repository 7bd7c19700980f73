// A mixture-of-experts layer for a few tokens: sifar_experts. gfx950 (MI355X) only.
//
// Of the weights, those of the experts that some token names have to be read once, and
// few tokens share them: bound by HBM bytes. Two launches, one for each product, with a
// row of 16 weights as the matrix instructions' first operand straight from memory and
// up to 64 tokens of the expert as columns:
//
//  in    a workgroup makes 16 elements of h for one expert that some token names: the
//        gate's rows and the up rows, its four waves a quarter of `hidden` each. Which
//        experts those are it finds in ids by itself (a bit each in LDS), so the grid has
//        no workgroup for an expert that nobody named, and no third launch plans it.
//        The first workgroup of an expert leaves its list of slots to the second launch.
//  out   a workgroup makes 16 elements of every token's output: its waves share the
//        experts, or parts of `inter` where those are fewer than waves, each slot's row
//        goes to LDS, and the slots of a token are summed in their order.
//
// h passes between the launches in fp32 (fp32) or as two bf16 elements whose sum is
// good to 2^-17 (16-bit types; bf16, because h in fp16 could overflow). fp16 weights
// meet it as two bf16 elements too, which hold their 11 bits exactly.
#include <hip/hip_runtime.h>

#include "operands.h"
#include "rows.h"
#include "tiles.h"

namespace sifar {
namespace {

constexpr int kInWaves = 4, kOutWaves = 8;
constexpr int kInThreads = kInWaves * kRowWave, kOutThreads = kOutWaves * kRowWave;
constexpr int kRows = 16;
constexpr int kMaxSlots = SIFAR_EXPERTS_MAX_SLOTS;
constexpr int kMaxExperts = SIFAR_ROUTE_MAX_EXPERTS;

// What the first launch leaves in the workspace: how many experts are named, and for the
// n-th of them its index and where its slots stand in the list.
struct Plan {
    int32_t named;
    int32_t pad[3];
};

struct ExpertsArgs {
    sifar_experts_args a;
    int32_t slots;   // tokens * topk
    int32_t named;   // experts that can be named at most
    int64_t at_list; // from the workspace's start, in int32: {expert, first, count} of the
                     // n-th behind Plan, then the list
    int64_t at_h;    // in bytes
};

__device__ __forceinline__ int local_expert(const sifar_experts_args &a, int slot) {
    const uint32_t e = static_cast<uint32_t>(a.ids[slot]) - static_cast<uint32_t>(a.first_expert);
    return e < static_cast<uint32_t>(a.experts) ? static_cast<int>(e) : -1;
}

// 64 bytes of each of 16 rows, a quarter a lane; behind `bytes` of a row zeros.
__device__ __forceinline__ U4 load_step(const unsigned char *row, int at, int bytes, bool whole) {
    if (whole) return *reinterpret_cast<const U4 *>(row + at);
    const U4 w = *reinterpret_cast<const U4 *>(row + (at < bytes ? at : 0));
    return at < bytes ? w : U4{0, 0, 0, 0};
}

__device__ __forceinline__ float act(float g, int activation) {
    // GELU's tanh form is x / (1 + exp(-2 y)) with tanh's argument y
    const float y = activation == SIFAR_EXPERTS_GELU
                        ? 0x1.988454p+0f * __builtin_fmaf(0x1.6e4e26p-5f * g * g, g, g)
                        : g;
    return g / (1.f + __builtin_amdgcn_exp2f(y * -0x1.715476p+0f));
}

// `rows` of 16 weights each (the gate's, the up ones) times up to 16 * TILES columns over
// the wave's steps of a row.
template <int D, int TILES, int AHEAD>
__device__ __forceinline__ void in_product(const unsigned char *const (&w)[2],
                                           const unsigned char *const (&x)[TILES], int from, int to,
                                           int bytes, F4 (&sum)[2][TILES]) {
    const int at = 16 * ((threadIdx.x & 63) >> 4);
    int s = from;
    const int whole = to * 64 <= bytes ? to : to - 1;  // steps that no row ends in
    for (; s + AHEAD <= whole; s += AHEAD) {
        U4 wa[AHEAD][2], xa[AHEAD][TILES];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
                wa[i][j] = *reinterpret_cast<const U4 *>(w[j] + 64 * (s + i) + at);
#pragma unroll
            for (int c = 0; c < TILES; ++c)
                xa[i][c] = *reinterpret_cast<const U4 *>(x[c] + 64 * (s + i) + at);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int c = 0; c < TILES; ++c) sum[j][c] = mma<D>(wa[i][j], xa[i][c], sum[j][c]);
    }
    for (; s < to; ++s) {
        U4 wa[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) wa[j] = load_step(w[j], 64 * s + at, bytes, s < whole);
#pragma unroll
        for (int c = 0; c < TILES; ++c) {
            const U4 xa = load_step(x[c], 64 * s + at, bytes, s < whole);
#pragma unroll
            for (int j = 0; j < 2; ++j) sum[j][c] = mma<D>(wa[j], xa, sum[j][c]);
        }
    }
}

// Columns base.. of the expert's slots: both products, the waves' parts joined, h stored.
template <int D, int TILES, int AHEAD>
__device__ __forceinline__ void in_columns(const ExpertsArgs &n, int expert, int row, const int *list,
                                           int base, int count, F4 (*parts)[2][4][kRowWave]) {
    constexpr int SIZE = D == SIFAR_FP32 ? 4 : 2;
    const sifar_experts_args &a = n.a;
    const int lane = threadIdx.x & 63, column = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int bytes = a.hidden * SIZE;
    const int mine = row + column < a.inter ? row + column : a.inter - 1;  // what is cut is not stored
    const unsigned char *matrix = static_cast<const unsigned char *>(a.w_in) +
                                  expert * a.w_in_stride * SIZE;
    const unsigned char *const w[2] = {
        matrix + static_cast<int64_t>(mine) * bytes,
        matrix + (static_cast<int64_t>(a.inter) + mine) * bytes};
    const unsigned char *x[TILES];
#pragma unroll
    for (int c = 0; c < TILES; ++c) {
        const int i = base + 16 * c + column;
        x[c] = static_cast<const unsigned char *>(a.x) +
               list[i < count ? i : base] / a.topk * a.x_stride * SIZE;
    }
    F4 sum[2][TILES];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int c = 0; c < TILES; ++c) sum[j][c] = F4{0.f, 0.f, 0.f, 0.f};
    const int steps = (bytes + 63) / 64, each = (steps + kInWaves - 1) / kInWaves;
    const int from = wave * each < steps ? wave * each : steps;
    in_product<D, TILES, AHEAD>(w, x, from, from + each < steps ? from + each : steps, bytes, sum);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int c = 0; c < TILES; ++c) parts[wave][j][c][lane] = sum[j][c];
    __syncthreads();
    // wave c joins the columns of tile c: lane (column, quarter) holds rows 4 quarter ..
    if (wave < TILES) {
        F4 g = parts[0][0][wave][lane], u = parts[0][1][wave][lane];
        for (int v = 1; v < kInWaves; ++v) {
            g += parts[v][0][wave][lane];
            u += parts[v][1][wave][lane];
        }
        F4 h;
#pragma unroll
        for (int r = 0; r < 4; ++r) h[r] = act(g[r], a.activation) * u[r];
        const int i = base + 16 * wave + column, at = row + 4 * (lane >> 4);
        if (i < count && at < a.inter) {  // inter is a multiple of 8
            unsigned char *to = static_cast<unsigned char *>(a.workspace) + n.at_h;
            const int64_t e = static_cast<int64_t>(list[i]) * a.inter + at;
            if constexpr (D == SIFAR_FP32) {
                *reinterpret_cast<F4 *>(to + 4 * e) = h;
            } else {
                typedef uint32_t U2 __attribute__((ext_vector_type(2)));
                const Split p = split<SIFAR_BF16>(h[0], h[1]), q = split<SIFAR_BF16>(h[2], h[3]);
                *reinterpret_cast<U2 *>(to + 2 * e) = U2{p.high, q.high};
                to += 2 * static_cast<int64_t>(n.slots) * a.inter;
                *reinterpret_cast<U2 *>(to + 2 * e) = U2{p.low, q.low};
            }
        }
    }
    __syncthreads();  // parts and, behind the last columns, nothing else is written again
}

template <int D>
__global__ void __launch_bounds__(kInThreads) in_kernel(const ExpertsArgs n) {
    __shared__ uint32_t bits[kMaxExperts / 32];
    __shared__ int list[kMaxSlots];
    __shared__ int count, before;
    __shared__ F4 parts[kInWaves][2][4][kRowWave];
    const sifar_experts_args &a = n.a;
    const int nth = blockIdx.y;

    // The experts of the slots: the nth that is named is this workgroup's.
    constexpr int EACH = kMaxSlots / kInThreads;
    int expert[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int slot = i * kInThreads + static_cast<int>(threadIdx.x);
        expert[i] = slot < n.slots ? local_expert(a, slot) : -1;
    }
    const int words = (a.experts + 31) / 32;
    if (static_cast<int>(threadIdx.x) < words) bits[threadIdx.x] = 0;
    if (threadIdx.x == 0) count = before = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (expert[i] >= 0) atomicOr(&bits[expert[i] / 32], 1u << (expert[i] & 31));
    __syncthreads();
    int mine = -1, named = 0;
    for (int w = 0; w < words; ++w) {
        uint32_t b = bits[w];
        const int here = __builtin_popcount(b);
        if (mine < 0 && nth < named + here) {
            for (int skip = nth - named; skip > 0; --skip) b &= b - 1;
            mine = 32 * w + __builtin_ctz(b);
        }
        named += here;
    }
    int32_t *plan = static_cast<int32_t *>(a.workspace);
    if (nth == 0 && blockIdx.x == 0 && threadIdx.x == 0) plan[0] = named;
    if (mine < 0) return;  // the same for the workgroup

    // Its slots, in any order: a column's sums do not depend on where it stands.
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (expert[i] == mine)
            list[atomicAdd(&count, 1)] = i * kInThreads + static_cast<int>(threadIdx.x);
        else if (expert[i] >= 0 && expert[i] < mine)
            atomicAdd(&before, 1);
    }
    __syncthreads();
    if (blockIdx.x == 0) {
        int32_t *mark = plan + 4 + 4 * nth;
        if (threadIdx.x == 0) {
            mark[0] = mine;
            mark[1] = before;
            mark[2] = count;
        }
        for (int i = threadIdx.x; i < count; i += kInThreads) plan[n.at_list + before + i] = list[i];
    }

    const int row = kRows * blockIdx.x, all = count;
    for (int base = 0; base < all; base += 64) {
        const int left = all - base;
        if (left <= 16) in_columns<D, 1, 8>(n, mine, row, list, base, all, parts);
        else if (left <= 32) in_columns<D, 2, 4>(n, mine, row, list, base, all, parts);
        else in_columns<D, 4, 2>(n, mine, row, list, base, all, parts);
    }
}

// h as the second operand: fp32, or what two bf16 elements add up to.
template <int D>
struct Hidden {
    U4 v[D == SIFAR_FP32 ? 1 : 2];
};

template <int D>
__device__ __forceinline__ F4 out_mma(const U4 &w, const Hidden<D> &h, F4 c) {
    if constexpr (D == SIFAR_FP32) {
        return mma<SIFAR_FP32>(w, h.v[0], c);
    } else if constexpr (D == SIFAR_BF16) {
        c = mma<SIFAR_BF16>(w, h.v[0], c);
        return mma<SIFAR_BF16>(w, h.v[1], c);
    } else {
        U4 high, low;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Split p = split<SIFAR_BF16>(low_half<SIFAR_FP16>(w[i]), high_half<SIFAR_FP16>(w[i]));
            high[i] = p.high;
            low[i] = p.low;
        }
        c = mma<SIFAR_BF16>(high, h.v[0], c);
        c = mma<SIFAR_BF16>(high, h.v[1], c);
        return mma<SIFAR_BF16>(low, h.v[0], c);
    }
}

// The columns base.. of an expert's slots over steps from..to of `inter`; each slot's sums
// go to its row of `rows`.
template <int D, int TILES, int AHEAD>
__device__ __forceinline__ void out_columns(const ExpertsArgs &n, int expert, int row,
                                            const int32_t *list, int base, int count, int from, int to,
                                            float *rows) {
    constexpr int SIZE = D == SIFAR_FP32 ? 4 : 2;
    const sifar_experts_args &a = n.a;
    const int lane = threadIdx.x & 63, column = lane & 15, at = 16 * (lane >> 4);
    const int bytes = a.inter * SIZE;
    const int mine = row + column < a.hidden ? row + column : a.hidden - 1;
    const unsigned char *w = static_cast<const unsigned char *>(a.w_out) +
                             expert * a.w_out_stride * SIZE + static_cast<int64_t>(mine) * bytes;
    const unsigned char *hidden = static_cast<const unsigned char *>(a.workspace) + n.at_h;
    const int64_t low = static_cast<int64_t>(n.slots) * bytes;  // behind the first elements
    const unsigned char *x[TILES];
    int slot[TILES];
#pragma unroll
    for (int c = 0; c < TILES; ++c) {
        const int i = base + 16 * c + column;
        slot[c] = list[i < count ? i : base];
        x[c] = hidden + static_cast<int64_t>(slot[c]) * bytes;
    }
    F4 sum[TILES];
#pragma unroll
    for (int c = 0; c < TILES; ++c) sum[c] = F4{0.f, 0.f, 0.f, 0.f};
    const auto load_hidden = [&](int c, int s, bool whole) {
        Hidden<D> h;
        h.v[0] = load_step(x[c], 64 * s + at, bytes, whole);
        if constexpr (D != SIFAR_FP32) h.v[1] = load_step(x[c] + low, 64 * s + at, bytes, whole);
        return h;
    };
    int s = from;
    const int whole = to * 64 <= bytes ? to : to - 1;
    for (; s + AHEAD <= whole; s += AHEAD) {
        U4 wa[AHEAD];
        Hidden<D> h[AHEAD][TILES];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            wa[i] = *reinterpret_cast<const U4 *>(w + 64 * (s + i) + at);
#pragma unroll
            for (int c = 0; c < TILES; ++c) h[i][c] = load_hidden(c, s + i, true);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int c = 0; c < TILES; ++c) sum[c] = out_mma<D>(wa[i], h[i][c], sum[c]);
    }
    for (; s < to; ++s) {
        const U4 wa = load_step(w, 64 * s + at, bytes, s < whole);
#pragma unroll
        for (int c = 0; c < TILES; ++c) sum[c] = out_mma<D>(wa, load_hidden(c, s, s < whole), sum[c]);
    }
#pragma unroll
    for (int c = 0; c < TILES; ++c)
        if (base + 16 * c + column < count)
            *reinterpret_cast<F4 *>(rows + slot[c] * kRows + 4 * (lane >> 4)) = sum[c];
}

// Parts that `inter` is cut into: waves that the experts leave idle, as long as all slots'
// rows of all parts fit.
__device__ __forceinline__ int parts_of(int named, int slots) {
    int parts = kOutWaves;
    while (parts > 1 && (parts * named > kOutWaves || parts * slots > kMaxSlots)) parts /= 2;
    return parts;
}

template <int D>
__global__ void __launch_bounds__(kOutThreads) out_kernel(const ExpertsArgs n) {
    extern __shared__ __attribute__((aligned(16))) float rows[];  // [parts][slots][kRows]
    constexpr int SIZE = D == SIFAR_FP32 ? 4 : 2;
    const sifar_experts_args &a = n.a;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), row = kRows * blockIdx.x;
    const int32_t *plan = static_cast<const int32_t *>(a.workspace);
    const int named = plan[0];
    const int parts = parts_of(named, n.slots);
    const int steps = (a.inter * SIZE + 63) / 64, each = (steps + parts - 1) / parts;
    for (int unit = wave; unit < named * parts; unit += kOutWaves) {
        const int nth = unit / parts, part = unit % parts;
        const int32_t *mark = plan + 4 + 4 * nth;
        const int expert = mark[0], count = mark[2];
        const int32_t *list = plan + n.at_list + mark[1];
        const int from = part * each < steps ? part * each : steps;
        const int to = from + each < steps ? from + each : steps;
        float *mine = rows + part * n.slots * kRows;
        for (int base = 0; base < count; base += 64) {
            const int left = count - base;
            if (left <= 16) out_columns<D, 1, 8>(n, expert, row, list, base, count, from, to, mine);
            else if (left <= 32) out_columns<D, 2, 4>(n, expert, row, list, base, count, from, to, mine);
            else out_columns<D, 4, 2>(n, expert, row, list, base, count, from, to, mine);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.tokens * kRows; i += kOutThreads) {
        const int t = i / kRows, r = i % kRows;
        if (row + r >= a.hidden) continue;
        float f = 0.f;
        for (int j = 0; j < a.topk; ++j) {
            const int slot = t * a.topk + j;
            if (local_expert(a, slot) < 0) continue;
            float y = rows[slot * kRows + r];
            for (int p = 1; p < parts; ++p) y += rows[(p * n.slots + slot) * kRows + r];
            f = __builtin_fmaf(a.weights[slot], y, f);
        }
        const int64_t at = t * a.out_stride + row + r;
        if constexpr (D == SIFAR_FP32) static_cast<float *>(a.out)[at] = f;
        else static_cast<uint16_t *>(a.out)[at] = static_cast<uint16_t>(pack16<D>(f, f));
    }
}

int64_t plan_words(int64_t slots) { return 4 + 4 * slots + slots; }

template <int D>
hipError_t launch(const sifar_experts_args &a, hipStream_t s) {
    ExpertsArgs n{};
    n.a = a;
    n.slots = a.tokens * a.topk;
    n.named = a.experts < n.slots ? a.experts : n.slots;
    n.at_list = 4 + 4 * static_cast<int64_t>(n.slots);
    n.at_h = (4 * plan_words(n.slots) + 255) / 256 * 256;
    in_kernel<D><<<dim3((a.inter + kRows - 1) / kRows, n.named), kInThreads, 0, s>>>(n);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int most = kOutWaves * n.slots < kMaxSlots ? kOutWaves * n.slots : kMaxSlots;
    out_kernel<D><<<(a.hidden + kRows - 1) / kRows, kOutThreads, most * kRows * 4, s>>>(n);
    return hipGetLastError();
}

bool good_sizes(int64_t tokens, int64_t topk, int64_t inter) {
    return tokens >= 0 && tokens <= SIFAR_EXPERTS_MAX_TOKENS && topk >= 1 &&
           topk <= SIFAR_ROUTE_MAX_TOPK && tokens * topk <= SIFAR_EXPERTS_MAX_SLOTS && inter >= 8 &&
           inter <= 65536 && inter % 8 == 0;
}

bool good(const sifar_experts_args &a) {
    if (!good_dtype(a.dtype) || !good_sizes(a.tokens, a.topk, a.inter)) return false;
    if (a.hidden < 8 || a.hidden > 65536 || a.hidden % 8) return false;
    if (a.experts < 1 || a.experts > SIFAR_ROUTE_MAX_EXPERTS || a.first_expert < 0) return false;
    if (a.activation != SIFAR_EXPERTS_SILU && a.activation != SIFAR_EXPERTS_GELU) return false;
    const int64_t matrix = static_cast<int64_t>(a.inter) * a.hidden;
    if (!good_stride(a.w_in_stride, a.experts, 2 * matrix) ||
        !good_stride(a.w_out_stride, a.experts, matrix))
        return false;
    if (a.tokens == 0) return true;
    if (!a.x || !a.ids || !a.weights || !a.w_in || !a.w_out || !a.out || !a.workspace) return false;
    for (const void *p : {a.x, a.w_in, a.w_out, static_cast<const void *>(a.out),
                          static_cast<const void *>(a.workspace)})
        if (!aligned16(p)) return false;
    if (!aligned4(a.ids) || !aligned4(a.weights)) return false;
    if (!good_stride(a.x_stride, a.tokens, a.hidden) ||
        !good_stride(a.out_stride, a.tokens, a.hidden))
        return false;
    const int64_t need = sifar_experts_workspace(a.tokens, a.topk, a.inter);
    if (a.workspace_bytes < need) return false;
    const uint64_t size = size_of(a.dtype), slots = static_cast<uint64_t>(a.tokens) * a.topk;
    const uint64_t last = static_cast<uint64_t>(a.experts - 1);
    const auto stride = [&](int64_t s) { return a.experts > 1 ? static_cast<uint64_t>(s) : 0; };
    const Rows out[] = {rows_of(a.out, a.dtype, a.tokens, a.out_stride, a.hidden),
                        span_of(a.workspace, static_cast<uint64_t>(need))};
    const Rows in[] = {rows_of(a.x, a.dtype, a.tokens, a.x_stride, a.hidden),
                       span_of(a.ids, 4 * slots), span_of(a.weights, 4 * slots),
                       span_of(a.w_in, size * (last * stride(a.w_in_stride) + 2 * matrix)),
                       span_of(a.w_out, size * (last * stride(a.w_out_stride) + matrix))};
    if (may_overlap(out[0], out[1])) return false;
    for (const Rows &o : out)
        for (const Rows &i : in)
            if (may_overlap(o, i)) return false;
    return true;
}

}  // namespace
}  // namespace sifar

extern "C" int64_t sifar_experts_workspace(int32_t tokens, int32_t topk, int32_t inter) {
    using namespace sifar;
    if (!good_sizes(tokens, topk, inter)) return SIFAR_EINVAL;
    const int64_t slots = static_cast<int64_t>(tokens) * topk;
    return (4 * plan_words(slots) + 255) / 256 * 256 + 4 * slots * inter;
}

extern "C" int sifar_experts(const sifar_experts_args *args, void *stream) {
    using namespace sifar;
    if (!args || !good(*args)) return SIFAR_EINVAL;
    const sifar_experts_args &a = *args;
    if (a.tokens == 0) return SIFAR_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = a.dtype == SIFAR_FP32   ? launch<SIFAR_FP32>(a, s)
                         : a.dtype == SIFAR_BF16 ? launch<SIFAR_BF16>(a, s)
                                                 : launch<SIFAR_FP16>(a, s);
    return e == hipSuccess ? SIFAR_OK : SIFAR_EHIP;
}
