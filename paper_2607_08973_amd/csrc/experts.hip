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
//        Where more than four tokens share the expert, their rows are read in order and
//        turned to the operand in LDS.
//  out   a workgroup makes 16 elements of every token's output: its waves share the
//        experts, or parts of `inter` where those are fewer than waves, each slot's row
//        goes to LDS, and the slots of a token are summed in their order. h lies in the
//        order of its loads, and two batches of them are in flight.
//
// h passes between the launches in fp32 (fp32) or as two bf16 elements whose sum is
// good to 2^-17 (16-bit types; bf16, because h in fp16 could overflow). fp16 weights
// meet it as two bf16 elements too, which hold their 11 bits exactly.
//
// Measured, bf16, us of the two launches: 16 tokens, 6 of 64 experts, 4096 x 1408 (41 of
// them named) 171 + 98, 5.5 and 4.8 TB/s; 64 tokens, 2 of 8, 4096 x 8192 220 + 174, 4.9 and
// 3.1 (h comes from the L2s in twice as many bytes); one token, 8 of 128, 2048 x 768 15 + 13, the
// latency of the ids or the plan and of two to six batches, and in the second launch the
// half of the CUs that its 128 workgroups leave idle. Reads of weights alone, 16 rows
// at a time, reach 6.4 TB/s.
#include <hip/hip_runtime.h>

#include "operands.h"
#include "rows.h"
#include "tiles.h"

namespace sifar {
namespace {

constexpr int kInWaves = 4, kOutWaves = 8;
constexpr int kInThreads = kInWaves * kRowWave, kOutThreads = kOutWaves * kRowWave;
constexpr int kRows = 16;
constexpr int kInAhead = 4, kOutAhead = 4;  // steps of a batch of loads, for 16 columns
constexpr int kFew = 4;  // columns up to which x is read as it is used (1, 4, 16: no change but
                         // at 16, where 64 tokens took 230 us for 217)
constexpr int kMaxSlots = SIFAR_EXPERTS_MAX_SLOTS;
constexpr int kMaxExperts = SIFAR_ROUTE_MAX_EXPERTS;

template <int N>
constexpr std::integral_constant<int, N> kInt{};

// What the first launch leaves in the workspace for the second, in int32: how many experts
// are named, and behind 4 words, 4 for each of them in ascending order: its index, the first
// of its slots in the list, their number. Then the list, slots by expert, then ascending.
struct ExpertsArgs {
    sifar_experts_args a;
    int32_t slots;   // tokens * topk
    int32_t named;   // experts that can be named at most
    int64_t at_list; // of the list, from the workspace's start, in int32
    int64_t at_h;    // in bytes
    int64_t h_bytes; // of a slot's h, or of its first elements
};

__device__ __forceinline__ int local_expert(const sifar_experts_args &a, int slot) {
    const uint32_t e = static_cast<uint32_t>(a.ids[slot]) - static_cast<uint32_t>(a.first_expert);
    return e < static_cast<uint32_t>(a.experts) ? static_cast<int>(e) : -1;
}

// How h lies in the workspace: slots ordered by expert, then ascending; sixteen of an expert
// (or what is left) make a tile, whose elements lie as the second product loads them: for
// each 64 bytes of its rows, for each quarter of them, every column's 16 bytes. So lanes
// of neighbouring columns read neighbouring bytes: where they read a row each, a load of 64
// lanes took 64 accesses to the cache instead of 8.
struct HiddenTile {
    int64_t at;
    int columns;
};
__device__ __forceinline__ HiddenTile hidden_tile(const ExpertsArgs &n, int before, int count,
                                                  int nth) {
    const int first = nth & ~15, left = count - first;
    return {(before + first) * n.h_bytes, left < 16 ? left : 16};
}
// Of element i of a column, from the tile's start, in bytes.
template <int SIZE>
__device__ __forceinline__ int hidden_at(int i, int column, int columns) {
    const int byte = i * SIZE;
    return (byte & ~15) * columns + 16 * column + (byte & 15);
}

// 64 bytes of each of 16 rows, a quarter a lane; behind `bytes` of a row zeros.
__device__ __forceinline__ U4 load_step(const unsigned char *row, int at, int bytes) {
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

// h as two bf16 elements. Above bf16's largest the first stays finite, so that the second,
// and with it what is infinite in fp32 or NaN, is all of the rest.
__device__ __forceinline__ Split split_h(float a, float b) {
    constexpr float most = 0x1.fep127f;
    const auto within = [](float f) { return __builtin_fminf(__builtin_fmaxf(f, -most), most); };
    Split s;
    s.high = pack16<SIFAR_BF16>(within(a), within(b));
    s.low = pack16<SIFAR_BF16>(a - low_half<SIFAR_BF16>(s.high), b - high_half<SIFAR_BF16>(s.high));
    return s;
}

// A batch of x: AHEAD steps of 16 * TILES rows. Read as an operand's lanes need it, each
// lane a row's 16 bytes, a load of 64 lanes takes 64 accesses to the cache, and the
// weights' own are as many as it has time for (64 tokens 246 us, by way of LDS 217). So
// lanes of neighbouring bytes read a row, and the wave's part of LDS turns them: 16 bytes of
// column c and quarter q of step s stand at place c ^ (4 s + q) of the 16 of (s, q), which
// keeps both sides off each other's banks.
template <int TILES, int AHEAD>
struct Turn {
    static constexpr int ROW = 4 * AHEAD;  // 16-byte pieces of a row
    static constexpr int LOADS = AHEAD * TILES;
    static __device__ __forceinline__ int place(int tile, int column, int piece) {
        return (tile * ROW + piece) * 16 + (column ^ (piece & 15));
    }
    static __device__ __forceinline__ void load(const unsigned char *const *rows, int at, int lane,
                                                U4 (&x)[LOADS]) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int f = i * kRowWave + lane;
            x[i] = *reinterpret_cast<const U4 *>(rows[f / ROW] + at + f % ROW * 16);
        }
    }
    static __device__ __forceinline__ void put(U4 *lds, int lane, const U4 (&x)[LOADS]) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int f = i * kRowWave + lane, row = f / ROW;
            lds[place(row / 16, row & 15, f % ROW)] = x[i];
        }
    }
    static __device__ __forceinline__ U4 get(const U4 *lds, int lane, int tile, int step) {
        return lds[place(tile, lane & 15, 4 * step + (lane >> 4))];
    }
};

// Two rows of 16 weights each (the gate's, the up ones) times up to 16 * TILES columns over
// the wave's steps of a row. TURNED: x by way of `lds`, from the addresses in `rows`.
template <int D, int TILES, int AHEAD, bool TURNED>
__device__ __forceinline__ void in_product(const unsigned char *const (&w)[2],
                                           const unsigned char *const *rows, int from, int to,
                                           int bytes, U4 *lds, F4 (&sum)[2][TILES]) {
    const int lane = threadIdx.x & 63, at = 16 * (lane >> 4);
    const unsigned char *x[TILES];
#pragma unroll
    for (int c = 0; c < TILES; ++c) x[c] = rows[16 * c + (lane & 15)];
    int s = from;
    const int whole = to * 64 <= bytes ? to : to - 1;  // steps that no row ends in
    for (; s + AHEAD <= whole; s += AHEAD) {
        U4 wa[AHEAD][2], xa[AHEAD * TILES];
        if constexpr (TURNED) Turn<TILES, AHEAD>::load(rows, 64 * s, lane, xa);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
                wa[i][j] = *reinterpret_cast<const U4 *>(w[j] + 64 * (s + i) + at);
            if constexpr (!TURNED)
#pragma unroll
                for (int c = 0; c < TILES; ++c)
                    xa[i * TILES + c] = *reinterpret_cast<const U4 *>(x[c] + 64 * (s + i) + at);
        }
        if constexpr (TURNED) {
            Turn<TILES, AHEAD>::put(lds, lane, xa);
            // other lanes of the wave read what this one wrote, and write it anew next time
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                for (int c = 0; c < TILES; ++c)
                    xa[i * TILES + c] = Turn<TILES, AHEAD>::get(lds, lane, c, i);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int c = 0; c < TILES; ++c)
                    sum[j][c] = mma<D>(wa[i][j], xa[i * TILES + c], sum[j][c]);
    }
    // what is left, a step in which rows end among it, also in one go
    for (; s < to; s += AHEAD) {
        U4 wa[AHEAD][2], xa[AHEAD][TILES];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int step = 64 * (s + i < to ? s + i : to - 1) + at;
#pragma unroll
            for (int j = 0; j < 2; ++j) wa[i][j] = load_step(w[j], step, bytes);
#pragma unroll
            for (int c = 0; c < TILES; ++c) xa[i][c] = load_step(x[c], step, bytes);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (s + i >= to) break;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int c = 0; c < TILES; ++c) sum[j][c] = mma<D>(wa[i][j], xa[i][c], sum[j][c]);
        }
    }
}

// Columns base.. of the expert's slots: both products, the waves' parts joined, h stored.
template <int D, int TILES, int AHEAD, bool TURNED>
__device__ __forceinline__ void in_columns(const ExpertsArgs &n, int expert, int row,
                                           const int *list, int base, int count, int before,
                                           F4 (*parts)[2][4][kRowWave],
                                           const unsigned char **rows) {
    constexpr int SIZE = D == SIFAR_FP32 ? 4 : 2;
    const sifar_experts_args &a = n.a;
    const int lane = threadIdx.x & 63, column = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int bytes = a.hidden * SIZE;
    // (what rows behind the last make is not stored)
    const int mine = row + column < a.inter ? row + column : a.inter - 1;
    const unsigned char *matrix = static_cast<const unsigned char *>(a.w_in) +
                                  expert * a.w_in_stride * SIZE;
    const unsigned char *const w[2] = {
        matrix + static_cast<int64_t>(mine) * bytes,
        matrix + (static_cast<int64_t>(a.inter) + mine) * bytes};
    // the columns' rows of x; columns behind the last slot repeat the first
    if (threadIdx.x < 16 * TILES) {
        const int i = base + static_cast<int>(threadIdx.x);
        rows[threadIdx.x] = static_cast<const unsigned char *>(a.x) +
                            list[i < count ? i : base] / a.topk * a.x_stride * SIZE;
    }
    __syncthreads();
    F4 sum[2][TILES];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int c = 0; c < TILES; ++c) sum[j][c] = F4{0.f, 0.f, 0.f, 0.f};
    const int steps = (bytes + 63) / 64, each = (steps + kInWaves - 1) / kInWaves;
    const int from = wave * each < steps ? wave * each : steps;
    in_product<D, TILES, AHEAD, TURNED>(w, rows, from, from + each < steps ? from + each : steps,
                                        bytes, reinterpret_cast<U4 *>(parts[wave]), sum);
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
            const HiddenTile tile = hidden_tile(n, before, count, i);
            unsigned char *to = static_cast<unsigned char *>(a.workspace) + n.at_h + tile.at +
                                hidden_at<SIZE>(at, i & 15, tile.columns);
            if constexpr (D == SIFAR_FP32) {
                *reinterpret_cast<F4 *>(to) = h;
            } else {
                typedef uint32_t U2 __attribute__((ext_vector_type(2)));
                const Split p = split_h(h[0], h[1]), q = split_h(h[2], h[3]);
                *reinterpret_cast<U2 *>(to) = U2{p.high, q.high};
                *reinterpret_cast<U2 *>(to + n.slots * n.h_bytes) = U2{p.low, q.low};
            }
        }
    }
    __syncthreads();  // parts and rows are written again
}

template <int D>
__global__ void __launch_bounds__(kInThreads, 4) in_kernel(const ExpertsArgs n) {
    __shared__ uint32_t bits[kMaxExperts / 32];
    __shared__ int list[kMaxSlots];
    __shared__ int here[kMaxSlots / kRowWave], below[kInWaves];
    __shared__ F4 parts[kInWaves][2][4][kRowWave];  // and, before the sums, x being turned
    __shared__ const unsigned char *rows[64];
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

    // Its slots in ascending order, as every workgroup of the expert lists them: h is laid
    // out by it. And how many slots other experts have before it.
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    uint64_t match[EACH];
    int lower = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        match[i] = __builtin_amdgcn_ballot_w64(expert[i] == mine);
        lower += __builtin_popcountll(
            __builtin_amdgcn_ballot_w64(expert[i] >= 0 && expert[i] < mine));
        if (lane == 0) here[i * kInWaves + wave] = __builtin_popcountll(match[i]);
    }
    if (lane == 0) below[wave] = lower;
    __syncthreads();
    int count = 0, before = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i)
#pragma unroll
        for (int w = 0; w < kInWaves; ++w) {
            if (w == wave && expert[i] == mine)
                list[count + __builtin_popcountll(match[i] & ((uint64_t{1} << lane) - 1))] =
                    i * kInThreads + static_cast<int>(threadIdx.x);
            count += here[i * kInWaves + w];
        }
#pragma unroll
    for (int w = 0; w < kInWaves; ++w) before += below[w];
    __syncthreads();
    if (blockIdx.x == 0) {
        int32_t *mark = plan + 4 + 4 * nth;
        if (threadIdx.x == 0) {
            mark[0] = mine;
            mark[1] = before;
            mark[2] = count;
        }
        for (int i = threadIdx.x; i < count; i += kInThreads)
            plan[n.at_list + before + i] = list[i];
    }

    const int row = kRows * blockIdx.x;
    for (int base = 0; base < count; base += 64) {
        const int left = count - base;
        const auto columns = [&](auto tiles, auto ahead, auto turned) {
            in_columns<D, decltype(tiles)::value, decltype(ahead)::value, decltype(turned)::value>(
                n, mine, row, list, base, count, before, parts, rows);
        };
        if (left <= kFew) columns(kInt<1>, kInt<8>, std::false_type{});
        else if (left <= 16) columns(kInt<1>, kInt<kInAhead>, std::true_type{});
        else if (left <= 32) columns(kInt<2>, kInt<kInAhead / 2>, std::true_type{});
        else columns(kInt<4>, kInt<kInAhead / 4>, std::true_type{});
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
            const Split p =
                split<SIFAR_BF16>(low_half<SIFAR_FP16>(w[i]), high_half<SIFAR_FP16>(w[i]));
            high[i] = p.high;
            low[i] = p.low;
        }
        c = mma<SIFAR_BF16>(high, h.v[0], c);
        c = mma<SIFAR_BF16>(high, h.v[1], c);
        return mma<SIFAR_BF16>(low, h.v[0], c);
    }
}

// Where in its steps a wave begins; it goes on from the first behind the last. Rows of
// weights lie a power of two apart, and workgroups that are all at the same step ask the
// same few memory channels at every moment; those of an XCD (every eighth) stay together,
// because they share h in its L2. 64 tokens over rows of 16 KB: 254 us in step, 204 so. (In
// the first product workgroups in step share DRAM pages: 246 us in step, 279 apart.)
__device__ __forceinline__ int turn_of(int steps, int batch) {
    const int turns = steps / batch, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int turn = static_cast<int>(blockIdx.x & 7) * turns / 8 + wave * turns / (8 * kOutWaves);
    return steps > 0 ? turn * batch : 0;
}

// The columns base.. of an expert's slots over steps from..to of `inter`; each slot's sums
// go to its row of `rows`. Is one of them not finite?
template <int D, int TILES, int AHEAD>
__device__ __forceinline__ bool out_columns(const ExpertsArgs &n, int expert, int row,
                                            const int32_t *list, int before, int base, int count,
                                            int from, int to, float *rows) {
    constexpr int SIZE = D == SIFAR_FP32 ? 4 : 2;
    const sifar_experts_args &a = n.a;
    const int lane = threadIdx.x & 63, column = lane & 15, at = 16 * (lane >> 4);
    const int bytes = a.inter * SIZE;
    const int mine = row + column < a.hidden ? row + column : a.hidden - 1;
    const unsigned char *w = static_cast<const unsigned char *>(a.w_out) +
                             expert * a.w_out_stride * SIZE + static_cast<int64_t>(mine) * bytes;
    const unsigned char *hidden = static_cast<const unsigned char *>(a.workspace) + n.at_h;
    const int64_t low = n.slots * n.h_bytes;  // behind the first elements
    const unsigned char *x[TILES];
    int step[TILES], slot[TILES];
#pragma unroll
    for (int c = 0; c < TILES; ++c) {
        const int i = base + 16 * c + column;
        slot[c] = list[i < count ? i : base];
        // behind the last tile, or its last column, the first one's
        const HiddenTile tile =
            hidden_tile(n, before, count, base + 16 * c < count ? base + 16 * c : base);
        x[c] = hidden + tile.at + 16 * (i < count ? column : 0) + at * tile.columns;
        step[c] = 64 * tile.columns;
    }
    F4 sum[TILES];
#pragma unroll
    for (int c = 0; c < TILES; ++c) sum[c] = F4{0.f, 0.f, 0.f, 0.f};
    const auto load_hidden = [&](int c, int s, auto whole) {
        Hidden<D> h;
        const bool in = decltype(whole)::value || 64 * s + at < bytes;
        const unsigned char *p = in ? x[c] + static_cast<int64_t>(s) * step[c] : hidden;
        h.v[0] = *reinterpret_cast<const U4 *>(p);
        if constexpr (D != SIFAR_FP32) h.v[1] = *reinterpret_cast<const U4 *>(p + low);
        if (!in) {
            h.v[0] = U4{0, 0, 0, 0};
            if constexpr (D != SIFAR_FP32) h.v[1] = U4{0, 0, 0, 0};
        }
        return h;
    };
    // Two batches of AHEAD steps: one is on its way while the other is multiplied.
    struct Batch {
        U4 w[AHEAD];
        Hidden<D> h[AHEAD][TILES];
    };
    const auto load = [&](Batch &t, int s) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            t.w[i] = *reinterpret_cast<const U4 *>(w + 64 * (s + i) + at);
#pragma unroll
            for (int c = 0; c < TILES; ++c) t.h[i][c] = load_hidden(c, s + i, std::true_type{});
        }
    };
    const auto multiply = [&](const Batch &t) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int c = 0; c < TILES; ++c) sum[c] = out_mma<D>(t.w[i], t.h[i][c], sum[c]);
    };
    // From `first` to `last`: whole batches, then what is left in one go, a step in which
    // rows end among it.
    const auto steps = [&](int first, int last) {
        const int whole = last * 64 <= bytes ? last : last - 1;
        int s = first;
        if (s + AHEAD <= whole) {
            Batch one, two;
            load(one, s);
            for (s += AHEAD; s + 2 * AHEAD <= whole; s += 2 * AHEAD) {
                load(two, s);
                multiply(one);
                load(one, s + AHEAD);
                multiply(two);
            }
            if (s + AHEAD <= whole) {
                load(two, s);
                s += AHEAD;
                multiply(one);
                multiply(two);
            } else {
                multiply(one);
            }
        }
        for (; s < last; s += AHEAD) {
            Batch t;
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int step = s + i < last ? s + i : last - 1;
                t.w[i] = load_step(w, 64 * step + at, bytes);
#pragma unroll
                for (int c = 0; c < TILES; ++c) t.h[i][c] = load_hidden(c, step, std::false_type{});
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if (s + i >= last) break;
#pragma unroll
                for (int c = 0; c < TILES; ++c) sum[c] = out_mma<D>(t.w[i], t.h[i][c], sum[c]);
            }
        }
    };
    const int middle = from + turn_of(to - from, AHEAD);
    steps(middle, to);
    if (middle > from) steps(from, middle);
#pragma unroll
    for (int c = 0; c < TILES; ++c)
        if (base + 16 * c + column < count)
            *reinterpret_cast<F4 *>(rows + slot[c] * kRows + 4 * (lane >> 4)) = sum[c];
    F4 all = sum[0];
#pragma unroll
    for (int c = 1; c < TILES; ++c) all += sum[c];
    const float any = __builtin_fabsf(all[0] + all[1] + (all[2] + all[3]));
    return __builtin_amdgcn_ballot_w64(!(any < __builtin_inff())) != 0;
}

// The columns' sums that are not finite, anew (16-bit types): an infinite weight, or in fp16
// its second element, meets the zeros and signs of second elements in the matrix
// instructions. Here weights and h are whole again; a lane takes four rows of its column.
// Sums that turn NaN end it at once; where all stay infinite, 64 tokens (2 of 8, 4096 x 8192)
// take 3.8 ms instead of 0.36.
template <int D>
__device__ __forceinline__ void strange_columns(const ExpertsArgs &n, int expert, int row,
                                                const int32_t *list, int before, int base,
                                                int count, int from, int to, float *rows) {
    const sifar_experts_args &a = n.a;
    const int column = threadIdx.x & 15, first = row + 4 * (threadIdx.x >> 4 & 3);
    const int bytes = a.inter * 2, end = 64 * to < bytes ? 64 * to : bytes;
    const unsigned char *w =
        static_cast<const unsigned char *>(a.w_out) + expert * a.w_out_stride * 2;
    const unsigned char *hidden = static_cast<const unsigned char *>(a.workspace) + n.at_h;
    const int last = base + 64 < count ? base + 64 : count;
#pragma unroll 1
    for (int tile = base; tile < last; tile += 16) {
        const bool in = tile + column < last;
        float *sums = rows + list[in ? tile + column : tile] * kRows + 4 * (threadIdx.x >> 4 & 3);
        const HiddenTile h = hidden_tile(n, before, count, tile);
        const unsigned char *x = hidden + h.at + 16 * (in ? column : 0);
#pragma unroll 1
        for (int r = 0; r < 4; ++r) {
            const int i = first + r < a.hidden ? first + r : a.hidden - 1;
            const unsigned char *mine = w + static_cast<int64_t>(i) * bytes;
            const bool odd = in && !(__builtin_fabsf(sums[r]) < __builtin_inff());
            float f = 0.f;
#pragma unroll 1
            for (int at = 64 * from; at < end; at += 16) {
                if (!__builtin_amdgcn_ballot_w64(odd && f == f)) break;  // NaN stays
                const unsigned char *p = x + static_cast<int64_t>(at) * h.columns;
                const U4 y = *reinterpret_cast<const U4 *>(mine + at);
                const U4 high = *reinterpret_cast<const U4 *>(p);
                const U4 low = *reinterpret_cast<const U4 *>(p + n.slots * n.h_bytes);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t p0 = high[k], p1 = low[k];
                    f = __builtin_fmaf(low_half<D>(y[k]),
                                       low_half<SIFAR_BF16>(p0) + low_half<SIFAR_BF16>(p1), f);
                    f = __builtin_fmaf(high_half<D>(y[k]),
                                       high_half<SIFAR_BF16>(p0) + high_half<SIFAR_BF16>(p1), f);
                }
            }
            if (odd) sums[r] = f;
        }
    }
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
    // what each slot adds with, loaded at once here rather than one by one at the end
    __shared__ float weight[kMaxSlots];
    __shared__ int8_t here[kMaxSlots];
    constexpr int SIZE = D == SIFAR_FP32 ? 4 : 2;
    const sifar_experts_args &a = n.a;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), row = kRows * blockIdx.x;
    const int32_t *plan = static_cast<const int32_t *>(a.workspace);
    // the first experts' marks with the number of them, before one of either is used
    const int lane = threadIdx.x & 63;
    int marks[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) marks[i] = plan[4 + 4 * (lane < n.named ? lane : 0) + i];
    const int named = plan[0];
    for (int i = threadIdx.x; i < n.slots; i += kOutThreads) {
        weight[i] = a.weights[i];
        here[i] = local_expert(a, i) >= 0;
    }
    const int parts = parts_of(named, n.slots);
    const int steps = (a.inter * SIZE + 63) / 64, each = (steps + parts - 1) / parts;
    for (int unit = wave; unit < named * parts; unit += kOutWaves) {
        const int nth = unit / parts, part = unit % parts;
        int mark[3];
#pragma unroll
        for (int i = 0; i < 3; ++i)
            mark[i] = nth < kRowWave ? __builtin_amdgcn_readlane(marks[i], nth)
                                     : plan[4 + 4 * nth + i];
        const int count = mark[2];
        const int32_t *list = plan + n.at_list + mark[1];
        const int from = part * each < steps ? part * each : steps;
        const int to = from + each < steps ? from + each : steps;
        float *mine = rows + part * n.slots * kRows;
        for (int base = 0; base < count; base += 64) {
            const int left = count - base;
            const auto columns = [&](auto tiles, auto ahead) {
                return out_columns<D, decltype(tiles)::value, decltype(ahead)::value>(
                    n, mark[0], row, list, mark[1], base, count, from, to, mine);
            };
            const bool strange = left <= 16   ? columns(kInt<1>, kInt<kOutAhead>)
                                 : left <= 32 ? columns(kInt<2>, kInt<kOutAhead / 2>)
                                              : columns(kInt<4>, kInt<kOutAhead / 4>);
            if constexpr (D != SIFAR_FP32)
                if (strange)
                    strange_columns<D>(n, mark[0], row, list, mark[1], base, count, from, to, mine);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.tokens * kRows; i += kOutThreads) {
        const int t = i / kRows, r = i % kRows;
        if (row + r >= a.hidden) continue;
        float f = 0.f;
        for (int j = 0; j < a.topk; ++j) {
            const int slot = t * a.topk + j;
            if (!here[slot]) continue;
            float y = rows[slot * kRows + r];
            for (int p = 1; p < parts; ++p) y += rows[(p * n.slots + slot) * kRows + r];
            f = __builtin_fmaf(weight[slot], y, f);
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
    n.h_bytes = static_cast<int64_t>(a.inter) * size_of(a.dtype);
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
    if (a.experts < 1 || a.experts > SIFAR_ROUTE_MAX_EXPERTS || a.first_expert < 0 ||
        a.first_expert > INT32_MAX - a.experts)
        return false;
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
