// A token from its logits and one given random number: sifar_sample. gfx950
// (MI355X) only.
//
// Two launches. scan_kernel reads every logit once and leaves, for each chunk (the
// 16 bytes of each of a wave's lanes), the maximum and, where the row needs it,
// the weights' sum. pick_kernel, a workgroup a row, finds the threshold of top-k,
// top-p and min-p and walks to the token in index order, reading again only
// chunks whose maximum says that they hold something to keep. A nucleus of many
// tokens takes two more passes over its row, which a workgroup makes in 60 us for
// 128256 logits; where few rows would leave the GPU idle meanwhile, two launches
// between spread them over several workgroups a row. (Where top-k comes with top-p,
// for whichever rows, no row's passes are spread.)
//
// Weights w = 2^((x - max) log2(e) / temperature) are 64-bit values rounded to
// units of 2^-42 and added as integers: sums do not depend on the order of
// addition, so histograms may be filled by atomics. A kept token counts one unit at
// least, so a border between two tokens is off by up to a unit for each before it (half
// a unit by rounding, 0.2 by the exponential). Without a filter it is a chunk's sum that
// is rounded to units, and the chunk's tokens share it. In 32 bits, where a running sum
// is off by some 1e-8, one draw in a thousand from a flat row of 100000 tokens would
// land on the neighbour.
//
// Bound: the 64-bit exponentials for many rows, latency of the two launches and
// of pick_kernel's barriers and loads for a few. Measured: 256 x 151936 bf16 (15 us at
// a copy's rate) scan 34 us, pick 84 for flat rows under top-p, of which 18 go to the
// window's histogram and 47 to the exact pass; in both kernels vector instructions of
// four cycles each fill 85 % of the SIMDs' time. 8 x 128256 fp32 under every filter 15
// us a call, 1 x 32000 without one 8 in a graph.
#include <hip/hip_runtime.h>

#include "exp2.h"
#include "rows.h"

namespace sifar {
namespace {

constexpr int kBatch = 4;                      // chunks a wave loads at a time
constexpr int kScanWaves = 4;                  // waves of a scan workgroup
constexpr int kThreads = 1024;                 // of a pick workgroup
constexpr int kPickWaves = kThreads / kRowWave;
constexpr int kLeastChunk = kRowWave * 4;      // logits of a chunk: 256 of 32 bits, 512 of 16
constexpr int kMaxChunks = SIFAR_SAMPLE_MAX_VOCAB / kLeastChunk;
constexpr int kBins = 64 + 26 * 64;            // log-linear bins of a 32-bit distance
constexpr int kList = 4096;                    // candidates kept in LDS
constexpr int kSmall = 256;                    // most candidates that are ranked by counting
constexpr int kPerBit = 64;                    // bins of a halving of the weight
// Passes over rows are spread for up to 128 rows of 65536 logits or more, where the call
// has no top-k. In a graph, us a call in one workgroup a row and spread: a wide nucleus in
// fp32 1 x 65536 49 and 35, 1 x 128256 75 and 37, 128 x 65536 56 and 55, 128 x 128256 92 and
// 78; in bf16 47 and 41, 70 and 41, 54 and 52, 83 and 72. A narrow one, for which the
// two launches find nothing to do: fp32 1 x 65536 12 and 16, 128 x 128256 27 and 33, bf16
// 1 x 65536 14 and 18. So a third is lost on the one to halve the other, which is not known
// before the launch.
constexpr int kSpreadRows = 128;
constexpr int kSpreadVocab = 65536;
constexpr int kSpreadMaxima = 160;             // most chunks, of any type, of a narrow nucleus
constexpr int kSpreadGroups = 256;             // workgroups of a spread launch: one a CU
constexpr int kUnitBits = 42;                  // a weight of 1 in units
constexpr uint64_t kUnitBase = 0x433ull << 52;  // the bits of 2^52: units are its last place
constexpr double kLog2e = 1.4426950408889634;
constexpr double kLn2 = 0.6931471805599453;
constexpr double kCut = 60.0;                  // weights below 2^-60 are 0
constexpr float kLowest = -3.402823466e38f;

// What the first spread launch finds out about a row, for the launches behind it, and
// the second for the third.
struct RowState {
    uint64_t row_units;
    uint32_t top, bound;
    uint32_t wide, spread;
    uint32_t above, least, found;  // the window
    uint32_t unused;
};

struct SampleArgs {
    sifar_sample_args a;
    int32_t chunks;  // of a row
    double *mass;    // [tokens][chunks] sums of weights relative to the chunk's maximum
    uint64_t *units; // [tokens][chunks], of what lies above a spread row's window
    float *max;      // [tokens][chunks]
    // spread rows, or null
    RowState *state; // [tokens]
    uint32_t *hist;  // [tokens][kBins]
    uint32_t *listed;                // [tokens] candidates in the window,
    uint32_t *list_key, *list_at;    // [tokens][kList]
    int32_t groups;  // workgroups of a row
};

// Order-preserving 32 bits of a number: a negative one's turned over, others' sign bit
// set. -0 counts as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}

__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(
        key ^ (static_cast<uint32_t>(static_cast<int32_t>(~key) >> 31) | 0x80000000u));
}

constexpr uint32_t kLowestKey = 0x00800000u;  // of the lowest finite fp32

// The least key whose logit is at least `limit`, and of a finite logit.
__device__ __forceinline__ uint32_t key_from(double limit) {
    const float f = static_cast<float>(limit);
    uint32_t k = key_of(f);
    if (static_cast<double>(f) < limit) ++k;
    return k < kLowestKey ? kLowestKey : k;
}

// The larger of two numbers; of a number and a quiet NaN, the number.
__device__ __forceinline__ float max32(float a, float b) {
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

// The same of three.
__device__ __forceinline__ float max32(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// How a row is drawn.
struct Draw {
    float temperature, top_p, min_p;
    int32_t top_k;
    bool greedy;
};

__device__ __forceinline__ Draw draw_of(const sifar_sample_args &a, int64_t t) {
    Draw d;
    d.temperature = a.temperature ? a.temperature[t] : 1.0f;
    d.greedy = !(d.temperature > 0.0f);
    d.top_k = a.top_k ? a.top_k[t] : 0;
    d.top_p = a.top_p ? a.top_p[t] : 1.0f;
    d.min_p = a.min_p ? a.min_p[t] : 0.0f;
    return d;
}

// 16 bytes of a row that need not be aligned to more than an element.
template <int D>
struct __attribute__((packed, aligned(sizeof(Stored<D>)))) Loose {
    U4 v;
};

template <int D>
constexpr int kVec = 16 / sizeof(Stored<D>);  // logits of a lane in a chunk
template <int D>
constexpr int kChunkOf = kRowWave * kVec<D>;

// The lane's logits of a chunk, as they are stored.
struct Raw {
    U4 v;
};

template <int D>
__device__ __forceinline__ float logit(const Raw &e, int i) {
    if constexpr (D == SIFAR_FP32) return __uint_as_float(e.v[i]);
    else if constexpr (D == SIFAR_BF16)
        return __uint_as_float(i & 1 ? e.v[i >> 1] & 0xFFFF0000u : e.v[i >> 1] << 16);
    else
        return widen<D>(i & 1 ? e.v[i >> 1] >> 16 : e.v[i >> 1] & 0xFFFFu);
}

// The same where v_max_f32 reads it, which would answer a signalling NaN with a NaN:
// quiet. (Half precision comes quiet from its conversion.)
template <int D>
__device__ __forceinline__ float quiet_logit(const Raw &e, int i) {
    const float x = logit<D>(e, i);
    return D == SIFAR_FP16 ? x : max32(x, x);
}

template <int D>
__device__ __forceinline__ Raw nothing() {  // -inf
    constexpr uint32_t w = D == SIFAR_FP32 ? 0xFF800000u : D == SIFAR_BF16 ? 0xFF80FF80u : 0xFC00FC00u;
    return Raw{U4{w, w, w, w}};
}

// -inf past the row. (A NaN stays: comparisons with it are false, and nothing below
// asks for less.) The lane that the row ends in loads the row's last 16 bytes and
// shifts them down; only rows shorter than that are read by element.
template <int D>
__device__ __forceinline__ Raw load_chunk(const Stored<D> *row, int vocab, int c, int lane) {
    const int at = c * kChunkOf<D> + lane * kVec<D>;
    if (at + kVec<D> <= vocab) return Raw{reinterpret_cast<const Loose<D> *>(row + at)->v};
    Raw e = nothing<D>();
    if (at >= vocab) return e;
    constexpr int bits = 8 * sizeof(Stored<D>);
    if (vocab >= kVec<D>) {
        const U4 v = reinterpret_cast<const Loose<D> *>(row + vocab - kVec<D>)->v;
        const int shift = (at + kVec<D> - vocab) * bits;  // 16 .. 112
        const unsigned __int128 got = __builtin_bit_cast(unsigned __int128, v) >> shift;
        const unsigned __int128 fill = __builtin_bit_cast(unsigned __int128, e.v) << (128 - shift);
        e.v = __builtin_bit_cast(U4, got | fill);
        return e;
    }
    unsigned __int128 all = __builtin_bit_cast(unsigned __int128, e.v);
#pragma unroll 1
    for (int i = vocab - at - 1; i >= 0; --i)
        all = (all << bits) | static_cast<uint32_t>(row[at + i]);
    e.v = __builtin_bit_cast(U4, all);
    return e;
}

// Four values reduced over the wave at once: lanes 16 i .. 16 i + 15 get the i-th
// one's. The lane swaps of the first two steps put two values' halves into one
// register.
template <class T, class Op>
__device__ __forceinline__ T wave_reduce4(const T (&v)[4], Op op) {
    const auto join32 = [&](T a, T b) {  // lower half of the lanes: a's, upper: b's
        if constexpr (sizeof(T) == 4) {
            const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, a),
                                                            __builtin_bit_cast(uint32_t, b),
                                                            false, false);
            const uint32_t x = r[0], y = r[1];  // (a vector's element has no address)
            return op(__builtin_bit_cast(T, x), __builtin_bit_cast(T, y));
        } else {
            const uint64_t x = __builtin_bit_cast(uint64_t, a), y = __builtin_bit_cast(uint64_t, b);
            const auto lo = __builtin_amdgcn_permlane32_swap(static_cast<uint32_t>(x),
                                                             static_cast<uint32_t>(y), false, false);
            const auto hi =
                __builtin_amdgcn_permlane32_swap(static_cast<uint32_t>(x >> 32),
                                                 static_cast<uint32_t>(y >> 32), false, false);
            return op(__builtin_bit_cast(T, (static_cast<uint64_t>(hi[0]) << 32) | lo[0]),
                      __builtin_bit_cast(T, (static_cast<uint64_t>(hi[1]) << 32) | lo[1]));
        }
    };
    const auto join16 = [&](T a, T b) {  // even rows of 16: a's, odd rows: b's
        if constexpr (sizeof(T) == 4) {
            const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, a),
                                                            __builtin_bit_cast(uint32_t, b),
                                                            false, false);
            const uint32_t x = r[0], y = r[1];  // (a vector's element has no address)
            return op(__builtin_bit_cast(T, x), __builtin_bit_cast(T, y));
        } else {
            const uint64_t x = __builtin_bit_cast(uint64_t, a), y = __builtin_bit_cast(uint64_t, b);
            const auto lo = __builtin_amdgcn_permlane16_swap(static_cast<uint32_t>(x),
                                                             static_cast<uint32_t>(y), false, false);
            const auto hi =
                __builtin_amdgcn_permlane16_swap(static_cast<uint32_t>(x >> 32),
                                                 static_cast<uint32_t>(y >> 32), false, false);
            return op(__builtin_bit_cast(T, (static_cast<uint64_t>(hi[0]) << 32) | lo[0]),
                      __builtin_bit_cast(T, (static_cast<uint64_t>(hi[1]) << 32) | lo[1]));
        }
    };
    return wave_reduce<16>(join16(join32(v[0], v[2]), join32(v[1], v[3])), op);
}

struct Max32 {
    __device__ __forceinline__ float operator()(float a, float b) const { return max32(a, b); }
};

// log2 of a weight. 0 at the maximum, which may be infinite; finite elsewhere.
__device__ __forceinline__ double log2_weight(float x, float max, double c) {
    const double z = (static_cast<double>(x) - static_cast<double>(max)) * c;
    return x == max ? 0.0 : z > -1000.0 ? z : -1000.0;
}

// Every chunk's maximum and, where the row needs it, the sum of its weights. What
// top-k keeps is summed when it is known, and so is what min-p alone keeps.
template <int D>
__global__ void __launch_bounds__(kRowWave *kScanWaves) scan_kernel(const SampleArgs n) {
    const sifar_sample_args &a = n.a;
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x;
    const int first = (blockIdx.y * kScanWaves + threadIdx.y) * kBatch;
    if (n.hist && blockIdx.y == 0) {  // for the launches behind this one
        for (int b = threadIdx.y * kRowWave + lane; b < kBins; b += kScanWaves * kRowWave)
            n.hist[t * kBins + b] = 0;
        if (threadIdx.y == 0 && lane == 0) n.listed[t] = 0;
    }
    if (first >= n.chunks) return;
    const Draw d = draw_of(a, t);
    const Stored<D> *row = static_cast<const Stored<D> *>(a.logits) + t * a.logits_stride;
    Raw raw[kBatch];
    float x[kBatch][kVec<D>], top[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) raw[b] = load_chunk<D>(row, a.vocab, first + b, lane);
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
        top[b] = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < kVec<D>; ++i) x[b][i] = quiet_logit<D>(raw[b], i);
#pragma unroll
        for (int i = 0; i < kVec<D>; i += 2) top[b] = max32(top[b], x[b][i], x[b][i + 1]);
    }
    const float mine = wave_reduce4(top, Max32{});
    const int c = first + (lane >> 4);
    const bool writes = (lane & 15) == 0 && c < n.chunks;
    if (writes) n.max[t * n.chunks + c] = mine;
    if (d.greedy || d.top_k > 0 || (d.min_p > 0.0f && !(d.top_p < 1.0f))) return;
    const double tau = static_cast<double>(d.temperature), scale = kLog2e / tau;
    double sum[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
        const float m = lane_value(mine, 16 * b);
        sum[b] = 0.0;
        if (m < __builtin_inff()) {
            const double max = static_cast<double>(m);
            const float least = max32(static_cast<float>(max - kCut * kLn2 * tau), kLowest);
            if ((static_cast<double>(least) - max) * scale < 1.0 - kCut) {
                // what is below the cut, or not there, counts at the cut, rounded to fp32:
                // 2^-59 at most, less than 2^-50 of the chunk's weight together, and
                // cheaper than leaving it out
#pragma unroll
                for (int i = 0; i < kVec<D>; ++i)
                    sum[b] += exp2_quick<0>(
                        static_cast<double>(max32(x[b][i], least)) - max, scale);
            } else {  // a temperature or a maximum for which no logit lies at the cut
#pragma unroll
                for (int i = 0; i < kVec<D>; ++i) {
                    sum[b] += exp2_quick<0>(static_cast<double>(max32(x[b][i], least)) - max,
                                            scale, x[b][i] >= least);
                }
            }
        } else {  // they share the weight
#pragma unroll
            for (int i = 0; i < kVec<D>; ++i) sum[b] += x[b][i] == m ? 1.0 : 0.0;
        }
    }
    const double all = wave_reduce4(sum, Add{});
    if (writes) n.mass[t * n.chunks + c] = mine > -__builtin_inff() ? all : 0.0;
}

// ---- pick_kernel -----------------------------------------------------------------

struct Shared {
    uint64_t hist[kBins];                // also the candidates in order
    uint64_t chunk_units[kMaxChunks];
    uint32_t chunk_ties[kMaxChunks];
    uint32_t chunk_key[kMaxChunks];      // of the chunk's maximum; 0: nothing is there
    uint32_t queue[kMaxChunks];          // chunks to be read
    uint32_t list_key[kList];            // candidates
    uint32_t list_at[kList];
    uint32_t rank[kSmall];
    uint64_t sums[kSmall];
    uint64_t wave_sum[kPickWaves];
    uint32_t wave_max[kPickWaves];
    uint64_t found_before;
    uint32_t found_bin;
    uint32_t list_size, queue_size;
    uint32_t first_top;    // the first chunk that holds the maximum
    uint32_t chosen;       // the token's chunk,
    uint64_t chosen_at;    // the units before the token in it
    uint64_t chosen_ties;  // and the ties before the chunk
};

__device__ __forceinline__ void add(uint64_t &sum, uint64_t x) {  // in LDS
    atomicAdd(reinterpret_cast<unsigned long long *>(&sum), static_cast<unsigned long long>(x));
}

// Inclusive sum over the lanes below: DPP moves within rows of 16, then the last
// lane of a row, and of the lower half, to the rows above. (By shuffles
// through LDS a call of 1 x 32000 took 3 us more: a row's walk has a dozen of these.)
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t add_from(uint64_t x) {
    const int lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(static_cast<uint32_t>(x)), CTRL,
                                               ROWS, 0xF, false);
    const int hi = __builtin_amdgcn_update_dpp(
        0, static_cast<int>(static_cast<uint32_t>(x >> 32)), CTRL, ROWS, 0xF, false);
    return x + ((static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32) |
                static_cast<uint32_t>(lo));
}

__device__ __forceinline__ uint64_t wave_scan(uint64_t x) {
    x = add_from<0x111, 0xF>(x);  // row_shr:1
    x = add_from<0x112, 0xF>(x);
    x = add_from<0x114, 0xF>(x);
    x = add_from<0x118, 0xF>(x);
    x = add_from<0x142, 0xA>(x);  // row_bcast:15 into rows 1 and 3
    x = add_from<0x143, 0xC>(x);  // row_bcast:31 into rows 2 and 3
    return x;
}

// Exclusive sum over the workgroup's threads, and the whole sum. FRESH: a barrier lies
// between this call and the one before, whose sums may otherwise still be read.
template <bool FRESH = false>
__device__ __forceinline__ uint64_t block_scan(Shared &s, uint64_t x, uint64_t &total) {
    const int wave = threadIdx.x >> 6;
    const uint64_t inc = wave_scan(x);
    if constexpr (!FRESH) __syncthreads();
    if ((threadIdx.x & 63) == 63) s.wave_sum[wave] = inc;
    __syncthreads();
    // the waves' sums, scanned by the 16 lanes of a row at once
    static_assert(kPickWaves == 16, "a row of lanes");
    uint64_t sums = s.wave_sum[threadIdx.x & 15];
    sums = add_from<0x111, 0xF>(sums);
    sums = add_from<0x112, 0xF>(sums);
    sums = add_from<0x114, 0xF>(sums);
    sums = add_from<0x118, 0xF>(sums);
    total = lane_value(sums, 15);
    const uint64_t through = lane_value(sums, __builtin_amdgcn_readfirstlane(wave));
    const uint64_t mine = lane_value(inc, 63);
    return through - mine + inc - x;
}

template <bool FRESH = false>
__device__ __forceinline__ uint64_t block_sum(Shared &s, uint64_t x) {
    uint64_t total;
    block_scan<FRESH>(s, x, total);
    return total;
}

__device__ __forceinline__ uint32_t block_max(Shared &s, uint32_t x) {  // called once
    x = wave_reduce(x, Max{});
    if ((threadIdx.x & 63) == 0) s.wave_max[threadIdx.x >> 6] = x;
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(
        wave_reduce<kPickWaves>(s.wave_max[threadIdx.x & (kPickWaves - 1)], Max{}));
}

// A row in pick_kernel.
template <int D>
struct Row {
    const Stored<D> *logits;
    int vocab, chunks;
    float max;
    double max64, scale;  // log2(e) / temperature
    float one;            // logits below it weigh one unit
    bool finite;          // the maximum is; otherwise the infinite logits share the weight

    // A weight in units above kUnitBase. (Garbage for logits below the cut.)
    __device__ __forceinline__ uint64_t units_near(float x, bool keep = true) const {
        const double w = exp2_quick<kUnitBits>(static_cast<double>(x) - max64, scale, keep);
        return __builtin_bit_cast(uint64_t, w + 0x1p52);
    }
    // Of a kept weight at least one, so that what may be drawn can be.
    __device__ __forceinline__ uint64_t units(uint32_t key) const {
        return units_of(value_of(key));
    }
    __device__ __forceinline__ uint64_t units_of(float x) const {
        if (!finite) return uint64_t{1} << kUnitBits;  // the same in every lane
        const uint64_t u = units_near(x) - kUnitBase;
        return u ? u : 1;
    }
};

// A row's chunks, or some of them.
struct Span {
    int first, end;
};

// The chunks whose maximum reaches `least`, in no order.
__device__ __forceinline__ uint32_t queue_chunks(Shared &s, Span span, uint32_t least) {
    // every thread has read the size of the queue before, and a barrier has passed since
    if (threadIdx.x == 0) s.queue_size = 0;
    __syncthreads();
    for (int c = span.first + threadIdx.x; c < span.end; c += kThreads)
        if (s.chunk_key[c] >= least) s.queue[atomicAdd(&s.queue_size, 1u)] = c;
    __syncthreads();
    return s.queue_size;
}

// Over the queued chunks: a wave loads four at a time, the next four while it works
// on these. f(logits of a lane, chunk) is called for each, and its sums, over the
// wave, go to done(sum, chunk) in one lane. The four take turns in one set of
// registers: the loop's body is what its instructions cost to fetch.
template <int D, class F, class Done>
__device__ __forceinline__ void each_batch(const Shared &s, const Row<D> &r, uint32_t size, F f,
                                           Done done) {
    const int lane = threadIdx.x & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // spread over the waves where there are few chunks
    const uint32_t each = size >= kBatch * kPickWaves ? kBatch : (size + kPickWaves - 1) / kPickWaves;
    uint32_t q = wave * each;
    if (q >= size) return;
    Raw next[kBatch];
    int c_next[kBatch];
    int n_next;
    const auto load = [&] {
        n_next = static_cast<int>(size - q < each ? size - q : each);
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            c_next[b] = b < n_next ? __builtin_amdgcn_readfirstlane(s.queue[q + b]) : 0;
            next[b] = b < n_next ? load_chunk<D>(r.logits, r.vocab, c_next[b], lane) : nothing<D>();
        }
    };
    load();
    while (true) {
        Raw x[kBatch];
        uint64_t sum[kBatch];
        const int c_mine = lane < 16 ? c_next[0] : lane < 32 ? c_next[1] : lane < 48 ? c_next[2]
                                                                                     : c_next[3];
        int c[kBatch];
        const int n = n_next;
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            x[b] = next[b];
            c[b] = c_next[b];
        }
        q += each * kPickWaves;
        const bool more = q < size;
        if (more) load();
#pragma unroll 1
        for (int b = 0; b < kBatch; ++b) {
            const uint64_t mine = f(x[0], c[0]);
#pragma unroll
            for (int i = 0; i + 1 < kBatch; ++i) {
                x[i] = x[i + 1];
                c[i] = c[i + 1];
                sum[i] = sum[i + 1];
            }
            sum[kBatch - 1] = mine;
        }
        const uint64_t all = wave_reduce4(sum, Add{});
        if ((lane & 15) == 0 && (lane >> 4) < n) done(all, c_mine);
        if (!more) return;
    }
}

// Where weights are sought: the row's chunks whose maximum reaches `least`, a chunk
// at a time (what goes through here often goes through each_batch instead: its
// body is four times as long)...
template <int D>
struct InRow {
    Shared &s;
    const Row<D> &r;
    template <class F>
    __device__ __forceinline__ void each(uint32_t least, F f) const {
        const int lane = threadIdx.x & 63;
        const float low = value_of(least);
        const uint32_t size = queue_chunks(s, Span{0, r.chunks}, least);
        for (uint32_t q = threadIdx.x >> 6; q < size; q += kPickWaves) {
            const int c = __builtin_amdgcn_readfirstlane(s.queue[q]);
            const Raw x = load_chunk<D>(r.logits, r.vocab, c, lane);
#pragma unroll
            for (int i = 0; i < kVec<D>; ++i) {
                const float l = logit<D>(x, i);
                if (l >= low) f(key_of(l), c * kChunkOf<D> + lane * kVec<D> + i);
            }
        }
    }
};

// ... or the candidates in LDS.
struct InList {
    const Shared &s;
    uint32_t size;
    template <class F>
    __device__ __forceinline__ void each(uint32_t least, F f) const {
        for (uint32_t i = threadIdx.x; i < size; i += kThreads)
            if (s.list_key[i] >= least) f(s.list_key[i], s.list_at[i]);
    }
};

// The logits of a lane in chunk c that lie in [low, high], into the list, in no order:
// one counter's addition and wait for the whole chunk.
template <int D>
__device__ __forceinline__ void to_list(Shared &s, const Raw &x, int c, float low, float high) {
    const int lane = threadIdx.x & 63;
    uint64_t in[kVec<D>], any = 0;
    uint32_t count = 0;
#pragma unroll
    for (int i = 0; i < kVec<D>; ++i) {
        in[i] = __ballot(logit<D>(x, i) >= low && logit<D>(x, i) <= high);
        any |= in[i];
    }
    if (!any) return;
#pragma unroll
    for (int i = 0; i < kVec<D>; ++i) count += static_cast<uint32_t>(__builtin_popcountll(in[i]));
    uint32_t at = 0;
    if (lane == 0) at = atomicAdd(&s.list_size, count);
    at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
    for (int i = 0; i < kVec<D>; ++i) {
        if (!in[i]) continue;  // the same in every lane
        if (__builtin_amdgcn_inverse_ballot_w64(in[i])) {
            const uint32_t place =
                at + __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(in[i] >> 32),
                                               __builtin_amdgcn_mbcnt_lo(
                                                   static_cast<uint32_t>(in[i]), 0));
            if (place < kList) {
                s.list_key[place] = key_of(logit<D>(x, i));
                s.list_at[place] = static_cast<uint32_t>(c * kChunkOf<D> + lane * kVec<D> + i);
            }
        }
        at += static_cast<uint32_t>(__builtin_popcountll(in[i]));
    }
}

// Candidates from key `least` to `most` into the list, in no order. False if they
// do not fit.
template <int D>
__device__ __forceinline__ bool collect(Shared &s, const Row<D> &r, uint32_t least, uint32_t most) {
    const float low = value_of(least), high = value_of(most);
    if (threadIdx.x == 0) s.list_size = 0;  // queue_chunks() waits
    const uint32_t size = queue_chunks(s, Span{0, r.chunks}, least);
    each_batch(s, r, size, [&](const Raw &x, int c) {
        to_list<D>(s, x, c, low, high);
        return uint64_t{0};
    }, [](uint64_t, int) {});
    __syncthreads();
    return s.list_size <= kList;
}

// The bin in which the running sum over bins reaches target (>= 1), and the sum
// before it; false if the whole sum does not reach it.
template <class B>
__device__ __forceinline__ bool find_bin(Shared &s, const B *hist, int bins, uint64_t target,
                                         uint32_t &bin, uint64_t &before) {
    static_assert(kBins <= 2 * kThreads, "two bins a thread");
    __syncthreads();
    const int b = 2 * threadIdx.x;
    const uint64_t v0 = b < bins ? hist[b] : 0, v1 = b + 1 < bins ? hist[b + 1] : 0;
    uint64_t total;
    const uint64_t run = block_scan<true>(s, v0 + v1, total);
    if (total < target) return false;  // the same in every thread
    if (run < target && target <= run + v0 + v1) {
        const bool second = target > run + v0;
        s.found_bin = second ? b + 1 : b;
        s.found_before = second ? run + v0 : run;
    }
    __syncthreads();
    bin = s.found_bin;
    before = s.found_before;
    return true;
}

__device__ __forceinline__ void clear_bins(Shared &s) {
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += kThreads) s.hist[b] = 0;
    __syncthreads();
}

// Log-linear bins of a 32-bit distance: its first 64 values, then 64 to an octave.
// The last one ends at 2^32 - 1.
__device__ __forceinline__ uint32_t far_bin(uint32_t d) {
    const int e = d < 64 ? 6 : 31 - __builtin_clz(d);
    return d < 64 ? d : 64 + (e - 6) * 64 + ((d >> (e - 6)) & 63);
}
__device__ __forceinline__ int bin_bits(uint32_t bin) { return bin < 64 ? 0 : (bin - 64) / 64; }
__device__ __forceinline__ uint32_t bin_start(uint32_t bin) {
    return bin < 64 ? bin : (64 + (bin & 63)) << bin_bits(bin);
}

struct Border {
    bool found;
    uint32_t key;     // of the element in which the running sum reaches the target
    uint64_t before;  // the sum over larger keys
};

// seek() inside the bin [lo, lo + 2^bits) of distances from `top`.
template <class From, class W>
__device__ __forceinline__ Border narrow(Shared &s, const From &from, uint32_t top, uint32_t floor,
                                         uint32_t lo, int bits, uint64_t before, uint64_t target,
                                         W weight) {
    while (bits > 0) {
        const int shift = bits > 10 ? bits - 10 : 0;
        const uint32_t last = lo + ((1u << bits) - 1);  // no more than 2^32 - 1
        uint32_t least = top >= last ? top - last : 0;
        if (least <= floor) least = floor + 1;
        clear_bins(s);
        from.each(least, [&](uint32_t k, int) {
            const uint32_t d = top - k;
            if (k <= top && d >= lo) add(s.hist[(d - lo) >> shift], weight(k));
        });
        uint32_t bin;
        uint64_t in;
        if (!find_bin(s, s.hist, 1024, target - before, bin, in)) return Border{false, 0, 0};
        before += in;
        lo += bin << shift;
        bits = shift;
    }
    return Border{true, top - lo, before};
}

// In descending order of keys from `top` down to, not including, `floor`: where
// does the running sum of weights reach target? Histograms over the distance
// d = top - key: first log-linear bins, then 1024 at a time inside the bin that
// was found.
template <class From, class W>
__device__ __forceinline__ Border seek(Shared &s, const From &from, uint32_t top, uint32_t floor,
                                       uint64_t target, W weight) {
    clear_bins(s);
    from.each(floor + 1, [&](uint32_t k, int) {
        add(s.hist[far_bin(top - k)], weight(k));
    });
    uint32_t bin;
    uint64_t before;
    if (!find_bin(s, s.hist, kBins, target, bin, before)) return Border{false, 0, 0};
    const int bits = bin_bits(bin);
    const uint32_t lo = bin_start(bin);
    if constexpr (!std::is_same_v<From, InList>) {
        if (bits > 0) {
            const uint32_t last = lo + ((1u << bits) - 1);
            uint32_t least = top >= last ? top - last : 0;
            if (least <= floor) least = floor + 1;
            if (collect(s, from.r, least, top - lo))
                return narrow(s, InList{s, s.list_size}, top, floor, lo, bits, before, target,
                              weight);
        }
    }
    return narrow(s, from, top, floor, lo, bits, before, target, weight);
}

// What is kept: keys above `key`, and of those equal to it the first `ties` in
// index order.
struct Keep {
    uint32_t key;
    uint32_t ties;
};
constexpr uint32_t kAllTies = 0xFFFFFFFFu;

// Sum of the kept weights that `from` holds.
template <int D, class From>
__device__ __forceinline__ uint64_t kept_units(Shared &s, const From &from, const Row<D> &r,
                                               Keep keep) {
    uint64_t sum = 0;
    uint64_t ties = 0;
    from.each(keep.key, [&](uint32_t k, int) {
        const bool above = k > keep.key;  // (two branches put the sums into memory)
        sum += above ? r.units(k) : 0;
        ties += !above;
    });
    const uint64_t all = block_sum(s, sum);
    uint64_t tied = block_sum(s, ties);
    if (tied > keep.ties) tied = keep.ties;
    return tied ? all + tied * r.units(keep.key) : all;
}

// The least whole number that is at least part * all, and 1.
__device__ __forceinline__ uint64_t share(float part, uint64_t all) {
    const double p = static_cast<double>(part) * static_cast<double>(all);
    const uint64_t t = p > 1.0 ? static_cast<uint64_t>(p) : 1;
    return static_cast<double>(t) < p ? t + 1 : t;
}

// The place of a random number in [0, all), and the part of a unit behind it; from 1 on the
// end of the last one. (1.0 times `all`, which a double need not hold to the unit, would
// be a place before the last tokens.)
struct Place {
    uint64_t at;
    double part;
};
__device__ __forceinline__ Place place(float u, uint64_t all) {
    if (!(u >= 1.0f)) {
        const double p = u > 0.0f ? static_cast<double>(u) * static_cast<double>(all) : 0.0;
        const uint64_t at = static_cast<uint64_t>(p);
        if (at < all) return Place{at, p - static_cast<double>(at)};
    }
    return Place{all - 1, 1.0};
}

// The fewest in order from `top` whose sum reaches target, of what `keep` leaves
// and `from` holds; `before` is the sum of what lies above that.
template <int D, class From>
__device__ __forceinline__ Keep reach(Shared &s, const From &from, const Row<D> &r, uint32_t top,
                                      uint64_t before, uint64_t target, Keep keep) {
    const bool open = keep.ties == kAllTies;
    const Border b = seek(s, from, top, open ? keep.key - 1 : keep.key, target - before,
                          [&](uint32_t k) { return r.units(k); });
    if (b.found) {
        keep = Keep{b.key, kAllTies};
        before += b.before;
    } else if (open) {  // all of it: the target was rounded up
        return keep;
    } else {  // among the first ties of the least key
        uint64_t mine = 0;
        from.each(keep.key + 1, [&](uint32_t k, int) { mine += r.units(k); });
        before += block_sum(s, mine);
    }
    const uint64_t w = r.units(keep.key);
    const uint64_t ties = (target - before + w - 1) / w;
    return Keep{keep.key, ties < keep.ties ? static_cast<uint32_t>(ties) : keep.ties};
}

// top-k, then top-p over what `from` holds: everything that may be kept. units:
// the weights' sum, where top-k keeps all of it (else it is added up).
template <int D, class From>
__device__ __forceinline__ Keep filter(Shared &s, const From &from, const Row<D> &r, const Draw &d,
                                       uint32_t top, uint64_t units, Keep keep) {
    if (d.top_k > 0) {
        uint64_t mine = 0;
        from.each(keep.key, [&](uint32_t, int) { ++mine; });
        const uint64_t k = static_cast<uint64_t>(d.top_k);
        if (block_sum(s, mine) > k) {
            const Border b = seek(s, from, top, keep.key - 1, k,
                                  [](uint32_t) { return uint64_t{1}; });
            keep = Keep{b.key, static_cast<uint32_t>(k - b.before)};
        }
        if (d.top_p < 1.0f) units = kept_units(s, from, r, keep);
    }
    return d.top_p < 1.0f ? reach(s, from, r, top, 0, share(d.top_p, units), keep) : keep;
}

// A nucleus of more tokens than the list holds. Sums in 32 bits give a window of
// logits that holds its border; one pass over the row then adds up, exactly, what
// lies above the window, chunk by chunk, and lists what lies inside.

// The two passes are bounded where temperature and maximum are ordinary.
template <int D>
__device__ __forceinline__ bool window_fits(const Row<D> &r) {
    return r.finite && r.scale > 1e-30 && r.scale < 1e30;
}

// First pass, over some chunks: the histogram, in LDS, cleared before. The whole row
// comes to 2^31.
template <int D>
__device__ __forceinline__ void window_bins(Shared &s, const Row<D> &r, Span span, uint32_t cut_key,
                                            uint64_t units) {
    const float cut = value_of(cut_key), scale = static_cast<float>(r.scale);
    const float unit = static_cast<float>(0x1p73 / static_cast<double>(units));
    uint32_t *hist = reinterpret_cast<uint32_t *>(s.hist);
    const uint32_t size = queue_chunks(s, span, cut_key);
    each_batch(s, r, size, [&](const Raw &x, int) {
#pragma unroll
        for (int i = 0; i < kVec<D>; ++i) {
            const float l = logit<D>(x, i);
            const float z = (l - r.max) * scale;
            const uint32_t w = static_cast<uint32_t>(__builtin_amdgcn_exp2f(z) * unit + 0.5f);
            const uint32_t bin = static_cast<uint32_t>(z * -static_cast<float>(kPerBit));
            if (l >= cut && w) atomicAdd(&hist[bin < kBins ? bin : kBins - 1], w);
        }
        return uint64_t{0};
    }, [](uint64_t, int) {});
}

struct Window {
    bool found;
    uint32_t above, least;  // keys: what is larger lies above, the border is least or more
};

// A window of 2^-16 of the row's weight to either side: what rounding and 32-bit
// exponentials leave is an order less, unless most of the row weighs next to nothing.
template <int D>
__device__ __forceinline__ Window window_of(Shared &s, const Row<D> &r, float part, uint32_t top,
                                            uint32_t cut_key) {
    const uint32_t *hist = reinterpret_cast<const uint32_t *>(s.hist);
    const double aim = static_cast<double>(part) * 0x1p31;
    uint32_t first, end;
    uint64_t unused;
    if (!find_bin(s, hist, kBins, aim > 0x1p15 + 1.0 ? static_cast<uint64_t>(aim - 0x1p15) : 1,
                  first, unused))
        return Window{false, 0, 0};
    if (!find_bin(s, hist, kBins, static_cast<uint64_t>(aim + 0x1p15), end, unused) ||
        end >= kBins - 1)
        return Window{false, 0, 0};
    Window w;
    w.above = first ? key_from(r.max64 - first / (kPerBit * r.scale)) : top;
    w.least = key_from(r.max64 - (end + 1) / (kPerBit * r.scale));
    if (w.least < cut_key) w.least = cut_key;
    // weights above the window are more than a unit
    w.found = w.least <= w.above && value_of(w.above) >= r.one;
    return w;
}

// Second pass, over some chunks: s.chunk_units of what lies above, the list of what
// lies inside.
template <int D>
__device__ __forceinline__ void window_sums(Shared &s, const Row<D> &r, Span span, const Window &w) {
    const float high = value_of(w.above), low = value_of(w.least);
    if (threadIdx.x == 0) s.list_size = 0;
    const uint32_t size = queue_chunks(s, span, w.least);
    each_batch(s, r, size, [&](const Raw &x, int c) {
        to_list<D>(s, x, c, low, high);
        uint64_t sum = 0;
#pragma unroll
        for (int i = 0; i < kVec<D>; ++i) {
            const float l = quiet_logit<D>(x, i);
            sum += r.units_near(max32(l, high), l > high);
        }
        sum -= kVec<D> * kUnitBase;  // modulo 2^64
        return sum;
    }, [&](uint64_t sum, int c) { s.chunk_units[c] = sum; });
    __syncthreads();
}

// The border, from the sums of every chunk and the list. False where the window misses
// it or does not fit the list: then nothing is decided.
template <int D>
__device__ __forceinline__ bool window_border(Shared &s, const Row<D> &r, float part,
                                              const Window &w, uint64_t units, Keep &keep) {
    const uint32_t listed = s.list_size;
    uint64_t mine = 0;
    for (int c = threadIdx.x; c < r.chunks; c += kThreads) mine += s.chunk_units[c];
    const uint64_t before = block_sum(s, mine);
    const uint64_t target = share(part, units);
    if (listed > kList || before >= target) return false;
    const InList list{s, listed};
    const uint64_t in = kept_units(s, list, r, Keep{w.least, kAllTies});
    if (before + in < target) return false;
    keep = reach(s, list, r, w.above, before, target, Keep{w.least, kAllTies});
    return true;
}

// Key, then lower index: sorts as the order of the draw.
__device__ __forceinline__ uint64_t order_of(uint32_t key, uint32_t at) {
    return (static_cast<uint64_t>(key) << 32) | static_cast<uint32_t>(~at);
}

// Few candidates, and nothing outside them kept: each is ranked by counting those
// above it, then every filter is a prefix of the order and every sum a scan. Four
// threads, or eight for up to 128 candidates, share one's comparisons.
template <int D>
__device__ __forceinline__ void draw_small(Shared &s, const Row<D> &r, const Draw &d, int n,
                                           uint32_t least, uint64_t units, float u, int32_t *out,
                                           float *prob) {
    const int tid = threadIdx.x;
    uint64_t *order = s.hist;           // as collected, then sorted
    uint64_t *sorted = s.hist + kSmall;
    uint64_t *kept = s.hist + 2 * kSmall;
    const int parts = n <= kSmall / 2 ? 2 * kThreads / kSmall : kThreads / kSmall;
    const int span = kThreads / parts;
    const int e = tid & (span - 1), part = n <= kSmall / 2 ? tid / (kSmall / 2) : tid / kSmall;
    const int share_of = (n + parts - 1) / parts;
    const int j0 = share_of * part, j1 = j0 + share_of < n ? j0 + share_of : n;
    if (tid < n) order[tid] = order_of(s.list_key[tid], s.list_at[tid]);
    if (tid < kSmall) {
        s.rank[tid] = 0;
        s.sums[tid] = 0;
    }
    __syncthreads();
    if (e < n) {
        const uint64_t mine = order[e];
        uint32_t above = 0;
#pragma unroll 4
        for (int j = j0; j < j1; ++j) above += order[j] > mine;
        if (above) atomicAdd(&s.rank[e], above);
    }
    __syncthreads();
    if (tid < n) sorted[s.rank[tid]] = order[tid];
    __syncthreads();
    const uint64_t mine = tid < n ? sorted[tid] : 0;
    const uint32_t key = static_cast<uint32_t>(mine >> 32);
    const uint64_t w = tid < n ? r.units(key) : 0;
    bool in = tid < n && (d.top_k <= 0 || tid < d.top_k);
    if (d.top_p < 1.0f) {
        uint64_t top_units;
        const uint64_t before = block_scan<true>(s, in ? w : 0, top_units);
        in = in && before < share(d.top_p, d.top_k > 0 ? top_units : units);
    }
    in = in && (key >= least || tid == 0);
    const uint64_t all = block_sum(s, in ? w : 0);
    if (tid < n) kept[tid] = in ? w : 0;
    __syncthreads();
    // in index order: the kept weight before each candidate
    const uint32_t at_e = e < n ? ~static_cast<uint32_t>(sorted[e]) : 0;
    if (e < n) {
        uint64_t sum = 0;
#pragma unroll 4
        for (int j = j0; j < j1; ++j)
            sum += ~static_cast<uint32_t>(sorted[j]) < at_e ? kept[j] : 0;
        if (sum) add(s.sums[e], sum);
    }
    __syncthreads();
    const uint64_t at = place(u, all).at;
    if (in && s.sums[tid] <= at && at < s.sums[tid] + w) {
        *out = static_cast<int32_t>(~static_cast<uint32_t>(mine));
        if (prob) {
            const double sum = __builtin_ldexp(static_cast<double>(all), -kUnitBits);
            *prob = static_cast<float>(exp2_64(log2_weight(value_of(key), r.max, r.scale)) / sum);
        }
    }
}

// What a workgroup knows of its row when it starts.
template <int D>
struct Begun {
    Draw d;
    Row<D> r;
    uint32_t top, my_key;  // of the row's maximum (0: nothing is there), of this thread's chunks'
    int c0, c1;            // a thread's chunks, in index order over the threads
};

template <int D>
__device__ __forceinline__ Begun<D> begin_row(Shared &s, const SampleArgs &n, int64_t t) {
    Begun<D> b;
    const int tid = threadIdx.x;
    b.d = draw_of(n.a, t);
    b.r.logits = static_cast<const Stored<D> *>(n.a.logits) + t * n.a.logits_stride;
    b.r.vocab = n.a.vocab;
    b.r.chunks = n.chunks;
    const int per = (n.chunks + kThreads - 1) / kThreads;
    b.c0 = tid * per < n.chunks ? tid * per : n.chunks;
    b.c1 = b.c0 + per < n.chunks ? b.c0 + per : n.chunks;
    b.my_key = 0;
    for (int c = b.c0; c < b.c1; ++c) {
        const float m = n.max[t * n.chunks + c];
        const uint32_t k = m > -__builtin_inff() ? key_of(m) : 0;
        s.chunk_key[c] = k;
        s.chunk_units[c] = 0;
        s.chunk_ties[c] = 0;
        b.my_key = k > b.my_key ? k : b.my_key;
    }
    for (int i = tid; i < kBins; i += kThreads) s.hist[i] = 0;
    b.top = block_max(s, b.my_key);
    return b;
}

// The limits of what a row keeps, and the kinds of rows.
struct Limits {
    Keep keep;           // by the cut
    uint32_t least;      // and min-p
    bool by_k, by_p;
    bool plain;          // every weight above the cut is kept: the scan's sums serve
    uint32_t bound;      // what top-k or top-p keeps is among the keys from here on (0: not known)
    bool wide;           // a nucleus of many tokens: no such bound
    bool spread;         // whose passes are launches of their own
    uint64_t row_units;  // the whole weight, where top-p starts from it
};

// From the maximum alone.
template <int D>
__device__ __forceinline__ Limits limit_row(const Draw &d, uint32_t top, Row<D> &r) {
    Limits l;
    r.max = value_of(top);
    r.max64 = static_cast<double>(r.max);
    r.finite = r.max < __builtin_inff();
    const double tau = static_cast<double>(d.temperature);
    r.scale = kLog2e / tau;
    r.one = value_of(key_from(r.max64 - kUnitBits * kLn2 * tau));
    l.keep = Keep{r.finite ? key_from(r.max64 - kCut * kLn2 * tau) : top, kAllTies};
    l.least = l.keep.key;
    // at an infinite temperature every weight is 1
    if (d.min_p > 0.0f && r.finite && d.temperature < __builtin_inff()) {
        const double p = d.min_p < 1.0f ? static_cast<double>(d.min_p) : 1.0;
        const uint32_t k = key_from(p < 1.0 ? r.max64 + log(p) * tau : r.max64);
        l.least = k > l.least ? k : l.least;
    }
    l.by_k = d.top_k > 0;
    l.by_p = d.top_p < 1.0f;
    l.plain = !l.by_k && !l.by_p && !(d.min_p > 0.0f);
    l.row_units = 0;
    l.bound = 0;
    l.wide = l.spread = false;
    return l;
}

// From the chunks' maxima and sums.
template <int D>
__device__ __forceinline__ void weigh_row(Shared &s, const SampleArgs &n, int64_t t,
                                          const Begun<D> &b, Limits &l) {
    const Draw &d = b.d;
    const Row<D> &r = b.r;
    if (l.plain || (l.by_p && !l.by_k)) {
        uint64_t mine = 0;
        for (int c = b.c0; c < b.c1; ++c) {
            if (s.chunk_key[c] < l.keep.key) continue;
            const double w = exp2_64(log2_weight(value_of(s.chunk_key[c]), r.max, r.scale)) *
                             n.mass[t * n.chunks + c];
            uint64_t units = static_cast<uint64_t>(
                __builtin_rint(__builtin_ldexp(w, kUnitBits)));
            units = units > 0 ? units : 1;
            if (l.plain) s.chunk_units[c] = units;
            mine += units;
        }
        if (!l.plain) l.row_units = block_sum<true>(s, mine);
    }
    // The chunks' maxima bound what is kept: the k-th largest of them (to a bin of the
    // histogram) has k tokens at or above it, and the one at which their own weights
    // reach top-p's share has that much at or above it. A row whose maxima do not reach it
    // has a wide nucleus. Under a top-k of as many tokens as there are chunks, or more, no
    // maximum says anything: the whole row is listed, or sorted out if it does not fit the
    // list (8 x 32000 bf16, 63 chunks, in a graph: top-k 50 13 us, 62 19, 63 39).
    if ((l.by_k && d.top_k < n.chunks) || (l.by_p && !l.by_k)) {
        for (int c = b.c0; c < b.c1; ++c)
            if (s.chunk_key[c] >= l.keep.key)
                add(s.hist[far_bin(b.top - s.chunk_key[c])],
                    l.by_k ? 1 : r.units(s.chunk_key[c]));
        uint32_t bin;
        uint64_t unused;
        if (find_bin(s, s.hist, kBins,
                     l.by_k ? static_cast<uint64_t>(d.top_k) : share(d.top_p, l.row_units), bin,
                     unused)) {
            const uint32_t last = bin_start(bin) + ((1u << bin_bits(bin)) - 1);
            l.bound = b.top > last ? b.top - last : 0;
            if (n.hist && !l.by_k) {
                // more than a few candidates take longer to list and sort out than spread
                // passes do: 55 us against 39 for 4 x 128256 in fp32. (A chunk of a 16-bit
                // type has twice the logits: its rows of up to 81920 never count as wide here.)
                uint64_t mine = 0;
                for (int c = b.c0; c < b.c1; ++c) mine += s.chunk_key[c] >= l.bound;
                l.wide = block_sum(s, mine) > kSpreadMaxima;
            }
        } else {
            l.wide = !l.by_k;
        }
        l.spread = l.wide && n.hist && window_fits(r);
    }
}

// The chunks of a row that a workgroup of a spread launch takes.
__device__ __forceinline__ Span span_of(const SampleArgs &n, int group) {
    const int each = (n.chunks + n.groups - 1) / n.groups;
    const int first = each * group < n.chunks ? each * group : n.chunks;
    return Span{first, first + each < n.chunks ? first + each : n.chunks};
}

// The first pass over such rows, spread: LDS histograms added up in memory.
template <int D>
__global__ void __launch_bounds__(kThreads) spread_bins_kernel(const SampleArgs n) {
    __shared__ Shared s;
    const int64_t t = blockIdx.y;
    Begun<D> b = begin_row<D>(s, n, t);
    if (b.top == 0 || b.d.greedy) {  // the same in every thread
        if (blockIdx.x == 0 && threadIdx.x == 0) n.state[t].spread = 0;
        return;
    }
    Limits l = limit_row(b.d, b.top, b.r);
    if (l.by_p) weigh_row(s, n, t, b, l);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        RowState *state = n.state + t;
        state->row_units = l.row_units;
        state->top = b.top;
        state->bound = l.bound;
        state->wide = l.wide;
        state->spread = l.spread;
    }
    if (!l.spread) return;
    clear_bins(s);
    window_bins(s, b.r, span_of(n, blockIdx.x), l.keep.key, l.row_units);
    __syncthreads();
    const uint32_t *hist = reinterpret_cast<const uint32_t *>(s.hist);
    for (int i = threadIdx.x; i < kBins; i += kThreads)
        if (hist[i]) atomicAdd(&n.hist[t * kBins + i], hist[i]);
}

// The second pass, spread: chunks' sums and the candidates inside the window.
template <int D>
__global__ void __launch_bounds__(kThreads) spread_sums_kernel(const SampleArgs n) {
    __shared__ Shared s;
    const int64_t t = blockIdx.y;
    const int tid = threadIdx.x;
    const RowState state = n.state[t];
    if (!state.spread) return;
    const Draw d = draw_of(n.a, t);
    Row<D> r;
    r.logits = static_cast<const Stored<D> *>(n.a.logits) + t * n.a.logits_stride;
    r.vocab = n.a.vocab;
    r.chunks = n.chunks;
    const Limits l = limit_row(d, state.top, r);
    const Span span = span_of(n, blockIdx.x);
    for (int c = span.first + tid; c < span.end; c += kThreads) {
        const float m = n.max[t * n.chunks + c];
        s.chunk_key[c] = m > -__builtin_inff() ? key_of(m) : 0;
        s.chunk_units[c] = 0;
    }
    uint32_t *hist = reinterpret_cast<uint32_t *>(s.hist);
    for (int i = tid; i < kBins; i += kThreads) hist[i] = n.hist[t * kBins + i];
    const Window w = window_of(s, r, d.top_p, state.top, l.keep.key);
    if (blockIdx.x == 0 && tid == 0) {
        n.state[t].above = w.above;
        n.state[t].least = w.least;
        n.state[t].found = w.found;
    }
    if (!w.found) return;
    window_sums(s, r, span, w);
    for (int c = span.first + tid; c < span.end; c += kThreads)
        n.units[t * n.chunks + c] = s.chunk_units[c];
    // a list that does not fit is counted, and noticed by its size
    const uint32_t size = s.list_size < kList ? s.list_size : kList;
    if (tid == 0) s.found_bin = atomicAdd(&n.listed[t], s.list_size);
    __syncthreads();
    const uint32_t at = s.found_bin;
    for (uint32_t i = tid; i < size; i += kThreads)
        if (at + i < kList) {
            n.list_key[t * kList + at + i] = s.list_key[i];
            n.list_at[t * kList + at + i] = s.list_at[i];
        }
}

// What the spread launches left, into LDS.
template <int D>
__device__ __forceinline__ void load_spread(Shared &s, const SampleArgs &n, int64_t t) {
    const uint32_t listed = n.listed[t];
    for (int c = threadIdx.x; c < n.chunks; c += kThreads)
        s.chunk_units[c] = n.units[t * n.chunks + c];
    for (uint32_t i = threadIdx.x; i < (listed < kList ? listed : kList); i += kThreads) {
        s.list_key[i] = n.list_key[t * kList + i];
        s.list_at[i] = n.list_at[t * kList + i];
    }
    if (threadIdx.x == 0) s.list_size = listed;
    __syncthreads();
}

// The border of a nucleus that the list does not hold, by its window. `spread`: the two
// passes were made already. False where nothing is decided.
template <int D>
__device__ __forceinline__ bool nucleus(Shared &s, const SampleArgs &n, int64_t t, const Row<D> &r,
                                        float part, uint32_t top, uint64_t units, bool spread,
                                        Keep &keep) {
    if (spread) {
        const RowState state = n.state[t];
        if (!state.found) return false;
        __syncthreads();
        load_spread<D>(s, n, t);
        return window_border(s, r, part, Window{true, state.above, state.least}, units, keep);
    }
    if (!window_fits(r)) return false;
    const Span all{0, r.chunks};
    clear_bins(s);
    window_bins(s, r, all, keep.key, units);
    const Window w = window_of(s, r, part, top, keep.key);
    if (!w.found) return false;
    window_sums(s, r, all, w);
    return window_border(s, r, part, w, units, keep);
}

template <int D>
__global__ void __launch_bounds__(kThreads) pick_kernel(const SampleArgs n) {
    __shared__ Shared s;
    const sifar_sample_args &a = n.a;
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float u = a.uniform[t];
    if (tid == 0) {
        s.first_top = kMaxChunks;
        s.chosen = 0;
        s.chosen_at = 0;
        s.chosen_ties = 0;
    }
    Begun<D> b = begin_row<D>(s, n, t);
    const Draw &d = b.d;
    Row<D> &r = b.r;
    r.max = value_of(b.top);
    const uint32_t top = b.top, my_key = b.my_key;
    const int c0 = b.c0, c1 = b.c1;
    if (top == 0) {  // nothing is there
        if (tid == 0) {
            a.out[t] = -1;
            if (a.probs) a.probs[t] = 0.0f;
        }
        return;
    }
    if (d.greedy) {
        if (my_key == top)
            for (int c = c0; c < c1; ++c)
                if (s.chunk_key[c] == top) {
                    atomicMin(&s.first_top, static_cast<uint32_t>(c));
                    break;
                }
        __syncthreads();
        if (wave != 0) return;
        const int c = __builtin_amdgcn_readfirstlane(s.first_top);
        const Raw x = load_chunk<D>(r.logits, r.vocab, c, lane);
        int here = kVec<D>;
#pragma unroll
        for (int i = kVec<D> - 1; i >= 0; --i)
            if (logit<D>(x, i) == r.max) here = i;
        const uint64_t hit = __ballot(here < kVec<D>);
        if (hit && lane == __builtin_ctzll(hit)) {
            a.out[t] = c * kChunkOf<D> + lane * kVec<D> + here;
            if (a.probs) a.probs[t] = 1.0f;
        }
        return;
    }
    Limits limits = limit_row(d, top, r);
    if (n.hist && limits.by_p) {
        const RowState state = n.state[t];
        limits.row_units = state.row_units;
        limits.bound = state.bound;
        limits.wide = state.wide;
        limits.spread = state.spread;
    } else {
        weigh_row(s, n, t, b, limits);
    }
    Keep keep = limits.keep;
    const uint32_t least = limits.least;
    const bool by_k = limits.by_k, by_p = limits.by_p, plain = limits.plain;
    const uint64_t row_units = limits.row_units;
    if (!plain) {
        // First the candidates above a bound that is known, if they are few.
        uint32_t from = by_p ? keep.key : least;
        from = limits.bound > from ? limits.bound : from;
        bool listed = !limits.wide && collect(s, r, from, top);
        const InList list{s, s.list_size};
        if (listed && list.size <= kSmall) {
            draw_small(s, r, d, static_cast<int>(list.size), least, row_units, u, a.out + t,
                       a.probs ? a.probs + t : nullptr);
            return;
        }
        if (listed) {
            keep = filter(s, list, r, d, top, row_units, Keep{from, kAllTies});
            if (least > keep.key) keep = Keep{least, kAllTies};
        } else if (by_p && !by_k && nucleus(s, n, t, r, d.top_p, top, row_units, limits.spread,
                                           keep)) {
            listed = least <= keep.key;  // else what is above the window counts too much
            if (!listed) keep = Keep{least, kAllTies};
        } else {
            if (by_k || by_p) keep = filter(s, InRow<D>{s, r}, r, d, top, row_units, keep);
            if (least > keep.key) keep = Keep{least, kAllTies};
        }
        if (listed) {
            InList{s, s.list_size}.each(keep.key, [&](uint32_t k, int at) {
                if (k > keep.key) add(s.chunk_units[at / kChunkOf<D>], r.units(k));
                else atomicAdd(&s.chunk_ties[at / kChunkOf<D>], 1u);
            });
        } else {
            __syncthreads();
            for (int c = c0; c < c1; ++c) s.chunk_units[c] = 0;
            const float low = value_of(keep.key);
            const uint32_t size = queue_chunks(s, Span{0, n.chunks}, keep.key);
            // a chunk's ties in the ten top bits of its sum, which weights leave free
            each_batch(s, r, size, [&](const Raw &x, int) {
                uint64_t sum = 0;
#pragma unroll
                for (int i = 0; i < kVec<D>; ++i) {
                    const float l = logit<D>(x, i);
                    if (l > low) sum += r.units_of(l);
                    sum += l == low ? uint64_t{1} << 54 : 0;
                }
                return sum;
            }, [&](uint64_t sum, int c) {
                s.chunk_units[c] = sum & ((uint64_t{1} << 54) - 1);
                s.chunk_ties[c] = static_cast<uint32_t>(sum >> 54);
            });
        }
        __syncthreads();
    }

    // The chunk of the token, in index order over the kept weights.
    uint64_t ties_before = 0, ties = 0;
    const uint64_t tie_units = r.units(keep.key);
    const auto kept_ties = [&](uint64_t before, int c) {  // of chunk c, `before` ties before it
        const uint64_t here = s.chunk_ties[c];
        const uint64_t left = keep.ties > before ? keep.ties - before : 0;
        return here < left ? here : left;
    };
    if (!plain) {
        for (int c = c0; c < c1; ++c) ties += s.chunk_ties[c];
        uint64_t tied;
        ties_before = block_scan<true>(s, ties, tied);  // behind the barrier above
    }
    uint64_t units = 0, run_ties = ties_before;
    for (int c = c0; c < c1; ++c) {
        units += s.chunk_units[c];
        if (plain) continue;
        units += kept_ties(run_ties, c) * tie_units;
        run_ties += s.chunk_ties[c];
    }
    uint64_t all;
    const uint64_t before = block_scan(s, units, all);
    const Place target = place(u, all);
    const uint64_t at = target.at;
    if (units && before <= at && at < before + units) {
        uint64_t run = before;
        run_ties = ties_before;
        for (int c = c0; c < c1; ++c) {
            const uint64_t here =
                s.chunk_units[c] + (plain ? 0 : kept_ties(run_ties, c) * tie_units);
            if (at < run + here) {
                s.chosen = c;
                s.chosen_at = at - run;
                s.chosen_ties = run_ties;
                break;
            }
            run += here;
            if (!plain) run_ties += s.chunk_ties[c];
        }
    }
    __syncthreads();
    if (wave != 0) return;

    // The token inside the chunk: which lane, then which of its logits. The sum of a chunk
    // of a row without filters came from the scan, rounded to units once, so its tokens
    // share it: by weights in units of 2^-42 of the chunk's maximum, the place in
    // proportion. In the row's units each would count one at least, and a chunk of light
    // tokens would end before its heavy ones.
    const int c = __builtin_amdgcn_readfirstlane(s.chosen);
    Row<D> inside = r;
    if (plain) inside.max64 = static_cast<double>(value_of(s.chunk_key[c]));
    const Raw x = load_chunk<D>(r.logits, r.vocab, c, lane);
    const float low_kept = value_of(keep.key);
    uint64_t w[kVec<D>], sum = 0, rank = s.chosen_ties;
    if (keep.ties != kAllTies) {
        uint64_t mine = 0;
#pragma unroll
        for (int i = 0; i < kVec<D>; ++i) mine += logit<D>(x, i) == low_kept;
        rank += wave_scan(mine) - mine;
    }
#pragma unroll
    for (int i = 0; i < kVec<D>; ++i) {
        const float l = logit<D>(x, i);
        const bool tie = l == low_kept;
        const bool in = l > low_kept || (tie && rank < keep.ties);
        rank += tie;
        w[i] = in ? inside.units_of(l) : 0;
        sum += w[i];
    }
    const uint64_t through = wave_scan(sum);
    uint64_t want = s.chosen_at;
    if (plain) {
        const uint64_t whole = lane_value(through, 63);
        const double share = static_cast<double>(whole) / static_cast<double>(s.chunk_units[c]);
        want = static_cast<uint64_t>((static_cast<double>(want) + target.part) * share);
        want = want < whole ? want : whole - 1;
    }
    uint64_t low = through - sum;
    int here = -1;
#pragma unroll
    for (int i = 0; i < kVec<D>; ++i) {
        if (w[i] && low <= want && want < low + w[i]) here = i;
        low += w[i];
    }
    const uint64_t hit = __ballot(here >= 0);  // one lane: want is below the chunk's sum
    const int from_lane = hit ? __builtin_ctzll(hit) : 0;
    const int i = lane_value(here, from_lane);
    const int token = c * kChunkOf<D> + from_lane * kVec<D> + (i < 0 ? 0 : i);
    if (lane == 0) {
        a.out[t] = token;
        if (a.probs) {
            const double weight = exp2_64(log2_weight(widen<D>(r.logits[token]), r.max, r.scale));
            const double whole = __builtin_ldexp(static_cast<double>(all), -kUnitBits);
            a.probs[t] = static_cast<float>(weight / whole);
        }
    }
}

// Byte offsets in the workspace, each a multiple of 16, for the most chunks that any
// type has.
struct Workspace {
    int64_t mass, units, max, state, hist, listed, list_key, list_at, end;
};

Workspace workspace_of(int32_t tokens, int32_t vocab) {
    const int64_t t = tokens, chunks = t * ((vocab + kLeastChunk - 1) / kLeastChunk);
    // of the batches that may be spread, so that a larger one's workspace serves them
    const int64_t rows = vocab < kSpreadVocab ? 0 : tokens < kSpreadRows ? tokens : kSpreadRows;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += (bytes + 15) / 16 * 16;
        return here;
    };
    Workspace w;
    w.mass = take(chunks * 8);
    w.max = take(chunks * 4);
    w.units = take(t ? chunks / t * rows * 8 : 0);
    w.state = take(rows * static_cast<int64_t>(sizeof(RowState)));
    w.hist = take(rows * kBins * 4);
    w.listed = take(rows * 4);
    w.list_key = take(rows * kList * 4);
    w.list_at = take(rows * kList * 4);
    w.end = at;
    return w;
}

template <int D>
hipError_t launch_sample(SampleArgs &n, hipStream_t s) {
    const sifar_sample_args &a = n.a;
    n.chunks = (a.vocab + kChunkOf<D> - 1) / kChunkOf<D>;
    const Workspace w = workspace_of(a.tokens, a.vocab);
    const auto at = [&](int64_t offset) {
        return static_cast<void *>(static_cast<char *>(a.workspace) + offset);
    };
    n.mass = static_cast<double *>(at(w.mass));
    n.max = static_cast<float *>(at(w.max));
    const bool spread =
        a.top_p && !a.top_k && a.tokens <= kSpreadRows && a.vocab >= kSpreadVocab;
    if (spread) {
        n.units = static_cast<uint64_t *>(at(w.units));
        n.state = static_cast<RowState *>(at(w.state));
        n.hist = static_cast<uint32_t *>(at(w.hist));
        n.listed = static_cast<uint32_t *>(at(w.listed));
        n.list_key = static_cast<uint32_t *>(at(w.list_key));
        n.list_at = static_cast<uint32_t *>(at(w.list_at));
        // a batch of chunks for each wave at least
        const int most = (n.chunks + kPickWaves * kBatch - 1) / (kPickWaves * kBatch);
        n.groups = kSpreadGroups / a.tokens < most ? kSpreadGroups / a.tokens : most;
    }
    const int per_group = kScanWaves * kBatch;
    const dim3 scan(a.tokens, (n.chunks + per_group - 1) / per_group);
    scan_kernel<D><<<scan, dim3(kRowWave, kScanWaves), 0, s>>>(n);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && spread) {
        const dim3 grid(n.groups, a.tokens);
        spread_bins_kernel<D><<<grid, kThreads, 0, s>>>(n);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        spread_sums_kernel<D><<<grid, kThreads, 0, s>>>(n);
        e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    pick_kernel<D><<<a.tokens, kThreads, 0, s>>>(n);
    return hipGetLastError();
}

bool good_sizes(int32_t tokens, int32_t vocab) {
    return tokens >= 0 && tokens <= SIFAR_ROWS_MAX_TOKENS && vocab >= 1 &&
           vocab <= SIFAR_SAMPLE_MAX_VOCAB;
}

bool good(const sifar_sample_args &a) {
    if (a.dtype < SIFAR_BF16 || a.dtype > SIFAR_FP32 || !good_sizes(a.tokens, a.vocab)) return false;
    if (a.tokens == 0) return true;
    if (!a.logits || !a.uniform || !a.out || !a.workspace) return false;
    const uint64_t size = a.dtype == SIFAR_FP32 ? 4 : 2;
    const auto at = [](const void *p) { return reinterpret_cast<uintptr_t>(p); };
    if (at(a.logits) % size || at(a.workspace) % 16) return false;
    const uint64_t tokens = static_cast<uint64_t>(a.tokens);
    const void *per_row[] = {a.uniform, a.temperature, a.top_k, a.top_p, a.min_p};
    for (const void *p : per_row)
        if (at(p) % 4) return false;
    if (at(a.out) % 4 || at(a.probs) % 4) return false;
    if (a.tokens > 1 && (a.logits_stride < a.vocab || a.logits_stride > (int64_t{1} << 40)))
        return false;
    const int64_t need = sifar_sample_workspace(a.tokens, a.vocab);
    if (a.workspace_bytes < need) return false;
    // What is written, apart from everything else.
    const Rows logits{at(a.logits), tokens, static_cast<uint64_t>(a.logits_stride) * size,
                      static_cast<uint64_t>(a.vocab) * size};
    const Rows work{at(a.workspace), 1, 0, static_cast<uint64_t>(need)};
    const Rows out[] = {Rows{at(a.out), 1, 0, tokens * 4}, Rows{at(a.probs), 1, 0, tokens * 4}, work};
    for (int i = 0; i < 3; ++i) {
        if (may_overlap(out[i], logits)) return false;
        for (const void *p : per_row)
            if (may_overlap(out[i], Rows{at(p), 1, 0, tokens * 4})) return false;
        for (int j = 0; j < i; ++j)
            if (may_overlap(out[i], out[j])) return false;
    }
    return true;
}

}  // namespace
}  // namespace sifar

extern "C" int64_t sifar_sample_workspace(int32_t tokens, int32_t vocab) {
    using namespace sifar;
    if (!good_sizes(tokens, vocab)) return SIFAR_EINVAL;
    return workspace_of(tokens, vocab).end;
}

extern "C" int sifar_sample(const sifar_sample_args *args, void *stream) {
    using namespace sifar;
    if (!args || !good(*args)) return SIFAR_EINVAL;
    if (args->tokens == 0) return SIFAR_OK;
    SampleArgs n{};
    n.a = *args;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = args->dtype == SIFAR_BF16   ? launch_sample<SIFAR_BF16>(n, s)
                         : args->dtype == SIFAR_FP16 ? launch_sample<SIFAR_FP16>(n, s)
                                                     : launch_sample<SIFAR_FP32>(n, s);
    return e == hipSuccess ? SIFAR_OK : SIFAR_EHIP;
}
