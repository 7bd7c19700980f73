// A token from its logits and one given random number: sifar_sample. gfx950
// (MI355X) only.
//
// Two launches. scan_kernel reads every logit once: a wave takes a chunk of 1024
// and leaves its maximum and, where the row needs it, its weights' sum.
// pick_kernel, a workgroup a row, finds the threshold of top-k, top-p and min-p
// and walks to the token in index order, reading again only chunks whose maximum
// says that they hold something to keep.
//
// Weights w = 2^((x - max) log2(e) / temperature) are 64-bit values rounded to
// units of 2^-42 and added as integers: sums do not depend on the order of
// addition, so histograms may be filled by atomics, and a border between two
// tokens is off by 2^-43 a token at most. In 32 bits a draw from a flat row of
// 100000 tokens would land on the neighbour once in a thousand times.
//
// Bound: HBM bytes of the logits for many rows, latency of the two launches and
// of pick_kernel's barriers for a few.
#include <hip/hip_runtime.h>

#include "exp2.h"
#include "rows.h"

namespace sifar {
namespace {

constexpr int kChunkElems = 1024;              // logits of a wave's chunk
constexpr int kPer = kChunkElems / kRowWave;   // of a lane
constexpr int kScanWaves = 4;                  // chunks of a scan workgroup
constexpr int kThreads = 1024;                 // of a pick workgroup
constexpr int kPickWaves = kThreads / kRowWave;
constexpr int kMaxChunks = SIFAR_SAMPLE_MAX_VOCAB / kChunkElems;
constexpr int kBins = 64 + 26 * 64;            // log-linear bins of a 32-bit distance
constexpr int kList = 8192;                    // candidates kept in LDS
constexpr int kSmall = 256;                    // most candidates that are ranked by counting
constexpr int kNucleus = 64;                   // chunk maxima a nucleus is first sought above
constexpr int kNucleusMass = 128;              // most p * sum / largest weight of such a row
constexpr int kPerBit = 64;                    // bins of a halving of the weight
constexpr int kUnitBits = 42;                  // a weight of 1 in units
constexpr double kLog2e = 1.4426950408889634;
constexpr double kLn2 = 0.6931471805599453;
constexpr double kCut = 60.0;                  // weights below 2^-60 are 0
static_assert(kMaxChunks <= kThreads, "a thread per chunk");

struct ChunkStat {
    double mass;  // sum of weights relative to the chunk's maximum
    float max;
    uint32_t unused;
};

struct SampleArgs {
    sifar_sample_args a;
    int32_t chunks;  // of a row
};

// Order-preserving 32 bits of a logit; 0 for one that is not there. -0 counts as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key >> 31 ? key & 0x7FFFFFFFu : ~key);
}

constexpr uint32_t kLowestKey = 0x00800000u;  // of the lowest finite fp32

// The least key whose logit is at least `limit`, and of a finite logit.
__device__ __forceinline__ uint32_t key_from(double limit) {
    float f = static_cast<float>(limit);
    uint32_t k = key_of(f);
    if (static_cast<double>(f) < limit) ++k;
    return k < kLowestKey ? kLowestKey : k;
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

// A wave's chunk: vectors of 16 bytes a lane, lanes adjacent. Element i of lane l
// is logit chunk_at<D>(c, l, i); one past the row, a NaN or -inf is -inf.
template <int D>
constexpr int kVecElems = 16 / sizeof(Stored<D>);

template <int D>
__device__ __forceinline__ int chunk_at(int c, int lane, int i) {
    constexpr int VE = kVecElems<D>;
    return c * kChunkElems + (i / VE) * (kRowWave * VE) + lane * VE + i % VE;
}

template <int D>
__device__ __forceinline__ void load_chunk(const Stored<D> *row, int vocab, int c, int lane,
                                           float (&x)[kPer]) {
    constexpr int VE = kVecElems<D>;
    const float none = -__builtin_inff();
#pragma unroll
    for (int v = 0; v < kPer / VE; ++v) {
        const int at = chunk_at<D>(c, lane, v * VE);
        if (at + VE <= vocab) {
            Eight<D> e;
            e.v[0] = reinterpret_cast<const Loose<D> *>(row + at)->v;
#pragma unroll
            for (int i = 0; i < VE; ++i) x[v * VE + i] = element<D>(e, i);
        } else {
#pragma unroll
            for (int i = 0; i < VE; ++i)
                x[v * VE + i] = at + i < vocab ? widen<D>(row[at + i]) : none;
        }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = x[i] > none ? x[i] : none;
}

// log2 of a weight. 0 at the maximum, which may be infinite; finite elsewhere.
__device__ __forceinline__ double log2_weight(float x, float max, double c) {
    const double z = (static_cast<double>(x) - static_cast<double>(max)) * c;
    return x == max ? 0.0 : z > -1100.0 ? z : -1100.0;
}

// The weight of a finite logit under a finite maximum, times 2^bits. Garbage, but
// finite, for logits far below the cut; -inf and NaN come out as the lowest
// finite logit.
__device__ __forceinline__ double weight(float x, double max, double scale, int bits) {
    const float y = fmaxf(x, -3.402823466e38f);
    const double z = (static_cast<double>(y) - max) * scale;
    const double i = __builtin_rint(z);
    return __builtin_ldexp(exp2_fraction9(z - i), static_cast<int>(i) + bits);
}

__device__ __forceinline__ double max64(double a, double b) {
    double r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

// A chunk's maximum and, where the row needs it, the sum of its weights. What
// top-k keeps is summed when it is known, and so is what min-p alone keeps.
template <int D>
__global__ void __launch_bounds__(kRowWave *kScanWaves) scan_kernel(const SampleArgs n) {
    const sifar_sample_args &a = n.a;
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x;
    const int c = blockIdx.y * kScanWaves + threadIdx.y;
    if (c >= n.chunks) return;
    const Draw d = draw_of(a, t);
    float x[kPer];
    load_chunk<D>(static_cast<const Stored<D> *>(a.logits) + t * a.logits_stride, a.vocab, c, lane,
                  x);
    const float none = -__builtin_inff();
    float m = none;
#pragma unroll
    for (int i = 0; i < kPer; ++i) m = fmaxf(m, x[i]);
    m = wave_reduce(m, Max{});
    double mass = 0.0;
    if (!d.greedy && d.top_k <= 0 && (d.top_p < 1.0f || !(d.min_p > 0.0f)) && m > none) {
        const double scale = kLog2e / static_cast<double>(d.temperature);
        if (m < __builtin_inff()) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const double w = weight(x[i], m, scale, 0);
                mass += x[i] > none ? w : 0.0;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i) mass += x[i] == m ? 1.0 : 0.0;
        }
        mass = wave_reduce(mass, Add{});
    }
    if (lane == 0)
        static_cast<ChunkStat *>(a.workspace)[t * n.chunks + c] = ChunkStat{mass, m, 0};
}

// ---- pick_kernel -----------------------------------------------------------------

struct Shared {
    uint64_t hist[kBins];                // also the candidates in order, or the chunks' ranks
    uint64_t chunk_units[kMaxChunks];
    uint32_t chunk_ties[kMaxChunks];
    uint32_t chunk_key[kMaxChunks];      // of the chunk's maximum
    uint32_t queue[kMaxChunks];          // chunks to be read
    uint32_t list_key[kList];            // candidates
    uint32_t list_at[kList];
    uint32_t rank[kThreads];
    uint64_t sums[kSmall];
    uint64_t wave_sum[kPickWaves];
    uint32_t wave_max[kPickWaves];
    uint64_t found_before;
    uint32_t found_bin;
    uint32_t list_size, queue_size;
    uint32_t bound;        // of the candidates
    uint32_t chosen;       // the token's chunk,
    uint64_t chosen_at;    // the units before the token in it
    uint64_t chosen_ties;  // and the ties before the chunk
};

__device__ __forceinline__ void add(uint64_t &sum, uint64_t x) {  // in LDS
    atomicAdd(reinterpret_cast<unsigned long long *>(&sum), static_cast<unsigned long long>(x));
}

// Inclusive sum over the lanes below: DPP moves within rows of 16, then the last
// lane of a row, and of the lower half, to the rows above. (Shuffles through LDS
// took six times as long, and a row's walk has a dozen of these.)
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

// Exclusive sum over the workgroup's threads, and the whole sum.
__device__ __forceinline__ uint64_t block_scan(Shared &s, uint64_t x, uint64_t &total) {
    const int wave = threadIdx.x >> 6;
    const uint64_t inc = wave_scan(x);
    __syncthreads();  // wave_sum may still be read from the call before
    if ((threadIdx.x & 63) == 63) s.wave_sum[wave] = inc;
    __syncthreads();
    uint64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kPickWaves; ++w) {
        const uint64_t v = s.wave_sum[w];
        before += w < wave ? v : 0;
        total += v;
    }
    return before + inc - x;
}

__device__ __forceinline__ uint64_t block_sum(Shared &s, uint64_t x) {
    uint64_t total;
    block_scan(s, x, total);
    return total;
}

__device__ __forceinline__ uint32_t block_max(Shared &s, uint32_t x) {
    x = wave_reduce(x, Max{});
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.wave_max[threadIdx.x >> 6] = x;
    __syncthreads();
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < kPickWaves; ++w) m = s.wave_max[w] > m ? s.wave_max[w] : m;
    return m;
}

// Key, then lower index: sorts as the order of the draw.
__device__ __forceinline__ uint64_t order_of(uint32_t key, uint32_t at) {
    return (static_cast<uint64_t>(key) << 32) | static_cast<uint32_t>(~at);
}

// Into s.rank[e]: how many of the first n values of `order` are above the e-th. Up
// to 256 values the workgroup splits each one's comparisons four ways.
__device__ __forceinline__ void rank_all(Shared &s, const uint64_t *order, int n) {
    const int span = n <= kThreads / 4 ? kThreads / 4 : n <= kThreads / 2 ? kThreads / 2 : kThreads;
    const int parts = kThreads / span;
    const int e = threadIdx.x & (span - 1), part = threadIdx.x / span;
    s.rank[threadIdx.x] = 0;
    __syncthreads();
    if (e < n) {
        const int each = (n + parts - 1) / parts;
        const int end = each * (part + 1) < n ? each * (part + 1) : n;
        const uint64_t mine = order[e];
        uint32_t above = 0;
#pragma unroll 4
        for (int j = each * part; j < end; ++j) above += order[j] > mine;
        atomicAdd(&s.rank[e], above);
    }
    __syncthreads();
}

// A row in pick_kernel.
template <int D>
struct Row {
    const Stored<D> *logits;
    int vocab, chunks;
    float max;
    double scale;  // log2(e) / temperature
    bool finite;   // the maximum is; otherwise the infinite logits share the weight

    // a weight in units; at least one, so that what may be drawn can be
    __device__ __forceinline__ double units_of(float x) const {
        return __builtin_rint(max64(weight(x, max, scale, kUnitBits), 1.0));
    }
    __device__ __forceinline__ uint64_t units(uint32_t key) const {
        return finite ? static_cast<uint64_t>(units_of(value_of(key))) : uint64_t{1} << kUnitBits;
    }
};

// The chunks whose maximum reaches `least`, in no order.
__device__ __forceinline__ uint32_t queue_chunks(Shared &s, int chunks, uint32_t least) {
    __syncthreads();
    if (threadIdx.x == 0) s.queue_size = 0;
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < chunks && s.chunk_key[threadIdx.x] >= least)
        s.queue[atomicAdd(&s.queue_size, 1u)] = threadIdx.x;
    __syncthreads();
    return s.queue_size;
}

// f(logits of a lane, chunk) over the queued chunks, a wave a chunk, the next one
// loaded while one is worked on.
template <int D, class F>
__device__ __forceinline__ void each_chunk(const Shared &s, const Row<D> &r, uint32_t size, F f) {
    const int lane = threadIdx.x & 63;
    uint32_t q = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (q >= size) return;
    float x[kPer], next[kPer];
    int c = __builtin_amdgcn_readfirstlane(s.queue[q]);
    load_chunk<D>(r.logits, r.vocab, c, lane, next);
    while (true) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) x[i] = next[i];
        const int at = c;
        q += kPickWaves;
        const bool more = q < size;
        if (more) {
            c = __builtin_amdgcn_readfirstlane(s.queue[q]);
            load_chunk<D>(r.logits, r.vocab, c, lane, next);
        }
        f(x, at);
        if (!more) return;
    }
}

// Where weights are sought: the row's chunks whose maximum reaches `least`...
template <int D>
struct InRow {
    Shared &s;
    const Row<D> &r;
    template <class F>
    __device__ __forceinline__ void each(uint32_t least, F f) const {
        const int lane = threadIdx.x & 63;
        const uint32_t size = queue_chunks(s, r.chunks, least);
        each_chunk(s, r, size, [&](const float(&x)[kPer], int c) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const uint32_t k = key_of(x[i]);
                if (k >= least) f(k, chunk_at<D>(c, lane, i));
            }
        });
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

__device__ __forceinline__ void to_list(Shared &s, uint32_t key, int at) {
    const uint32_t i = atomicAdd(&s.list_size, 1u);
    if (i < kList) {
        s.list_key[i] = key;
        s.list_at[i] = static_cast<uint32_t>(at);
    }
}

// Candidates from key `least` to `most` into the list, in no order. False if they
// do not fit.
template <int D>
__device__ __forceinline__ bool collect(Shared &s, const InRow<D> &from, uint32_t least,
                                        uint32_t most) {
    if (threadIdx.x == 0) s.list_size = 0;  // each() waits before it reads or adds
    from.each(least, [&](uint32_t k, int at) {
        if (k <= most) to_list(s, k, at);
    });
    __syncthreads();
    return s.list_size <= kList;
}

// The bin in which the running sum over bins reaches target (>= 1), and the sum
// before it; false if the whole sum does not reach it.
__device__ __forceinline__ bool find_bin(Shared &s, int bins, uint64_t target, uint32_t &bin,
                                         uint64_t &before) {
    static_assert(kBins <= 2 * kThreads, "two bins a thread");
    __syncthreads();
    const int b = 2 * threadIdx.x;
    const uint64_t v0 = b < bins ? s.hist[b] : 0, v1 = b + 1 < bins ? s.hist[b + 1] : 0;
    uint64_t total;
    const uint64_t run = block_scan(s, v0 + v1, total);
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
        const uint32_t last = lo + ((1u << bits) - 1);  // no more than 2^32 - 1: see seek()
        uint32_t least = top >= last ? top - last : 0;
        if (least <= floor) least = floor + 1;
        clear_bins(s);
        from.each(least, [&](uint32_t k, int) {
            const uint32_t d = top - k;
            if (k <= top && d >= lo) add(s.hist[(d - lo) >> shift], weight(k));
        });
        uint32_t bin;
        uint64_t in;
        if (!find_bin(s, 1024, target - before, bin, in)) return Border{false, 0, 0};
        before += in;
        lo += bin << shift;
        bits = shift;
    }
    return Border{true, top - lo, before};
}

// In descending order of keys from `top` down to, not including, `floor`: where
// does the running sum of weights reach target? Histograms over the distance
// d = top - key: first log-linear bins, 64 to an octave, over all 32 bits, then
// 1024 at a time inside the bin that was found.
template <class From, class W>
__device__ __forceinline__ Border seek(Shared &s, const From &from, uint32_t top, uint32_t floor,
                                       uint64_t target, W weight) {
    clear_bins(s);
    from.each(floor + 1, [&](uint32_t k, int) {
        const uint32_t d = top - k;
        const int e = d < 64 ? 6 : 31 - __builtin_clz(d);
        const uint32_t bin = d < 64 ? d : 64 + (e - 6) * 64 + ((d >> (e - 6)) & 63);
        add(s.hist[bin], weight(k));
    });
    uint32_t bin;
    uint64_t before;
    if (!find_bin(s, kBins, target, bin, before)) return Border{false, 0, 0};
    // the last bin of 64 << 25 distances ends at 2^32 - 1
    const int bits = bin < 64 ? 0 : (bin - 64) / 64;
    const uint32_t lo = bin < 64 ? bin : (64 + (bin & 63)) << bits;
    if constexpr (!std::is_same_v<From, InList>) {
        if (bits > 0) {
            const uint32_t last = lo + ((1u << bits) - 1);
            uint32_t least = top >= last ? top - last : 0;
            if (least <= floor) least = floor + 1;
            if (collect(s, from, least, top - lo))
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
        if (k > keep.key) sum += r.units(k);
        else ++ties;
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
// lies above the window, chunk by chunk, and lists what lies inside. False where
// the window misses or does not fit: then nothing is decided.
template <int D>
__device__ __forceinline__ bool window(Shared &s, const Row<D> &r, float part, uint32_t top,
                                       uint64_t units, Keep &keep) {
    if (!r.finite || !(r.scale > 1e-30 && r.scale < 1e30)) return false;
    const float cut = value_of(keep.key), scale = static_cast<float>(r.scale);
    // the whole row comes to 2^31
    const float unit = static_cast<float>(0x1p73 / static_cast<double>(units));
    clear_bins(s);
    const uint32_t size = queue_chunks(s, r.chunks, keep.key);
    each_chunk(s, r, size, [&](const float(&x)[kPer], int) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const float z = (x[i] - r.max) * scale;
            const uint32_t w = static_cast<uint32_t>(__builtin_amdgcn_exp2f(z) * unit + 0.5f);
            const uint32_t bin = static_cast<uint32_t>(z * -static_cast<float>(kPerBit));
            if (x[i] >= cut && w)
                atomicAdd(reinterpret_cast<uint32_t *>(&s.hist[bin < kBins ? bin : kBins - 1]), w);
        }
    });
    // A window of 2^-10 of the row's weight to either side: rounded weights are off by
    // half a unit each, 2^-12 of it for the largest vocabulary.
    const double aim = static_cast<double>(part) * 0x1p31;
    uint32_t first, end;
    uint64_t unused;
    if (!find_bin(s, kBins, aim > 0x1p21 + 1.0 ? static_cast<uint64_t>(aim - 0x1p21) : 1, first,
                  unused))
        return false;
    if (!find_bin(s, kBins, static_cast<uint64_t>(aim + 0x1p21), end, unused) ||
        end >= kBins - 1)
        return false;
    const double max = static_cast<double>(r.max);
    const uint32_t above = first ? key_from(max - first / (kPerBit * r.scale)) : top;
    uint32_t least = key_from(max - (end + 1) / (kPerBit * r.scale));
    if (least < keep.key) least = keep.key;
    if (least > above) return false;
    const float high = value_of(above), low = value_of(least);
    if (threadIdx.x == 0) s.list_size = 0;
    const uint32_t again = queue_chunks(s, r.chunks, least);
    const int lane = threadIdx.x & 63;
    each_chunk(s, r, again, [&](const float(&x)[kPer], int c) {
        double sum = 0.0;  // whole numbers below 2^53: exact
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            sum = __builtin_fma(r.units_of(x[i]), x[i] > high ? 1.0 : 0.0, sum);
            if (x[i] >= low && x[i] <= high) to_list(s, key_of(x[i]), chunk_at<D>(c, lane, i));
        }
        sum = wave_reduce(sum, Add{});
        if (lane == 0) s.chunk_units[c] = static_cast<uint64_t>(sum);
    });
    __syncthreads();
    const uint32_t listed = s.list_size;
    const int tid = threadIdx.x;
    const uint64_t before = block_sum(s, tid < r.chunks ? s.chunk_units[tid] : 0);
    const uint64_t target = share(part, units);
    if (listed > kList || before >= target) return false;
    const InList list{s, listed};
    const uint64_t in = kept_units(s, list, r, Keep{least, kAllTies});
    if (before + in < target) return false;
    keep = reach(s, list, r, above, before, target, Keep{least, kAllTies});
    return true;
}

// Few candidates, and nothing outside them kept: ranked by counting, then every
// filter is a prefix of the order and every sum a scan.
template <int D>
__device__ __forceinline__ void draw_small(Shared &s, const Row<D> &r, const Draw &d, int n,
                                           uint32_t least, uint64_t units, float u, int32_t *out,
                                           float *prob) {
    const int tid = threadIdx.x;
    uint64_t *order = s.hist;           // as collected, then sorted
    uint64_t *sorted = s.hist + kSmall;
    uint64_t *kept = s.hist + 2 * kSmall;
    if (tid < n) order[tid] = order_of(s.list_key[tid], s.list_at[tid]);
    rank_all(s, order, n);
    if (tid < n) sorted[s.rank[tid]] = order[tid];
    if (tid < kSmall) s.sums[tid] = 0;
    __syncthreads();
    const uint64_t mine = tid < n ? sorted[tid] : 0;
    const uint32_t key = static_cast<uint32_t>(mine >> 32);
    const uint64_t w = tid < n ? r.units(key) : 0;
    bool in = tid < n && (d.top_k <= 0 || tid < d.top_k);
    uint64_t top_units;
    const uint64_t before = block_scan(s, in ? w : 0, top_units);
    if (d.top_p < 1.0f) in = in && before < share(d.top_p, d.top_k > 0 ? top_units : units);
    in = in && (key >= least || tid == 0);
    uint64_t all;
    block_scan(s, in ? w : 0, all);
    if (tid < kSmall) kept[tid] = in ? w : 0;
    __syncthreads();
    // in index order: the kept weight before each candidate, four threads to one
    const int e = tid & (kSmall - 1), part = tid / kSmall;
    const uint32_t at_e = e < n ? ~static_cast<uint32_t>(sorted[e]) : 0;
    if (e < n) {
        const int each = (n + 3) / 4;
        const int end = each * (part + 1) < n ? each * (part + 1) : n;
        uint64_t sum = 0;
#pragma unroll 4
        for (int j = each * part; j < end; ++j)
            sum += ~static_cast<uint32_t>(sorted[j]) < at_e ? kept[j] : 0;
        add(s.sums[e], sum);
    }
    __syncthreads();
    uint64_t at = u > 0.0f ? static_cast<uint64_t>(static_cast<double>(u < 1.0f ? u : 1.0f) *
                                                   static_cast<double>(all))
                           : 0;
    if (at >= all) at = all - 1;
    if (in && s.sums[tid] <= at && at < s.sums[tid] + w) {
        *out = static_cast<int32_t>(at_e);
        if (prob) {
            const double sum = __builtin_ldexp(static_cast<double>(all), -kUnitBits);
            *prob = static_cast<float>(exp2_64(log2_weight(value_of(key), r.max, r.scale)) / sum);
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads) pick_kernel(const SampleArgs n) {
    __shared__ Shared s;
    const sifar_sample_args &a = n.a;
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Draw d = draw_of(a, t);
    const float u = a.uniform[t];
    const ChunkStat *stats = static_cast<const ChunkStat *>(a.workspace) + t * n.chunks;

    Row<D> r;
    r.logits = static_cast<const Stored<D> *>(a.logits) + t * a.logits_stride;
    r.vocab = a.vocab;
    r.chunks = n.chunks;
    const float none = -__builtin_inff();
    ChunkStat mine{0.0, none, 0};
    if (tid < n.chunks) mine = stats[tid];
    const uint32_t my_key = mine.max > none ? key_of(mine.max) : 0;
    if (tid < n.chunks) {
        s.chunk_key[tid] = my_key;
        s.chunk_units[tid] = 0;
        s.chunk_ties[tid] = 0;
    }
    if (tid == 0) {
        s.chosen = 0;
        s.chosen_at = 0;
        s.chosen_ties = 0;
    }
    const uint32_t top = block_max(s, my_key);
    if (top == 0) {  // nothing is there
        if (tid == 0) {
            a.out[t] = -1;
            if (a.probs) a.probs[t] = 0.0f;
        }
        return;
    }
    r.max = value_of(top);
    r.finite = r.max < __builtin_inff();
    r.scale = d.greedy ? 0.0 : kLog2e / static_cast<double>(d.temperature);

    uint64_t units = 0;   // of this thread's chunk
    Keep keep{top, 1};
    bool plain = false;   // every weight above the cut is kept: the scan's sums serve
    if (!d.greedy) {
        const double max = static_cast<double>(r.max), tau = static_cast<double>(d.temperature);
        keep = Keep{r.finite ? key_from(max - kCut * kLn2 * tau) : top, kAllTies};
        uint32_t least = keep.key;  // of min-p
        // at an infinite temperature every weight is 1
        if (d.min_p > 0.0f && r.finite && d.temperature < __builtin_inff()) {
            const double p = d.min_p < 1.0f ? static_cast<double>(d.min_p) : 1.0;
            const uint32_t k = key_from(p < 1.0 ? max + log(p) * tau : max);
            least = k > least ? k : least;
        }
        if (tid < n.chunks && my_key >= keep.key && mine.mass > 0.0) {
            units = static_cast<uint64_t>(__builtin_rint(
                __builtin_ldexp(mine.mass * exp2_64(log2_weight(mine.max, r.max, r.scale)),
                                kUnitBits)));
            units = units > 0 ? units : 1;
        }
        const bool by_k = d.top_k > 0, by_p = d.top_p < 1.0f;
        plain = !by_k && !by_p && !(d.min_p > 0.0f);
        if (!plain) {
            const uint64_t row_units = by_p && !by_k ? block_sum(s, units) : 0;
            // First the candidates above a bound that is known: min-p's, or the rank-th
            // largest of the chunks' maxima, above which there are at least `rank`. That is
            // enough for top-k, and likely for a nucleus, unless its weight says that it
            // holds more tokens.
            uint32_t from = by_p ? keep.key : least;
            const int rank = by_k ? d.top_k : kNucleus;
            const bool wide =
                by_p && !by_k &&
                static_cast<double>(d.top_p) * static_cast<double>(row_units) >
                    static_cast<double>(kNucleusMass) * __builtin_ldexp(1.0, kUnitBits);
            if ((by_k || (by_p && !wide)) && rank < n.chunks) {
                if (tid < n.chunks) s.hist[tid] = order_of(my_key, tid);
                rank_all(s, s.hist, n.chunks);
                if (tid < n.chunks && s.rank[tid] == static_cast<uint32_t>(rank - 1))
                    s.bound = my_key;
                __syncthreads();
                from = s.bound > from ? s.bound : from;
            }
            bool listed = !wide && collect(s, InRow<D>{s, r}, from, top);
            const InList list{s, s.list_size};
            if (listed && by_p && !by_k && from > keep.key)
                listed = kept_units(s, list, r, Keep{from, kAllTies}) >=
                         share(d.top_p, row_units);
            if (listed && list.size <= kSmall) {
                draw_small(s, r, d, static_cast<int>(list.size), least, row_units, u, a.out + t,
                           a.probs ? a.probs + t : nullptr);
                return;
            }
            if (listed) {
                keep = filter(s, list, r, d, top, row_units, Keep{from, kAllTies});
                if (least > keep.key) keep = Keep{least, kAllTies};
            } else if (by_p && !by_k && window(s, r, d.top_p, top, row_units, keep)) {
                listed = least <= keep.key;  // else what is above the window counts too much
                if (!listed) keep = Keep{least, kAllTies};
            } else {
                if (by_k || by_p)
                    keep = filter(s, InRow<D>{s, r}, r, d, top, row_units, keep);
                if (least > keep.key) keep = Keep{least, kAllTies};
            }
            if (listed) {
                InList{s, s.list_size}.each(keep.key, [&](uint32_t k, int at) {
                    if (k > keep.key) add(s.chunk_units[at / kChunkElems], r.units(k));
                    else atomicAdd(&s.chunk_ties[at / kChunkElems], 1u);
                });
            } else {
                __syncthreads();
                if (tid < n.chunks) s.chunk_units[tid] = 0;
                const uint32_t size = queue_chunks(s, n.chunks, keep.key);
                each_chunk(s, r, size, [&](const float(&x)[kPer], int c) {
                    uint64_t sum = 0;
                    uint32_t ties = 0;
#pragma unroll
                    for (int i = 0; i < kPer; ++i) {
                        const uint32_t k = key_of(x[i]);
                        if (k > keep.key) sum += r.units(k);
                        ties += k == keep.key;
                    }
                    sum = wave_reduce(sum, Add{});
                    ties = wave_reduce(ties, Add{});
                    if (lane == 0) {
                        s.chunk_units[c] = sum;
                        s.chunk_ties[c] = ties;
                    }
                });
            }
            __syncthreads();
            units = tid < n.chunks ? s.chunk_units[tid] : 0;
        }
    }

    // The chunk of the token, in index order over the kept weights.
    uint64_t ties_before = 0;
    if (!plain) {
        const uint64_t ties = d.greedy ? (my_key == top ? 1 : 0)
                                       : tid < n.chunks ? s.chunk_ties[tid] : 0;
        uint64_t tied;
        ties_before = block_scan(s, ties, tied);
        const uint64_t left = keep.ties > ties_before ? keep.ties - ties_before : 0;
        const uint64_t kept = ties < left ? ties : left;
        if (kept) units += kept * (d.greedy ? 1 : r.units(keep.key));
    }
    uint64_t all;
    const uint64_t before = block_scan(s, units, all);
    uint64_t at = u > 0.0f ? static_cast<uint64_t>(static_cast<double>(u < 1.0f ? u : 1.0f) *
                                                   static_cast<double>(all))
                           : 0;
    if (at >= all) at = all - 1;
    if (units && before <= at && at < before + units) {
        s.chosen = tid;
        s.chosen_at = at - before;
        s.chosen_ties = ties_before;
    }
    __syncthreads();
    if (wave != 0) return;

    // The token inside the chunk: which vector of the lanes, then which lane, then which
    // element.
    const int c = __builtin_amdgcn_readfirstlane(s.chosen);
    uint64_t want = s.chosen_at;
    uint64_t ties_run = s.chosen_ties;
    float x[kPer];
    load_chunk<D>(r.logits, r.vocab, c, lane, x);
    constexpr int VE = kVecElems<D>;
    int token = -1, last = -1;
#pragma unroll
    for (int v = 0; v < kPer / VE; ++v) {
        uint64_t w[VE], sum = 0;
        uint32_t ties = 0;
#pragma unroll
        for (int i = 0; i < VE; ++i) ties += key_of(x[v * VE + i]) == keep.key;
        uint64_t rank = ties_run;
        if (keep.ties != kAllTies) {
            const uint64_t tie_scan = wave_scan(ties);
            rank += tie_scan - ties;
            ties_run += lane_value(tie_scan, 63);
        }
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            const uint32_t k = key_of(x[v * VE + i]);
            const bool tie = k == keep.key;
            const bool in = k > keep.key || (tie && rank < keep.ties);
            rank += tie;
            w[i] = !in ? 0 : d.greedy ? 1 : r.units(k);
            sum += w[i];
        }
        const uint64_t scan = wave_scan(sum);
        uint64_t low = scan - sum;
        int here = -1, kept = -1;
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            if (w[i] && low <= want && want < low + w[i]) here = chunk_at<D>(c, lane, v * VE + i);
            if (w[i]) kept = chunk_at<D>(c, lane, v * VE + i);
            low += w[i];
        }
        const uint64_t hit = __ballot(here >= 0), any = __ballot(kept >= 0);
        if (any) last = lane_value(kept, 63 - __builtin_clzll(any));
        if (hit) {
            token = lane_value(here, __builtin_ctzll(hit));
            break;
        }
        want -= lane_value(scan, 63);
    }
    if (token < 0) token = last < 0 ? 0 : last;  // the chunk's own sum was rounded up
    if (lane == 0) {
        a.out[t] = token;
        if (a.probs) {
            const double w = exp2_64(log2_weight(widen<D>(r.logits[token]), r.max, r.scale));
            const double sum = __builtin_ldexp(static_cast<double>(all), -kUnitBits);
            a.probs[t] = d.greedy ? 1.0f : static_cast<float>(w / sum);
        }
    }
}

template <int D>
hipError_t launch_sample(const SampleArgs &n, hipStream_t s) {
    const dim3 scan(n.a.tokens, (n.chunks + kScanWaves - 1) / kScanWaves);
    scan_kernel<D><<<scan, dim3(kRowWave, kScanWaves), 0, s>>>(n);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    pick_kernel<D><<<n.a.tokens, kThreads, 0, s>>>(n);
    return hipGetLastError();
}

int32_t chunks_of(int32_t vocab) { return (vocab + kChunkElems - 1) / kChunkElems; }

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
    return static_cast<int64_t>(tokens) * chunks_of(vocab) * static_cast<int64_t>(sizeof(ChunkStat));
}

extern "C" int sifar_sample(const sifar_sample_args *args, void *stream) {
    using namespace sifar;
    if (!args || !good(*args)) return SIFAR_EINVAL;
    if (args->tokens == 0) return SIFAR_OK;
    SampleArgs n{};
    n.a = *args;
    n.chunks = chunks_of(args->vocab);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = args->dtype == SIFAR_BF16   ? launch_sample<SIFAR_BF16>(n, s)
                         : args->dtype == SIFAR_FP16 ? launch_sample<SIFAR_FP16>(n, s)
                                                     : launch_sample<SIFAR_FP32>(n, s);
    return e == hipSuccess ? SIFAR_OK : SIFAR_EHIP;
}
