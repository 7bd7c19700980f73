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
constexpr int kList = 4096;                    // candidates kept in LDS
constexpr int kNucleus = 64;                   // chunk maxima a nucleus is first sought above
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
    // top-k rows add up their own few weights, min-p rows those above a known logit
    if (!d.greedy && d.top_k <= 0 && !(d.min_p > 0.0f && !(d.top_p < 1.0f)) && m > none) {
        const double scale = kLog2e / static_cast<double>(d.temperature);
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            mass += x[i] > none ? exp2_64(log2_weight(x[i], m, scale)) : 0.0;
        mass = wave_reduce(mass, Add{});
    }
    if (lane == 0)
        static_cast<ChunkStat *>(a.workspace)[t * n.chunks + c] = ChunkStat{mass, m, 0};
}

// ---- pick_kernel -----------------------------------------------------------------

struct Shared {
    uint64_t hist[kBins];
    uint64_t chunk_units[kMaxChunks];
    uint32_t chunk_ties[kMaxChunks];
    uint32_t chunk_key[kMaxChunks];  // of the chunk's maximum
    uint32_t list_key[kList];
    uint32_t list_at[kList];
    uint64_t wave_sum[kPickWaves];
    uint32_t wave_max[kPickWaves];
    uint64_t found_before;
    uint32_t found_bin;
    uint32_t list_size;
    uint32_t bound;      // of the candidates
    uint32_t chosen;     // the token's chunk,
    uint64_t chosen_at;  // the units before the token in it
    uint64_t chosen_ties;  // and the ties before the chunk
};

__device__ __forceinline__ void add(uint64_t &sum, uint64_t x) {  // in LDS
    atomicAdd(reinterpret_cast<unsigned long long *>(&sum), static_cast<unsigned long long>(x));
}

__device__ __forceinline__ uint64_t shuffle_up(uint64_t x, int by) {
    return __shfl_up(static_cast<unsigned long long>(x), by);
}

__device__ __forceinline__ uint64_t wave_scan(uint64_t x, int lane) {  // inclusive
#pragma unroll
    for (int by = 1; by < kRowWave; by *= 2) {
        const uint64_t y = shuffle_up(x, by);
        if (lane >= by) x += y;
    }
    return x;
}

// Exclusive sum over the workgroup's threads, and the whole sum.
__device__ __forceinline__ uint64_t block_scan(Shared &s, uint64_t x, uint64_t &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t inc = wave_scan(x, lane);
    __syncthreads();  // wave_sum may still be read from the call before
    if (lane == 63) s.wave_sum[wave] = inc;
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

// A row in pick_kernel.
template <int D>
struct Row {
    const Stored<D> *logits;
    int vocab, chunks;
    float max;
    double scale;  // log2(e) / temperature

    // a weight in units; at least one, so that what may be drawn can be
    __device__ __forceinline__ uint64_t units(uint32_t key) const {
        const double t = log2_weight(value_of(key), max, scale);
        const double i = __builtin_rint(t);
        const double w =
            __builtin_ldexp(exp2_fraction(t - i), static_cast<int>(i) + kUnitBits);
        const uint64_t u = __builtin_bit_cast(uint64_t, w + 0x1p52) & ((uint64_t{1} << 52) - 1);
        return u > 0 ? u : 1;
    }
};

// Where weights are sought: the row's chunks whose maximum reaches `least`...
template <int D>
struct InRow {
    const Shared &s;
    const Row<D> &r;
    template <class F>
    __device__ __forceinline__ void each(uint32_t least, F f) const {
        const int lane = threadIdx.x & 63;
        for (int c = threadIdx.x >> 6; c < r.chunks; c += kPickWaves) {
            if (s.chunk_key[c] < least) continue;
            float x[kPer];
            load_chunk<D>(r.logits, r.vocab, c, lane, x);
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const uint32_t k = key_of(x[i]);
                if (k >= least) f(k, chunk_at<D>(c, lane, i));
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

// Candidates from key `least` to `most` into the list, in no order. False if they
// do not fit.
template <class From>
__device__ __forceinline__ bool collect(Shared &s, const From &from, uint32_t least, uint32_t most) {
    __syncthreads();
    if (threadIdx.x == 0) s.list_size = 0;
    __syncthreads();
    from.each(least, [&](uint32_t k, int at) {
        if (k > most) return;
        const uint32_t i = atomicAdd(&s.list_size, 1u);
        if (i < kList) {
            s.list_key[i] = k;
            s.list_at[i] = static_cast<uint32_t>(at);
        }
    });
    __syncthreads();
    return s.list_size <= kList;
}

// The bin in which the running sum over bins reaches target (>= 1, at most the
// whole sum), and the sum before it.
__device__ __forceinline__ void find_bin(Shared &s, int bins, uint64_t target, uint32_t &bin,
                                         uint64_t &before) {
    constexpr int each = (kBins + kThreads - 1) / kThreads;
    __syncthreads();
    uint64_t v[each], sum = 0;
#pragma unroll
    for (int i = 0; i < each; ++i) {
        const int b = threadIdx.x * each + i;
        v[i] = b < bins ? s.hist[b] : 0;
        sum += v[i];
    }
    uint64_t total;
    uint64_t run = block_scan(s, sum, total);
#pragma unroll
    for (int i = 0; i < each; ++i) {
        if (run < target && target <= run + v[i]) {
            s.found_bin = threadIdx.x * each + i;
            s.found_before = run;
        }
        run += v[i];
    }
    __syncthreads();
    bin = s.found_bin;
    before = s.found_before;
}

__device__ __forceinline__ void clear_bins(Shared &s) {
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += kThreads) s.hist[b] = 0;
    __syncthreads();
}

struct Border {
    uint32_t key;     // of the element in which the running sum reaches the target
    uint64_t before;  // the sum over larger keys
};

// In descending order of keys from `top` down to, not including, `floor`: where
// does the running sum of weights reach target? The whole sum has to reach it.
// Histograms over the distance d = top - key: first log-linear bins, 64 to an
// octave, over all 32 bits, then 1024 at a time inside the bin that was found.
template <class From, class W>
__device__ __forceinline__ Border narrow(Shared &s, const From &from, uint32_t top, uint32_t floor,
                                         uint32_t lo, int bits, uint64_t before, uint64_t target,
                                         W weight) {
    while (bits > 0) {
        const int shift = bits > 10 ? bits - 10 : 0;
        const uint32_t last = lo + ((1u << bits) - 1);  // d of the bin's end
        uint32_t least = last >= lo && top >= last ? top - last : 0;
        if (least <= floor) least = floor + 1;
        clear_bins(s);
        from.each(least, [&](uint32_t k, int) {
            const uint32_t d = top - k;
            if (k <= top && d >= lo) add(s.hist[(d - lo) >> shift], weight(k));
        });
        uint32_t bin;
        uint64_t in;
        find_bin(s, 1024, target - before, bin, in);
        before += in;
        lo += bin << shift;
        bits = shift;
    }
    return Border{top - lo, before};
}

template <class From, class W>
__device__ __forceinline__ Border seek(Shared &s, const From &from, bool in_list, uint32_t top,
                                       uint32_t floor, uint64_t target, W weight) {
    clear_bins(s);
    from.each(floor + 1, [&](uint32_t k, int) {
        const uint32_t d = top - k;
        const int e = d < 64 ? 6 : 31 - __builtin_clz(d);
        const uint32_t bin = d < 64 ? d : 64 + (e - 6) * 64 + ((d >> (e - 6)) & 63);
        add(s.hist[bin], weight(k));
    });
    uint32_t bin;
    uint64_t before;
    find_bin(s, kBins, target, bin, before);
    const int bits = bin < 64 ? 0 : (bin - 64) / 64;
    const uint32_t lo = bin < 64 ? bin : (64 + (bin & 63)) << bits;
    if (bits == 0) return Border{top - lo, before};
    if (!in_list) {
        const uint32_t last = lo + ((1u << bits) - 1);
        uint32_t least = last >= lo && top >= last ? top - last : 0;
        if (least <= floor) least = floor + 1;
        if (collect(s, from, least, top - lo))
            return narrow(s, InList{s, s.list_size}, top, floor, lo, bits, before, target, weight);
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
    uint64_t all, tied;
    block_scan(s, sum, all);
    block_scan(s, ties, tied);
    if (tied > keep.ties) tied = keep.ties;
    return tied ? all + tied * r.units(keep.key) : all;
}

// top-k, then top-p over what `from` holds: everything that may be kept. units:
// the weights' sum, if known (else 0).
template <int D, class From>
__device__ __forceinline__ void filter(Shared &s, const From &from, bool in_list, const Row<D> &r,
                                       const Draw &d, uint32_t top, uint64_t units, Keep &keep) {
    if (d.top_k > 0) {
        uint64_t mine = 0, there;
        from.each(keep.key, [&](uint32_t, int) { ++mine; });
        block_scan(s, mine, there);
        const uint64_t k = static_cast<uint64_t>(d.top_k);
        if (there > k) {
            const Border b = seek(s, from, in_list, top, keep.key - 1, k,
                                  [](uint32_t) { return uint64_t{1}; });
            keep = Keep{b.key, static_cast<uint32_t>(k - b.before)};
        }
        units = 0;
    }
    if (!(d.top_p < 1.0f)) return;
    const uint64_t all = units ? units : kept_units(s, from, r, keep);
    const double part = static_cast<double>(d.top_p) * static_cast<double>(all);
    uint64_t target = part > 1.0 ? static_cast<uint64_t>(part) : 1;
    if (static_cast<double>(target) < part) ++target;
    const auto weight = [&](uint32_t k) { return r.units(k); };
    // the weight above the least kept key decides whether the border lies there
    uint64_t mine = 0, above;
    from.each(keep.key + 1, [&](uint32_t k, int) { mine += r.units(k); });
    block_scan(s, mine, above);
    if (target > above) {
        const uint64_t w = r.units(keep.key);
        const uint64_t ties = (target - above + w - 1) / w;
        if (ties < keep.ties) keep.ties = static_cast<uint32_t>(ties);
        return;
    }
    const Border b = seek(s, from, in_list, top, keep.key, target, weight);
    const uint64_t w = r.units(b.key);
    keep = Keep{b.key, static_cast<uint32_t>((target - b.before + w - 1) / w)};
}

template <int D>
__global__ void __launch_bounds__(kThreads) pick_kernel(const SampleArgs n) {
    __shared__ Shared s;
    const sifar_sample_args &a = n.a;
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Draw d = draw_of(a, t);
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
    r.scale = d.greedy ? 0.0 : kLog2e / static_cast<double>(d.temperature);

    uint64_t units = 0;  // of this thread's chunk
    Keep keep{top, 1};
    bool by_row = false;  // what is kept is not in the list
    bool plain = false;   // every weight above the cut is kept: the scan's sums serve
    if (!d.greedy) {
        const double max = static_cast<double>(r.max), tau = static_cast<double>(d.temperature);
        const bool finite = r.max < __builtin_inff();
        keep = Keep{finite ? key_from(max - kCut * kLn2 * tau) : top, kAllTies};
        uint32_t least = keep.key;  // of min-p
        // at an infinite temperature every weight is 1
        if (d.min_p > 0.0f && finite && d.temperature < __builtin_inff()) {
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
        const bool filtered = d.top_k > 0 || d.top_p < 1.0f;
        plain = !filtered && !(d.min_p > 0.0f);
        if (filtered) {
            uint64_t all;
            block_scan(s, units, all);  // top-p's sum; 0 where top-k comes first
            // Candidates above the rank-th largest chunk maximum: at least `rank` of them, so
            // enough for top-k, and likely for a nucleus.
            const int rank = d.top_k > 0 ? d.top_k : kNucleus;
            uint32_t from = keep.key;
            if (rank < n.chunks) {
                int larger = 0;
                for (int c = 0; c < n.chunks; ++c)
                    larger += s.chunk_key[c] > my_key || (s.chunk_key[c] == my_key && c < tid);
                if (tid < n.chunks && larger == rank - 1) s.bound = my_key;
                __syncthreads();
                from = s.bound > from ? s.bound : from;
            }
            bool listed = collect(s, InRow<D>{s, r}, from, top);
            if (listed && d.top_k <= 0 && from > keep.key)
                listed = static_cast<double>(kept_units(s, InList{s, s.list_size}, r,
                                                        Keep{from, kAllTies})) >=
                         static_cast<double>(d.top_p) * static_cast<double>(all) + 1.0;
            if (listed) {
                keep.key = from;
                filter(s, InList{s, s.list_size}, true, r, d, top, d.top_k > 0 ? 0 : all, keep);
            } else {
                filter(s, InRow<D>{s, r}, false, r, d, top, d.top_k > 0 ? 0 : all, keep);
            }
            if (least > keep.key) keep = Keep{least, kAllTies};
            if (listed) {
                InList{s, s.list_size}.each(keep.key, [&](uint32_t k, int at) {
                    if (k > keep.key) add(s.chunk_units[at / kChunkElems], r.units(k));
                    else atomicAdd(&s.chunk_ties[at / kChunkElems], 1u);
                });
            }
            by_row = !listed;
        } else if (!plain) {
            keep = Keep{least, kAllTies};
            by_row = true;
        }
        if (by_row) {
            for (int c = wave; c < n.chunks; c += kPickWaves) {
                if (s.chunk_key[c] < keep.key) continue;
                float x[kPer];
                load_chunk<D>(r.logits, r.vocab, c, lane, x);
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
            }
        }
        if (!plain) {
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
    const float u = a.uniform[t];
    uint64_t at = u > 0.0f ? static_cast<uint64_t>(
                                 static_cast<double>(u < 1.0f ? u : 1.0f) * static_cast<double>(all))
                           : 0;
    if (at >= all) at = all - 1;
    if (units && before <= at && at < before + units) {
        s.chosen = tid;
        s.chosen_at = at - before;
        s.chosen_ties = ties_before;
    }
    __syncthreads();
    if (wave != 0) return;

    // The token inside the chunk.
    const int c = s.chosen;
    const uint64_t want = s.chosen_at;
    uint64_t ties_run = s.chosen_ties, run = 0;
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
        const uint64_t tie_scan = wave_scan(ties, lane);
        uint64_t rank = ties_run + tie_scan - ties;
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            const uint32_t k = key_of(x[v * VE + i]);
            const bool tie = k == keep.key;
            const bool in = k > keep.key || (tie && rank < keep.ties);
            rank += tie;
            w[i] = !in ? 0 : d.greedy ? 1 : r.units(k);
            sum += w[i];
        }
        const uint64_t scan = wave_scan(sum, lane);
        uint64_t low = run + scan - sum;
        int here = -1, kept = -1;
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            if (w[i] && low <= want && want < low + w[i]) here = chunk_at<D>(c, lane, v * VE + i);
            if (w[i]) kept = chunk_at<D>(c, lane, v * VE + i);
            low += w[i];
        }
        const int found = static_cast<int>(wave_reduce(static_cast<uint32_t>(here + 1), Max{})) - 1;
        const int tail = static_cast<int>(wave_reduce(static_cast<uint32_t>(kept + 1), Max{})) - 1;
        if (token < 0) token = found;
        if (tail >= 0) last = tail;
        run += lane_value(scan, 63);
        ties_run += lane_value(tie_scan, 63);
    }
    if (token < 0) token = last;  // the chunk's own sum was rounded up
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
